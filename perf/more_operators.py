"""Operators of an MoE layer kept in 16 bits, and of its activations kept in 8 bits for the backward pass, as cases that can be
timed and compared.

The experts' products on bf16 tensors (forward, the input's and the weights' gradients, rows in the order of their experts);
checkpoints of activations in 8 bits (E4M3 levels, a power of two per 32 values of a row) and back; the experts' activation with
its checkpoint, and its gradient from that; the weights' gradient from a checkpoint of the input. Each case is computed in plain
torch operations in 32 bits, or, where `own` is true, by the framework's entry points. Activations are N(0, 1) with 0.1% of the
channels x50 and a mean that is not zero, weights N(0, 0.02^2), gradients N(0, 1e-3^2); tokens choose their experts by a power law.
"""

from __future__ import annotations

import math

import torch

own = False

LARGEST = 3 * 32768 * 5120 * 4096  # multiplications of the largest case


def listed():
    return [
        # one token through the two experts it chose, a small model's FFN: launch latency
        {"name": "experts-token", "op": "product", "pass": "fwd", "tokens": 1, "k": 2, "groups": 8, "N": 1312, "K": 512, "out": "bf16"},
        # a decode step of the 7.9B MoE model, 7 sequences: bound by reading the chosen experts' weights
        {"name": "experts-decode", "op": "product", "pass": "fwd", "tokens": 7, "k": 6, "groups": 64, "N": 1408, "K": 2048, "out": "bf16"},
        # its training micro-batch, forward
        {"name": "experts-fwd", "op": "product", "pass": "fwd", "tokens": 16384, "k": 6, "groups": 64, "N": 1408, "K": 2048, "out": "bf16"},
        # the input's gradient
        {"name": "experts-grad-x", "op": "product", "pass": "dx", "tokens": 16384, "k": 6, "groups": 64, "N": 1408, "K": 2048, "out": "bf16"},
        # the weights' gradient, kept in fp32 for the optimizer
        {"name": "experts-grad-w", "op": "product", "pass": "dw", "tokens": 16384, "k": 6, "groups": 64, "N": 1408, "K": 2048, "out": "f32"},
        # a whole step of experts with no size that a tile divides (a short batch, odd widths), fp32 results
        {"name": "experts-odd", "op": "product", "pass": "all", "tokens": 1683, "k": 2, "groups": 16, "N": 1313, "K": 515, "out": "f32"},
        # a whole step of few wide experts, one GPU's share of a large model
        {"name": "experts-wide", "op": "product", "pass": "all", "tokens": 16384, "k": 2, "groups": 8, "N": 4096, "K": 5120, "out": "bf16"},
        # the weights' gradient where the forward pass kept its input in 8 bits
        {"name": "grad-w-saved", "op": "saved", "tokens": 16384, "k": 6, "groups": 64, "N": 1408, "K": 2048, "out": "f32"},
        # a 1 GiB tensor to 8 bits and back, the quantizer benchmark's size
        {"name": "save-1gib", "op": "save", "rows": 32768, "cols": 16384, "dtype": "bf16"},
        # an fp32 tensor of odd sizes (rows of a packed batch, a width no block divides)
        {"name": "save-odd", "op": "save", "rows": 4099, "cols": 1411, "dtype": "f32"},
        # squared ReLU of the 7.9B model's experts at the training micro-batch: forward with the checkpoint, then backward from it
        {"name": "act-train", "op": "act", "kind": "relu2", "rows": 98304, "cols": 1408, "dtype": "bf16"},
        # gated SiLU in fp32, odd sizes
        {"name": "act-gated-odd", "op": "act", "kind": "swiglu", "rows": 4099, "cols": 1411, "dtype": "f32"},
    ]


def _log(rng, lo, hi, mult=1):
    """A multiple of `mult`, spread over the logarithm of lo..hi."""
    return max(mult, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi))) / mult)) * mult)


def draw(rng):
    op = rng.choice(["product", "product", "product", "product", "saved", "save", "act", "act"])
    while True:
        if op in ("product", "saved"):
            groups = rng.choice([1, 4, 8, 16, 40, 64, 128])
            c = {"op": op, "tokens": _log(rng, 1, 32768), "k": rng.choice([k for k in (1, 2, 4, 6, 8) if k <= groups]), "groups": groups,
                 "N": _log(rng, 64, 8192, rng.choice([1, 8, 64])), "K": _log(rng, 64, 8192, rng.choice([1, 8, 64])),
                 "out": rng.choice(["bf16", "f32"])}
            if op == "product":
                c["pass"] = rng.choice(["fwd", "fwd", "dx", "dw", "all"])
            passes = 3 if c.get("pass") == "all" else 1
            if passes * c["tokens"] * c["k"] * c["N"] * c["K"] <= LARGEST and groups * c["N"] * c["K"] <= 1 << 28:
                return c
        elif op == "save":
            c = {"op": op, "rows": _log(rng, 1, 32768), "cols": _log(rng, 32, 16384, rng.choice([1, 8, 32])),
                 "dtype": rng.choice(["bf16", "bf16", "f32"])}
            if c["rows"] * c["cols"] <= 1 << 28:
                return c
        else:
            c = {"op": op, "kind": rng.choice(["relu2", "swiglu"]), "rows": _log(rng, 1, 131072),
                 "cols": _log(rng, 32, 8192, rng.choice([1, 8, 32])), "dtype": rng.choice(["bf16", "bf16", "f32"])}
            if c["rows"] * c["cols"] <= 1 << 27:
                return c


# ---------------------------------------------------------------------------------------------------
# Inputs
# ---------------------------------------------------------------------------------------------------


def _normal(g, std, *shape):
    return torch.randn(*shape, generator=g, device="cuda") * std


def _acts(g, rows, cols):
    x = torch.randn(rows, cols, generator=g, device="cuda")
    ch = torch.randperm(cols, generator=g, device="cuda")[: max(1, round(0.001 * cols))]
    x[:, ch] *= 50.0
    return x + 0.25


def _loads(g, tokens, k, groups):
    """Rows per expert: every token takes k different ones, popular ones more often."""
    liked = -1.1 * torch.log(torch.arange(1, groups + 1, device="cuda", dtype=torch.float32))
    liked = liked[torch.randperm(groups, generator=g, device="cuda")]
    noise = -torch.log(-torch.log(torch.rand(tokens, groups, generator=g, device="cuda").clamp(1e-6, 1 - 1e-6)))
    ids = torch.topk(liked + noise, k, dim=1).indices
    return torch.bincount(ids.reshape(-1), minlength=groups)


def prepare(case, seed):
    g = torch.Generator(device="cuda").manual_seed(seed * 6151 + 17)
    s, op = dict(case), case["op"]
    dt = {"bf16": torch.bfloat16, "f32": torch.float32}[case.get("dtype", "bf16")]
    if op in ("product", "saved"):
        rows, N, K = case["tokens"] * case["k"], case["N"], case["K"]
        loads = _loads(g, case["tokens"], case["k"], case["groups"])
        s["offsets"] = torch.cat([torch.zeros_like(loads[:1]), loads.cumsum(0)])
        s["counts"] = loads.tolist()
        what = case.get("pass", "dw")
        if what != "dx":
            s["x"] = _acts(g, rows, K).bfloat16()
        if what != "fwd":
            s["dy"] = _normal(g, 1e-3, rows, N).bfloat16()
        if what != "dw":
            s["w"] = _normal(g, 0.02, case["groups"] * N, K).bfloat16()
    elif op == "save":
        s["x"] = _acts(g, case["rows"], case["cols"]).to(dt)
    else:
        wide = case["cols"] * (2 if case["kind"] == "swiglu" else 1)
        s["u"] = _normal(g, 1.0, case["rows"], wide).to(dt)
        s["da"] = _normal(g, 1e-3, case["rows"], case["cols"]).to(dt)
    s["dt"], s["odt"] = dt, torch.float32 if case.get("out") == "f32" else torch.bfloat16
    return s


# ---------------------------------------------------------------------------------------------------
# One pass
# ---------------------------------------------------------------------------------------------------


def run(state):
    return (_run_own if own else _run_plain)(state)


def _run_own(s):
    from paper_2606_20381_amd import ufp4 as U

    op = s["op"]
    if op == "save":
        return U.checkpoint8_load(U.checkpoint8_save(s["x"]), s["dt"])
    if op == "act":
        a, kept = U.activation(s["u"], s["kind"], save=True)
        du, again = U.activation_bwd(s["da"], kept, s["kind"])
        return {"a": a, "du": du, "again": again}
    if op == "saved":
        return U.bf16_gemm_bwd_dw_grouped(s["dy"], U.checkpoint8_save(s["x"]), s["offsets"], s["odt"])
    out, what = {}, s["pass"]
    if what in ("fwd", "all"):
        out["y"] = U.bf16_gemm_fwd_y_grouped(s["x"], s["w"], s["offsets"], s["odt"])
    if what in ("dx", "all"):
        out["dx"] = U.bf16_gemm_bwd_dx_grouped(s["dy"], s["w"], s["offsets"], s["odt"])
    if what in ("dw", "all"):
        out["dw"] = U.bf16_gemm_bwd_dw_grouped(s["dy"], s["x"], s["offsets"], s["odt"])
    return out


def _eight(x):
    """x's values in 8 bits: per 32 of a row the smallest power of two 2^e with max|x| <= 448 2^e (e >= -124), levels of E4M3."""
    cols = x.shape[1]
    v = torch.nn.functional.pad(x.float(), (0, -cols % 32)).view(x.shape[0], -1, 32)
    m, p = torch.frexp(v.abs().amax(-1, keepdim=True))
    e = (p - 9 + (m > 0.875).to(p.dtype)).clamp(min=-124)
    v = torch.ldexp(v, -e)
    bits = (torch.frexp(v).exponent - 4).clamp(min=-9)  # the last of four significant bits, 2^-9 in the subnormal range
    v = torch.ldexp(torch.round(torch.ldexp(v, -bits)), bits)
    return torch.ldexp(v, e).view(x.shape[0], -1)[:, :cols]


def _eight_parts(u, kind):
    """A gated activation's input has two halves, each in blocks of its own."""
    return _eight(u) if kind == "relu2" else torch.cat([_eight(p) for p in u.chunk(2, 1)], 1)


def _act(u, kind):
    if kind == "relu2":
        return u.clamp(min=0).square()
    g, v = u.chunk(2, 1)
    return g / (1 + torch.exp(-g)) * v


def _act_grad(da, u, kind):
    if kind == "relu2":
        return 2 * u.clamp(min=0) * da
    g, v = u.chunk(2, 1)
    s = 1 / (1 + torch.exp(-g))
    return torch.cat([da * v * s * (1 + g * (1 - s)), da * g * s], 1)


def _run_plain(s):
    op = s["op"]
    if op == "save":
        return _eight(s["x"]).to(s["dt"])
    if op == "act":
        kept, da = _eight_parts(s["u"], s["kind"]), s["da"].float()
        return {"a": _act(s["u"].float(), s["kind"]).to(s["dt"]), "du": _act_grad(da, kept, s["kind"]).to(s["dt"]),
                "again": _act(kept, s["kind"]).to(s["dt"])}
    if op == "saved":
        dy, x = s["dy"].float().split(s["counts"]), _eight(s["x"]).split(s["counts"])
        return torch.stack([d.t() @ v for d, v in zip(dy, x)]).to(s["odt"])
    out, what, counts = {}, s["pass"], s["counts"]
    w = s["w"].float().split(s["N"]) if what != "dw" else None
    if what in ("fwd", "all"):
        out["y"] = torch.cat([x @ m.t() for x, m in zip(s["x"].float().split(counts), w)]).to(s["odt"])
    if what in ("dx", "all"):
        out["dx"] = torch.cat([d @ m for d, m in zip(s["dy"].float().split(counts), w)]).to(s["odt"])
    if what in ("dw", "all"):
        out["dw"] = torch.stack([d.t() @ x for d, x in zip(s["dy"].float().split(counts), s["x"].float().split(counts))]).to(s["odt"])
    return out


# ---------------------------------------------------------------------------------------------------
# What a pass cannot do without
# ---------------------------------------------------------------------------------------------------


def _chosen(case):
    """How many experts have rows, on average over the power law's draws (each token's k choices taken as independent of the others')."""
    share = [(i + 1) ** -1.1 for i in range(case["groups"])]
    each = [min(1.0, case["k"] * v / sum(share)) for v in share]
    return max(case["k"], round(sum(1.0 - (1.0 - p) ** case["tokens"] for p in each)))


def work(case):
    op = case["op"]
    if op in ("product", "saved"):
        rows, N, K, groups = case["tokens"] * case["k"], case["N"], case["K"], case["groups"]
        o = 4 if case["out"] == "f32" else 2
        x, dy, w, mul = rows * K, rows * N, _chosen(case) * N * K, rows * N * K
        if op == "saved":  # x is read, and its checkpoint written and read
            return {"bytes": 2 * x + 2 * x * 33 // 32 + 2 * dy + groups * N * K * o, "flops": 2 * mul}
        moved = {"fwd": 2 * (x + w) + dy * o, "dx": 2 * (dy + w) + x * o, "dw": 2 * (x + dy) + groups * N * K * o,
                 "all": 2 * (x + dy + w) + (x + dy + groups * N * K) * o}
        return {"bytes": moved[case["pass"]], "flops": 2 * mul * (3 if case["pass"] == "all" else 1)}
    n, b = case["rows"] * case["cols"], 4 if case["dtype"] == "f32" else 2
    if op == "save":  # x read, the checkpoint written and read, its values written
        return {"bytes": 2 * n * b + 2 * n * 33 // 32, "flops": 4 * n}
    wide = 2 * n if case["kind"] == "swiglu" else n
    # u read, a and the checkpoint written; da and the checkpoint read, du and a written
    return {"bytes": 2 * wide * b + 3 * n * b + 2 * wide * 33 // 32, "flops": 20 * n}


# ---------------------------------------------------------------------------------------------------
# The definitions in 64 bits
# ---------------------------------------------------------------------------------------------------


def _eight64(x):
    """The 8-bit values by search: the scale by trial of powers of two, the level from the middles between neighbours (a middle
    belongs to the level with the even number)."""
    at = torch.tensor([n * 2.0**-9 if n < 8 else (8 + n % 8) * 2.0 ** (n // 8 - 10) for n in range(127)], dtype=torch.float64, device=x.device)
    middle = (at[1:] + at[:-1]) / 2
    rows, cols = x.shape
    t = torch.zeros(rows, (cols + 31) // 32 * 32, dtype=torch.float64, device=x.device)
    t[:, :cols] = x
    t = t.view(rows, -1, 32)
    top = t.abs().max(dim=2, keepdim=True).values
    e = torch.ceil(torch.log2(top.clamp(min=1e-300) / 448.0))
    e = torch.where(448.0 * torch.exp2(e - 1) >= top, e - 1, torch.where(448.0 * torch.exp2(e) < top, e + 1, e)).clamp(min=-124.0)
    a = (t.abs() / torch.exp2(e)).contiguous()
    low = torch.searchsorted(middle, a)  # middles below a
    n = low + ((low % 2 == 1) & (middle[low.clamp(max=125)] == a)).long()
    return (torch.sign(t) * at[n] * torch.exp2(e)).view(rows, -1)[:, :cols]


def _silu64(g):
    return g * torch.sigmoid(g), torch.sigmoid(g) + g * torch.sigmoid(g) * torch.sigmoid(-g)


def exact(case, seed):
    s, op = prepare(case, seed), case["op"]
    if op == "save":
        return _eight64(s["x"])
    if op == "act":
        n, u, da = case["cols"], s["u"].double(), s["da"].double()
        kept = torch.empty_like(u)
        for at in range(0, u.shape[1], n):
            kept[:, at : at + n] = _eight64(s["u"][:, at : at + n])
        if case["kind"] == "relu2":
            up, kp = torch.relu(u), torch.relu(kept)
            return {"a": up * up, "du": kp * da * 2.0, "again": kp * kp}
        f, slope = _silu64(kept[:, :n])
        du = torch.empty_like(kept)
        du[:, :n] = slope * kept[:, n:] * da
        du[:, n:] = f * da
        return {"a": _silu64(u[:, :n])[0] * u[:, n:], "du": du, "again": f * kept[:, n:]}
    rows, N, K, groups = case["tokens"] * case["k"], case["N"], case["K"], case["groups"]
    what = case.get("pass", "dw")
    out = {}
    if what in ("fwd", "all"):
        out["y"] = torch.zeros(rows, N, dtype=torch.float64, device="cuda")
    if what in ("dx", "all"):
        out["dx"] = torch.zeros(rows, K, dtype=torch.float64, device="cuda")
    if what in ("dw", "all"):
        out["dw"] = torch.zeros(groups, N, K, dtype=torch.float64, device="cuda")
    kept = _eight64(s["x"]) if op == "saved" else None
    ends = s["offsets"].tolist()
    for e in range(groups):
        at = slice(ends[e], ends[e + 1])
        if "y" in out:
            out["y"][at] = s["x"][at].double() @ s["w"][e * N : (e + 1) * N].double().T
        if "dx" in out:
            out["dx"][at] = s["dy"][at].double() @ s["w"][e * N : (e + 1) * N].double()
        if "dw" in out:
            out["dw"][e] = s["dy"][at].double().T @ (s["x"][at].double() if kept is None else kept[at])
    return out["dw"] if op == "saved" else out
