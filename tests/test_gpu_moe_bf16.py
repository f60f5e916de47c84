"""The MoE layer step with its products in bf16, the gated activation, and activations kept in 8 bits: one operator's output at a time
against 64 bits on the tensors before it, gradients of the whole layer against differences, and captured in a graph.

Tolerance: an output in bf16 is off by its rounding, 2^-8 of itself, and fp32 sums of R terms by R 2^-23 of the sum of magnitudes, below
1e-5 of the largest output here; the norm's gradients, behind two roundings to bf16 of every element they sum, by 2% of their norm.
"""

import pytest
import torch

from paper_2606_20381_amd import moe
from paper_2606_20381_amd import ufp4 as U

pytestmark = pytest.mark.gpu

BF = torch.bfloat16


def _close(got, ref, k=2.0**-8, abs_scale=1e-5):
    if not ref.numel():
        return
    err = (got.double() - ref).abs()
    assert bool((err <= k * ref.abs() + abs_scale * ref.abs().max()).all()), float((err / ref.abs().max()).max())


def _act(u, kind):
    """a and its derivative's parts."""
    if kind == "relu2":
        r = torch.relu(u)
        return r * r, (2 * r,)
    g, v = u.chunk(2, 1)
    s = torch.sigmoid(g)
    return g * s * v, (v * (s + g * s * (1 - s)), g * s)


def _inputs(tokens, experts, k, H, F, activation, seed, drop=False):
    g = torch.Generator(device="cuda").manual_seed(seed)

    def normal(*shape, std=1.0):
        return torch.randn(*shape, generator=g, device="cuda") * std

    wide = F * (2 if activation == "swiglu" else 1)
    s = {"x": normal(tokens, H).to(BF), "dout": normal(tokens, H).to(BF), "gamma": 1 + 0.1 * normal(H), "beta": 0.1 * normal(H),
         "w1": normal(experts * wide, H, std=0.1).to(BF), "w2": normal(experts * H, F, std=0.1).to(BF),
         "ids": torch.topk(normal(tokens, experts), k, dim=1).indices, "gate": torch.softmax(normal(tokens, k), 1)}
    if drop:
        s["ids"][torch.rand(tokens, k, generator=g, device="cuda") < 0.2] = -1
    return s


@pytest.mark.parametrize("save8", [False, True])
@pytest.mark.parametrize("activation", ["relu2", "swiglu"])
@pytest.mark.parametrize("tokens,experts,k,H,F,drop", [(1, 4, 2, 128, 256, False), (100, 8, 2, 72, 131, True), (900, 4, 3, 264, 136, False),
                                                       (64, 70, 1, 40, 33, True)])
def test_layer_against_plain(tokens, experts, k, H, F, drop, activation, save8):
    s = _inputs(tokens, experts, k, H, F, activation, tokens, drop)
    layer = moe.MoELayer(experts, H, F, k, precision="bf16", activation=activation, save8=save8)
    layer.load_weights(s["w1"], s["w2"])
    out = layer.forward(s["x"], s["ids"], s["gate"], s["gamma"], s["beta"])
    _, _, _, mean, rstd, offsets, rows, hs, u, a, y = layer.saved
    grads = layer.backward(s["dout"])
    off = offsets.tolist()
    assert off[-1] == int((s["ids"] >= 0).sum())
    h = U.layer_norm(s["x"], s["gamma"], s["beta"])[0]
    exact_hs = U.moe_dispatch(h, rows, offsets)
    if save8:
        assert a is None
        hs, u, y = (U.checkpoint8_load(t) for t in (hs, u, y))
        for kept, ref in ((hs, exact_hs),):  # what is kept is within half a step, 2^-4, or of the block's smallest step
            err = (kept[: off[-1]].double() - ref[: off[-1]].double()).abs()
            assert bool((err <= 2.0**-4 * ref[: off[-1]].double().abs() + 2.0**-17 * ref.double().abs().max()).all())
    else:
        assert torch.equal(hs, exact_hs)
    wide = F * (2 if activation == "swiglu" else 1)
    dy = U.moe_dispatch(s["dout"], rows, offsets, s["gate"])
    dhs = torch.zeros(tokens * k, H, dtype=BF, device="cuda")
    forward = torch.zeros(tokens * k, H, dtype=torch.float64, device="cuda")
    for e in range(experts):
        at = slice(off[e], off[e + 1])
        w1e, w2e = s["w1"][e * wide : (e + 1) * wide].double(), s["w2"][e * H : (e + 1) * H].double()
        exact_u = (exact_hs[at].double() @ w1e.t())
        if not save8:
            _close(u[at], exact_u)
        ae, slopes = _act(u[at].double(), activation)
        ae = ae.to(BF)
        if not save8:
            _close(a[at], ae.double(), 2.0**-7)
            _close(y[at], a[at].double() @ w2e.t())
        forward[at] = y[at].double()
        _close(grads["w2"][e], dy[at].double().t() @ (ae if save8 else a[at]).double(), 2.0**-8 if save8 else 1e-5)
        da = (dy[at].double() @ w2e).to(BF).double()
        du = torch.cat([p * da for p in slopes], 1).to(BF)
        # da may differ in its last bit from the kernel's: the gradients behind it as a whole
        ref = du.double().t() @ hs[at].double()
        assert float((grads["w1"][e].double() - ref).norm()) <= 0.01 * float(ref.norm()) + 1e-12
        dhs[at] = (du.double() @ w1e).to(BF)
    flat = rows.long()
    picked = torch.where((flat >= 0)[:, :, None], forward[flat.clamp(min=0)], 0.0)
    if not save8:
        _close(out, (picked * s["gate"].double()[:, :, None]).sum(1), 2.0**-7)
    _close(grads["gate"], (picked * s["dout"].double()[:, None]).sum(2), 1e-5)
    dh = torch.where((flat >= 0)[:, :, None], dhs.double()[flat.clamp(min=0)], 0.0).sum(1)
    xh = (s["x"].double() - mean.double()[:, None]) * rstd.double()[:, None]
    t = dh * s["gamma"].double()
    dx = rstd.double()[:, None] * (t - t.mean(1, keepdim=True) - xh * (t * xh).mean(1, keepdim=True))
    for got, ref in ((grads["x"], dx), (grads["gamma"], (dh * xh).sum(0)), (grads["beta"], dh.sum(0))):
        assert float((got.double() - ref).norm()) <= 0.02 * float(ref.norm()) + 1e-12


@pytest.mark.parametrize("precision", ["mxfp4", "bf16"])
def test_kept_in_8_bits_changes_little(precision):
    """Gradients from 8-bit activations against those from bf16 ones: every kept value is within 2^-4 of itself, errors of either sign, so
    the gradients' norms differ by less than that."""
    s = _inputs(600, 8, 2, 256, 384, "swiglu", 3)
    grads = []
    for save8 in (False, True):
        layer = moe.MoELayer(8, 256, 384, 2, precision=precision, activation="swiglu", save8=save8)
        layer.load_weights(s["w1"], s["w2"])
        out = layer.forward(s["x"], s["ids"], s["gate"], s["gamma"], s["beta"])
        grads.append(dict(layer.backward(s["dout"], stochastic=False), out=out))
    assert torch.equal(grads[0]["out"], grads[1]["out"])
    limit = 2.0**-4 if precision == "bf16" else 0.2  # in 4 bits a kept value can move a code to the next level
    for n, ref in grads[0].items():
        assert float((grads[1][n].double() - ref.double()).norm()) <= limit * float(ref.double().norm()), n


def test_gradients_by_differences():
    """The layer's loss <dout, out> along a random direction of every input, in differences that bf16's rounding of out leaves meaningful:
    steps of a few percent, central, averaged over all outputs."""
    s = _inputs(512, 4, 2, 128, 192, "swiglu", 8)
    layer = moe.MoELayer(4, 128, 192, 2, precision="bf16", activation="swiglu")
    g = torch.Generator(device="cuda").manual_seed(1)

    def loss(t):
        layer.load_weights(t["w1"].to(BF), t["w2"].to(BF))
        out = layer.forward(t["x"].to(BF), t["ids"], t["gate"], t["gamma"], t["beta"])
        return float((out.double() * s["dout"].double()).sum())

    loss(s)
    grads = layer.backward(s["dout"])
    for n, scale in (("x", 0.05), ("w1", 0.005), ("w2", 0.005), ("gate", 0.05), ("gamma", 0.05), ("beta", 0.05)):
        grad = grads[n].reshape(s[n].shape).double()
        way = torch.sign(grad) * torch.rand(s[n].shape, generator=g, device="cuda").double()  # downhill in every place: a large difference
        up, down = dict(s), dict(s)
        up[n], down[n] = (s[n].double() + scale * way), (s[n].double() - scale * way)
        if n in ("gate", "gamma", "beta"):
            up[n], down[n] = up[n].float(), down[n].float()
        taken = (up[n].to(BF).double() - down[n].to(BF).double()) if n in ("x", "w1", "w2") else up[n].double() - down[n].double()
        want = float((grad * taken).sum())
        assert abs(loss(up) - loss(down) - want) <= 0.05 * abs(want), n


def test_command():
    """The command runs in every form (how far the loss falls is not looked at)."""
    base = ["--steps", "3", "--tokens", "512", "--experts", "4", "--hidden", "128", "--ffn", "128"]
    for more in (["--precision", "bf16"], ["--precision", "bf16", "--activation", "swiglu", "--save8"], ["--activation", "swiglu", "--save8"]):
        losses = moe.main(base + more)
        assert len(losses) == 3 and all(v == v and v < float("inf") for v in losses)


def test_refusals():
    for kw in (dict(precision="fp8"), dict(activation="gelu")):
        with pytest.raises(ValueError):
            moe.MoELayer(4, 128, 128, 2, **kw)
    layer = moe.MoELayer(2, 100, 60, 1, precision="bf16", activation="swiglu")  # any sizes in bf16
    with pytest.raises(ValueError):
        layer.load_weights(torch.zeros(2 * 60, 100, dtype=BF, device="cuda"), torch.zeros(200, 60, dtype=BF, device="cuda"))


def test_binding_refusals():
    """What only tensors on a GPU reach."""
    bf = lambda *s: torch.zeros(*s, dtype=BF, device="cuda")  # noqa: E731
    off = torch.zeros(3, dtype=torch.int64, device="cuda")
    x, w, dy = bf(4, 8), bf(32, 8), bf(4, 16)
    kept = U.checkpoint8_save(x)
    bad = [lambda: U.bf16_gemm_fwd_y_grouped(x.float(), w, off), lambda: U.bf16_gemm_fwd_y_grouped(x, w.float(), off),
           lambda: U.bf16_gemm_fwd_y_grouped(x, bf(31, 8), off), lambda: U.bf16_gemm_fwd_y_grouped(x, bf(32, 9), off),
           lambda: U.bf16_gemm_fwd_y_grouped(x, w, off.int()), lambda: U.bf16_gemm_fwd_y_grouped(x, w, off[:1]),
           lambda: U.bf16_gemm_fwd_y_grouped(x, w, off[::2]), lambda: U.bf16_gemm_fwd_y_grouped(x, w, off, torch.float16),
           lambda: U.bf16_gemm_fwd_y_grouped(x, w, off, out=bf(4, 15)), lambda: U.bf16_gemm_fwd_y_grouped(x.t(), w, off),
           lambda: U.bf16_gemm_fwd_y_grouped(x, w, off.cpu()), lambda: U.bf16_gemm_bwd_dx_grouped(x, w, off),
           lambda: U.bf16_gemm_bwd_dw_grouped(dy, x[:3], off), lambda: U.bf16_gemm_bwd_dw_grouped(dy, kept, off, out=bf(2, 16, 9)),
           lambda: U.bf16_gemm_bwd_dw_grouped(dy[:3], kept, off), lambda: U.checkpoint8_save(x.half()),
           lambda: U.checkpoint8_save(x, out=U.checkpoint8_save(bf(5, 8))), lambda: U.checkpoint8_load(kept, torch.float16),
           lambda: U.checkpoint8_load(kept, out=bf(4, 9)), lambda: U.activation(x, out=bf(4, 9)), lambda: U.activation(bf(4, 9), "swiglu"),
           lambda: U.activation(x, out=torch.zeros(4, 8, device="cuda")), lambda: U.activation_bwd(x, bf(4, 9)),
           lambda: U.activation_bwd(x, x.float()), lambda: U.activation_bwd(x, x, "swiglu"), lambda: U.activation_bwd(x[:3], kept),
           lambda: U.activation_bwd(x, kept, out=bf(3, 8)), lambda: U.activation_bwd(x.expand(2, 4, 8), kept)]
    for n, call in enumerate(bad):
        with pytest.raises(ValueError):
            call()
            pytest.fail(f"call {n} was taken")
    with pytest.raises(U.UFP4Error):
        U.bf16_gemm_fwd_y_grouped(x, bf(1025 * 16, 8), torch.zeros(1026, dtype=torch.int64, device="cuda"))


def test_graph_replays():
    """Forward and backward captured once, replayed on other inputs and routes with eager work in between; two graphs at once."""
    tokens, experts, k, H, F = 257, 8, 2, 256, 384
    weights = _inputs(1, experts, k, H, F, "swiglu", 2)

    def draw(seed):
        s = _inputs(tokens, experts, k, H, F, "swiglu", seed)
        return {n: s[n] for n in ("x", "dout", "ids", "gate")}

    def layer():
        made = moe.MoELayer(experts, H, F, k, precision="bf16", activation="swiglu", save8=True)
        made.load_weights(weights["w1"], weights["w2"])
        return made

    def step(made, s):
        out = made.forward(s["x"], s["ids"], s["gate"], weights["gamma"], weights["beta"])
        return dict(made.backward(s["dout"]), out=out)

    eager, graphs = layer(), []
    for n in range(2):
        still, made = draw(n), layer()
        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):
            step(made, still)
        torch.cuda.current_stream().wait_stream(side)
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            got = step(made, still)
        graphs.append((graph, still, got))
    for r in range(3):
        wants = []
        for n, (graph, still, got) in enumerate(graphs):
            fresh = draw(10 * r + n + 5)
            for name in still:
                still[name].copy_(fresh[name])
            wants.append(step(eager, fresh))
        streams = [torch.cuda.Stream(), torch.cuda.Stream()]
        torch.cuda.synchronize()
        for s, (graph, _, _) in zip(streams, graphs):  # at the same time
            with torch.cuda.stream(s):
                graph.replay()
        torch.cuda.synchronize()
        for want, (_, _, got) in zip(wants, graphs):
            for name in want:
                assert torch.equal(got[name], want[name]), name
