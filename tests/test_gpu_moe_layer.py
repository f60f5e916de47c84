"""The MoE layer step (paper_2606_20381_amd.moe): every operator together, against the same layer in 64 bits on the values that the
quantizers give, and a few steps of training.

Tolerance: Q of the intermediate tensors is taken from the kernels' own bf16 tensors (a bf16 rounding can move a value to another
level), so what is compared is one operator's output at a time: fp32 sums as in the product tests plus bf16's 2^-8 of the result.
"""

import pytest
import torch

from paper_2606_20381_amd import moe
from paper_2606_20381_amd import ufp4 as U

pytestmark = pytest.mark.gpu

BF = torch.bfloat16


def _q(x):
    """x's rows as microscaled values, 64 bits."""
    return U.mxfp4_dequantize(U.mxfp4_quantize(x)).double()


def _qt(x, mask):
    """x's columns, each expert's tokens filled up to whole blocks and rotated."""
    pad = -x.shape[0] % 32
    x = torch.nn.functional.pad(x, (0, 0, 0, pad))
    return U.mxfp4_dequantize(U.mxfp4_quantize(x, transpose=True, rht=True, sign_mask=mask)).double()


def _close(got, ref, k=2.0**-8, abs_scale=1e-5):
    if not ref.numel():  # an expert without tokens
        return
    err = (got.double() - ref).abs()
    assert bool((err <= k * ref.abs() + abs_scale * ref.abs().max()).all()), float(err.max())


@pytest.mark.parametrize("tokens,experts,k,drop", [(1, 4, 2, False), (100, 8, 2, True), (300, 4, 3, False), (64, 16, 1, True)])
def test_layer_against_plain(tokens, experts, k, drop):
    H, F = 128, 256
    g = torch.Generator(device="cuda").manual_seed(tokens)

    def normal(*shape, std=1.0):
        return torch.randn(*shape, generator=g, device="cuda") * std

    x, dout = normal(tokens, H).to(BF), normal(tokens, H).to(BF)
    w1, w2 = normal(experts * F, H, std=0.1).to(BF), normal(experts * H, F, std=0.1).to(BF)
    gamma, beta = 1 + 0.1 * normal(H), 0.1 * normal(H)
    ids = torch.topk(normal(tokens, experts), k, dim=1).indices
    if drop:
        ids[torch.rand(tokens, k, generator=g, device="cuda") < 0.2] = -1
    gate = torch.softmax(normal(tokens, k), 1)
    layer = moe.MoELayer(experts, H, F, k)
    layer.load_weights(w1, w2)
    out = layer.forward(x, ids, gate, gamma, beta)
    grads = layer.backward(dout, stochastic=False)
    _, _, _, mean, rstd, offsets, rows, hs, u, a, y = layer.saved
    off = offsets.tolist()
    assert off[-1] == int((ids >= 0).sum())

    h = U.layer_norm(x, gamma, beta)[0]
    mask = layer.sign_mask
    dy = U.moe_dispatch(dout, rows, offsets, gate)
    dhs = torch.zeros(tokens * k, H, dtype=BF, device="cuda")
    for e in range(experts):
        s = slice(off[e], off[e + 1])
        tokens_of = [t for t in range(tokens) for j in range(k) if int(ids[t, j]) == e]
        assert torch.equal(hs[s], h[tokens_of])
        w1e, w2e = w1[e * F : (e + 1) * F], w2[e * H : (e + 1) * H]
        _close(u[s], _q(hs[s]) @ _q(w1e).t())
        assert torch.equal(a[s], torch.relu(u[s]) ** 2)
        _close(y[s], _q(a[s]) @ _q(w2e).t())
        _close(grads["w2"][e], _qt(dy[s], mask) @ _qt(a[s], mask).t(), 1e-5)
        da = (_q(dy[s]) @ _q(w2e.t().contiguous()).t()).to(BF)
        du = torch.relu(u[s]) * 2 * da
        # da may differ in its last bit from the kernel's, and a code with it: the weight gradient as a whole
        ref = _qt(du, mask) @ _qt(hs[s], mask).t()
        assert float((grads["w1"][e].double() - ref).norm()) <= 0.02 * float(ref.norm()) + 1e-12
        dhs[s] = (_q(du) @ _q(w1e.t().contiguous()).t()).to(BF)
    flat = rows.long()
    picked = torch.where((flat >= 0)[:, :, None], y.double()[flat.clamp(min=0)], 0.0)
    _close(out, (picked * gate.double()[:, :, None]).sum(1), 2.0**-7)
    _close(grads["gate"], (picked * dout.double()[:, None]).sum(2), 1e-5)
    dh = torch.where((flat >= 0)[:, :, None], dhs.double()[flat.clamp(min=0)], 0.0).sum(1)
    xh = (x.double() - mean.double()[:, None]) * rstd.double()[:, None]
    t = dh * gamma.double()
    dx = rstd.double()[:, None] * (t - t.mean(1, keepdim=True) - xh * (t * xh).mean(1, keepdim=True))
    assert float((grads["x"].double() - dx).norm()) <= 0.02 * float(dx.norm())
    assert float((grads["gamma"].double() - (dh * xh).sum(0)).norm()) <= 0.02 * float((dh * xh).sum(0).norm()) + 1e-12
    assert float((grads["beta"].double() - dh.sum(0)).norm()) <= 0.02 * float(dh.sum(0).norm()) + 1e-12


def test_training_lowers_the_loss():
    """The gradients point downhill: the loss against a fixed target falls at every few steps."""
    losses = moe.main(["--steps", "12", "--tokens", "1024", "--experts", "8", "--hidden", "256", "--ffn", "256"])
    assert losses[-1] < 0.8 * losses[0] and all(b < a for a, b in zip(losses[::4], losses[4::4]))


def test_refusals():
    with pytest.raises(ValueError):
        moe.MoELayer(4, 100, 128, 2)
    layer = moe.MoELayer(2, 128, 128, 1)
    with pytest.raises(ValueError):
        layer.load_weights(torch.zeros(128, 128, dtype=BF, device="cuda"), torch.zeros(256, 128, dtype=BF, device="cuda"))


def test_graph_replays():
    """Forward and backward captured once, replayed on other inputs, with eager work in between; on a stream of their own."""
    tokens, experts, k, H, F = 257, 8, 2, 256, 384
    g = torch.Generator(device="cuda").manual_seed(4)

    def draw():
        return {"x": torch.randn(tokens, H, generator=g, device="cuda").to(BF),
                "dout": torch.randn(tokens, H, generator=g, device="cuda").to(BF),
                "ids": torch.topk(torch.rand(tokens, experts, generator=g, device="cuda"), k, dim=1).indices,
                "gate": torch.rand(tokens, k, generator=g, device="cuda")}

    gamma, beta = torch.ones(H, device="cuda"), torch.zeros(H, device="cuda")
    layer = moe.MoELayer(experts, H, F, k)
    layer.load_weights(torch.randn(experts * F, H, generator=g, device="cuda").to(BF),
                       torch.randn(experts * H, F, generator=g, device="cuda").to(BF))

    def step(s):
        out = layer.forward(s["x"], s["ids"], s["gate"], gamma, beta)
        return dict(layer.backward(s["dout"], seed=7), out=out)

    still = draw()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step(still)
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = step(still)
    for _ in range(4):
        fresh = draw()
        want = step(fresh)
        for n in still:
            still[n].copy_(fresh[n])
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        for n in want:
            assert torch.equal(want[n], got[n]), n
