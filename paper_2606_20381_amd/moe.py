"""One mixture-of-experts layer of a training step on the library's operators: norm, tokens sorted by expert, the experts' two
products in microscaled 4 bits, the way back with the gate weights, and every gradient.

    h = layer_norm(x); each token's k experts: u = Q(h) Q(W1_e)^T, a = relu(u)^2, y = Q(a) Q(W2_e)^T
    out = sum_j gate_j y_j            (the residual stays with the caller)

The operands follow the comparison recipe (Table 1): E2M1 levels, gradients rounded stochastically, the block-16 RHT on the
operands of the weight gradients. Nothing waits for the GPU: the experts' loads stay there, buffers are sized by their bounds.

    python -m paper_2606_20381_amd.moe        # a few steps of a small layer towards a fixed target: loss and time per step
"""

from __future__ import annotations

import argparse
import time

import torch

from . import ufp4 as U

BF16 = torch.bfloat16


class MoELayer:
    """A layer of `experts` experts hidden -> ffn -> hidden, k per token. ffn and hidden are multiples of 128. Weights are bf16
    tensors of the caller's: w1 [experts * ffn, hidden], w2 [experts * hidden, ffn]; `load_weights` quantizes them (both ways) and is
    called again after they change. `forward` keeps what `backward` needs in `self.saved`."""

    def __init__(self, experts: int, hidden: int, ffn: int, k: int, sign_mask: int = 0x6A09):
        if hidden % 128 or ffn % 128:
            raise ValueError("hidden and ffn must be multiples of 128")
        self.experts, self.hidden, self.ffn, self.k, self.sign_mask = experts, hidden, ffn, k, sign_mask
        self.w1 = self.w2 = self.saved = None

    def load_weights(self, w1: torch.Tensor, w2: torch.Tensor):
        e, h, f = self.experts, self.hidden, self.ffn
        if tuple(w1.shape) != (e * f, h) or tuple(w2.shape) != (e * h, f):
            raise ValueError(f"w1 must be {(e * f, h)} and w2 {(e * h, f)}")
        self.w1 = U.mxfp4_quantize_dual(w1, out_rows=self.w1 and self.w1[0], out_cols=self.w1 and self.w1[1])
        self.w2 = U.mxfp4_quantize_dual(w2, out_rows=self.w2 and self.w2[0], out_cols=self.w2 and self.w2[1])

    def _rows(self, x, offsets, **kw):
        """x's rows by expert, each expert's from a panel: the left operand of the forward product and of the input's gradient."""
        bound = -(-(x.shape[0] + 127 * self.experts) // 128) * 128
        return U.mxfp4_quantize_grouped(x, offsets, bound, transpose=False, **kw)

    def _cols(self, x, offsets, **kw):
        """x transposed, the tokens of each expert filled up to whole blocks: an operand of the weights' gradient."""
        bound = -(-(x.shape[0] + 31 * self.experts) // 32) * 32
        return U.mxfp4_quantize_grouped(x, offsets, bound, transpose=True, rht=True, sign_mask=self.sign_mask, **kw)

    def forward(self, x, ids, gate, gamma, beta, eps: float = 1e-5):
        """out [tokens, hidden] of x [tokens, hidden] bf16, ids [tokens, k] (int32 or int64; outside 0 .. experts - 1: dropped), gate
        [tokens, k] fp32."""
        h, mean, rstd = U.layer_norm(x, gamma, beta, eps=eps)
        offsets, rows, _ = U.moe_sort(ids, self.experts)
        hs = U.moe_dispatch(h, rows, offsets)
        n = hs.shape[0]
        u = U.mxfp4_gemm_fwd_y_grouped(self._rows(hs, offsets), self.w1[0], offsets, n, BF16)
        a = torch.relu(u).square_()
        y = U.mxfp4_gemm_fwd_y_grouped(self._rows(a, offsets), self.w2[0], offsets, n, BF16)
        out = U.moe_combine(y, rows, gate)
        self.saved = (x, gate, gamma, mean, rstd, offsets, rows, hs, u, a, y)
        return out

    def backward(self, dout, seed: int = 0, stochastic: bool = True):
        """Gradients of the last forward: a dict of x and gate, gamma, beta (fp32), w1 [experts, ffn, hidden] and w2 [experts, hidden,
        ffn] (fp32)."""
        x, gate, gamma, mean, rstd, offsets, rows, hs, u, a, y = self.saved
        n = hs.shape[0]
        sr = dict(rounding=U.SR if stochastic else U.RTNE, seed=seed)
        dy, dgate = U.moe_combine_bwd(dout, y, rows, offsets, gate)
        dw2 = U.mxfp4_gemm_bwd_dw_grouped(self._cols(dy, offsets, stream_id=1, **sr), self._cols(a, offsets), offsets)
        da = U.mxfp4_gemm_bwd_dx_grouped(self._rows(dy, offsets, stream_id=0, **sr), self.w2[1], offsets, n, BF16)
        du = torch.relu(u).mul_(2.0).mul_(da)
        dw1 = U.mxfp4_gemm_bwd_dw_grouped(self._cols(du, offsets, stream_id=3, **sr), self._cols(hs, offsets), offsets)
        dhs = U.mxfp4_gemm_bwd_dx_grouped(self._rows(du, offsets, stream_id=2, **sr), self.w1[1], offsets, n, BF16)
        dh = U.moe_combine(dhs, rows)  # the dispatch's gradient
        dx, dgamma, dbeta = U.layer_norm_bwd(dh, x, gamma, mean, rstd)
        return {"x": dx, "gate": dgate, "gamma": dgamma, "beta": dbeta, "w1": dw1, "w2": dw2}


def main(argv=None) -> list[float]:
    p = argparse.ArgumentParser(description="A few training steps of one MoE layer in microscaled 4 bits")
    p.add_argument("--tokens", type=int, default=4096)
    p.add_argument("--experts", type=int, default=16)
    p.add_argument("--hidden", type=int, default=512)
    p.add_argument("--ffn", type=int, default=1024)
    p.add_argument("--k", type=int, default=2)
    p.add_argument("--steps", type=int, default=20)
    p.add_argument("--lr", type=float, default=0.02)
    a = p.parse_args(argv)
    g = torch.Generator(device="cuda").manual_seed(0)

    def normal(*shape, std=1.0):
        return torch.randn(*shape, generator=g, device="cuda") * std

    layer = MoELayer(a.experts, a.hidden, a.ffn, a.k)
    w1, w2 = normal(a.experts * a.ffn, a.hidden, std=a.hidden**-0.5), normal(a.experts * a.hidden, a.ffn, std=a.ffn**-0.5)
    gamma, beta = torch.ones(a.hidden, device="cuda"), torch.zeros(a.hidden, device="cuda")
    x = normal(a.tokens, a.hidden).to(BF16)
    score, ids = torch.topk(normal(a.tokens, a.experts), a.k, dim=1)
    gate = torch.softmax(score, 1)
    target = (normal(a.tokens, a.hidden, std=0.5) + x).float()
    losses = []
    for step in range(a.steps):
        if step == 1:
            torch.cuda.synchronize()
            began = time.perf_counter()
        layer.load_weights(w1.to(BF16), w2.to(BF16))
        d = x + layer.forward(x, ids, gate, gamma, beta).float() - target
        losses.append(d.square().mean())
        grads = layer.backward((d * (2.0 / a.hidden)).to(BF16), seed=step)
        for w, dw in ((w1, grads["w1"]), (w2, grads["w2"]), (gamma, grads["gamma"]), (beta, grads["beta"])):
            w.sub_(dw.reshape(w.shape), alpha=a.lr)
    torch.cuda.synchronize()
    ms = (time.perf_counter() - began) / max(1, a.steps - 1) * 1e3 if a.steps > 1 else float("nan")
    losses = [float(v) for v in losses]
    print(f"{a.tokens} tokens, {a.k} of {a.experts} experts, {a.hidden} -> {a.ffn}: loss {losses[0]:.4f} -> {losses[-1]:.4f}, "
          f"{ms:.2f} ms a step")
    return losses


if __name__ == "__main__":
    main()
