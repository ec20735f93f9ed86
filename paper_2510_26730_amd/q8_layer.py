"""One MoE layer with 8-bit experts, made of the operators beside the layer: routing from logits, 8-bit products, weighted sum.

    layer = Q8Layer(w13, w2, top_k=6, max_tokens=1056, sigmoid=True, bias=balance_bias, n_groups=8, groups_kept=3, group_best=2)
    out = layer(hidden, logits)

The weights are quantised once, a scale for every output channel; tokens and activations in every call, a scale for every row.  A
call only enqueues kernels (it may be captured into a graph) and leaves its routing in ``ids``, ``w``, ``counts``, ``offsets``,
``perm`` and ``inv_perm``.  ``python -m paper_2510_26730_amd.q8_layer`` runs a layer of one of the synthetic shapes.
"""
from __future__ import annotations

import argparse
import contextlib

import torch

from . import binding as ef


def quantise(w):
    """Weights [.., N, K] on the device -> codes int8 of the same shape, rows 64 bytes aligned (read faster than at 16), and scales [.., N]."""
    *lead, K = w.shape
    codes = torch.empty(*lead, (K + 63) // 64 * 64, dtype=torch.int8, device=w.device)
    scales = torch.empty(*lead, dtype=torch.float32, device=w.device)
    ef.ef_quant_rows(w.reshape(-1, K), codes.view(-1, codes.shape[-1]), scales.view(-1), stream=torch.cuda.current_stream(w.device))
    return codes[..., :K], scales


class Q8Layer:
    """w13 [E, 2F, d]: gate rows, then up rows; w2 [E, d, F] (16- or 32-bit floats).  `bias` and the keyword arguments are those of
    ef_route_scores.  Buffers are sized for max_tokens tokens and shared by the calls: one call at a time."""

    def __init__(self, w13, w2, top_k, max_tokens, *, bias=None, act_dtype=torch.bfloat16, **route):
        (E, F2, d), dev = w13.shape, w13.device
        if w2.shape != (E, d, F2 // 2) or F2 % 2:
            raise ef.EfError(ef.EF_EINVAL, "Q8Layer: w13 must be [E, 2F, d] and w2 [E, d, F]")
        self.E, self.d, self.k, self.max_tokens, self.bias, self.route = E, d, top_k, max_tokens, bias, route
        self.w13, self.s13 = quantise(w13)
        self.w2, self.s2 = quantise(w2)
        n, i32 = max_tokens * top_k, dict(dtype=torch.int32, device=dev)
        self._ids, self._w = torch.empty(n, **i32), torch.empty(n, dtype=torch.float32, device=dev)
        self.counts, self.offsets = torch.empty(E, **i32), torch.empty(E + 1, **i32)
        self._perm, self._inv_perm = torch.empty(n, **i32), torch.empty(n, **i32)
        self._act = torch.empty(n, F2 // 2, dtype=act_dtype, device=dev)
        self._y = torch.empty(n, d, dtype=torch.float32, device=dev)
        work = ef.ef_route_scores_work(max_tokens, E, top_k, route.get("n_groups", 1), route.get("groups_kept", 1))
        x = torch.empty(max_tokens, d, dtype=act_dtype, device=dev)
        up = ef.ef_matmul_q8_work(x, self.w13, self.s13, self._act, rows=self._perm, row_div=top_k, offsets=self.offsets, swiglu=True)
        down = ef.ef_matmul_q8_work(self._act, self.w2, self.s2, self._y, offsets=self.offsets)
        self._work = torch.empty(max(work, up, down, 1), dtype=torch.uint8, device=dev)

    def __call__(self, hidden, logits, out=None, stream=None):
        """hidden [T, d], logits [T, E] -> out [T, d] (in hidden's type unless given).  With `stream`, all of it runs there, on inputs that are
        ready there, and an out that is not given belongs to that stream."""
        T, k = hidden.shape[0], self.k
        if T > self.max_tokens:
            raise ef.EfError(ef.EF_EINVAL, f"Q8Layer: {T} tokens, buffers for {self.max_tokens}")
        # routing takes its tokens and experts from the logits; the views below have room for hidden's
        if hidden.shape != (T, self.d) or logits.shape != (T, self.E) or (out is not None and out.shape != (T, self.d)):
            raise ef.EfError(ef.EF_EINVAL, f"Q8Layer: hidden {tuple(hidden.shape)} and logits {tuple(logits.shape)} (and out, if given) do not fit "
                                           f"{self.E} experts of {self.d}")
        s = torch.cuda.current_stream(hidden.device) if stream is None else stream
        if out is None:
            # on the stream that writes it: memory of another stream's may still be in use there
            on = contextlib.nullcontext() if stream is None else torch.cuda.stream(torch.cuda.ExternalStream(s, hidden.device) if isinstance(s, int) else s)
            with on:
                out = torch.empty(T, self.d, dtype=hidden.dtype, device=hidden.device)
        n = T * k
        self.ids, self.w, self.perm, self.inv_perm = self._ids[:n].view(T, k), self._w[:n].view(T, k), self._perm[:n], self._inv_perm[:n]
        act, y = self._act[:n], self._y[:n]
        ef.ef_route_scores(logits, self.bias, self.ids, self.w, self.counts, self.offsets, self.perm, self.inv_perm, self._work, stream=s,
                           **self.route)
        ef.ef_matmul_q8(hidden, self.w13, self.s13, act, self._work, offsets=self.offsets, rows=self.perm, row_div=k, swiglu=True, stream=s)
        ef.ef_matmul_q8(act, self.w2, self.s2, y, self._work, offsets=self.offsets, stream=s)
        ef.ef_combine(y, self.w, self.inv_perm, out, stream=s)
        return out


def main():
    from . import synth
    ap = argparse.ArgumentParser(description="time one MoE layer with 8-bit experts")
    ap.add_argument("--shape", default="deepseek_v2_lite", choices=[n for n in synth.CONFIGS])
    ap.add_argument("--tokens", type=int, default=32)
    ap.add_argument("--steps", type=int, default=50)
    a = ap.parse_args()
    c = synth.CONFIGS[a.shape]
    torch.manual_seed(0)
    w13 = torch.randn(c.E, 2 * c.F, c.d, device="cuda", dtype=torch.bfloat16).mul_(0.02)
    w2 = torch.randn(c.E, c.d, c.F, device="cuda", dtype=torch.bfloat16).mul_(0.02)
    layer = Q8Layer(w13, w2, c.k, a.tokens, renorm=bool(c.renorm))
    x = torch.randn(a.tokens, c.d, device="cuda", dtype=torch.bfloat16)
    logits = torch.randn(a.tokens, c.E, device="cuda")
    out = layer(x, logits)
    t = torch.randint(a.tokens, (1,)).item()      # one token against the unquantised weights
    want = torch.zeros(c.d, device="cuda")
    for e, w in zip(layer.ids[t].tolist(), layer.w[t].tolist()):
        g, u = (w13[e].float() @ x[t].float()).chunk(2)
        want += w * (w2[e].float() @ (torch.nn.functional.silu(g) * u))
    begin, end = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
    begin.record()
    for _ in range(a.steps):
        layer(x, logits, out)
    end.record()
    torch.cuda.synchronize()
    print(f"{a.shape}, {a.tokens} tokens: {begin.elapsed_time(end) / a.steps * 1e3:.1f} us a layer, {layer.counts.count_nonzero().item()} of {c.E} experts "
          f"in use; token {t} is {(out[t].float() - want).norm() / want.norm():.4f} from the unquantised weights")


if __name__ == "__main__":
    main()
