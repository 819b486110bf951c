"""A linear-attention block as it is served with weights of 4 bits, on the operators of ``libconvtune.so``.

    x -> norm, to 8 bits -> project to q, k, v, the gate z and the steps -> linear attention with a
      decay for each head -> norm of each head, gated by z, to 8 bits -> project out, plus x

Five calls on one stream (``ct_norm_run`` twice, ``ct_mx_linear_run`` twice, ``ct_decay_attention_run``),
and where offsets may leave rows out a clear of the attention's output before the second norm: the
columns of the first product are read in place through row pitches, activations go from call to call in
8 bits with a scale for 32 of them, and the residual is added in the last product's epilogue. States
live in slots that the caller hands out, as a :class:`~.sequence.SequenceBlock`'s do, and a block is
served alike (``sequence.serve``): packed prompts of unequal lengths, single tokens of many sequences and
rows of no sequence go through the same code, a call allocates nothing and may be captured into a HIP
graph.

Usage: ``python -m paper_2008_03602_amd.linear_attention [--model 1024] [--tokens 2048] [--sequences 8]``:
packed prompts and a decode loop of a block with random weights; prints one JSON line.
"""
from __future__ import annotations

import argparse
import json
import math
import sys

import torch

from . import _lib as L
from .sequence import _stream, serve

EPS = 1e-5


def _rows(rows, cols, fmt):
    """Buffers of microscaled rows, elements and scales, all 0."""
    return (torch.zeros(rows, L.mx_row_bytes(cols, fmt), dtype=torch.uint8, device="cuda"),
            torch.zeros(rows, L.mx_scale_bytes(cols), dtype=torch.uint8, device="cuda"))


class LinearAttentionBlock:
    """The block's weights, its state slots and its buffers.

    ``model`` columns of x, ``heads`` heads of ``value`` columns each, which share ``groups`` pairs of
    queries and keys of ``key`` columns. ``max_rows``: the most token rows of one call.
    """

    def __init__(self, model: int, heads: int = 16, groups: int = 16, key: int = 64, value: int = 64, slots: int = 8,
                 max_rows: int = 2048, seed: int = 0):
        if value % 32:
            raise ValueError("a head's value columns are whole blocks of 32")
        L.ct_init(0)
        self.model, self.heads, self.groups, self.key, self.value = model, heads, groups, key, value
        self.slots, self.max_rows, self.dtype = slots, max_rows, torch.bfloat16
        gen = torch.Generator(device="cuda")
        gen.manual_seed(seed)

        def normal(*shape, std=1.0, mean=0.0, dt=torch.float32):
            return (torch.randn(shape, generator=gen, device="cuda") * std + mean).to(dt)

        def quantised(w):
            q, scales = _rows(w.shape[0], w.shape[1], L.MX_E2M1)
            L.ct_mx_quantise_run(L.make_mx(w.shape[0], w.shape[1], L.DT_BF16, L.MX_E2M1), w, q, scales, _stream())
            return q, scales

        # columns of the first product: q, k, v, z, steps, each from a 16-byte group on
        widths = (groups * key, groups * key, heads * value, heads * value, heads)
        self.starts = [sum((w + 7) // 8 * 8 for w in widths[:i]) for i in range(6)]
        self.columns, self.inner = self.starts[5], heads * value
        self.w_in = quantised(normal(self.columns, model, std=model ** -0.5, dt=self.dtype))
        self.w_out = quantised(normal(model, self.inner, std=self.inner ** -0.5, dt=self.dtype))
        self.norm_in, self.norm_out = normal(model, mean=1.0, std=0.1), normal(self.inner, mean=1.0, std=0.1)
        self.b_step, self.a = normal(heads, mean=-3.0, std=0.5), -torch.exp(normal(heads, std=0.5))
        self.state = torch.zeros(slots, heads, key, value, device="cuda")
        self._x = _rows(max_rows, model, L.MX_E4M3)
        self._p = torch.empty(max_rows, self.columns, dtype=self.dtype, device="cuda")
        self._o = torch.empty(max_rows, self.inner, dtype=self.dtype, device="cuda")
        self._g = _rows(max_rows, self.inner, L.MX_E4M3)
        self._workspaces = []  # each larger than the ones before; all of them, for graphs keep their addresses

    def reset(self) -> None:
        """Forgets every slot."""
        self.state.zero_()

    def sequences(self, rows: int, count: int, max_len: int = 0, offsets=None, slots=None) -> L.ct_sequences:
        """Packed sequences over the block's slots (``offsets``, ``slots``: int32 device tensors)."""
        for t, n in ((offsets, count + 1), (slots, count)):
            if t is not None and (t.dtype != torch.int32 or not t.is_cuda or t.shape != (n,) or not t.is_contiguous()):
                raise ValueError("offsets and slots are contiguous int32 device tensors of count + 1 and count values")
        return L.make_sequences(rows, count, self.slots, max_len, offsets, slots)

    def plan(self, seqs: L.ct_sequences) -> dict:
        """The calls' descriptions for these rows, and a workspace of what they need. Workspaces are
        kept as long as the block: a graph that was captured with one goes on using it."""
        m, dt, cols = seqs.tokens, L.DT_BF16, self.columns
        if m > self.max_rows:
            raise ValueError("%d rows, but the block's buffers hold %d" % (m, self.max_rows))
        p = {"seqs": seqs,
             "norm": L.make_norm(m, self.model, dt, L.MX_E4M3, eps=EPS),
             "in": L.make_mx_linear(m, cols, self.model, L.MX_E4M3, L.MX_E2M1, dt),
             "attention": L.make_decay_attention(self.heads, self.groups, self.key, self.value, dt, scale=self.key ** -0.5,
                                                 ldq=cols, ldk=cols, ldv=cols, lddelta=cols),
             "heads": L.make_norm(m, self.inner, dt, L.MX_E4M3, groups=self.heads, eps=EPS, ldz=cols),
             "out": L.make_mx_linear(m, self.model, self.inner, L.MX_E4M3, L.MX_E2M1, dt, res=L.RES_ADD)}
        need = max([L.ct_mx_linear_workspace(p[k]) for k in ("in", "out")] +
                   [L.ct_decay_attention_workspace(p["attention"], seqs), 16])
        if not self._workspaces or self._workspaces[-1].numel() < need:
            self._workspaces.append(torch.empty(need, dtype=torch.uint8, device="cuda"))
        p["ws"] = self._workspaces[-1]
        return p

    def run(self, plan: dict, x: torch.Tensor, y: torch.Tensor) -> torch.Tensor:
        """One pass over x (rows x model) into y on the current stream; the slots move on. The
        calls follow each other on one stream, so they share a workspace. Rows of no sequence
        come out as they went in, those with an infinity or NaN as NaN."""
        for t in (x, y):
            if t.dtype != self.dtype or not t.is_cuda or t.shape != (plan["seqs"].tokens, self.model) or \
                    not t.is_contiguous():
                raise ValueError("x and y are contiguous device tensors of rows x model in bfloat16")
        st, ws, s = _stream(), plan["ws"], plan["seqs"]
        q, k, v, z, step = (self._p[:, a:] for a in self.starts[:5])
        L.ct_norm_run(plan["norm"], x, None, None, self.norm_in, None, self._x[0], self._x[1], st)
        L.ct_mx_linear_run(plan["in"], *self._x, *self.w_in, None, None, self._p, ws, st)
        if s.offsets:  # the attention writes no row of no sequence, and the norm takes them all
            self._o[:s.tokens].zero_()
        L.ct_decay_attention_run(plan["attention"], s, q, k, v, step, self.b_step, self.a, self.state, self.state, self._o,
                                 ws, st)
        L.ct_norm_run(plan["heads"], self._o, None, None, self.norm_out, z, self._g[0], self._g[1], st)
        L.ct_mx_linear_run(plan["out"], *self._g, *self.w_out, None, x, y, ws, st)
        return y


def main(argv=None) -> int:
    ap = argparse.ArgumentParser()
    ap.add_argument("--model", type=int, default=1024)
    ap.add_argument("--heads", type=int, default=16)
    ap.add_argument("--groups", type=int, default=16, help="pairs of queries and keys that the heads share")
    ap.add_argument("--key", type=int, default=64)
    ap.add_argument("--value", type=int, default=64)
    ap.add_argument("--tokens", type=int, default=4096, help="rows of all prompts together")
    ap.add_argument("--sequences", type=int, default=8)
    ap.add_argument("--steps", type=int, default=64, help="tokens that every sequence decodes after its prompt")
    a = ap.parse_args(argv)
    if not torch.cuda.is_available():
        print("linear_attention: needs an MI355X", file=sys.stderr)
        return 1
    n = a.sequences
    weights = [i + 1 for i in range(n)]  # unequal lengths
    lens = [a.tokens * w // sum(weights) for w in weights]
    lens[-1] += a.tokens - sum(lens)
    block = LinearAttentionBlock(a.model, a.heads, a.groups, a.key, a.value, slots=n, max_rows=max(a.tokens, n))
    r = serve(block, lens, a.steps)
    ok = bool(torch.isfinite(r["prompt"].float()).all()) and bool(torch.isfinite(r["steps"].float()).all())
    print(json.dumps({"model": a.model, "heads": a.heads, "groups": a.groups, "key": a.key, "value": a.value, "lens": lens,
                      "prompt_ms": round(r["prompt_ms"], 3), "prompt_tokens_per_s": round(a.tokens / r["prompt_ms"] * 1e3),
                      "step_us": round(r["step_us"], 1), "tokens_per_s": round(n / r["step_us"] * 1e6),
                      "finite": ok}), flush=True)
    return 0 if ok and math.isfinite(r["prompt_ms"]) else 1


if __name__ == "__main__":
    sys.exit(main())
