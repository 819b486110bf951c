"""A recurrent sequence block as it is served, on the operators of ``libconvtune.so``.

    x -> project in (two halves: u, z) -> causal convolution and SiLU along the tokens of u
      -> project to (low rank step, b, c) -> project the step up -> selective scan, gated by z
      -> project out, plus x

Six calls on one stream (``ct_linear_run`` four times, ``ct_causal_conv_run``, ``ct_scan_run``), and
where offsets may leave rows out a clear of the scan's output before it: the halves and slices are
read in place through row pitches, and the residual is added in the last product's epilogue. Histories and states live in slots that the
caller hands out, so prompts of unequal lengths, single tokens of many sequences and rows that
belong to no sequence go through the same code. Buffers are made once for the most rows that a
call may bring, workspaces with the plans, and a call allocates nothing: it may be captured into
a HIP graph.

Usage: ``python -m paper_2008_03602_amd.sequence [--model 1024] [--tokens 2048] [--sequences 8]``:
packed prompts and a decode loop of a block with random weights; prints one JSON line.
"""
from __future__ import annotations

import argparse
import json
import math
import sys
import time

import torch

from . import _lib as L

CODES = {torch.float32: L.DT_F32, torch.bfloat16: L.DT_BF16}


def _stream() -> int:
    return torch.cuda.current_stream().cuda_stream


class SequenceBlock:
    """The block's weights, its state slots and its buffers.

    ``model`` rows of x, ``inner`` convolved and scanned channels with ``states`` states each,
    step sizes through ``rank`` columns. ``max_rows``: the most token rows of one call.
    """

    def __init__(self, model: int, inner: int, states: int = 16, rank: int = 64, width: int = 4, slots: int = 8,
                 max_rows: int = 2048, dtype=torch.bfloat16, seed: int = 0):
        L.ct_init(0)
        self.model, self.inner, self.states, self.rank, self.width = model, inner, states, rank, width
        self.slots, self.max_rows, self.dtype = slots, max_rows, dtype
        gen = torch.Generator(device="cuda")
        gen.manual_seed(seed)

        def normal(*shape, std=1.0, mean=0.0, dt=torch.float32):
            return (torch.randn(shape, generator=gen, device="cuda") * std + mean).to(dt)

        self.w_in = normal(2 * inner, model, std=model ** -0.5, dt=dtype)
        self.w_conv, self.b_conv = normal(inner, width, std=width ** -0.5), normal(inner, std=0.1)
        self.w_x = normal(rank + 2 * states, inner, std=inner ** -0.5, dt=dtype)
        self.w_step = normal(inner, rank, std=rank ** -0.5, dt=dtype)
        self.b_step = normal(inner, mean=-4.6, std=0.5)
        self.a = -torch.arange(1, states + 1, device="cuda", dtype=torch.float32).repeat(inner, 1)
        self.skip = torch.ones(inner, device="cuda")
        self.w_out = normal(model, inner, std=inner ** -0.5, dt=dtype)
        # what a sequence leaves behind: its last rows before the convolution, its states
        self.history = torch.zeros(slots, width - 1, inner, dtype=dtype, device="cuda")
        self.state = torch.zeros(slots, inner, states, device="cuda")

        def rows(cols):
            return torch.empty(max_rows, cols, dtype=dtype, device="cuda")

        self._xz, self._u, self._p = rows(2 * inner), rows(inner), rows(rank + 2 * states)
        self._step, self._y = rows(inner), rows(inner)
        self._workspaces = []  # each larger than the ones before; all of them, for graphs keep their addresses

    def reset(self) -> None:
        """Forgets every slot."""
        self.history.zero_()
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
        m, dt, width = seqs.tokens, CODES[self.dtype], self.rank + 2 * self.states
        if m > self.max_rows:
            raise ValueError("%d rows, but the block's buffers hold %d" % (m, self.max_rows))
        p = {"seqs": seqs,
             "in": L.make_linear(m, 2 * self.inner, self.model, dt, dt),
             "conv": L.make_causal_conv(self.inner, self.width, dt, L.ACT_SILU, ldx=2 * self.inner),
             "x": L.make_linear(m, width, self.inner, dt, dt),
             "step": L.make_linear(m, self.inner, self.rank, dt, dt, ldx=width),
             "scan": L.make_scan(self.inner, self.states, 1, dt, softplus=True, ldb=width, ldc=width,
                                 ldz=2 * self.inner),
             "out": L.make_linear(m, self.model, self.inner, dt, dt, res=L.RES_ADD)}
        need = max([L.ct_linear_workspace(p[k]) for k in ("in", "x", "step", "out")] +
                   [L.ct_scan_workspace(p["scan"], seqs), 16])
        if not self._workspaces or self._workspaces[-1].numel() < need:
            self._workspaces.append(torch.empty(need, dtype=torch.uint8, device="cuda"))
        p["ws"] = self._workspaces[-1]
        return p

    def run(self, plan: dict, x: torch.Tensor, y: torch.Tensor) -> torch.Tensor:
        """One pass over x (rows x model) into y on the current stream; the slots move on. The
        calls follow each other on one stream, so they share a workspace. Rows of no sequence
        come out as they went in."""
        for t in (x, y):
            if t.dtype != self.dtype or not t.is_cuda or t.shape != (plan["seqs"].tokens, self.model) or \
                    not t.is_contiguous():
                raise ValueError("x and y are contiguous device tensors of rows x model in the block's type")
        st, ws, s = _stream(), plan["ws"], plan["seqs"]
        z, b, c = self._xz[:, self.inner:], self._p[:, self.rank:], self._p[:, self.rank + self.states:]
        L.ct_linear_run(plan["in"], x, self.w_in, None, None, self._xz, ws, st)
        L.ct_causal_conv_run(plan["conv"], s, self._xz, self.w_conv, self.b_conv, self.history, self.history, self._u, st)
        L.ct_linear_run(plan["x"], self._u, self.w_x, None, None, self._p, ws, st)
        L.ct_linear_run(plan["step"], self._p, self.w_step, None, None, self._step, ws, st)
        if s.offsets:  # the scan writes no row of no sequence, and the last product takes them all
            self._y[:s.tokens].zero_()
        L.ct_scan_run(plan["scan"], s, self._u, self._step, self.b_step, self.a, b, c, self.skip, z, self.state,
                      self.state, self._y, ws, st)
        L.ct_linear_run(plan["out"], self._y, self.w_out, None, x, y, ws, st)
        return y


def serve(block: SequenceBlock, lens, steps: int, seed: int = 1) -> dict:
    """Packed prompts of the given lengths, then `steps` tokens of every sequence from a captured
    graph (tanh of a step's output, which stays bounded, is the next one's input); returns the
    outputs and the times."""
    tokens, count = sum(lens), len(lens)
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    x = torch.randn(tokens, block.model, generator=gen, device="cuda").to(block.dtype)
    off = torch.tensor([sum(lens[:i]) for i in range(count + 1)], dtype=torch.int32, device="cuda")
    slots = torch.randperm(block.slots, generator=gen, device="cuda")[:count].to(torch.int32).contiguous()
    prompt = block.plan(block.sequences(tokens, count, max(lens), off, slots))
    step = block.plan(block.sequences(count, count, 1, None, slots))
    y = torch.empty_like(x)
    last = (off[1:].long() - 1).clamp(min=0)
    some = (off[1:] > off[:-1])[:, None]  # a sequence without a prompt starts from zeros
    a, b = (torch.empty(count, block.model, dtype=block.dtype, device="cuda") for _ in range(2))
    block.run(prompt, x, y)  # loads the kernels; the passes that count follow
    block.run(step, a.zero_(), b)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        block.run(step, a, b)
        a.copy_(torch.tanh(b))
    block.reset()
    torch.cuda.synchronize()
    t0 = time.perf_counter()
    block.run(prompt, x, y)
    torch.cuda.synchronize()
    t1 = time.perf_counter()
    a.copy_(torch.where(some, torch.tanh(y[last]), 0) if tokens else a.zero_())
    out = [a.clone()]
    torch.cuda.synchronize()
    t2 = time.perf_counter()
    for _ in range(steps):
        graph.replay()
        out.append(a.clone())
    torch.cuda.synchronize()
    t3 = time.perf_counter()
    return {"prompt": y, "steps": torch.stack(out), "prompt_ms": (t1 - t0) * 1e3,
            "step_us": (t3 - t2) / max(steps, 1) * 1e6}


def main(argv=None) -> int:
    ap = argparse.ArgumentParser()
    ap.add_argument("--model", type=int, default=1024)
    ap.add_argument("--inner", type=int, default=2048)
    ap.add_argument("--tokens", type=int, default=4096, help="rows of all prompts together")
    ap.add_argument("--sequences", type=int, default=8)
    ap.add_argument("--steps", type=int, default=64, help="tokens that every sequence decodes after its prompt")
    ap.add_argument("--dtype", choices=("bf16", "f32"), default="bf16")
    a = ap.parse_args(argv)
    if not torch.cuda.is_available():
        print("sequence: needs an MI355X", file=sys.stderr)
        return 1
    n = a.sequences
    weights = [i + 1 for i in range(n)]  # unequal lengths
    lens = [a.tokens * w // sum(weights) for w in weights]
    lens[-1] += a.tokens - sum(lens)
    block = SequenceBlock(a.model, a.inner, slots=n, max_rows=max(a.tokens, n),
                          dtype=torch.bfloat16 if a.dtype == "bf16" else torch.float32)
    r = serve(block, lens, a.steps)
    ok = bool(torch.isfinite(r["prompt"].float()).all()) and bool(torch.isfinite(r["steps"].float()).all())
    print(json.dumps({"model": a.model, "inner": a.inner, "dtype": a.dtype, "lens": lens,
                      "prompt_ms": round(r["prompt_ms"], 3), "prompt_tokens_per_s": round(a.tokens / r["prompt_ms"] * 1e3),
                      "step_us": round(r["step_us"], 1), "tokens_per_s": round(n / r["step_us"] * 1e6),
                      "finite": ok}), flush=True)
    return 0 if ok and math.isfinite(r["prompt_ms"]) else 1


if __name__ == "__main__":
    sys.exit(main())
