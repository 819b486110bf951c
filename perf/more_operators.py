"""What the operators of a linear-attention block are timed on: calls of a user's program, through the public entry points.

Four operators, which together are one such block as it is served with weights of 4 bits:

* ``norm``: the root-mean-square norm of rows or of a row's heads, with the residual's addition before it, a gate
  behind it, and rows of 8 or 4 bits with block scales among its outputs (``ct_norm_run``);
* ``quantise``: rows to microscaled floating point, blocks of 32 values with a power of two as their scale, and back
  to the values they stand for (``ct_mx_quantise_run``, ``ct_mx_values_run``);
* ``mx_linear``: the product of such rows, with bias, activation and residual in its epilogue (``ct_mx_linear_run``);
  a pass quantises its activations, as a user's program does, and takes weights that were quantised before;
* ``attention``: linear attention with a decay for each head over packed sequences, its states in slots: prompts of
  many tokens, and single tokens (``ct_decay_attention_run``).

Microscaled rows are returned as the values they stand for. A case's ``lens`` is the lengths of packed sequences as a
text, or ``count`` x ``len`` equal ones (``len`` 1: a decode step). The plain forms are elementary torch operations
in 32 bits, the sums of the decays' logarithms in 64.
"""
import math

import torch

own = False

ACTS = ("none", "relu", "relu6", "silu", "gelu")
RES = ("none", "add", "add_act")  # no residual; act(v) + r; act(v + r)
EPS = 1e-5
CHUNK = 64  # tokens that the plain attention takes at a time
# microscaled elements: the largest value, its exponent, the smallest normal exponent, bits of the fraction
MX = {"mx8": (448.0, 8, -6, 3), "mx4": (6.0, 2, 0, 1)}
BLOCK = 32


def listed():
    return [
        # one token's row, the residual added and kept: the smallest call, latency counts
        {"name": "norm_one_token", "op": "norm", "rows": 1, "cols": 2048, "groups": 1, "dtype": "bf16", "out": "bf16",
         "residual": True, "gate": False},
        # a prompt of 8192 tokens: the norm of each of 32 heads, gated, to 8 bits for the projection behind it
        {"name": "norm_heads_gated_8bit", "op": "norm", "rows": 8192, "cols": 4096, "groups": 32, "dtype": "bf16",
         "out": "mx8", "residual": False, "gate": True},
        # a projection's weights to 4 bits, when they are loaded
        {"name": "quantise_weights_4bit", "op": "quantise", "rows": 8192, "cols": 4096, "dtype": "bf16", "format": "mx4"},
        # fp32 rows whose last block is not whole, to 8 bits
        {"name": "quantise_odd_f32", "op": "quantise", "rows": 1021, "cols": 515, "dtype": "f32", "format": "mx8"},
        # a decode step of 24 sequences through a wide projection with the residual: the weight's bytes
        {"name": "mx_linear_decode", "op": "mx_linear", "m": 24, "n": 4096, "k": 8192, "x": "mx8", "w": "mx4",
         "out": "bf16", "act": "none", "bias": False, "res": "add"},
        # a prompt of 8192 tokens: the matrix cores
        {"name": "mx_linear_prompt", "op": "mx_linear", "m": 8192, "n": 8192, "k": 4096, "x": "mx8", "w": "mx4",
         "out": "bf16", "act": "silu", "bias": True, "res": "none"},
        # both operands in 4 bits, ragged in every size
        {"name": "mx_linear_odd", "op": "mx_linear", "m": 1021, "n": 1277, "k": 515, "x": "mx4", "w": "mx4",
         "out": "f32", "act": "relu", "bias": True, "res": "add_act"},
        # a decode step of 8 sequences: latency
        {"name": "attention_step_small", "op": "attention", "count": 8, "len": 1, "heads": 16, "groups": 16, "key": 64,
         "value": 64, "dtype": "bf16", "decay": "token", "step": False},
        # a decode step of 128 sequences: the states' bytes
        {"name": "attention_step_large", "op": "attention", "count": 128, "len": 1, "heads": 16, "groups": 16,
         "key": 128, "value": 128, "dtype": "bf16", "decay": "token", "step": False},
        # one long prompt with few heads, so the work has to be split over the tokens
        {"name": "attention_long", "op": "attention", "count": 1, "len": 16384, "heads": 16, "groups": 16, "key": 128,
         "value": 128, "dtype": "bf16", "decay": "token", "step": False},
        # packed prompts of unequal lengths; the heads share 4 pairs of queries and keys, and the step scales the input
        {"name": "attention_ragged_shared", "op": "attention", "lens": "2047,0,1,517,3891,96,1640", "heads": 32,
         "groups": 4, "key": 128, "value": 64, "dtype": "bf16", "decay": "token", "step": True},
        # fp32 with odd sizes and one decay for each head at every token
        {"name": "attention_odd_f32", "op": "attention", "lens": "333,1,444", "heads": 10, "groups": 5, "key": 40,
         "value": 72, "dtype": "f32", "decay": "head", "step": False},
    ]


def _log_int(rng, lo, hi):
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def _size(rng, lo, hi):
    """A size over the logarithm of its range: a multiple of 64 half the time, of 8 or any otherwise."""
    v = _log_int(rng, lo, hi)
    g = rng.choice((64, 64, 8, 1))
    return max(lo, v // g * g)


def _draw_lens(rng, tokens, most):
    """Up to `most` unequal lengths that sum to about `tokens`, an empty or a single-token one among them."""
    n = rng.randrange(1, most + 1)
    part = [rng.random() + 0.02 for _ in range(n)]
    lens = [int(tokens * p / sum(part)) for p in part]
    for special in (0, 1):
        if rng.random() < 0.3:
            lens.insert(rng.randrange(len(lens) + 1), special)
    return ",".join(str(v) for v in lens)


def draw(rng):
    op = rng.choice(("norm", "quantise", "mx_linear", "mx_linear", "attention", "attention", "attention"))
    if op == "norm":
        groups = rng.choice((1, 1, 1, 4, 16, 32))
        out = rng.choice(("bf16", "f32", "mx8", "mx8", "mx4"))
        if groups > 1:  # whole blocks to a head
            cols = groups * rng.choice((32, 64, 96, 128, 256))
        else:
            cols = _size(rng, 32, 16384)
        return {"op": op, "rows": _log_int(rng, 1, max(1, min(16384, (8192 * 4096) // cols))), "cols": cols,
                "groups": groups, "dtype": rng.choice(("bf16", "bf16", "f32")), "out": out,
                "residual": rng.random() < 0.6, "gate": rng.random() < 0.4}
    if op == "quantise":
        cols = _size(rng, 32, 16384)
        return {"op": op, "rows": _log_int(rng, 1, max(1, min(16384, (8192 * 4096) // cols))), "cols": cols,
                "dtype": rng.choice(("bf16", "bf16", "f32")), "format": rng.choice(("mx8", "mx4"))}
    if op == "mx_linear":
        while True:
            case = {"op": op, "m": _log_int(rng, 1, 16384), "n": _size(rng, 16, 8192), "k": _size(rng, 32, 8192),
                    "x": rng.choice(("mx8", "mx8", "mx4")), "w": rng.choice(("mx4", "mx4", "mx8")),
                    "out": rng.choice(("bf16", "bf16", "f32")), "act": rng.choice(ACTS), "bias": rng.random() < 0.7,
                    "res": rng.choice(RES)}
            cost = work(case)
            if cost["flops"] <= 5e11 and cost["bytes"] <= 2.5e8:
                return case
    step = rng.random() < 0.35
    groups = rng.choice((1, 2, 4, 8, 16))
    heads = groups * rng.choice((1, 1, 2, 4))
    key = rng.choice((16, 32, 64, 64, 128, 128, 256, rng.randrange(8, 257)))
    value = rng.choice((32, 64, 64, 128, 128, 256, rng.randrange(8, 257)))
    case = {"op": op, "heads": heads, "groups": groups, "key": key, "value": value,
            "dtype": rng.choice(("bf16", "bf16", "f32")), "decay": rng.choice(("token", "token", "head")),
            "step": rng.random() < 0.3}
    case["step"] = case["step"] and case["decay"] == "token"
    each = heads * key * value
    if step:
        case.update(count=_log_int(rng, 1, max(1, min(256, 128 * 16 * 128 * 128 // each))), len=1)
        return case
    tokens = _log_int(rng, 32, max(64, min(16384, 16384 * 16 * 128 * 128 // (2 * each))))
    if rng.random() < 0.4:
        count = rng.randrange(1, 5)
        case.update(count=count, len=max(2, tokens // count))
    else:
        case["lens"] = _draw_lens(rng, tokens, 8)
    return case


# ---------------------------------------------------------------- inputs
def _dtype(text):
    return torch.bfloat16 if text == "bf16" else torch.float32


def _lens(case):
    if "lens" in case:
        return [int(v) for v in case["lens"].split(",")]
    return [case.get("len", 0)] * case.get("count", 0)


def _pitch(cols, dtype):
    """Row pitch of a projection's output: whole 16-byte groups."""
    g = 16 // torch.empty(0, dtype=dtype).element_size()
    return (cols + g - 1) // g * g


class _Draw:
    def __init__(self, seed):
        self.gen = torch.Generator(device="cuda")
        self.gen.manual_seed(seed)

    def normal(self, *shape, mean=0.0, std=1.0, dtype=torch.float32):
        return (torch.randn(shape, generator=self.gen, device="cuda") * std + mean).to(dtype)

    def order(self, n):
        return torch.randperm(n, generator=self.gen, device="cuda").to(torch.int32)


def _inputs(case, seed):
    d = _Draw(seed)
    if case["op"] == "norm":
        rows, cols, dt = case["rows"], case["cols"], _dtype(case["dtype"])
        return {"x": d.normal(rows, cols, dtype=dt), "w": d.normal(cols, mean=1.0, std=0.2),
                "res": d.normal(rows, cols, std=2.0, dtype=dt) if case["residual"] else None,
                "z": d.normal(rows, cols, dtype=dt) if case["gate"] else None}
    if case["op"] == "quantise":
        return {"x": d.normal(case["rows"], case["cols"], std=case["cols"] ** -0.5, dtype=_dtype(case["dtype"]))}
    if case["op"] == "mx_linear":
        m, n, k, out = case["m"], case["n"], case["k"], _dtype(case["out"])
        return {"x": d.normal(m, k, dtype=torch.bfloat16), "w": d.normal(n, k, std=k ** -0.5, dtype=torch.bfloat16),
                "bias": d.normal(n, std=0.5) if case["bias"] else None,
                "res": d.normal(m, n, dtype=out) if case["res"] != "none" else None}
    lens, dt, heads, groups = _lens(case), _dtype(case["dtype"]), case["heads"], case["groups"]
    tokens, count, key, value = sum(lens), len(lens), case["key"], case["value"]
    # states in slots of a larger pool, the sequences' own slots in no order
    s = {"lens": lens, "slots": d.order(count + 3)[:count].contiguous(), "num_slots": count + 3,
         "offsets": torch.tensor([sum(lens[:i]) for i in range(count + 1)], dtype=torch.int32, device="cuda")}
    # queries, keys, values and steps are columns of one projection, each from a 16-byte group on
    widths = (groups * key, groups * key, heads * value, heads)
    starts = [sum(_pitch(w, dt) for w in widths[:i]) for i in range(5)]
    p = d.normal(tokens, starts[4], dtype=dt)
    s["q"], s["k"], s["v"], s["delta"] = (p[:, a:a + w] for a, w in zip(starts, widths))
    if case["decay"] == "token":  # steps of 0.001 to 0.1 after the softplus, rates of 0.5 to 16
        s["dt_bias"] = d.normal(heads, mean=-4.6, std=0.8)
        s["a"] = -torch.exp(d.normal(heads, mean=1.0, std=0.8))
    else:  # one decay a head, from 31/32 towards 1
        s["delta"] = s["dt_bias"] = None
        s["a"] = torch.log1p(-torch.exp2(-5.0 - 7.0 * torch.rand(heads, generator=d.gen, device="cuda")))
    s["state"] = d.normal(s["num_slots"], heads, key, value)
    return s


def _workspace(nbytes):
    return torch.empty(nbytes, dtype=torch.uint8, device="cuda") if nbytes else None


def _rows_of(rows, cols, fmt):
    """Buffers of microscaled rows: codes, a byte or half of one each in whole blocks, and scales in groups of four."""
    blocks = (cols + BLOCK - 1) // BLOCK
    return (torch.empty(rows, blocks * (BLOCK if fmt == "mx8" else BLOCK // 2), dtype=torch.uint8, device="cuda"),
            torch.empty(rows, (blocks + 3) // 4 * 4, dtype=torch.uint8, device="cuda"))


def _plan(case, s):
    """What a user's program keeps from call to call: descriptions, workspaces, outputs, quantised weights."""
    from paper_2008_03602_amd import _lib as L
    L.ct_init(0)
    code = {torch.float32: L.DT_F32, torch.bfloat16: L.DT_BF16, "mx8": L.MX_E4M3, "mx4": L.MX_E2M1}
    if case["op"] == "norm":
        rows, cols, dt = case["rows"], case["cols"], s["x"].dtype
        plan = {"sum": torch.empty_like(s["x"]) if case["residual"] else None, "scales": None}
        if case["out"] in MX:
            plan["y"], plan["scales"] = _rows_of(rows, cols, case["out"])
            plan["values"] = torch.empty(rows, cols, dtype=torch.bfloat16, device="cuda")
            plan["mx"] = L.make_mx(rows, cols, L.DT_BF16, code[case["out"]])
        else:
            plan["y"] = torch.empty(rows, cols, dtype=_dtype(case["out"]), device="cuda")
        plan["op"] = L.make_norm(rows, cols, code[dt], code[case["out"] if case["out"] in MX else plan["y"].dtype],
                                 groups=case["groups"], eps=EPS)
        return plan
    if case["op"] == "quantise":
        q, scales = _rows_of(case["rows"], case["cols"], case["format"])
        return {"op": L.make_mx(case["rows"], case["cols"], code[s["x"].dtype], code[case["format"]]), "q": q,
                "scales": scales, "values": torch.empty_like(s["x"])}
    if case["op"] == "mx_linear":
        m, n, k = case["m"], case["n"], case["k"]
        x, xs = _rows_of(m, k, case["x"])
        w, ws = _rows_of(n, k, case["w"])
        L.ct_mx_quantise_run(L.make_mx(n, k, L.DT_BF16, code[case["w"]]), s["w"], w, ws,
                             torch.cuda.current_stream().cuda_stream)
        y = torch.empty(m, n, dtype=_dtype(case["out"]), device="cuda")
        op = L.make_mx_linear(m, n, k, code[case["x"]], code[case["w"]], code[y.dtype], act=ACTS.index(case["act"]),
                              res=RES.index(case["res"]))
        return {"mx": L.make_mx(m, k, L.DT_BF16, code[case["x"]]), "op": op, "x": x, "xs": xs, "w": w, "ws": ws, "y": y,
                "scratch": _workspace(L.ct_mx_linear_workspace(op))}
    dt = s["q"].dtype
    tokens, pitch = s["q"].shape[0], s["q"].stride(0)
    seqs = L.make_sequences(tokens, len(s["lens"]), s["num_slots"], max_len=max(s["lens"]),
                            offsets=s["offsets"] if "lens" in case else None, slots=s["slots"])
    op = L.make_decay_attention(case["heads"], case["groups"], case["key"], case["value"], code[dt], code[dt],
                                softplus=case["decay"] == "token", step_input=case["step"], scale=case["key"] ** -0.5,
                                ldq=pitch, ldk=pitch, ldv=pitch, lddelta=pitch)
    return {"op": op, "seqs": seqs, "scratch": _workspace(L.ct_decay_attention_workspace(op, seqs)),
            "o": torch.empty(tokens, case["heads"] * case["value"], dtype=dt, device="cuda"),
            "state": torch.zeros_like(s["state"])}


def prepare(case, seed):
    state = {"case": case, "in": _inputs(case, seed)}
    if own:
        state["plan"] = _plan(case, state["in"])
    elif case["op"] == "mx_linear":  # the weights' values, which 16 bits hold exactly
        state["in"]["wv"] = _plain_mx(state["in"]["w"].float(), case["w"]).bfloat16()
    return state


# ---------------------------------------------------------------- one pass
def run(state):
    case, s = state["case"], state["in"]
    if not own:
        return {"norm": _plain_norm, "quantise": _plain_quantise, "mx_linear": _plain_mx_linear,
                "attention": _plain_attention}[case["op"]](case, s)
    from paper_2008_03602_amd import _lib as L
    p = state["plan"]
    stream = torch.cuda.current_stream().cuda_stream
    if case["op"] == "norm":
        L.ct_norm_run(p["op"], s["x"], s["res"], p["sum"], s["w"], s["z"], p["y"], p["scales"], stream)
        if "mx" in p:
            L.ct_mx_values_run(p["mx"], p["y"], p["scales"], p["values"], stream)
        return {"y": p["values"] if "mx" in p else p["y"], "sum": p["sum"]}
    if case["op"] == "quantise":
        L.ct_mx_quantise_run(p["op"], s["x"], p["q"], p["scales"], stream)
        L.ct_mx_values_run(p["op"], p["q"], p["scales"], p["values"], stream)
        return p["values"]
    if case["op"] == "mx_linear":
        L.ct_mx_quantise_run(p["mx"], s["x"], p["x"], p["xs"], stream)
        L.ct_mx_linear_run(p["op"], p["x"], p["xs"], p["w"], p["ws"], s["bias"], s["res"], p["y"], p["scratch"], stream)
        return p["y"]
    L.ct_decay_attention_run(p["op"], p["seqs"], s["q"], s["k"], s["v"], s["delta"], s["dt_bias"], s["a"], s["state"],
                             p["state"], p["o"], p["scratch"], stream)
    return {"o": p["o"], "state": p["state"]}


def _act(v, name):
    if name == "relu":
        return torch.clamp(v, min=0)
    if name == "relu6":
        return torch.clamp(v, min=0, max=6)
    if name == "silu":
        return v / (1 + torch.exp(-v))
    if name == "gelu":
        return 0.5 * v * (1 + torch.erf(v * 0.5 ** 0.5))
    return v


def _pow2(e):
    """2^e for whole e of -126 to 127, exactly."""
    return ((e + 127) << 23).view(torch.float32)


def _exponent(v):
    """floor(log2 v) of normal values, as the bits of v say."""
    return ((v.view(torch.int32) >> 23) & 255) - 127


def _plain_mx(v, fmt):
    """The values that rows stand for once they are microscaled: a block's scale is the power of two that brings its
    largest value's exponent to the largest one of the format; elements are rounded to nearest even and saturate."""
    top, top_e, low_e, bits = MX[fmt]
    rows, cols = v.shape
    blocks = (cols + BLOCK - 1) // BLOCK
    full = torch.zeros(rows, blocks * BLOCK, device="cuda")
    full[:, :cols] = v
    full = full.reshape(rows, blocks, BLOCK)
    e = torch.clamp(_exponent(full.abs().amax(2, keepdim=True)) - top_e, min=-126)
    scale = _pow2(e)
    t = full / scale
    step = _pow2(torch.clamp(_exponent(t.abs()), min=low_e) - bits)
    t = torch.clamp(torch.round(t / step) * step, -top, top)
    return (t * scale).reshape(rows, -1)[:, :cols]


def _plain_norm(case, s):
    rows, cols, groups = case["rows"], case["cols"], case["groups"]
    h = s["x"].float()
    if s["res"] is not None:
        h = h + s["res"].float()
    v = h.reshape(rows, groups, cols // groups)
    v = (v / torch.sqrt((v * v).mean(2, keepdim=True) + EPS)).reshape(rows, cols) * s["w"]
    if s["z"] is not None:
        v = v * _act(s["z"].float(), "silu")
    y = _plain_mx(v, case["out"]).bfloat16() if case["out"] in MX else v.to(_dtype(case["out"]))
    return {"y": y, "sum": h.to(s["x"].dtype) if s["res"] is not None else None}


def _plain_quantise(case, s):
    return _plain_mx(s["x"].float(), case["format"]).to(s["x"].dtype)


def _plain_mx_linear(case, s):
    v = torch.mm(_plain_mx(s["x"].float(), case["x"]), s["wv"].float().t())
    if s["bias"] is not None:
        v = v + s["bias"]
    if case["res"] == "add_act":
        v = v + s["res"].float()
    v = _act(v, case["act"])
    if case["res"] == "add":
        v = v + s["res"].float()
    return v.to(_dtype(case["out"]))


def _sequences_of_equal_length(case, s):
    """(token rows [sequences, length], slots) of sequences that a plain form takes at once."""
    dev = s["q"].device
    if "lens" not in case:
        rows = torch.arange(case["count"] * case["len"], device=dev).reshape(case["count"], case["len"])
        return [(rows, s["slots"].long())]
    starts = s["offsets"].tolist()
    return [(torch.arange(starts[i], starts[i + 1], device=dev)[None], s["slots"][i:i + 1].long())
            for i in range(len(s["lens"]))]


def _plain_attention(case, s):
    heads, groups, key, value = case["heads"], case["groups"], case["key"], case["value"]
    o = torch.empty(s["q"].shape[0], heads * value, dtype=s["q"].dtype, device="cuda")
    state = torch.zeros_like(s["state"])
    for rows, slots in _sequences_of_equal_length(case, s):
        h = s["state"][slots]
        for at in range(0, rows.shape[1], CHUNK):
            r = rows[:, at:at + CHUNK]
            n, c = r.shape
            q, k = (s[x][r].float().reshape(n, c, groups, key).repeat_interleave(heads // groups, 2).transpose(1, 2)
                    for x in ("q", "k"))
            v = s["v"][r].float().reshape(n, c, heads, value).transpose(1, 2)
            dt = torch.ones(n, c, heads, device="cuda")
            if s["delta"] is not None:
                t = s["delta"][r].float() + s["dt_bias"]
                dt = torch.clamp(t, min=0) + torch.log1p(torch.exp(-torch.abs(t)))
            g = torch.cumsum(torch.clamp(dt * s["a"], max=0).double(), 1).transpose(1, 2)
            dt = dt.transpose(1, 2) if case["step"] else torch.ones_like(g, dtype=torch.float32)
            past = torch.ones(c, c, dtype=torch.bool, device="cuda").tril()
            decay = torch.where(past, g[..., :, None] - g[..., None, :], -math.inf).float().exp() * dt[..., None, :]
            p = torch.matmul(q, k.transpose(2, 3).contiguous()) * decay
            y = torch.matmul(p, v) + torch.matmul(q, h) * g.float().exp()[..., None]
            o[r] = (y * key ** -0.5).transpose(1, 2).reshape(n, c, heads * value).to(o.dtype)
            w = (g[..., -1:] - g).float().exp() * dt
            h = h * g[..., -1:, None].float().exp() + torch.matmul((k * w[..., None]).transpose(2, 3).contiguous(), v)
        state[slots] = h
    return {"o": o, "state": state}


# ---------------------------------------------------------------- what a pass cannot do without
def _mx_bytes(rows, cols, fmt):
    return rows * ((cols + BLOCK - 1) // BLOCK) * (33.0 if fmt == "mx8" else 17.0)


def _bytes_of(name):
    return 2 if name == "bf16" else 4


def work(case):
    if case["op"] == "norm":
        n = case["rows"] * case["cols"]
        e = _bytes_of(case["dtype"])
        out = _mx_bytes(case["rows"], case["cols"], case["out"]) if case["out"] in MX else n * _bytes_of(case["out"])
        return {"bytes": float(e * n * (1 + 2 * case["residual"] + case["gate"]) + out + 4 * case["cols"]),
                "flops": n * (4.0 + case["residual"] + 5 * case["gate"])}
    if case["op"] == "quantise":
        n = case["rows"] * case["cols"]
        # the codes written, and the values they stand for
        return {"bytes": 2.0 * _bytes_of(case["dtype"]) * n + _mx_bytes(case["rows"], case["cols"], case["format"]),
                "flops": 4.0 * n}
    if case["op"] == "mx_linear":
        m, n, k, o = case["m"], case["n"], case["k"], _bytes_of(case["out"])
        outs = 2 if case["res"] != "none" else 1
        return {"bytes": 2.0 * m * k + _mx_bytes(n, k, case["w"]) + o * m * n * outs + 4.0 * n * case["bias"],
                "flops": 2.0 * m * n * k}
    lens, e = _lens(case), _bytes_of(case["dtype"])
    tokens, count, each = sum(lens), len(lens), case["heads"] * case["key"] * case["value"]
    columns = 2 * case["groups"] * case["key"] + 2 * case["heads"] * case["value"]
    columns += case["heads"] if case["decay"] == "token" else 0
    return {"bytes": float(e * tokens * columns + 8 * count * each), "flops": 4.0 * tokens * each}


# ---------------------------------------------------------------- the definitions in 64 bits
def exact(case, seed):
    s = _inputs(case, seed)
    f = torch.float64
    if case["op"] == "norm":
        h = s["x"].to(f) + (s["res"].to(f) if s["res"] is not None else 0.0)
        parts = h.reshape(case["rows"], case["groups"], -1)
        y = (parts * torch.rsqrt(parts.square().mean(-1, keepdim=True) + EPS)).reshape(h.shape) * s["w"].to(f)
        y = y if s["z"] is None else y * _act64(s["z"].to(f), "silu")
        return {"y": _mx64(y, case["out"]) if case["out"] in MX else y, "sum": h if s["res"] is not None else None}
    if case["op"] == "quantise":
        return _mx64(s["x"].to(f), case["format"])
    if case["op"] == "mx_linear":
        v = _mx64(s["x"].to(f), case["x"]) @ _mx64(s["w"].to(f), case["w"]).t().contiguous()
        v = v if s["bias"] is None else v + s["bias"].to(f)
        r = s["res"].to(f) if s["res"] is not None else 0.0
        early, late = (r, 0.0) if case["res"] == "add_act" else (0.0, r)
        return _act64(v + early, case["act"]) + late
    heads, groups, key, value = case["heads"], case["groups"], case["key"], case["value"]
    o = torch.zeros(s["q"].shape[0], heads, value, dtype=f, device="cuda")
    state = torch.zeros(s["state"].shape, dtype=f, device="cuda")
    lens, slots = s["lens"], s["slots"].tolist()
    starts = [sum(lens[:i]) for i in range(len(lens))]
    # sequences side by side, longest first, so that those still running at a step are the first ones
    order = sorted(range(len(lens)), key=lambda i: -lens[i])
    index = torch.tensor([slots[i] for i in order], device="cuda")
    held = s["state"][index].to(f)
    head = torch.arange(heads, device="cuda") // (heads // groups)
    for t in range(max(lens)):
        alive = sum(1 for v in lens if v > t)
        rows = torch.tensor([starts[i] + t for i in order[:alive]], device="cuda")
        q, k = (s[x][rows].to(f).reshape(alive, groups, key)[:, head] for x in ("q", "k"))
        v = s["v"][rows].to(f).reshape(alive, heads, value)
        dt = torch.ones(alive, heads, dtype=f, device="cuda")
        if s["delta"] is not None:
            dt = torch.nn.functional.softplus(s["delta"][rows].to(f) + s["dt_bias"].to(f), threshold=700.0)
        a = torch.exp(torch.clamp(dt * s["a"].to(f), max=0.0))
        k = k * dt[..., None] if case["step"] else k
        held[:alive] = a[..., None, None] * held[:alive] + k[..., :, None] * v[..., None, :]
        o[rows] = (q[..., :, None] * held[:alive]).sum(2) * key ** -0.5
    state[index] = held
    return {"o": o.reshape(-1, heads * value), "state": state}


def _two_to64(e):
    return ((e.long() + 1023) << 52).view(torch.float64)  # exactly, which a power function need not be


def _mx64(v, fmt):
    top, top_e, low_e, bits = MX[fmt]
    out = torch.zeros_like(v)
    for c in range(0, v.shape[1], BLOCK):
        b = v[:, c:c + BLOCK]
        _, e = torch.frexp(b.abs().amax(1, keepdim=True))  # the largest is m 2^e with m in [1/2, 1)
        scale = _two_to64(e - 1 - top_e)
        t = b / scale
        _, e = torch.frexp(t)
        step = _two_to64(torch.clamp(e - 1, min=low_e) - bits)
        out[:, c:c + BLOCK] = torch.clamp(torch.round(t / step) * step, -top, top) * scale
    return out


def _act64(v, name):
    if name == "silu":
        return v * torch.sigmoid(v)
    if name == "gelu":
        return torch.nn.functional.gelu(v)
    if name in ("relu", "relu6"):
        return torch.nn.functional.relu6(v) if name == "relu6" else torch.relu(v)
    return v
