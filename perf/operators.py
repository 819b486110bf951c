"""What the sequence-block operators are timed on: calls of a user's program, through the public entry points.

Three operators, which together are one recurrent sequence block as it is served:

* ``linear``: a matrix product with bias, activation and residual in its epilogue (``ct_linear_run``);
* ``conv``: the short causal depthwise convolution along the tokens of packed sequences, with the
  values before a sequence's start held in state slots (``ct_causal_conv_run``);
* ``scan``: the selective state space scan over packed sequences, with its state in slots
  (``ct_scan_run``).

Sequences are packed: token rows of all sequences one after another. A case's ``lens`` is the lengths
as a text, or ``count`` x ``len`` equal ones (``len`` 1: a decode step). The plain forms are elementary
torch operations in 32 bits.
"""
import math

import torch

own = False

ACTS = ("none", "relu", "relu6", "silu", "gelu")
RES = ("none", "add", "add_act")  # no residual; act(v) + r; act(v + r)
LOW_RANK = 64  # columns before B and C in the projection that they are slices of


def listed():
    return [
        # one token of one sequence through a projection: the smallest call, latency counts
        {"name": "linear_one_token", "op": "linear", "m": 1, "n": 2048, "k": 1024, "dtype": "bf16", "out": "bf16",
         "act": "silu", "bias": True, "res": "none"},
        # a decode step of 24 sequences through a wide projection with the residual: the weight's bytes
        {"name": "linear_decode", "op": "linear", "m": 24, "n": 4096, "k": 8192, "dtype": "bf16", "out": "bf16",
         "act": "none", "bias": False, "res": "add"},
        # a prompt of 8192 tokens: the matrix cores
        {"name": "linear_prompt", "op": "linear", "m": 8192, "n": 8192, "k": 4096, "dtype": "bf16", "out": "bf16",
         "act": "gelu", "bias": True, "res": "none"},
        # MobileNet-v2's expansion 32 -> 192 at 28 x 28, batch 16, as a product with its folded normalisation
        # and ReLU6: x and y's bytes
        {"name": "linear_pointwise", "op": "linear", "m": 12544, "n": 192, "k": 32, "dtype": "bf16", "out": "f32",
         "act": "relu6", "bias": True, "res": "none"},
        # fp32 with no aligned row: ragged in every size
        {"name": "linear_odd_f32", "op": "linear", "m": 1021, "n": 1277, "k": 515, "dtype": "f32", "out": "f32",
         "act": "relu", "bias": True, "res": "add_act"},
        # a decode step of 32 sequences
        {"name": "conv_step", "op": "conv", "count": 32, "len": 1, "channels": 2048, "width": 4, "dtype": "f32",
         "act": "silu", "bias": True},
        # packed prompts of unequal lengths, one of them empty and one of a single token
        {"name": "conv_ragged", "op": "conv", "lens": "2047,0,1,517,3891,96,1640", "channels": 4096, "width": 4,
         "dtype": "bf16", "act": "silu", "bias": True},
        # a decode step of 8 sequences: latency
        {"name": "scan_step_small", "op": "scan", "count": 8, "len": 1, "channels": 2048, "states": 16, "groups": 1,
         "dtype": "bf16", "z": True},
        # a decode step of 256 sequences: the states' bytes
        {"name": "scan_step_large", "op": "scan", "count": 256, "len": 1, "channels": 4096, "states": 16, "groups": 1,
         "dtype": "bf16", "z": True},
        # one long prompt: few channels, so the work has to be split over the tokens
        {"name": "scan_long", "op": "scan", "count": 1, "len": 16384, "channels": 2048, "states": 16, "groups": 1,
         "dtype": "bf16", "z": True},
        # packed prompts of unequal lengths
        {"name": "scan_ragged", "op": "scan", "lens": "2047,0,1,517,3891,96,1640", "channels": 4096, "states": 16,
         "groups": 1, "dtype": "bf16", "z": True},
        # fp32 with odd sizes, grouped B and C and no gate
        {"name": "scan_odd_f32", "op": "scan", "lens": "333,1,444", "channels": 1005, "states": 13, "groups": 5,
         "dtype": "f32", "z": False},
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
    while True:
        case = _draw(rng)
        if 3072 not in case.values() and 3072 not in _lens(case):
            return case


def _draw(rng):
    op = rng.choice(("linear", "linear", "conv", "scan", "scan"))
    if op == "linear":
        while True:
            case = {"op": op, "m": _log_int(rng, 1, 16384), "n": _size(rng, 16, 8192), "k": _size(rng, 16, 8192),
                    "dtype": rng.choice(("bf16", "bf16", "bf16", "f32")), "out": rng.choice(("bf16", "f32")),
                    "act": rng.choice(ACTS), "bias": rng.random() < 0.7, "res": rng.choice(RES)}
            most = 5e11 if case["dtype"] == "bf16" else 3e10
            cost = work(case)
            if cost["flops"] <= most and cost["bytes"] <= 4e8:
                return case
    step = rng.random() < 0.35
    dtype = rng.choice(("bf16", "bf16", "f32"))
    case = {"op": op}
    channels = _size(rng, 64, 8192 if step or op == "conv" else 4096)
    if op == "conv":
        case.update(channels=channels, width=rng.choice((2, 3, 4, 4, 4)), dtype=dtype,
                    act=rng.choice(("silu", "silu", "none")), bias=rng.random() < 0.8)
    else:
        groups = rng.choice((1, 1, 2, 4))
        channels = channels // groups * groups
        states = rng.choice((8, 13, 16, 16, 16, 32, 64))
        case.update(channels=channels, states=states, groups=groups, dtype=dtype, z=rng.random() < 0.7)
    per_token = channels * case.get("states", 16)
    if step:
        most = min(256, int(256 * 4096 * 16 / per_token))
        case.update(count=_log_int(rng, 1, max(1, most)), len=1)
    else:
        most = min(16384, int(8192 * 4096 * 16 / per_token))
        tokens = _log_int(rng, 32, max(64, most))
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
    if case["op"] == "linear":
        m, n, k, dt, out = case["m"], case["n"], case["k"], _dtype(case["dtype"]), _dtype(case["out"])
        return {"x": d.normal(m, k, dtype=dt), "w": d.normal(n, k, std=k ** -0.5, dtype=dt),
                "bias": d.normal(n, std=0.5) if case["bias"] else None,
                "res": d.normal(m, n, dtype=out) if case["res"] != "none" else None}
    lens, ch, dt = _lens(case), case["channels"], _dtype(case["dtype"])
    tokens, count = sum(lens), len(lens)
    # states in slots of a larger pool, the sequences' own slots in no order
    s = {"lens": lens, "slots": d.order(count + 3)[:count].contiguous(), "num_slots": count + 3,
         "offsets": torch.tensor([sum(lens[:i]) for i in range(count + 1)], dtype=torch.int32, device="cuda")}
    # x and the gate are the two halves of one projection
    xz = d.normal(tokens, 2 * _pitch(ch, dt), dtype=dt)
    s["x"], z = xz[:, :ch], xz[:, _pitch(ch, dt):_pitch(ch, dt) + ch]
    if case["op"] == "conv":
        w = case["width"]
        s.update(w=d.normal(ch, w, std=w ** -0.5), bias=d.normal(ch, std=0.3) if case["bias"] else None,
                 state=d.normal(s["num_slots"], w - 1, ch, dtype=dt))
        return s
    n, g = case["states"], case["groups"]
    bc = d.normal(tokens, _pitch(LOW_RANK + 2 * g * n, dt), dtype=dt)
    s.update(z=z if case["z"] else None, dt=d.normal(tokens, ch, dtype=dt),
             # steps of 0.001 to 0.1 after the softplus, decay rates of 1 to the number of states
             dt_bias=d.normal(ch, mean=-4.6, std=0.8),
             a=-(torch.arange(1, n + 1, device="cuda") * torch.exp(d.normal(ch, n, std=0.2))).contiguous(),
             b=bc[:, LOW_RANK:LOW_RANK + g * n], c=bc[:, LOW_RANK + g * n:LOW_RANK + 2 * g * n],
             d=d.normal(ch, mean=1.0, std=0.1), state=d.normal(s["num_slots"], ch, n, std=0.3))
    return s


def _plan(case, s):
    """What a user's program keeps from call to call: the operator's description, its workspace, the output."""
    from paper_2008_03602_amd import _lib as L
    L.ct_init(0)
    code = {torch.float32: L.DT_F32, torch.bfloat16: L.DT_BF16}
    if case["op"] == "linear":
        y = torch.empty(case["m"], case["n"], dtype=_dtype(case["out"]), device="cuda")
        p = L.make_linear(case["m"], case["n"], case["k"], code[s["x"].dtype], code[y.dtype],
                          act=ACTS.index(case["act"]), res=RES.index(case["res"]))
        return {"op": p, "y": y, "ws": _workspace(L.ct_linear_workspace(p))}
    x = s["x"]
    y = torch.empty(x.shape, dtype=x.dtype, device="cuda")
    seqs = L.make_sequences(x.shape[0], len(s["lens"]), s["num_slots"], max_len=max(s["lens"]),
                            offsets=s["offsets"] if "lens" in case else None, slots=s["slots"])
    plan = {"seqs": seqs, "y": y, "state": torch.zeros_like(s["state"])}
    if case["op"] == "conv":
        plan["op"] = L.make_causal_conv(case["channels"], case["width"], code[x.dtype], act=ACTS.index(case["act"]),
                                        ldx=x.stride(0))
    else:
        plan["op"] = L.make_scan(case["channels"], case["states"], case["groups"], code[x.dtype], softplus=True,
                                 ldu=x.stride(0), ldb=s["b"].stride(0), ldc=s["c"].stride(0), ldz=x.stride(0))
        plan["ws"] = _workspace(L.ct_scan_workspace(plan["op"], seqs))
    return plan


def _workspace(nbytes):
    return torch.empty(nbytes, dtype=torch.uint8, device="cuda") if nbytes else None


def prepare(case, seed):
    state = {"case": case, "in": _inputs(case, seed)}
    if own:
        state["plan"] = _plan(case, state["in"])
    return state


# ---------------------------------------------------------------- one pass
def run(state):
    case, s = state["case"], state["in"]
    if not own:
        return {"linear": _plain_linear, "conv": _plain_conv, "scan": _plain_scan}[case["op"]](case, s)
    from paper_2008_03602_amd import _lib as L
    p = state["plan"]
    stream = torch.cuda.current_stream().cuda_stream
    if case["op"] == "linear":
        L.ct_linear_run(p["op"], s["x"], s["w"], s["bias"], s["res"], p["y"], p["ws"], stream)
        return p["y"]
    if case["op"] == "conv":
        L.ct_causal_conv_run(p["op"], p["seqs"], s["x"], s["w"], s["bias"], s["state"], p["state"], p["y"], stream)
    else:
        L.ct_scan_run(p["op"], p["seqs"], s["x"], s["dt"], s["dt_bias"], s["a"], s["b"], s["c"], s["d"], s["z"],
                      s["state"], p["state"], p["y"], p["ws"], stream)
    return {"y": p["y"], "state": p["state"]}


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


def _plain_linear(case, s):
    v = torch.mm(s["x"].float(), s["w"].float().t())
    if s["bias"] is not None:
        v = v + s["bias"]
    if case["res"] == "add_act":
        v = v + s["res"].float()
    v = _act(v, case["act"])
    if case["res"] == "add":
        v = v + s["res"].float()
    return v.to(_dtype(case["out"]))


def _groups_of_equal_length(case, s):
    """(token rows [sequences, length], slots) of sequences that a plain form takes at once."""
    dev = s["x"].device
    if "lens" not in case:
        rows = torch.arange(case["count"] * case["len"], device=dev).reshape(case["count"], case["len"])
        return [(rows, s["slots"].long())]
    out, at = [], 0
    for i, n in enumerate(s["lens"]):
        out.append((torch.arange(at, at + n, device=dev).reshape(1, n), s["slots"][i:i + 1].long()))
        at += n
    return out


def _plain_conv(case, s):
    y = torch.empty(s["x"].shape, dtype=s["x"].dtype, device="cuda")
    state = torch.zeros_like(s["state"])
    w = case["width"]
    for rows, slots in _groups_of_equal_length(case, s):
        x = torch.cat([s["state"][slots], s["x"][rows]], dim=1).float()
        n = rows.shape[1]
        v = torch.zeros(rows.shape + (case["channels"],), device="cuda")
        for j in range(w):
            v = v + x[:, j:j + n] * s["w"][:, j]
        if s["bias"] is not None:
            v = v + s["bias"]
        y[rows] = _act(v, case["act"]).to(y.dtype)
        state[slots] = x[:, n:].to(state.dtype)
    return {"y": y, "state": state}


def _plain_scan(case, s):
    y = torch.empty(s["x"].shape, dtype=s["x"].dtype, device="cuda")
    state = torch.zeros_like(s["state"])
    n, g, ch = case["states"], case["groups"], case["channels"]
    for rows, slots in _groups_of_equal_length(case, s):
        count, length = rows.shape
        h = s["state"][slots]
        if length:
            v = s["dt"][rows].float() + s["dt_bias"]
            dt = torch.clamp(v, min=0) + torch.log1p(torch.exp(-torch.abs(v)))
            u = s["x"][rows].float()
            b = s["b"][rows].float().reshape(count, length, g, 1, n)
            c = s["c"][rows].float().reshape(count, length, g, 1, n)
            decay = torch.exp(dt.unsqueeze(-1) * s["a"])
            hs = ((dt * u).reshape(count, length, g, ch // g, 1) * b).reshape(count, length, ch, n)
            for t in range(length):
                h = torch.addcmul(hs[:, t], decay[:, t], h)
                hs[:, t] = h
            del decay
            v = (hs.reshape(count, length, g, ch // g, n) * c).sum(-1).reshape(count, length, ch) + s["d"] * u
            del hs
            if s["z"] is not None:
                v = v * _act(s["z"][rows].float(), "silu")
            y[rows] = v.to(y.dtype)
        state[slots] = h
    return {"y": y, "state": state}


# ---------------------------------------------------------------- what a pass cannot do without
def work(case):
    e = 2 if case["dtype"] == "bf16" else 4
    if case["op"] == "linear":
        m, n, k, o = case["m"], case["n"], case["k"], 2 if case["out"] == "bf16" else 4
        outs = 2 if case["res"] != "none" else 1
        return {"bytes": float(e * (m * k + n * k) + o * m * n * outs + 4 * n * case["bias"]),
                "flops": 2.0 * m * n * k}
    lens, ch = _lens(case), case["channels"]
    tokens, count = sum(lens), len(lens)
    if case["op"] == "conv":
        w = case["width"]
        return {"bytes": float(e * ch * (2 * tokens + 2 * count * (w - 1)) + 4 * ch * (w + case["bias"])),
                "flops": 2.0 * tokens * ch * w}
    n, g = case["states"], case["groups"]
    rows = 4 if case["z"] else 3
    return {"bytes": float(e * tokens * (rows * ch + 2 * g * n) + 8 * count * ch * n + 4 * ch * (n + 2)),
            "flops": 7.0 * tokens * ch * n + 12.0 * tokens * ch}


# ---------------------------------------------------------------- the definition in 64 bits
def exact(case, seed):
    s = _inputs(case, seed)
    f = torch.float64
    if case["op"] == "linear":
        v = s["x"].to(f) @ s["w"].to(f).t().contiguous()
        v = v if s["bias"] is None else v + s["bias"].to(f)
        r = s["res"].to(f) if s["res"] is not None else 0.0
        early, late = (r, 0.0) if case["res"] == "add_act" else (0.0, r)
        return _act64(v + early, case["act"]) + late
    y = torch.zeros(s["x"].shape, dtype=f, device="cuda")
    state = torch.zeros(s["state"].shape, dtype=f, device="cuda")
    lens, slots = s["lens"], s["slots"].tolist()
    starts = [sum(lens[:i]) for i in range(len(lens))]
    # sequences side by side, longest first, so that those still running at a step are the first ones
    order = sorted(range(len(lens)), key=lambda i: -lens[i])
    index = torch.tensor([slots[i] for i in order], device="cuda")
    held = s["state"][index].to(f)
    for t in range(max(lens)):
        alive = sum(1 for v in lens if v > t)
        rows = torch.tensor([starts[i] + t for i in order[:alive]], device="cuda")
        if case["op"] == "conv":
            window = torch.cat([held[:alive], s["x"][rows].to(f).unsqueeze(1)], dim=1)
            v = (window * s["w"].to(f).t()).sum(1)
            v = v if s["bias"] is None else v + s["bias"].to(f)
            y[rows] = _act64(v, case["act"])
            held[:alive] = window[:, 1:]
        else:
            per = case["channels"] // case["groups"]
            n = case["states"]
            step = torch.nn.functional.softplus(s["dt"][rows].to(f) + s["dt_bias"].to(f), threshold=700.0)
            u = s["x"][rows].to(f)
            b = s["b"][rows].to(f).reshape(alive, -1, n).repeat_interleave(per, dim=1)
            c = s["c"][rows].to(f).reshape(alive, -1, n).repeat_interleave(per, dim=1)
            held[:alive] = torch.exp(step[..., None] * s["a"].to(f)) * held[:alive] + (step * u)[..., None] * b
            v = (c * held[:alive]).sum(-1) + s["d"].to(f) * u
            if s["z"] is not None:
                v = v * _act64(s["z"][rows].to(f), "silu")
            y[rows] = v
    state[index] = held
    return {"y": y, "state": state}


def _act64(v, name):
    if name == "silu":
        return v * torch.sigmoid(v)
    if name == "gelu":
        return torch.nn.functional.gelu(v)
    if name in ("relu", "relu6"):
        return torch.nn.functional.relu6(v) if name == "relu6" else torch.relu(v)
    return v
