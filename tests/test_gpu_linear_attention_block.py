"""The linear-attention block: each of its calls against 64 bits from what the call before it left, and
what passes, plans, graphs and slots leave to each other."""
import pytest
import torch

from paper_2008_03602_amd import _lib as L
from paper_2008_03602_amd.linear_attention import EPS, LinearAttentionBlock, main
from paper_2008_03602_amd.sequence import serve
from gpu_util import device_ready, note
from test_gpu_linear_attention import B, D, ROUND, U, attention64, check_rows, dropped, gen, normal, values_of, within

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _device():
    device_ready()
    yield


def normed(x, parts, w, z=None):
    """The norm in 64 bits and its bound, as the norm's own test works it out."""
    rows, cols = x.shape
    v = x.double().reshape(rows, parts, -1)
    n = cols // parts
    y = (v / torch.sqrt((v * v).mean(2, keepdim=True) + EPS)).reshape(rows, cols) * w.cpu().double()
    rel = (n / 2 + 12) * U * torch.ones_like(y)
    if z is not None:
        z = z.double()
        y, rel = y * z / (1 + torch.exp(-z)), rel + (2 * z.abs() + 8) * U
    return y, rel * y.abs()


def product(x, w, res=None):
    """The product of values in 64 bits and its bound."""
    y, bound = x @ w.t(), dropped(x, w) + (x.shape[1] + 4) * U * (x.abs() @ w.abs().t())
    if res is not None:
        y = y + res.double()
        bound = bound + U * y.abs()
    return y, bound + ROUND[B] * (y.abs() + bound)


def check_pass(block, plan, off, slots, x, what):
    """One pass, each call's output against 64 bits from its inputs as the block's buffers hold them."""
    note(what)
    m = x.shape[0]
    before = block.state.cpu()
    xd, y = x.cuda(), torch.full((m, block.model), float("nan"), dtype=B, device="cuda")
    block.run(plan, xd, y)
    torch.cuda.synchronize()
    c, s = block.starts, {}
    q8, s8 = (t[:m].cpu() for t in block._x)
    check_rows(q8, s8, *normed(x, 1, block.norm_in), L.MX_E4M3, what + ": norm")
    w_in, w_out = (values_of(w[0].cpu(), w[1].cpu(), k, L.MX_E2M1) for w, k in ((block.w_in, block.model), (block.w_out, block.inner)))
    p = block._p[:m].cpu()
    within(p, *product(values_of(q8, s8, block.model, L.MX_E4M3), w_in), what + ": project in")
    widths = (block.groups * block.key, block.groups * block.key, block.inner, block.inner, block.heads)
    s["q"], s["k"], s["v"], z, s["delta"] = (p[:, a:a + n] for a, n in zip(c, widths))
    s["dt_bias"], s["a"], s["state"] = block.b_step.cpu(), block.a.cpu(), before
    ref, bound, new, nbound = attention64(s, off, slots, block.key ** -0.5, False, True, B)
    o = block._o[:m].cpu()
    inside = torch.zeros(m, dtype=torch.bool)
    inside[int(off[0]):int(off[-1])] = True
    within(o[inside], ref[inside], bound[inside], what + ": attention")
    assert (o[~inside] == 0).all()
    within(block.state, new, nbound, what + ": states")
    g8, gs = (t[:m].cpu() for t in block._g)
    check_rows(g8, gs, *normed(o, block.heads, block.norm_out, z), L.MX_E4M3, what + ": norm of heads")
    within(y, *product(values_of(g8, gs, block.inner, L.MX_E4M3), w_out, x), what + ": project out")
    assert torch.equal(y.cpu()[~inside], x[~inside]), what + ": rows of nobody"
    return y


@pytest.mark.parametrize("heads,groups,key,value", [(4, 4, 64, 64), (6, 2, 24, 32), (2, 1, 128, 96), (3, 3, 16, 160)])
def test_block_passes(heads, groups, key, value):
    block = LinearAttentionBlock(200, heads, groups, key, value, slots=6, max_rows=300)
    g = gen(heads)
    lens = [70, 0, 1, 130, 64]
    off = torch.tensor([3 + sum(lens[:i]) for i in range(6)], dtype=torch.int32)
    slots = torch.tensor([4, 0, 2, 5, 1], dtype=torch.int32)
    plan = block.plan(block.sequences(275, 5, 0, off.cuda(), slots.cuda()))
    for i in range(2):
        check_pass(block, plan, off, slots, normal(g, 275, 200, dtype=B), "packed prompts, pass %d" % i)
    step = block.plan(block.sequences(5, 5, 1, None, slots.cuda()))
    for i in range(2):
        check_pass(block, step, torch.arange(6), slots, normal(g, 5, 200, dtype=B), "single tokens, pass %d" % i)


def test_prompts_then_tokens_from_a_graph():
    """A prompt in one pass and its tokens one by one end alike; replays are the eager steps' bits."""
    block = LinearAttentionBlock(256, 4, 2, 32, 32, slots=3, max_rows=256)
    lens = [40, 0, 23]
    note("serve")
    first = serve(block, lens, 6)
    state = block.state.clone()
    again = serve(block, lens, 6)
    assert torch.equal(first["steps"], again["steps"]) and torch.equal(first["prompt"], again["prompt"])
    assert torch.equal(state, block.state)
    # the same steps without a graph, on another stream
    g = torch.Generator(device="cuda")
    g.manual_seed(1)
    x = torch.randn(63, 256, generator=g, device="cuda").to(B)
    off = torch.tensor([0, 40, 40, 63], dtype=torch.int32, device="cuda")
    slots = torch.randperm(3, generator=g, device="cuda").to(torch.int32).contiguous()
    block.reset()
    torch.cuda.synchronize()
    with torch.cuda.stream(torch.cuda.Stream()):
        y = torch.empty_like(x)
        block.run(block.plan(block.sequences(63, 3, 40, off, slots)), x, y)
        plan = block.plan(block.sequences(3, 3, 1, None, slots))
        a, b = torch.tanh(y[[39, 0, 62]]), torch.empty(3, 256, dtype=B, device="cuda")
        a[1] = 0
        outs = [a.clone()]
        for _ in range(6):
            block.run(plan, a, b)
            a = torch.tanh(b)
            outs.append(a.clone())
        torch.cuda.synchronize()
    assert torch.equal(torch.stack(outs), first["steps"]) and torch.equal(block.state, state)


def test_captured_steps_outlive_plans_of_longer_prompts():
    block = LinearAttentionBlock(64, 1, 1, 64, 64, slots=2, max_rows=8192)
    plan = block.plan(block.sequences(4096, 1))
    x = normal(gen(1), 4096, 64, dtype=B).cuda()
    y = torch.empty_like(x)
    note("a captured prompt in pieces")
    assert L.ct_decay_attention_workspace(plan["attention"], plan["seqs"]) > 16
    block.run(plan, x, y)
    block.reset()
    block.run(plan, x, y)
    want, state = y.clone(), block.state.clone()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        block.run(plan, x, y)
    longer = block.plan(block.sequences(8192, 1))
    assert longer["ws"].numel() > plan["ws"].numel()
    others = [torch.full((plan["ws"].numel() + 4096 * i,), 7, dtype=torch.uint8, device="cuda") for i in range(8)]
    for _ in range(3):
        block.reset()
        y.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(y, want) and torch.equal(block.state, state)
    assert all((o == 7).all() for o in others)


def test_the_command_serves(capsys):
    assert main(["--model", "256", "--heads", "4", "--groups", "2", "--key", "32", "--value", "32", "--tokens", "300",
                 "--sequences", "3", "--steps", "4"]) == 0
    assert '"finite": true' in capsys.readouterr().out


def test_block_refuses_what_its_buffers_do_not_hold():
    with pytest.raises(ValueError):
        LinearAttentionBlock(64, 2, 2, 16, 40)
    block = LinearAttentionBlock(64, 2, 2, 16, 32, slots=2, max_rows=16)
    with pytest.raises(ValueError):
        block.plan(block.sequences(17, 1))
    with pytest.raises(ValueError):
        block.sequences(4, 1, offsets=torch.zeros(2, dtype=torch.int64, device="cuda"))
    plan = block.plan(block.sequences(4, 1))
    with pytest.raises(ValueError):
        block.run(plan, torch.zeros(4, 64, device="cuda"), torch.zeros(4, 64, dtype=B, device="cuda"))
