"""The sequence block (seven operator calls) in fp32 against the same block in 64 bits on the CPU,
over packed prompts, single tokens and rows of no sequence, eager and from a captured graph."""
import pytest
import torch

from paper_2008_03602_amd import _lib as L
from paper_2008_03602_amd.sequence import SequenceBlock, main, serve
from gpu_util import device_ready, note

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _device():
    device_ready()
    yield


class Block64:
    """The block's mathematics, token by token, from its weights."""

    def __init__(self, b):
        self.b = b
        for k in ("w_in", "w_conv", "b_conv", "w_x", "w_step", "b_step", "a", "skip", "w_out"):
            setattr(self, k, getattr(b, k).double().cpu())
        self.hist, self.h = {}, {}

    def token(self, slot, x):
        n, b = self.b.inner, self.b
        hist = self.hist.get(slot, torch.zeros(b.width - 1, n, dtype=torch.float64))
        h = self.h.get(slot, torch.zeros(n, b.states, dtype=torch.float64))
        x = x.double()
        xz = self.w_in @ x
        win = torch.cat([hist, xz[None, :n]])
        self.hist[slot] = win[1:]
        v = (win * self.w_conv.t()).sum(0) + self.b_conv
        u = v / (1 + torch.exp(-v))
        p = self.w_x @ u
        dt = torch.nn.functional.softplus(self.w_step @ p[:b.rank] + self.b_step, threshold=700.0)
        bb, c = p[b.rank:b.rank + b.states], p[b.rank + b.states:]
        self.h[slot] = torch.exp(dt[:, None] * self.a) * h + (dt * u)[:, None] * bb
        y = self.h[slot] @ c + self.skip * u
        z = xz[n:]
        return self.w_out @ (y * z / (1 + torch.exp(-z))) + x


# Products of up to 96 terms with sums of magnitudes of order 10, through four of them one after
# another and recurrences of up to 60 steps: 2^-24 times some thousands.
TOL = 5e-4


def _block(**kw):
    return SequenceBlock(48, 96, states=16, rank=8, slots=6, max_rows=160, dtype=torch.float32, **kw)


def test_packed_prompts_then_tokens_match_64_bits():
    block = _block()
    ref = Block64(block)
    lens, slots = [60, 0, 1, 33], [4, 2, 5, 0]
    g = torch.Generator().manual_seed(3)
    x = torch.randn(100, 48, generator=g)
    off = torch.tensor([3, 63, 63, 64, 97], dtype=torch.int32).cuda()  # rows 0-2 and 97-99 belong to nobody
    y = torch.full((100, 48), 7.0, device="cuda")
    note("sequence block: packed prompts")
    dev_slots = torch.tensor(slots, dtype=torch.int32).cuda()
    block.run(block.plan(block.sequences(100, 4, 0, off, dev_slots)), x.cuda(), y)
    got = y.cpu()
    for s, b, e in ((4, 3, 63), (5, 63, 64), (0, 64, 97)):
        for t in range(b, e):
            want = ref.token(s, x[t])
            assert (got[t].double() - want).abs().max() < TOL, (s, t)
    assert torch.equal(block.state[1].cpu(), torch.zeros(96, 16)) and torch.equal(block.state[3].cpu(), torch.zeros(96, 16))
    note("sequence block: tokens, one sequence without a slot")
    step_slots = torch.tensor([0, -1, 4, 2], dtype=torch.int32).cuda()
    plan = block.plan(block.sequences(4, 4, 1, None, step_slots))
    y4 = torch.empty(4, 48, device="cuda")
    for _ in range(5):
        xt = torch.randn(4, 48, generator=g)
        block.run(plan, xt.cuda(), y4)
        got = y4.cpu()
        for i, s in enumerate((0, None, 4, 2)):
            if s is not None:
                assert (got[i].double() - ref.token(s, xt[i])).abs().max() < TOL, s


def test_serving_is_the_same_from_a_graph_and_by_hand():
    block = _block(seed=2)
    lens = [40, 17, 60]
    r = serve(block, lens, 6)
    block.reset()
    gen = torch.Generator(device="cuda")
    gen.manual_seed(1)
    x = torch.randn(117, 48, generator=gen, device="cuda")
    slots = torch.randperm(6, generator=gen, device="cuda")[:3].to(torch.int32).contiguous()
    off = torch.tensor([0, 40, 57, 117], dtype=torch.int32, device="cuda")
    y = torch.empty_like(x)
    block.run(block.plan(block.sequences(117, 3, 60, off, slots)), x, y)
    assert torch.equal(y, r["prompt"])
    a = torch.tanh(y[[39, 56, 116]])
    plan = block.plan(block.sequences(3, 3, 1, None, slots))
    for i in range(6):
        b = torch.empty_like(a)
        block.run(plan, a, b)
        a = torch.tanh(b)
        assert torch.equal(a, r["steps"][i + 1]), i


def test_wrong_buffers_are_refused():
    block = _block()
    plan = block.plan(block.sequences(4, 4, 1))
    x = torch.zeros(4, 48, device="cuda")
    for bad in (x.bfloat16(), x[:3], torch.zeros(4, 96, device="cuda")[:, ::2], x.cpu()):
        with pytest.raises(ValueError):
            block.run(plan, bad, torch.empty_like(x))
    with pytest.raises(ValueError):
        block.plan(block.sequences(161, 1))
    with pytest.raises(ValueError):
        block.sequences(4, 2, 0, torch.zeros(2, dtype=torch.int32, device="cuda"))
    with pytest.raises(ValueError):
        block.sequences(4, 2, 0, None, torch.zeros(2, dtype=torch.int64, device="cuda"))


def test_command_line(capsys):
    assert main(["--model", "256", "--inner", "512", "--tokens", "300", "--sequences", "3", "--steps", "4"]) == 0
    assert '"finite": true' in capsys.readouterr().out
    assert L.ct_last_error() is not None
