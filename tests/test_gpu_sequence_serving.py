"""The sequence block as a program serves with it: what passes, plans and graphs leave to each other."""
import pytest
import torch

from paper_2008_03602_amd import _lib as L
from paper_2008_03602_amd.sequence import SequenceBlock, serve
from gpu_util import device_ready, note

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _device():
    device_ready()
    yield


def test_a_captured_step_outlives_plans_of_longer_prompts():
    """A step whose products use a workspace is replayed after a plan that needed a larger one."""
    block = SequenceBlock(48, 4096, states=16, rank=8, slots=6, max_rows=512, dtype=torch.float32)
    step = block.plan(block.sequences(4, 4, 1))
    need = max(L.ct_linear_workspace(step[k]) for k in ("in", "x", "step", "out"))
    assert need > 16
    x, y = torch.randn(4, 48, device="cuda"), torch.empty(4, 48, device="cuda")
    note("sequence block: a step with a workspace")
    block.run(step, x, y)
    block.reset()
    block.run(step, x, y)
    want, state = y.clone(), block.state.clone()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        block.run(step, x, y)
    plan = block.plan(block.sequences(512, 1))
    assert plan["ws"].numel() > step["ws"].numel()
    others = [torch.full((step["ws"].numel() + 4096 * i,), 7, dtype=torch.uint8, device="cuda") for i in range(8)]
    for _ in range(3):
        block.reset()
        y.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(y, want) and torch.equal(block.state, state)
    assert all((o == 7).all() for o in others)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_rows_of_no_sequence_pass_through(dtype):
    """Nothing of an earlier pass, or of memory that was never written, is left in them."""
    block = SequenceBlock(48, 96, states=16, rank=8, slots=6, max_rows=160, dtype=dtype)
    for t in (block._xz, block._u, block._p, block._step, block._y):
        t.fill_(float("nan"))
    g = torch.Generator().manual_seed(5)
    off = torch.tensor([3, 63, 63, 64, 97], dtype=torch.int32).cuda()  # rows 0-2 and 97-99 belong to nobody
    nobody = [0, 1, 2, 97, 98, 99]
    packed, full = block.plan(block.sequences(100, 4, 0, off)), block.plan(block.sequences(100, 2))
    for i in range(2):
        x = torch.randn(100, 48, generator=g).to(dtype).cuda()
        y = torch.full_like(x, float("nan"))
        note("sequence block: rows of nobody, pass %d" % i)
        block.run(packed, x, y)
        assert torch.equal(y[nobody], x[nobody]), i
        assert torch.isfinite(y).all() and not torch.equal(y[3:97], x[3:97])
        block.run(full, torch.randn(100, 48, generator=g).to(dtype).cuda(), y)  # leaves every row of the buffers full
        assert torch.isfinite(y).all()


@pytest.mark.parametrize("lens", [[20, 0, 7, 0], [0, 9], [0, 0, 0]])
def test_sequences_without_a_prompt_start_from_zeros(lens):
    block = SequenceBlock(48, 96, states=16, rank=8, slots=6, max_rows=160, dtype=torch.float32)
    note("sequence block: prompts %s" % lens)
    r = serve(block, lens, 3)
    steps = r["steps"]
    assert torch.isfinite(steps).all()
    alone = serve(block, [0], 3)["steps"][:, 0]  # the same sequence with nobody beside it
    at = 0
    for i, n in enumerate(lens):
        if n:
            at += n
            assert torch.equal(steps[0, i], torch.tanh(r["prompt"][at - 1]))
        else:
            assert not steps[0, i].any()
            assert torch.equal(steps[:, i], alone)
