"""The sequence block's host side: what its plans hold. Nothing here runs a kernel or needs a device."""
import gc
import weakref

import torch

from paper_2008_03602_amd import _lib as L
from paper_2008_03602_amd import sequence as S


def _block(**kw):
    """A block without its weights and buffers, which a plan does not look at."""
    b = S.SequenceBlock.__new__(S.SequenceBlock)
    b.model, b.inner, b.states, b.rank, b.width, b.slots, b.max_rows, b.dtype = 48, 4096, 16, 8, 4, 6, 4096, torch.float32
    b._ws, b._workspaces = None, []
    for k, v in kw.items():
        setattr(b, k, v)
    return b


def test_a_plan_keeps_its_workspace_when_a_larger_one_is_made(monkeypatch):
    made, empty = [], torch.empty

    def on_the_cpu(*a, **kw):
        t = empty(*a, **{k: v for k, v in kw.items() if k != "device"})
        made.append((t.numel(), weakref.ref(t)))
        return t

    monkeypatch.setattr(S.torch, "empty", on_the_cpu)
    block = _block()
    step = block.plan(L.make_sequences(4, 4, 6, 1))
    need = max(L.ct_linear_workspace(step[k]) for k in ("in", "x", "step", "out"))
    assert need > 16 and made[0][0] >= need  # its products split their reductions
    prompt = block.plan(L.make_sequences(4096, 1, 6))
    assert len(made) == 2 and made[1][0] > made[0][0]
    again = block.plan(L.make_sequences(8, 8, 6, 1))
    gc.collect()
    assert made[0][1]() is not None and made[1][1]() is not None and len(made) == 2
    # and past the plans, which a graph does not keep
    del step, prompt, again
    gc.collect()
    assert made[0][1]() is not None and made[1][1]() is not None


def test_addresses_may_be_of_any_kind_of_int():
    class Address(int):
        pass

    a = Address(0x1000)
    assert L._ptr(a) == 0x1000 and L._ptr(None) is None and L._ptr(torch.empty(1)) > 0
    assert L._ws(a, 64) == (0x1000, 64)
    none = L.make_linear(0, 24, 16, L.DT_BF16, L.DT_F32)
    L.ct_linear_run(none, a, a, a, a, a, a, 0, 64)


def test_long_reductions_and_long_prompts_need_their_workspaces():
    """What the refusals of a wrong workspace are tested on."""
    assert L.ct_linear_workspace(L.make_linear(96, 64, 16384, L.DT_BF16, L.DT_F32)) > 0
    assert L.ct_scan_workspace(L.make_scan(256, 16, 1, 1), L.make_sequences(8192, 1, 1)) > 0
