"""Refusals of the sequence-block operators: wrong arguments give CT_E_ARG with a reason,
before anything of a device is touched (nothing here initialises one)."""
import ctypes

import pytest

from paper_2008_03602_amd import _lib as L

OK = 0x1000  # an address that no call here reaches


def refused(call, what):
    with pytest.raises(L.CtError) as e:
        call()
    assert e.value.code == L.CT_E_ARG and what in str(e.value), str(e.value)


def linear(**kw):
    a = dict(m=4, n=24, k=16, dtype=L.DT_BF16, out_dtype=L.DT_F32)
    a.update(kw)
    return L.make_linear(**a)


def run_linear(op, x=OK, w=OK, bias=OK, res=OK, y=OK, ws=None, ws_bytes=0):
    L.ct_linear_run(op, x, w, bias, res, y, ws, 0, ws_bytes)


@pytest.mark.parametrize("field,value,what", [
    ("m", -1, "negative"), ("n", -1, "negative"), ("k", -5, "negative"), ("dtype", 2, "dtype"), ("out_dtype", 7, "dtype"),
    ("m", 0x7FFFFFFF, "too many"), ("n", 0x7FFFF000, "too many"), ("act", 5, "activation"), ("act", -1, "activation"), ("res", 3, "residual"), ("reserved", 1, "reserved"),
    ("ldx", 15, "pitch"), ("ldw", 15, "pitch"), ("ldy", 23, "pitch"), ("ldx", (4 << 20) // 2 + 1, "4 MiB"),
    ("ldw", (4 << 20) // 2 + 1, "4 MiB"), ("ldy", (1 << 31) + 1, "pitch")])
def test_linear_refuses_a_wrong_description(field, value, what):
    op = linear()
    setattr(op, field, value)
    refused(lambda: run_linear(op), what)
    refused(lambda: L.ct_linear_workspace(op), what)


def test_linear_refuses_wrong_arrays():
    refused(lambda: run_linear(linear(), x=None), "null")
    refused(lambda: run_linear(linear(), w=None), "null")
    refused(lambda: run_linear(linear(), y=None), "null")
    refused(lambda: run_linear(linear(res=L.RES_ADD), res=None), "null")
    refused(lambda: run_linear(linear(res=L.RES_ADD, ldr=23)), "pitch")
    refused(lambda: run_linear(linear(), x=OK + 1), "aligned")
    refused(lambda: run_linear(linear(dtype=L.DT_F32), w=OK + 2), "aligned")
    refused(lambda: run_linear(linear(), bias=OK + 2), "aligned")
    refused(lambda: run_linear(linear(), y=OK + 2), "aligned")
    h = L.lib()
    assert h.ct_linear_run(None, OK, OK, None, None, OK, None, 0, None) == L.CT_E_ARG
    op = linear()
    assert h.ct_linear_workspace(ctypes.byref(op), None) == L.CT_E_ARG


def test_nothing_to_do_needs_no_device():
    run_linear(linear(m=0), x=None, y=None)
    run_linear(linear(n=0), y=None)
    assert L.ct_linear_workspace(linear(m=0)) == 0
    none = L.make_sequences(0, 0)
    L.ct_causal_conv_run(L.make_causal_conv(8, 4, 0), none, None, None, None, None, None, None)
    L.ct_scan_run(L.make_scan(8, 4, 1, 0), none, None, None, None, None, None, None, None, None, None, None, None)
    assert L.ct_scan_workspace(L.make_scan(8, 4, 1, 0), none) == 0


def test_valid_calls_need_an_initialised_device():
    seqs = L.make_sequences(6, 2, 2)
    for call in (lambda: run_linear(linear()),
                 lambda: L.ct_causal_conv_run(L.make_causal_conv(8, 4, 1), seqs, OK, OK, OK, OK, OK, OK),
                 lambda: L.ct_scan_run(L.make_scan(8, 4, 2, 1), seqs, OK, OK, OK, OK, OK, OK, OK, OK, OK, OK, OK)):
        with pytest.raises(L.CtError) as e:
            call()
        assert e.value.code == L.CT_E_NOINIT


SEQS = [(dict(tokens=-1, count=2), "negative"), (dict(tokens=4, count=-2), "negative"),
        (dict(tokens=4, count=2, num_slots=-1), "negative"), (dict(tokens=4, count=2, max_len=-1), "negative"),
        (dict(tokens=5, count=2, num_slots=2), "multiple"), (dict(tokens=5, count=0), "multiple"),
        (dict(tokens=0x7FFFFFF0, count=1), "too many"), (dict(tokens=8, count=0x7FFFFFF0, offsets=OK), "too many"),
        (dict(tokens=4, count=2, num_slots=1), "slots"), (dict(tokens=4, count=2, offsets=OK + 2), "misaligned"),
        (dict(tokens=4, count=2, num_slots=2, slots=OK + 1), "misaligned")]


@pytest.mark.parametrize("kw,what", SEQS)
def test_sequences_are_checked(kw, what):
    seqs = L.make_sequences(**kw)
    refused(lambda: L.ct_causal_conv_run(L.make_causal_conv(8, 4, 1), seqs, OK, OK, OK, OK, OK, OK), what)
    scan = L.make_scan(8, 4, 2, 1)
    refused(lambda: L.ct_scan_run(scan, seqs, OK, OK, OK, OK, OK, OK, OK, OK, OK, OK, OK), what)
    if what != "slots":
        refused(lambda: L.ct_scan_workspace(scan, seqs), what)


@pytest.mark.parametrize("field,value,what", [
    ("channels", -1, "negative"), ("width", 1, "width"), ("width", 9, "width"), ("dtype", 2, "dtype"),
    ("act", L.ACT_GELU, "activation"), ("ldx", 7, "pitch"), ("ldy", 7, "pitch")])
def test_causal_conv_refuses_a_wrong_description(field, value, what):
    op = L.make_causal_conv(8, 4, 1)
    setattr(op, field, value)
    refused(lambda: L.ct_causal_conv_run(op, L.make_sequences(6, 2, 2), OK, OK, OK, OK, OK, OK), what)


def test_causal_conv_refuses_wrong_arrays():
    op, seqs = L.make_causal_conv(8, 4, 1), L.make_sequences(6, 2, 2)
    good = dict(x=OK, w=OK, bias=OK, state_in=OK, state_out=OK, y=OK)
    for name, value, what in (("x", None, "null"), ("w", None, "null"), ("y", None, "null"), ("x", OK + 1, "aligned"),
                              ("state_in", OK + 1, "aligned"), ("bias", OK + 2, "aligned")):
        refused(lambda: L.ct_causal_conv_run(op, seqs, **dict(good, **{name: value})), what)


@pytest.mark.parametrize("field,value,what", [
    ("channels", -2, "negative"), ("states", 0, "states"), ("states", 257, "states"), ("groups", 0, "groups"),
    ("groups", 3, "groups"), ("dtype", -1, "dtype"), ("softplus", 2, "flag"), ("reserved", 1, "flag"),
    ("ldu", 7, "pitch"), ("lddelta", 7, "pitch"), ("ldb", 7, "pitch"), ("ldc", 7, "pitch"), ("ldy", 7, "pitch"),
    ("ldz", 7, "pitch"), ("ldu", (2 << 20) + 1, "4 MiB"), ("lddelta", (2 << 20) + 1, "4 MiB"),
    ("ldy", (2 << 20) + 1, "4 MiB"), ("ldz", (2 << 20) + 1, "4 MiB")])
def test_scan_refuses_a_wrong_description(field, value, what):
    op = L.make_scan(8, 4, 2, 1)
    setattr(op, field, value)
    refused(lambda: L.ct_scan_run(op, L.make_sequences(6, 2, 2), OK, OK, OK, OK, OK, OK, OK, OK, OK, OK, OK), what)


def test_scan_refuses_wrong_arrays_and_workspaces():
    op, seqs = L.make_scan(8, 4, 2, 1), L.make_sequences(6, 2, 2)
    good = dict(u=OK, delta=OK, dt_bias=OK, a=OK, b=OK, c=OK, d_skip=OK, z=OK, state_in=OK, state_out=OK, y=OK)
    for name in ("u", "delta", "a", "b", "c", "y"):
        refused(lambda: L.ct_scan_run(op, seqs, **dict(good, **{name: None})), "null")
    for name in ("u", "z", "y"):
        refused(lambda: L.ct_scan_run(op, seqs, **dict(good, **{name: OK + 1})), "aligned")
    for name in ("dt_bias", "a", "d_skip", "state_in", "state_out"):
        refused(lambda: L.ct_scan_run(op, seqs, **dict(good, **{name: OK + 2})), "aligned")


def test_workspaces_are_checked():
    op = linear(m=96, n=64, k=16384)
    need = L.ct_linear_workspace(op)
    if need:
        refused(lambda: run_linear(op), "workspace")
        refused(lambda: run_linear(op, ws=OK, ws_bytes=need - 1), "workspace")
        refused(lambda: run_linear(op, ws=OK + 4, ws_bytes=need), "16-byte")
    scan, seqs = L.make_scan(256, 16, 1, 1), L.make_sequences(8192, 1, 1)
    need = L.ct_scan_workspace(scan, seqs)
    if need:
        arrays = (OK,) * 11
        refused(lambda: L.ct_scan_run(scan, seqs, *arrays), "workspace")
        refused(lambda: L.ct_scan_run(scan, seqs, *arrays, OK, 0, need - 1), "workspace")
        refused(lambda: L.ct_scan_run(scan, seqs, *arrays, OK + 8, 0, need), "16-byte")
