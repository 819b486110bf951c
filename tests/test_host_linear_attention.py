"""Refusals of the linear-attention-block operators: wrong arguments give CT_E_ARG with a reason,
before anything of a device is touched (nothing here initialises one)."""
import ctypes
import random

import pytest

from paper_2008_03602_amd import _lib as L

OK = 0x1000  # an address that no call here reaches
BIG = (1 << 31) + 16


def refused(call, what):
    with pytest.raises(L.CtError) as e:
        call()
    assert e.value.code == L.CT_E_ARG and what in str(e.value), str(e.value)


def changed(op, **fields):
    for k, v in fields.items():
        setattr(op, k, v)
    return op


# ------------------------------------------------------------------ microscaled rows
def mx(**kw):
    return changed(L.make_mx(4, 100, L.DT_BF16, L.MX_E4M3), **kw)


def both_ways(op, x=OK, q=OK, scales=OK):
    return (lambda: L.ct_mx_quantise_run(op, x, q, scales), lambda: L.ct_mx_values_run(op, q, scales, x))


def test_rows_are_whole_blocks_and_scales_whole_groups():
    assert [L.mx_row_bytes(c, L.MX_E4M3) for c in (0, 1, 32, 33, 100)] == [0, 32, 32, 64, 128]
    assert [L.mx_row_bytes(c, L.MX_E2M1) for c in (0, 1, 32, 33, 100)] == [0, 16, 16, 32, 64]
    assert [L.mx_scale_bytes(c) for c in (0, 1, 128, 129)] == [0, 4, 4, 8]


@pytest.mark.parametrize("fields,what", [
    (dict(rows=-1), "negative"), (dict(cols=-1), "negative"), (dict(rows=0x7FFFFFFF), "too many"),
    (dict(cols=0x7FFFFFFF), "too many"), (dict(dtype=2), "dtype"), (dict(format=0), "format"), (dict(format=4), "format"),
    (dict(ldx=99), "pitch"), (dict(ldq=112), "pitch"), (dict(ldq=130), "16 bytes"), (dict(lds=0), "pitch"),
    (dict(lds=6), "scales 4"), (dict(ldq=BIG), "pitch")])
def test_mx_refuses_a_wrong_description(fields, what):
    for call in both_ways(mx(**fields)):
        refused(call, what)


def test_mx_refuses_wrong_arrays():
    for arrays, what in ((dict(x=None), "null"), (dict(q=None), "null"), (dict(scales=None), "null"),
                         (dict(x=OK + 1), "element"), (dict(q=OK + 8), "aligned to 16"), (dict(scales=OK + 2), "scales to 4")):
        for call in both_ways(mx(), **arrays):
            refused(call, what)
    assert L.lib().ct_mx_quantise_run(None, OK, OK, OK, None) == L.CT_E_ARG


# ------------------------------------------------------------------ product
def product(**kw):
    return changed(L.make_mx_linear(4, 24, 100, L.MX_E4M3, L.MX_E2M1, L.DT_BF16), **kw)


def run_product(op, x=OK, xs=OK, w=OK, wsc=OK, bias=OK, res=OK, y=OK, ws=None, ws_bytes=0):
    L.ct_mx_linear_run(op, x, xs, w, wsc, bias, res, y, ws, 0, ws_bytes)


@pytest.mark.parametrize("fields,what", [
    (dict(m=-1), "negative"), (dict(n=-1), "negative"), (dict(k=-1), "negative"), (dict(m=0x7FFFFFFF), "too many"),
    (dict(k=0x7FFFFFFF), "too many"), (dict(x_format=1), "format"), (dict(w_format=4), "format"),
    (dict(out_dtype=2), "dtype"), (dict(act=5), "activation"), (dict(act=-1), "activation"), (dict(res=3), "residual"),
    (dict(ldx=112), "pitch"), (dict(ldw=48), "pitch"), (dict(ldw=72), "16 bytes"), (dict(ldxs=2), "pitch"),
    (dict(ldws=5), "scales 4"), (dict(ldy=23), "pitch"), (dict(res=1, ldr=23), "pitch"),
    (dict(ldx=(4 << 20) + 16), "4 MiB"), (dict(ldw=(4 << 20) + 16), "4 MiB"), (dict(ldws=(4 << 20) + 4), "4 MiB")])
def test_product_refuses_a_wrong_description(fields, what):
    op = product(**fields)
    refused(lambda: run_product(op), what)
    refused(lambda: L.ct_mx_linear_workspace(op), what)


def test_product_refuses_wrong_arrays_and_workspaces():
    for arrays, what in ((dict(x=None), "null"), (dict(xs=None), "null"), (dict(w=None), "null"), (dict(wsc=None), "null"),
                         (dict(y=None), "null"), (dict(x=OK + 4), "aligned to 16"), (dict(w=OK + 8), "aligned to 16"),
                         (dict(xs=OK + 1), "scales to 4"), (dict(wsc=OK + 2), "scales to 4"), (dict(y=OK + 1), "element"),
                         (dict(bias=OK + 2), "element")):
        refused(lambda: run_product(product(), **arrays), what)
    refused(lambda: run_product(product(res=L.RES_ADD), res=None), "null")
    refused(lambda: run_product(product(res=L.RES_ADD), res=OK + 1), "element")
    op = L.make_mx_linear(96, 64, 32768, L.MX_E4M3, L.MX_E2M1, L.DT_BF16)
    need = L.ct_mx_linear_workspace(op)
    assert need > 0
    refused(lambda: run_product(op), "workspace")
    refused(lambda: run_product(op, ws=OK, ws_bytes=need - 1), "workspace")
    refused(lambda: run_product(op, ws=OK + 4, ws_bytes=need), "16-byte")
    assert L.lib().ct_mx_linear_workspace(ctypes.byref(op), None) == L.CT_E_ARG
    assert L.lib().ct_mx_linear_run(None, *[OK] * 7, None, 0, None) == L.CT_E_ARG


# ------------------------------------------------------------------ norm
def norm(**kw):
    return changed(L.make_norm(4, 96, L.DT_BF16, kw.pop("out", L.DT_BF16), groups=kw.pop("groups", 1)), **kw)


def run_norm(op, x=OK, res=OK, sum=OK, w=OK, z=OK, y=OK, scales=OK):
    L.ct_norm_run(op, x, res, sum, w, z, y, scales)


@pytest.mark.parametrize("fields,what", [
    (dict(rows=-1), "negative"), (dict(cols=-1), "negative"), (dict(rows=0x7FFFFFFF), "too many"),
    (dict(groups=0), "groups"), (dict(groups=5), "groups"), (dict(dtype=2), "dtype"), (dict(out=4), "output type"),
    (dict(out=-1), "output type"), (dict(eps=-1.0), "eps"), (dict(eps=float("nan")), "eps"), (dict(ldx=95), "pitch"),
    (dict(ldres=95), "pitch"), (dict(ldsum=95), "pitch"), (dict(ldz=95), "pitch"), (dict(ldy=95), "pitch"),
    (dict(out=L.MX_E4M3, ldy=80), "pitch"), (dict(out=L.MX_E2M1, ldy=56), "16 bytes"), (dict(out=L.MX_E2M1, lds=2), "pitch"),
    (dict(out=L.MX_E4M3, groups=2), "whole blocks")])
def test_norm_refuses_a_wrong_description(fields, what):
    refused(lambda: run_norm(norm(**fields)), what)


def test_norm_refuses_wrong_arrays():
    for arrays, what in ((dict(x=None), "null"), (dict(y=None), "null"), (dict(x=OK + 1), "element"),
                         (dict(res=OK + 1), "element"), (dict(sum=OK + 1), "element"), (dict(z=OK + 1), "element"),
                         (dict(w=OK + 2), "element"), (dict(y=OK + 1), "element")):
        refused(lambda: run_norm(norm(), **arrays), what)
    for arrays, what in ((dict(scales=None), "null"), (dict(y=OK + 8), "aligned to 16"), (dict(scales=OK + 1), "scales to 4")):
        refused(lambda: run_norm(norm(out=L.MX_E4M3), **arrays), what)
    assert L.lib().ct_norm_run(None, *[OK] * 7, None) == L.CT_E_ARG


# ------------------------------------------------------------------ attention
def attention(**kw):
    return changed(L.make_decay_attention(4, 2, 16, 24, L.DT_BF16), **kw)


ARRAYS = dict(q=OK, k=OK, v=OK, delta=OK, dt_bias=OK, a=OK, state_in=OK, state_out=OK, o=OK)


def run_attention(op, seqs=None, ws=None, ws_bytes=0, **kw):
    L.ct_decay_attention_run(op, seqs or L.make_sequences(6, 2, 2), **dict(ARRAYS, **kw), ws=ws, ws_bytes=ws_bytes)


@pytest.mark.parametrize("fields,what", [
    (dict(heads=-2), "negative"), (dict(groups=0), "groups"), (dict(groups=3), "groups"), (dict(key_dim=0), "dimension"),
    (dict(key_dim=257), "dimension"), (dict(value_dim=0), "dimension"), (dict(value_dim=257), "dimension"),
    (dict(dtype=2), "dtype"), (dict(delta_dtype=-1), "dtype"), (dict(softplus=2), "flag"), (dict(step_input=-1), "flag"),
    (dict(reserved=1), "flag"), (dict(ldq=31), "pitch"), (dict(ldk=31), "pitch"), (dict(ldv=95), "pitch"),
    (dict(ldo=95), "pitch"), (dict(lddelta=3), "pitch"), (dict(ldq=(2 << 20) + 1), "4 MiB"),
    (dict(ldk=(2 << 20) + 1), "4 MiB"), (dict(ldv=(2 << 20) + 1), "4 MiB"), (dict(ldo=(2 << 20) + 1), "4 MiB")])
def test_attention_refuses_a_wrong_description(fields, what):
    op = attention(**fields)
    refused(lambda: run_attention(op), what)
    if "lddelta" not in fields:
        refused(lambda: L.ct_decay_attention_workspace(op, L.make_sequences(6, 2, 2)), what)


def test_attention_refuses_wrong_arrays_and_workspaces():
    for name in ("q", "k", "v", "a", "o"):
        refused(lambda: run_attention(attention(), **{name: None}), "null")
    for name in ("q", "k", "v", "delta", "o"):
        refused(lambda: run_attention(attention(), **{name: OK + 1}), "element")
    for name in ("dt_bias", "a", "state_in", "state_out"):
        refused(lambda: run_attention(attention(), **{name: OK + 2}), "element")
    refused(lambda: run_attention(attention(), delta=None), "without delta")
    refused(lambda: run_attention(attention(), seqs=L.make_sequences(6, 2, 1)), "slots")
    op, seqs = L.make_decay_attention(2, 2, 128, 128, L.DT_BF16), L.make_sequences(65536, 1, 1)
    need = L.ct_decay_attention_workspace(op, seqs)
    if need:
        refused(lambda: run_attention(op, seqs), "workspace")
        refused(lambda: run_attention(op, seqs, OK, need - 1), "workspace")
        refused(lambda: run_attention(op, seqs, OK + 8, need), "16-byte")
    assert L.lib().ct_decay_attention_run(None, None, *[OK] * 9, None, 0, None) == L.CT_E_ARG
    assert L.lib().ct_decay_attention_workspace(ctypes.byref(op), ctypes.byref(seqs), None) == L.CT_E_ARG


@pytest.mark.parametrize("kw,what", [
    (dict(tokens=-1, count=2), "negative"), (dict(tokens=4, count=2, max_len=-1), "negative"),
    (dict(tokens=5, count=2, num_slots=2), "multiple"), (dict(tokens=0x7FFFFFF0, count=1), "too many"),
    (dict(tokens=4, count=2, num_slots=2, offsets=OK + 2), "misaligned")])
def test_attention_checks_its_sequences(kw, what):
    seqs = L.make_sequences(**kw)
    refused(lambda: run_attention(attention(), seqs), what)
    refused(lambda: L.ct_decay_attention_workspace(attention(), seqs), what)


# ------------------------------------------------------------------ all of them
def test_nothing_to_do_needs_no_device():
    L.ct_mx_quantise_run(mx(rows=0), None, None, None)
    L.ct_mx_values_run(L.make_mx(4, 0, L.DT_BF16, L.MX_E4M3), None, None, None)
    run_product(L.make_mx_linear(0, 24, 100, 2, 3, 1), x=None, y=None)
    run_norm(norm(rows=0), x=None, y=None)
    none = L.make_sequences(0, 0)
    run_attention(attention(), none, **{k: None for k in ARRAYS})
    run_attention(L.make_decay_attention(0, 1, 16, 16, 1), **{k: None for k in ARRAYS})
    assert L.ct_mx_linear_workspace(L.make_mx_linear(0, 24, 1 << 20, 2, 3, 1)) == 0
    assert L.ct_decay_attention_workspace(attention(), none) == 0


def test_valid_calls_need_an_initialised_device():
    for call in (*both_ways(mx()), lambda: run_product(product()), lambda: run_norm(norm()), lambda: run_attention(attention())):
        with pytest.raises(L.CtError) as e:
            call()
        assert e.value.code == L.CT_E_NOINIT


def test_addresses_may_be_of_any_kind_of_int():
    class Address(int):
        pass

    assert L._addresses(Address(OK), None) == [OK, None]


def test_pieces_of_bad_offsets_have_places_in_the_workspace():
    """A sequence's pieces are numbered from start / piece + s on. Whatever the offsets hold, the rows stay
    in 0..tokens and the places of a sequence's pieces, the last one's too, below tokens / piece + count."""
    rng = random.Random(3)
    for _ in range(2000):
        count, piece = rng.randint(1, 9), 64 * rng.randint(1, 4)
        tokens = rng.choice((0, 1, piece - 1, piece, rng.randint(1, 3000)))
        offsets = [rng.choice((rng.randint(-100, tokens + 100), rng.randint(0, tokens), -2**31, 2**31 - 1)) for _ in range(count + 1)]
        total = tokens // piece + count
        for s in range(count):
            begin = min(max(offsets[s], 0), tokens)
            end = min(max(offsets[s + 1], begin), tokens)
            unit = begin // piece + s
            pieces = (end - begin + piece - 1) // piece
            assert 0 <= begin <= end <= tokens and unit < total and unit + pieces - 1 < total
