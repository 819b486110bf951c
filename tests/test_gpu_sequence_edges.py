"""The sequence-block operators where values are infinite or zero and sizes take each kernel, against
their formulas in 64 bits."""
import pytest
import torch

from paper_2008_03602_amd import _lib as L
from gpu_util import device_ready, note
from test_gpu_sequence import B, CODE, F, check_conv, check_scan, layout, scan64, scan_inputs, stream, within

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _device():
    device_ready()
    yield


def scan(s, off, slots, dtype, uniform, softplus=True):
    """y and the new states of scan_inputs `s`."""
    channels, states, tokens = s["u"].shape[1], s["a"].shape[1], s["u"].shape[0]
    op = L.make_scan(channels, states, s["groups"], CODE[dtype], softplus)
    seqs = L.make_sequences(tokens, len(slots), s["state"].shape[0], 0, None if uniform else off.cuda(), slots.cuda())
    c = {k: v.cuda() if torch.is_tensor(v) else v for k, v in s.items()}
    y, out = torch.empty_like(c["u"]), c["state"].clone()
    ws = torch.full((max(1, L.ct_scan_workspace(op, seqs)),), 255, dtype=torch.uint8, device="cuda")
    L.ct_scan_run(op, seqs, c["u"], c["delta"], c["dt_bias"], c["a"], c["b"], c["c"], c["d"], c["z"], c["state"], out, y,
                  ws, stream())
    torch.cuda.synchronize()
    return y, out


def same_kinds(got, ref, bound, what):
    """NaN, infinities (with their signs) and finite values in the same places, and these within their bound."""
    got = got.detach().cpu().double()
    assert torch.equal(torch.isnan(got), torch.isnan(ref)), what + ": NaN in other places"
    inf = torch.isinf(ref)
    assert torch.equal(torch.isinf(got), inf), what + ": infinities in other places"
    assert torch.equal(got[inf], ref[inf]), what + ": signs of infinities"
    fine = torch.isfinite(ref)
    worst = ((got - ref).abs()[fine] / (bound[fine] + 1e-38)).max().item()
    assert worst <= 1.0, "%s: error %.2f times the bound" % (what, worst)


SPARE = [1, 3, 4, 5, 7, 8, 9, 13, 16, 17, 24, 33, 40, 64, 100, 132, 200]


@pytest.mark.parametrize("dtype", [B, F])
@pytest.mark.parametrize("states,lens,channels", [
    (n, lens, 70) for n in SPARE for lens in ([1] * 5, [12, 0, 5], [190, 0, 70])] + [
    (n, [40] * 30, 1100) for n in SPARE if n <= 40])  # enough for lanes of eight and 16 states
def test_scan_infinities_are_the_same_of_any_number_of_states(states, lens, channels, dtype):
    """An infinite input, step, state and coefficient: what the formula makes of them, whether or not a
    lane has states to spare. b, c, d and the inputs are positive, so that no infinities cancel."""
    uniform = len(set(lens)) == 1
    off, slots, n, tokens = layout(lens, seed=states)
    s = scan_inputs(tokens, channels, states, 1, dtype, n, states)
    for k in ("u", "b", "c", "d", "z"):
        s[k] = s[k].abs() + 0.1
    s["a"], s["state"] = -0.05 - 0.1 * torch.rand(s["a"].shape), s["state"].abs()
    inf = float("inf")
    s["u"][1, 3], s["delta"][0, 11], s["u"][tokens - 1, 5] = inf, inf, inf
    s["state"][int(slots[0]), 17, states - 1] = inf
    s["z"][2, 23] = inf
    note("scan of infinities: %s ch%d n%d %s" % (lens, channels, states, dtype))
    y, out = scan(s, off, slots, dtype, uniform)
    y64, new, ybound, nbound = scan64(s, off, slots, True, dtype)
    assert torch.isinf(y64).sum() >= 3 and torch.isfinite(y64).any()
    same_kinds(out, new, nbound, "state")
    same_kinds(y, y64, ybound, "y")


@pytest.mark.parametrize("states,channels", [(16, 66), (13, 66), (40, 66), (16, 4100)])
@pytest.mark.parametrize("lens", [[50, 190], [50, 350], [400]])  # 240 rows are a few chunks
def test_scan_of_cut_sequences_neither_over_nor_underflows_on_its_own(lens, states, channels):
    """Decays of a whole chunk leave fp32 where those of its tokens and the states do not."""
    off, slots, n, tokens = layout(lens, seed=1)
    inf, ln2 = float("inf"), 0.6931471805599453
    s = scan_inputs(tokens, channels, states, 1, F, n, 7)
    for k in ("b", "c", "d", "z"):
        s[k] = s[k].abs() + 0.1
    s["dt_bias"].zero_()
    s["a"] = -0.01 - 0.02 * torch.rand(channels, states)
    s["delta"] = 0.1 * torch.rand(tokens, channels)
    # channel 1: the states grow by 4.1 bits a token, but there is nothing to grow until the last eight
    s["a"][1], s["delta"][:, 1] = 4.1 * ln2, 1.0
    s["u"][:, 1] = 0.0
    for e in off[1:].tolist():
        s["u"][e - 8:e, 1] = 0.5
    s["state"][:, 1] = 0.0
    # channel 2: infinite states that are forgotten by 6 bits a token
    s["a"][2], s["delta"][:, 2] = -6.0 * ln2, 1.0
    s["state"][:, 2] = inf
    # channel 3: states of 2^-120 that grow by 4.1 bits a token, 45 tokens long
    s["a"][3], s["delta"][:, 3], s["u"][:, 3] = 4.1 * ln2, 0.0, 0.0
    for b in off[:-1].tolist():
        s["delta"][b:b + 45, 3] = 1.0
    s["state"][:, 3] = 2.0 ** -120
    note("scan over chunks: %s ch%d n%d" % (lens, channels, states))
    y, out = scan(s, off, slots, F, False, softplus=False)
    few = torch.cat([torch.arange(40), torch.arange(channels - 20, channels)])  # the reference's channels
    part = {k: v[..., few] if k in ("u", "delta", "z") else v[few] if k in ("dt_bias", "a", "d") else
            v[:, few] if k == "state" else v for k, v in s.items()}
    y64, new, ybound, nbound = scan64(part, off, slots, False, F)
    used = slots.long()
    assert torch.isinf(new[used][:, 2]).all() and torch.isfinite(new[used][:, [1, 3]]).all()
    same_kinds(out[:, few], new, nbound, "state")
    same_kinds(y[:, few], y64, ybound, "y")


# ------------------------------------------------------------------ sizes that take each kernel
@pytest.mark.parametrize("dtype", [B, F])
@pytest.mark.parametrize("states,groups,channels", [(16, 1, 2050), (13, 2, 2052), (32, 2, 1030), (20, 1, 1030), (64, 1, 516),
                                                    (40, 2, 516), (100, 1, 260), (128, 2, 520), (200, 1, 520), (256, 2, 260)])
def test_scan_of_single_tokens_two_sequences_a_wave(states, groups, channels, dtype):
    """As many waves as that takes (16 for each SIMD), and an odd number of sequences."""
    lanes = 4 if states <= 16 else 8 if states <= 32 else 16
    count = 16 * 1024 * 64 // (lanes * channels) + 1
    count += 1 - count % 2
    check_scan([1] * count, channels, states, groups, dtype, uniform=True, seed=states, unused=(0, 3))


@pytest.mark.parametrize("dtype", [B, F])
@pytest.mark.parametrize("states", [4, 8, 12, 20, 24, 28, 36, 60, 68, 132, 252])
def test_scan_of_single_tokens_with_lanes_to_spare(states, dtype):
    """States of whole quads that leave whole lanes without any."""
    check_scan([1] * 3, 36, states, 2, dtype, uniform=True, seed=states)


@pytest.mark.parametrize("dtype", [B, F])
@pytest.mark.parametrize("width", range(2, 9))
def test_conv_of_an_odd_number_of_channels(width, dtype):
    """An element a lane, every width."""
    check_conv([0, 1, width - 1, width, 16, 17, 33], 41, width, dtype, seed=width)
    check_conv([1] * 5, 41, width, dtype, uniform=True, seed=width + 1, unused=(2,))
    check_conv([21] * 3, 41, width, dtype, uniform=True, in_place=True, seed=width + 2)


@pytest.mark.parametrize("dtype", [B, F])
@pytest.mark.parametrize("lens,channels,states,chunk", [([9001, 0, 4530], 2050, 16, 64), ([13600], 2048, 13, 64),
                                                        ([5000, 1, 3333], 6000, 16, 96), ([4000, 3000], 2049, 40, 96)])
def test_scan_chunks_of_several_stages(lens, channels, states, chunk, dtype):
    """Chunks that are longer than what is staged at a time, the last of them ragged."""
    uniform = len(set(lens)) == 1 and len(lens) > 1
    off, slots, n, tokens = layout(lens, seed=3)
    s = scan_inputs(tokens, channels, states, 1, dtype, n, 9)
    chunks = sum(-(-l // chunk) for l in lens) if uniform else tokens // chunk + len(lens)
    op = L.make_scan(channels, states, 1, CODE[dtype])
    seqs = L.make_sequences(tokens, len(lens), n, 0, None if uniform else off.cuda())
    assert L.ct_scan_workspace(op, seqs) == chunks * channels * (states + 1) * 4
    note("scan of long chunks: %s ch%d n%d %s" % (lens, channels, states, dtype))
    y, out = scan(s, off, slots, dtype, uniform)
    few = torch.tensor([0, 1, 63, 64, 257, channels // 2, channels - 2, channels - 1])  # the reference's channels
    part = {k: v[..., few] if k in ("u", "delta", "z") else v[few] if k in ("dt_bias", "a", "d") else
            v[:, few] if k == "state" else v for k, v in s.items()}
    y64, new, ybound, nbound = scan64(part, off, slots, True, dtype)
    within(out[:, few], new, nbound, "state")
    within(y[:, few], y64, ybound, "y")


def test_errors_that_other_calls_left_are_not_the_operators():
    """An earlier HIP error that nobody took makes no later call fail."""
    hip = L.lib()  # its own runtime, through which the symbols are found
    x, w = torch.ones(4, 8, device="cuda"), torch.ones(16, 8, device="cuda")
    y, conv, out = torch.zeros(4, 16, device="cuda"), torch.zeros(4, 8, device="cuda"), torch.zeros(4, 8, device="cuda")
    seqs = L.make_sequences(4, 1, 1)
    one, taps, a = torch.ones(8, device="cuda"), torch.ones(8, 2, device="cuda"), -torch.ones(8, 4, device="cuda")
    op = L.make_scan(8, 4, 2, L.DT_F32)
    ws = torch.empty(max(1, L.ct_scan_workspace(op, seqs)), dtype=torch.uint8, device="cuda")
    torch.cuda.synchronize()
    st = stream()
    try:
        for call in (lambda: L.ct_linear_run(L.make_linear(4, 16, 8, L.DT_F32, L.DT_F32), x, w, None, None, y, None, st),
                     lambda: L.ct_causal_conv_run(L.make_causal_conv(8, 2, L.DT_F32), seqs, x, taps, None, None, None, conv, st),
                     lambda: L.ct_scan_run(op, seqs, x, x, one, a, x, x, None, None, None, None, out, ws, st)):
            assert hip.hipSetDevice(1 << 20) != 0  # refused on the host
            call()
    finally:
        hip.hipGetLastError()
    assert (y == 8).all() and (conv[1:] == 2).all() and torch.isfinite(out).all() and (out > 0).all()
