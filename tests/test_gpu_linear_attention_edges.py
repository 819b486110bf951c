"""The linear-attention-block operators where a small error shows: outputs beside the borders of a
rounding, values and scales at the ends of their ranges, every tile of the product and every kernel of
the attention's pieces. References are the formulas in 64 bits."""
import pytest
import torch

from paper_2008_03602_amd import _lib as L
from paper_2008_03602_amd.linear_attention import LinearAttentionBlock
import test_gpu_linear_attention as block
from gpu_util import device_ready, note
from test_gpu_linear_attention import (B, CODE, D, F, FORMATS, INF, NAN, PAIRS, ROUND, U, attention_inputs, check_attention,
                                       check_norm, codes_of, dropped, mx_buffers, quantise64, random_rows, run_plain, values_of)
from test_gpu_sequence import gen, normal, stream, within
from test_host_linear_attention_plans import TILES

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _device():
    device_ready()
    yield


# ------------------------------------------------------------------ norm
@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("dtype", [B, F])
@pytest.mark.parametrize("rows,cols,groups,residual,gate", [
    (1024, 4096, 32, False, True), (512, 4096, 1, True, True), (2048, 1000, 1, True, False), (300, 8192, 2, False, True),
    (60, 16384, 1, False, True), (60, 20000, 1, True, True)])
def test_norm_rounds_as_the_formula_beside_the_borders(rows, cols, groups, residual, gate, dtype, fmt):
    """Elements and scales equal those of the formula in 64 bits (of h, which is fp32), everywhere: both sides are
    within 2^-44, and of 4 million elements one would be that near to a border once in 2^17 runs."""
    note("norm beside borders %dx%d/%d %s format %d" % (rows, cols, groups, dtype, fmt))
    g = gen(rows + cols)
    x, res = normal(g, rows, cols, dtype=dtype), normal(g, rows, cols, std=2.0, dtype=dtype)
    z, w = normal(g, rows, cols, std=4.0, dtype=dtype), normal(g, cols, mean=1.0, std=0.2)
    q, s = mx_buffers(rows, cols, fmt)
    xd = x.cuda()
    L.ct_norm_run(L.make_norm(rows, cols, CODE[dtype], fmt, groups, 1e-5), xd, res.cuda() if residual else None,
                  xd if residual else None, w.cuda(), z.cuda() if gate else None, q, s, stream())
    torch.cuda.synchronize()
    h = (x.float() + res.float() if residual else x.float())
    if residual:
        assert torch.equal(xd.cpu(), h.to(dtype))
    v = h.double().reshape(rows, groups, -1)
    y = (v / torch.sqrt((v * v).mean(2, keepdim=True) + torch.tensor(1e-5).double())).reshape(rows, cols) * w.double()
    if gate:
        y = y * z.double() / (1 + torch.exp(-z.double()))
    code, scale, _ = quantise64(y, fmt)
    assert torch.equal(s.cpu().long(), scale), "%d scales" % int((s.cpu().long() != scale).sum())
    got = codes_of(q.cpu(), cols, fmt)
    assert torch.equal(got, code), "%d elements" % int((got != code).sum())


@pytest.mark.parametrize("out", [B, F, *FORMATS])
@pytest.mark.parametrize("dtype", [B, F])
def test_norm_of_tiny_values_without_eps(dtype, out):
    """Values whose squares are below fp32, and some whose reciprocal root mean square is above it."""
    for std in (1e-21, 1e-25, 1e-36, 1e-38, *((1e-42,) if dtype == F else ())):
        for rows, cols, groups in ((5, 96, 3), (3, 515, 1), (2, 4100, 1), (2, 20000, 1)):
            if groups == 1 or out in (B, F) or cols // groups % 32 == 0:
                check_norm(rows, cols, dtype, out, groups, std=std, eps=0.0, seed=cols)


@pytest.mark.parametrize("dtype", [B, F])
def test_norm_of_huge_values(dtype):
    """Values whose squares are past fp32 and whose norm is not."""
    for std in (1e21, 1e36):
        check_norm(3, 200, dtype, F, std=std, residual=False, seed=2)
        check_norm(3, 200, dtype, L.MX_E4M3, std=std, residual=False, seed=2)


# ------------------------------------------------------------------ product
def far_rows(g, m, n, k, fx, fw):
    """Rows of x and w whose blocks' scales lie anywhere, such that those of a block of both make up for each
    other: products of normal size."""
    xq, xs, _ = random_rows(g, m, k, fx)
    wq, wsc, _ = random_rows(g, n, k, fw)
    blocks = (k + 31) // 32
    ends = torch.tensor([0, 1, 2, 3, 5, 8, 9, 10, 60, 127, 200, 245, 246, 247, 249, 252, 253, 254])
    s = ends[torch.randint(0, len(ends), (blocks,), generator=g)]
    for scales, centre in ((xs, s), (wsc, 254 - s)):
        near = centre + torch.randint(-2, 3, (scales.shape[0], blocks), generator=g)
        scales[:, :blocks] = near.clamp(0, 254).to(torch.uint8).cuda()
    return xq, xs, values_of(xq.cpu(), xs.cpu(), k, fx), wq, wsc, values_of(wq.cpu(), wsc.cpu(), k, fw)


def check_far(m, n, k, fx, fw, out, nan=True):
    note("mx product of far scales m%d n%d k%d formats %d %d -> %s" % (m, n, k, fx, fw, out))
    xq, xs, x, wq, wsc, w = far_rows(gen(m + n + k), m, n, k, fx, fw)
    want, mag = x @ w.t(), x.abs() @ w.abs().t()
    assert 1e-3 < float(mag.median()) < 1e12
    if nan:  # a block without an element that is not 0 is NaN all the same
        row = L.mx_row_bytes(32, fx)
        xq[m // 2, :row] = 0
        xs[m // 2, 0] = 255
        wsc[n // 3, (k + 31) // 32 - 1] = 255
        want[m // 2], want[:, n // 3] = NAN, NAN
    op = L.make_mx_linear(m, n, k, fx, fw, CODE[out])
    ws = torch.full((max(16, L.ct_mx_linear_workspace(op)),), 255, dtype=torch.uint8, device="cuda")
    y = torch.full((m, n), NAN, dtype=out, device="cuda")
    L.ct_mx_linear_run(op, xq, xs, wq, wsc, None, None, y, ws, stream())
    torch.cuda.synchronize()
    # exact products, k sums in fp32; what the matrix cores drop for bf16
    bound = (k + 4) * U * mag + (dropped(x, w) if out == B else 0.0)
    within(y, want, bound + ROUND[out] * (want.abs() + bound), "far scales m%d n%d k%d %d %d %s" % (m, n, k, fx, fw, out))


@pytest.mark.parametrize("out", [B, F])
@pytest.mark.parametrize("fx,fw", PAIRS)
@pytest.mark.parametrize("m,n,k", [(1, 16, 32), (5, 33, 129), (20, 40, 96), (33, 48, 1000), (130, 70, 515), (200, 260, 4000),
                                   (20, 24, 9000)])
def test_product_of_scales_that_make_up_for_each_other(m, n, k, fx, fw, out):
    check_far(m, n, k, fx, fw, out)


@pytest.mark.parametrize("fx,fw", PAIRS)
def test_product_of_blocks_of_zeros_with_any_scale(fx, fw):
    """Scales of blocks that are all 0 change nothing, to the bit."""
    g = gen(8)
    xq, xs, x = random_rows(g, 70, 256, fx)
    wq, wsc, w = random_rows(g, 66, 256, fw)
    row = L.mx_row_bytes(32, fx)
    xq[:, 2 * row:3 * row], xq[5] = 0, 0
    y, z = (torch.empty(70, 66, device="cuda") for _ in range(2))
    op = L.make_mx_linear(70, 66, 256, fx, fw, L.DT_F32)
    for scale, to in ((127, y), (0, z), (254, z)):
        xs[:, 2], xs[5] = scale, scale
        L.ct_mx_linear_run(op, xq, xs, wq, wsc, None, None, to, None, stream())
        torch.cuda.synchronize()
        assert to is y or torch.equal(y, z)
    assert (y[5] == 0).all()


@pytest.mark.parametrize("fx,fw", PAIRS)
@pytest.mark.parametrize("m,n,k", [(20, 24, 600), (70, 66, 1000), (40, 70, 9000), (2000, 2010, 200), (2900, 2200, 168)])
def test_product_of_far_scales_leaves_the_bits_of_other_rows(m, n, k, fx, fw):
    g = gen(m + k)
    xq, xs, _ = random_rows(g, m, k, fx)
    wq, wsc, _ = random_rows(g, n, k, fw)
    op = L.make_mx_linear(m, n, k, fx, fw, L.DT_F32)
    ws = torch.full((max(16, L.ct_mx_linear_workspace(op)),), 255, dtype=torch.uint8, device="cuda")
    ys = []
    for far in (False, True):
        if far:
            xs[m // 2, 0], xs[1, 3], xs[3, (k + 31) // 32 - 1], xs[5, 1], wsc[n // 2, 2] = 1, 255, 254, 0, 250
        y = torch.empty(m, n, device="cuda")
        L.ct_mx_linear_run(op, xq, xs, wq, wsc, None, None, y, ws, stream())
        torch.cuda.synchronize()
        ys.append(y.cpu())
    same = torch.ones(m, n, dtype=torch.bool)
    same[[m // 2, 1, 3, 5]], same[:, n // 2] = False, False
    assert torch.equal(ys[0][same], ys[1][same])
    assert torch.isnan(ys[1][1]).all() and torch.isfinite(ys[1][same]).all()


def dropped_there(x, w):
    """What `dropped` gives, worked out on the device: large products take the CPU minutes."""
    m, k = x.shape
    xa, wa = (torch.nn.functional.pad(t.abs(), (0, -k % 8)).reshape(t.shape[0], -1, 8).cuda() for t in (x, w))
    out = torch.empty(m, w.shape[0], dtype=D, device="cuda")
    for i in range(m):
        out[i] = (xa[i][None] * wa).amax(2).sum(1)
    return 7 * 2.0 ** -13 * out.cpu()


@pytest.mark.parametrize("fx,fw", PAIRS)
@pytest.mark.parametrize("m,n,k,out", [t[:4] for t in TILES])
def test_product_on_every_tile(m, n, k, out, fx, fw, monkeypatch):
    """Every kernel, whole and ragged tiles, the reduction in one and in slices, rows and columns apart; which
    sizes reach which is checked where they are listed."""
    monkeypatch.setattr(block, "dropped", dropped_there)
    yp = n + (5 if m < 3000 else 0)
    block.check_product(m, n, k, fx, fw, B if out == "bf16" else F, act=(m + k) % 5, res=1 + n % 2, seed=m + n, yp=yp,
                        sp=L.mx_scale_bytes(k) + 4, in_place=m % 2 == 1)


@pytest.mark.parametrize("fx,fw", PAIRS)
@pytest.mark.parametrize("m,n,k", [t[:3] for t in TILES if t[3] == "f32"])
def test_product_of_far_scales_on_every_exact_tile(m, n, k, fx, fw):
    check_far(m, n, k, fx, fw, F)


# ------------------------------------------------------------------ attention
@pytest.mark.parametrize("dtype", [B, F])
@pytest.mark.parametrize("key,value", [(64, 64), (64, 128), (128, 64), (128, 128), (256, 64), (256, 128), (250, 130), (256, 256)])
def test_attention_in_pieces_of_every_shape(key, value, dtype):
    """Each kernel of the pieces' ends, rows on 16 bytes and off them, the state written where it is read."""
    for pad in (0, 3):
        assert check_attention([600], 2, 1, key, value, dtype, in_place=True, pad=pad, seed=key + value) > 0
    assert check_attention([330, 0, 5, 260], 2, 2, key, value, dtype, in_place=True, step_input=True, seed=key, lead=2) > 0


@pytest.mark.parametrize("dtype", [B, F])
@pytest.mark.parametrize("name,bad", [("v", NAN), ("v", INF), ("k", NAN), ("k", -INF), ("q", NAN), ("delta", NAN), ("state", NAN),
                                      ("state", INF)])
def test_attention_in_pieces_keeps_infinities_and_nan_behind_their_token(name, bad, dtype):
    """What a token's value reaches crosses the pieces behind it and nothing else: a sequence of nine pieces, the
    value at the first and last row of one, inside one, at the sequence's ends, or in its state."""
    heads, key, value, lens = 3, 32, 40, [40, 520, 90]
    op = L.make_decay_attention(heads, heads, key, value, CODE[dtype], L.DT_F32)
    seqs = L.make_sequences(sum(lens), 3, 3, 520, torch.zeros(4, dtype=torch.int32, device="cuda"))
    assert L.ct_decay_attention_workspace(op, seqs) // (heads * (key * 2 * value * 4 + 4)) >= 9
    s = attention_inputs(gen(4), sum(lens), heads, heads, key, value, 3, dtype, F)
    clean, cs = run_plain(s, lens, heads, heads, key, value, dtype, s["state"])
    for t in (40, 40 + 192, 40 + 255, 40 + 300, 559) if name != "state" else (40,):
        note("attention in pieces: %s %s at token %d %s" % (name, bad, t, dtype))
        d = {k: v.clone() if v is not None else None for k, v in s.items()}
        reached = torch.zeros(sum(lens), heads, value, dtype=torch.bool)
        rstate = torch.zeros(3, heads, key, value, dtype=torch.bool)
        if name == "state":
            d["state"][1, 1, 5, 7] = bad
            reached[t:560, 1, 7] = rstate[1, 1, 5, 7] = True
        else:
            d[name][t, {"v": value + 7, "delta": 1}.get(name, key + 5)] = bad  # of the second head
            if name == "q":
                reached[t, 1] = True
            elif name == "v":
                reached[t:560, 1, 7] = rstate[1, 1, :, 7] = True
            else:
                reached[t:560, 1] = True
                rstate[1, 1, 5 if name == "k" else slice(None)] = True
        got, gs = run_plain(d, lens, heads, heads, key, value, dtype, d["state"])
        flat = reached.reshape(sum(lens), -1)
        assert torch.equal(got[~flat], clean[~flat]) and torch.equal(gs[~rstate], cs[~rstate]), (name, bad, t)
        assert not torch.isfinite(got[flat]).any() and not torch.isfinite(gs[rstate]).any(), (name, bad, t)


@pytest.mark.parametrize("dtype", [B, F])
def test_attention_in_pieces_forgets_behind_an_infinite_rate(dtype):
    """A decay of 0 inside a piece, at its first row and its last: what was before leaves nothing."""
    heads, key, value, lens = 2, 32, 32, [600]
    s = attention_inputs(gen(6), 600, heads, heads, key, value, 1, dtype, F)
    for rows in ([100], [128], [191], [0, 64, 599]):
        d = dict(s, delta=s["delta"].clone())
        d["delta"][rows, 1] = INF
        o, st = run_plain(d, lens, heads, heads, key, value, dtype, s["state"])
        ref, bound, new, nbound = block.attention64({**d, "delta": d["delta"].clamp(max=1e4)}, torch.tensor([0, 600]), torch.tensor([0]),
                                                    1.0, False, True, dtype)
        within(o, ref, bound, "forgetting at %s" % rows)
        within(st, new, nbound, "forgetting at %s: state" % rows)


# ------------------------------------------------------------------ the block
def test_rows_of_nobody_may_hold_anything():
    """Infinities and NaN in rows of no sequence leave every other row, of a sequence or not, and the states as
    they are without them; the rows themselves come out NaN."""
    net = LinearAttentionBlock(256, 4, 2, 32, 64, slots=4, max_rows=300)
    off = torch.tensor([5, 75, 75, 200, 233], dtype=torch.int32, device="cuda")
    plan = net.plan(net.sequences(240, 4, 125, off))
    x = normal(gen(3), 240, 256, dtype=B)
    wild = x.clone()
    wild[2, 7], wild[234, 0], wild[236] = INF, -INF, NAN
    note("a block with infinities and NaN in rows of nobody")
    outs = []
    for t in (x, wild, x):
        net.reset()
        y = torch.empty(240, 256, dtype=B, device="cuda")
        net.run(plan, t.cuda(), y)
        outs.append((y.cpu(), net.state.cpu()))
    others = torch.ones(240, dtype=torch.bool)
    others[[2, 234, 236]] = False
    assert torch.equal(outs[0][0], outs[2][0]) and torch.equal(outs[0][1], outs[2][1])
    assert torch.equal(outs[1][0][others], outs[0][0][others]) and torch.equal(outs[1][1], outs[0][1])
    assert torch.isnan(outs[1][0][~others]).all()
    inside = torch.zeros(240, dtype=torch.bool)
    inside[5:233] = True
    assert torch.equal(outs[0][0][~inside], x[~inside]) and torch.isfinite(outs[0][0].float()).all()
