"""The linear-attention-block operators where a small error shows: outputs beside the borders of a
rounding, values and scales at the ends of their ranges, every tile of the product and every kernel of
the attention's pieces. References are the formulas in 64 bits."""
import pytest
import torch

from paper_2008_03602_amd import _lib as L
from gpu_util import device_ready, note
from test_gpu_linear_attention import B, CODE, D, F, FORMATS, check_norm, codes_of, mx_buffers, quantise64
from test_gpu_sequence import gen, normal, stream

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
