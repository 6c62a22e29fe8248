"""The mean of a row, where its last bit counts: rows without variance, and rows whose offset is far above their spread."""
import pytest
import torch

from _rows import N_ROW, U32, within

pytestmark = pytest.mark.gpu
DTS = [torch.float32, torch.float16, torch.bfloat16]
WIDTHS = [3, 7, 13, 14, 15, 26, 30, 41, 45, 60, 120, 256, 450, 513, 1000, 1025, 2050, 4095]


def _affine(c):
    g = torch.Generator(device="cuda").manual_seed(c)
    return 1 + 0.3 * torch.randn(c, generator=g, device="cuda"), 0.3 * torch.randn(c, generator=g, device="cuda")


@pytest.mark.parametrize("dtype", DTS)
@pytest.mark.parametrize("c", WIDTHS)
@pytest.mark.parametrize("eps", [0.0, 1e-5])
def test_rows_without_variance(dtype, c, eps):
    """x - mean is 0 for every element, so y is the bias and the statistics are the value and 1 / sqrt(eps) (2^-126 for no eps)."""
    import paper_2311_12862_amd as sp
    values = [2.5, -2.5, 1000.0, 60000.0, 8192.0, 0.1, -1 / 3, 1e-3, 123.456]
    if dtype != torch.float16:
        values += [1e30, -1e-12, 1.0000001e10, 3e-30]
    x = torch.tensor(values, dtype=torch.float64, device="cuda").to(dtype)[:, None].expand(-1, c).contiguous()
    w, b = _affine(c)
    y, stats = sp.layer_norm_fwd(x, w, b, eps)
    assert torch.equal(y, b.to(dtype).expand_as(y))
    assert torch.equal(stats[:, 0], x[:, 0].float())
    r = max(eps, 2.0 ** -126) ** -0.5
    assert (stats[:, 1].double() / r - 1).abs().max().item() <= 4 * U32
    _, dw, _, _ = sp.layer_norm_bwd(torch.ones_like(x), x, stats, w)
    assert (dw == 0).all()                      # (x - mean is 0 there as well)


@pytest.mark.parametrize("dtype", DTS)
@pytest.mark.parametrize("c", WIDTHS)
def test_offset_far_above_the_spread(dtype, c):
    """The error of a first mean m0 is taken out by the mean of the differences.  With a the error of a sum of a row, s = mean |x - m|
    and e0 = a mean |x| that of m0: x - m0 rounds by 2^-24 of itself, the mean of these is off by a (s + e0), and so is the corrected
    mean; mean (x - m0)^2 - (m - m0)^2 by a (var + 2 e0^2)."""
    import paper_2311_12862_amd as sp
    g = torch.Generator(device="cuda").manual_seed(c)
    x = torch.randn(64, c, generator=g, device="cuda")
    x = torch.cat([100 + x, -1000 + 4 * x, 3000 + 0.5 * x, 60000 + 64 * x, 10 + 0.01 * x]).to(dtype)
    w, b = _affine(c)
    eps = 1e-5
    y, stats = sp.layer_norm_fwd(x, w, b, eps)
    v, w, b = x.double(), w.double(), b.double()
    m = v.mean(1, keepdim=True)
    dev = v - m
    var = dev.square().mean(1, keepdim=True)
    r = (var + eps) ** -0.5
    want = dev * r * w + b
    a = N_ROW * U32
    s, e0 = dev.abs().mean(1, keepdim=True), a * v.abs().mean(1, keepdim=True)
    dm = a * (s + e0)
    dr = r * (a * (var + 2 * e0.square()) * r.square() + 4 * U32)
    tol = w.abs() * (dev.abs() * dr + r * (dm + 4 * U32 * (dev.abs() + e0))) + 4 * U32 * ((dev * r * w).abs() + b.abs())
    within(y, want, tol, dtype)
    within(stats, torch.cat([m, r], 1), torch.cat([dm + 2 * U32 * m.abs(), dr], 1))


def test_rows_that_are_not_finite():
    import paper_2311_12862_amd as sp
    for dtype in DTS:
        for c in (15, 64, 1000):
            x = torch.full((6, c), 2.5, dtype=dtype, device="cuda")
            x[1, 2], x[2, 3], x[3, 4] = float("inf"), float("-inf"), float("nan")
            x[4, 5], x[4, 6] = float("inf"), float("-inf")
            y, stats = sp.layer_norm_fwd(x)
            assert (y[0] == 0).all() and (y[5] == 0).all() and torch.isnan(y[1:5]).all()
            assert stats[1, 0] == float("inf") and stats[2, 0] == float("-inf") and torch.isnan(stats[3:5, 0]).all()
            assert torch.isnan(stats[1:5, 1]).all()


def test_squares_that_overflow():
    """Differences beyond 2^64: 1 / std counts as 0."""
    import paper_2311_12862_amd as sp
    for c in (15, 64, 1000):
        x = torch.full((3, c), 1e20, device="cuda")
        x[1, ::2] = -1e20
        w, b = _affine(c)
        y, stats = sp.layer_norm_fwd(x, w, b)
        assert torch.equal(y, b.expand_as(y)) and stats[1, 1] == 0 and torch.equal(stats[0, 0], x[0, 0])
