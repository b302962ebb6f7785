"""Layer norm of rows that lie far from zero beside their deviation."""
import pytest
import torch

from tests.clear_util import gen, norm_ref, randn

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("value", [3.0, 100.0, 1000.0, 1e4, 1234.567, -0.1])
@pytest.mark.parametrize("cols", [5, 109, 119, 120, 200, 333, 1000, 1023, 3001, 9999, 16400, 20011])
def test_constant_rows_have_no_deviation(cols, value):
    """All entries equal: y is the bias, the mean that value and rstd 1/sqrt(eps), whatever 1/cols rounds to.  The first mean is off
    by 2^-18 of the value at most (64 roundings); of that, 2^-18 is left once the mean of the differences is taken off, and 2^-17 of
    its square in the variance."""
    from paper_2604_09975_amd import clear as K
    g = gen(cols)
    x = torch.full((3, cols), value, device="cuda")
    w, b = 1 + 0.2 * randn(g, cols), 0.2 * randn(g, cols)
    y, mean, rstd = K.ckks_clear_layer_norm(x, w, b, 1e-5)
    first = 2.0**-18 * abs(float(x[0, 0]))
    off = 2.0**-18 * first * 1e-5**-0.5
    assert torch.equal(mean, x[:, 0].contiguous())
    assert ((rstd.double() * 1e-5**0.5 - 1).abs() <= 2.0**-20 + 2.0**-17 * first * first / 1e-5).all()
    assert ((y.double() - b.double()).abs() <= off * w.double().abs() + 2.0**-23 * b.double().abs() + 1e-30).all()
    dy = randn(g, 3, cols)
    dx, dw, _ = K.ckks_clear_layer_norm_grad(dy, x, mean, rstd, w)
    assert not dw.any()
    gw = dy.double() * w.double()
    want = 1e-5**-0.5 * (gw - gw.mean(1, keepdim=True))
    assert ((dx.double() - want).abs() <= 2.0**-18 * 1e-5**-0.5 * (gw.abs() + gw.abs().mean(1, keepdim=True))).all()


@pytest.mark.parametrize("cols", [7, 119, 700, 3001, 9999, 16400])
def test_offsets_large_beside_the_deviation(cols):
    """x = 4096 + d with d in steps of 2^-11: exact in 32 bits, deviation about 1.  What the mean loses to the sum's size must not
    show: differences and squares are sums of small terms, 2^-18 is 64 of their roundings; the differences from the first mean,
    which is off by up to 2^-18 * 4096 = 2^-6, are whole multiples of its last place up to one rounding, 2^-24 * 8, each."""
    from paper_2604_09975_amd import clear as K
    g = gen(cols)
    d = (randn(g, 40, cols) * 2048).round() / 2048
    x = 4096 + d
    assert torch.equal(x - 4096, d)
    w, b = 1 + 0.2 * randn(g, cols), 0.2 * randn(g, cols)
    y, mean, rstd = K.ckks_clear_layer_norm(x, w, b, 1e-5)
    want, m64, r64, xh = norm_ref(x, w, b, 1e-5)
    assert ((mean.double() - m64[:, 0]).abs() <= 2.0**-12 + 2.0**-17).all()       # half a last place of 4096, and the sums
    assert ((rstd.double() - r64[:, 0]).abs() <= 2.0**-17 * r64[:, 0]).all()
    wd = w.double().abs()
    assert ((y.double() - want).abs() <= 2.0**-17 * wd * (1 + xh.abs()) * (1 + r64) + 2.0**-22 * (want.abs() + b.double().abs())).all()
