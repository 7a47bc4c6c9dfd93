"""Arguments that the layer norm's entry points refuse on the host (no GPU is needed)."""
import pytest

from paper_2505_03254_b200 import binding, build

A = 0x1000          # an aligned non-null address; never dereferenced by these calls
F32, BF16, F16 = 0, 1, 2


@pytest.fixture(scope="module")
def lib():
    build.build()
    return binding.lib()


def test_forward(lib):
    def f(x=A, t=F32, m=4, n=64, xp=64, w=A, b=A, pt=F32, eps=1e-5, y=A, yp=64, mean=A, rstd=A):
        return lib.prom_layer_norm(x, t, m, n, xp, w, b, pt, eps, y, yp, mean, rstd, None)
    assert f(m=0) == f(m=0, x=None, y=None) == binding.PROM_OK
    assert f(t=3) == f(t=-1) == f(pt=7) == binding.PROM_ERR_RANGE
    assert f(eps=-1.0) == f(eps=float("nan")) == f(eps=float("inf")) == binding.PROM_ERR_RANGE
    assert f(m=-1) == f(m=1 << 31) == f(n=0) == f(n=65537, xp=1 << 20, yp=1 << 20) == binding.PROM_ERR_SHAPE
    assert f(xp=63) == f(yp=63) == f(xp=-64) == binding.PROM_ERR_SHAPE
    assert f(x=None) == f(y=None) == binding.PROM_ERR_NULL
    assert f(x=A + 2) == f(y=A + 1) == f(w=A + 2) == f(b=A + 1) == f(mean=A + 2) == f(rstd=A + 1) == binding.PROM_ERR_ALIGN
    assert f(t=BF16, x=A + 1) == f(t=F16, pt=F16, w=A + 1) == binding.PROM_ERR_ALIGN
    assert f(x=A, y=A, xp=64, yp=72) == binding.PROM_ERR_SHAPE          # in place takes one pitch


def test_codes(lib):
    def f(x=A, t=F32, m=4, n=64, xp=64, w=A, b=A, pt=F32, eps=1e-5, q=A, gamma=A, scale=A, mean=None, rstd=None):
        return lib.prom_layer_norm_i8(x, t, m, n, xp, w, b, pt, eps, q, gamma, scale, mean, rstd, None)
    assert f(m=0) == f(m=0, x=None, q=None, gamma=None, scale=None) == binding.PROM_OK
    assert f(q=None) == f(gamma=None) == f(scale=None) == f(x=None) == binding.PROM_ERR_NULL
    assert f(gamma=A + 1) == f(scale=A + 2) == f(mean=A + 2) == binding.PROM_ERR_ALIGN
    assert f(t=9) == f(eps=-0.5) == binding.PROM_ERR_RANGE
    assert f(n=0) == f(xp=1) == binding.PROM_ERR_SHAPE


def test_backward(lib):
    def f(dy=A, x=2 * A, t=F32, m=4, n=64, dyp=64, xp=64, w=A, pt=F32, mean=A, rstd=A, dx=3 * A, dxp=64, dw=A, db=A, ws=A, wb=1 << 30):
        return lib.prom_layer_norm_backward(dy, x, t, m, n, dyp, xp, w, pt, mean, rstd, dx, dxp, dw, db, ws, wb, None)
    assert f(dx=None, dw=None, db=None) == f(m=0, dw=None, db=None) == binding.PROM_OK          # nothing is wanted
    assert f(t=3) == f(pt=-1) == binding.PROM_ERR_RANGE
    assert f(m=-1) == f(n=0) == f(n=65537, dyp=1 << 20, xp=1 << 20, dxp=1 << 20) == binding.PROM_ERR_SHAPE
    assert f(dyp=63) == f(xp=63) == f(dxp=63) == binding.PROM_ERR_SHAPE
    assert f(dx=A, dxp=72) == f(dx=2 * A, dxp=72) == binding.PROM_ERR_SHAPE
    assert f(dy=None) == f(x=None) == f(mean=None) == f(rstd=None) == f(ws=None) == binding.PROM_ERR_NULL
    assert f(dy=A + 2) == f(dx=A + 1) == f(dw=A + 2) == f(db=A + 1) == f(mean=A + 2) == f(ws=A + 8) == binding.PROM_ERR_ALIGN
    assert binding.layer_norm_backward_workspace_bytes(0, 64) == binding.layer_norm_backward_workspace_bytes(4, 0) == 0
