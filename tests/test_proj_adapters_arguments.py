"""Arguments that the projection with adapters refuses on the host (no GPU is needed)."""
import ctypes as C

import pytest

from paper_2505_03254_b200 import binding, build

A = 0x1000          # an aligned non-null address; never dereferenced by these calls


@pytest.fixture(scope="module")
def lib():
    build.build()
    return binding.lib()


def test_refusals(lib):
    def f(x=A, batch=4, rows=1, cin=64, w=A, cout=32, alpha=A, gamma=A, ad=(A, A, A, 1, 2, 8), which=A, y=2 * A, yt=1, yp=32, ws=A, wb=1 << 30):
        table = C.byref(binding.PromAdapters(*ad)) if ad else None
        return lib.prom_pw_proj_adapters(x, batch, rows, cin, w, cout, alpha, gamma, table, which, y, yt, yp, ws, wb, None)
    assert f(batch=0) == f(batch=0, x=None, y=None, ad=None) == binding.PROM_OK
    assert f(batch=-1) == f(rows=0) == f(cin=0) == f(cout=0) == f(cin=4112) == f(cout=4104, yp=4104) == binding.PROM_ERR_SHAPE
    assert f(rows=1 << 31) == f(batch=1 << 16, rows=1 << 16) == f(yp=31) == binding.PROM_ERR_SHAPE
    assert f(ad=(A, A, A, 1, -1, 8)) == f(ad=(A, A, A, 1, 2, 0)) == f(ad=(A, A, A, 1, 2, 257)) == binding.PROM_ERR_SHAPE
    assert f(yt=3) == f(yt=-1) == f(ad=(A, A, A, 0, 2, 8)) == f(ad=(A, A, A, 3, 2, 8)) == binding.PROM_ERR_RANGE
    assert f(cin=24) == f(cin=8) == f(cout=12) == binding.PROM_ERR_UNSUPPORTED
    for k in ("x", "w", "alpha", "gamma", "y", "which", "ws"):
        assert f(**{k: None}) == binding.PROM_ERR_NULL, k
    assert f(ad=(None, A, A, 1, 2, 8)) == f(ad=(A, None, A, 1, 2, 8)) == binding.PROM_ERR_NULL
    assert f(x=A + 8) == f(w=A + 4) == f(y=2 * A + 1) == f(alpha=A + 2) == f(gamma=A + 1) == binding.PROM_ERR_ALIGN
    assert f(which=A + 2) == f(ws=A + 8) == f(ad=(A + 8, A, A, 1, 2, 8)) == f(ad=(A, A + 2, A, 1, 2, 8)) == binding.PROM_ERR_ALIGN
    assert f(ad=(A, A, A + 2, 1, 2, 8)) == f(y=A) == binding.PROM_ERR_ALIGN
    assert f(wb=16) == binding.PROM_ERR_WORKSPACE


def test_workspace_bytes(lib):
    size = binding.pw_proj_adapters_workspace_bytes
    assert size(0, 1, 8) == size(4, 0, 8) == size(4, 1, 0) == size(4, 1, 257) == size(1 << 16, 1 << 16, 8) == 0
    assert size(1, 1, 1) > 0 and size(100, 7, 16) >= size(700, 1, 16) > size(300, 1, 16)
