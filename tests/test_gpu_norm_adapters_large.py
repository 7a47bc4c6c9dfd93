"""Layer norm and the projection with adapters where offsets pass 32 bits: matrices of more than 2^32 values, and slices of a
wider buffer whose rows lie that far apart.  The first and the last rows and some between are compared with the formulas in
64 bits, with the bounds of the tests of ordinary sizes."""
import numpy as np
import pytest
import torch

from paper_2505_03254_b200 import binding, build

pytestmark = pytest.mark.gpu

U = 2.0 ** -24


@pytest.fixture(scope="module", autouse=True)
def _lib():
    build.build()
    binding.last_device_status()
    yield
    torch.cuda.empty_cache()
    assert binding.last_device_status() == binding.PROM_OK


def _rows(m):
    return torch.tensor([0, 1, m // 3, m // 2 + 1, m - 300, m - 257, m - 2, m - 1], device="cuda")


def _norm(xs, w, b):
    xd = xs.double()
    mean = xd.mean(1, keepdim=True)
    rstd = 1 / torch.sqrt(((xd - mean) ** 2).mean(1, keepdim=True) + 1e-5)
    slack = 256 * U * ((xd.abs().amax(1, keepdim=True) + mean.abs()) * rstd + 1) * (w.double().abs() + 1)
    return (xd - mean) * rstd * w.double() + b.double(), mean, rstd, slack


@pytest.mark.parametrize("m,n", [(1_100_000, 4096), (34_000_000, 131)])
def test_norm_of_more_than_2_to_the_32_values(m, n):
    g = torch.Generator(device="cuda").manual_seed(1)
    x = torch.empty((m, n), dtype=torch.bfloat16, device="cuda").normal_(generator=g)
    w, b = 1 + 0.2 * torch.randn(n, device="cuda", generator=g), 0.2 * torch.randn(n, device="cuda", generator=g)
    at = _rows(m)
    y, mean, rstd = binding.layer_norm(x, w, b)
    want, mu, rs, slack = _norm(x[at], w, b)
    assert bool(((y[at].double() - want).abs() <= slack + 2.0 ** -8 * want.abs() * 1.001).all())
    del y
    q, gamma, scale = binding.layer_norm_i8(x, w, b)
    small = binding.layer_norm_i8(x[at].contiguous(), w, b)
    assert torch.equal(q[at], small[0]) and torch.equal(gamma[at], small[1]) and torch.equal(scale[at], small[2])
    del q
    # dy is x, and dx takes its place
    gd = x[at].double() * w.double()
    xh = (x[at].double() - mean[at].double()[:, None]) * rstd[at].double()[:, None]
    dx_want = rstd[at].double()[:, None] * (gd - gd.mean(1, keepdim=True) - xh * (gd * xh).mean(1, keepdim=True))
    top = xh.abs().amax(1, keepdim=True) + 1
    lim = 256 * U * rstd[at].double()[:, None] * gd.abs().amax(1, keepdim=True) * top * top + 2.0 ** -8 * dx_want.abs() * 1.001
    db_want = torch.zeros(n, dtype=torch.float64, device="cuda")
    size = torch.zeros(n, dtype=torch.float64, device="cuda")
    for lo in range(0, m, 1 << 20):
        part = x[lo:lo + (1 << 20)].double()
        db_want += part.sum(0)
        size += part.abs().sum(0)
        del part
    dw, db = torch.empty_like(w), torch.empty_like(b)
    binding.layer_norm_backward(x, x, w, mean, rstd, out=(x, dw, db))
    assert bool(((x[at].double() - dx_want).abs() <= lim).all())
    # a thread's running sum has up to m / 148 terms here: u of each partial sum, which is at most the sum of sizes / 148
    assert bool(((db.double() - db_want).abs() <= (m / 148) * U * size / 148 + 256 * U * size).all())


def test_rows_far_apart():
    m, n, pitch = 5, 512, 1_000_000_008
    buf = torch.empty(4 * pitch + n, dtype=torch.bfloat16, device="cuda")
    x = buf.as_strided((m, n), (pitch, 1))
    x.copy_(torch.randn((m, n), device="cuda"))
    w, b = torch.ones(n, device="cuda"), torch.zeros(n, device="cuda")
    want, _, _, slack = _norm(x, w, b)
    codes = binding.layer_norm_i8(x, w, b)
    assert all(torch.equal(p, q) for p, q in zip(codes, binding.layer_norm_i8(x.contiguous(), w, b)))
    binding.layer_norm(x, w, b, out=(x, None, None))
    assert bool(((x.double() - want).abs() <= slack + 2.0 ** -8 * want.abs() * 1.001).all())


@pytest.mark.parametrize("m,cin,cout", [(1_100_000, 4096, 8), (1_100_000, 32, 4096)])
def test_projection_of_more_than_2_to_the_32_values(m, cin, cout):
    g = torch.Generator(device="cuda").manual_seed(2)
    n, rank = 3, 4
    x = torch.empty((m, cin), dtype=torch.int8, device="cuda").random_(-127, 128, generator=g)
    w = torch.randint(-1, 2, (cout, cin), device="cuda", generator=g).to(torch.int8)
    alpha = torch.rand(cout, device="cuda", generator=g) * 0.05 + 0.01
    gamma = torch.rand(m, device="cuda", generator=g) + 0.5
    a = (torch.randn((n, rank, cin), device="cuda", generator=g) / cin ** 0.5).bfloat16()
    b = torch.randn((n, cout, rank), device="cuda", generator=g).bfloat16()
    scale = torch.rand(n, device="cuda", generator=g) + 0.5
    which = torch.randint(-1, n, (m,), device="cuda", generator=g).int()
    y = binding.pw_proj_adapters(x, m, binding.pack_ternary(w), cout, alpha, gamma, a, b, scale, which)
    at = _rows(m)
    f = (gamma[at].double() / 127)[:, None]
    xs = x[at].double()
    base = (xs @ w.double().T) * alpha.double() * f
    want, lim = base.clone(), 8 * U * base.abs()
    for k, r in enumerate(at.tolist()):
        i = int(which[r])
        if i >= 0:
            t, t0 = xs[k] @ a[i].double().T, xs[k].abs() @ a[i].double().abs().T
            want[k] += float(scale[i]) * float(f[k]) * (b[i].double() @ t)
            lim[k] += float(scale[i]) * float(f[k]) * (512 * U * (b[i].double().abs() @ (t0 + t.abs())) + 2.0 ** -16 * (b[i].double().abs() @ t.abs()))
    assert bool(((y[at].double() - want).abs() <= lim + 2.0 ** -8 * 1.001 * (want.abs() + lim)).all())
