"""Layer norm where the number of rows chooses the kernel: the same rows in calls of a few rows and of thousands, every row
compared, in the three types.  With S multiprocessors, calls of 8 S rows and more of whole 16-byte pieces take a warp per row (in
registers up to 64 or 128 pieces, in shared memory above), rows that start anywhere take groups of threads, and few rows a block each.

Tolerances are those of the formula: u = 2^-24, 256 u of a row's largest term, plus half a step of the output's type.  Codes
and their statistics are compared bit for bit with the definition: sums in binary64 (exact here for the mean of 16-bit
values), a division, one rounding to binary32."""
import pytest
import torch

from paper_2505_03254_b200 import binding, build

pytestmark = pytest.mark.gpu

U = 2.0 ** -24
TYPES = [torch.float32, torch.bfloat16, torch.float16]
EPS = 1e-5


@pytest.fixture(scope="module", autouse=True)
def _lib():
    build.build()
    binding.last_device_status()
    yield
    assert binding.last_device_status() == binding.PROM_OK


def _many():
    """Rows from which on a warp takes each, and a few more."""
    return 8 * torch.cuda.get_device_properties(0).multi_processor_count + 37


def _statistics(x, eps=EPS):
    xd = x.double()
    n = torch.full((len(x), 1), float(x.shape[1]), dtype=torch.float64, device="cuda")     # (by a number, a product with its inverse)
    mean = xd.sum(1, keepdim=True) / n
    var = torch.square(xd - mean).sum(1, keepdim=True) / n
    return mean, 1 / torch.sqrt(var + eps)


def _codes(x, w, b, eps=EPS):
    """(q, gamma, scale, mean, rstd) of the definition."""
    mean, rstd = (t.float() for t in _statistics(x, eps))
    y = (x.float() - mean) * rstd
    y = y * w.float()
    y = y + b.float()
    gamma = y.abs().amax(1)
    scale = torch.full_like(gamma, 127.0) / gamma.clamp(min=1e-5)
    return torch.round(y * scale[:, None]).clamp(-128, 127).to(torch.int8), gamma, scale, mean[:, 0], rstd[:, 0]


def _run_codes(x, w, b, eps=EPS):
    stats = tuple(torch.empty(x.shape[0], device="cuda") for _ in range(2))
    return (*binding.layer_norm_i8(x, w, b, eps, stats=stats), *stats)


def _rows_apart(x, by):
    """The same values with `by` more between the rows' starts."""
    m, n = x.shape
    buf = torch.full((m, n + by), 7.0, dtype=x.dtype, device="cuda")
    buf[:, :n] = x
    return buf[:, :n]


def _halfway_rows(n, dtype):
    """Rows whose mean is 1.5 + (2 i + 1) 2^-24, halfway between two binary32 numbers: 1.5, and (2 i + 1) n 2^-24 in two values."""
    rows = torch.full((200, n), 1.5, dtype=torch.float64)
    for i in range(200):
        d = (2 * i + 1) * n
        low = (n & -n) << 8             # d in pieces of eight bits at most
        rows[i, 3], rows[i, n // 2], rows[i, n - 1] = 4.5, d % low * U, d // low * low * U
    got = rows.to(dtype)
    assert torch.equal(got.double(), rows)
    return got.cuda()


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("n", [328, 392, 1568, 2624])
def test_statistics_do_not_depend_on_the_number_of_rows(n, dtype):
    """A division by n and no product with its rounded inverse: a constant row's mean is its value, and a mean halfway between two
    binary32 numbers is rounded to the even one, however many rows there are and wherever they start."""
    g = torch.Generator().manual_seed(n)
    whole = torch.randint(1, 257, (200, 1), generator=g).double().expand(200, n).to(dtype).cuda()
    x = torch.cat([_halfway_rows(n, dtype), whole, torch.randn((200, n), generator=g).to(dtype).cuda()])
    x = x.repeat(-(-_many() // len(x)), 1)
    w, b = (1 + 0.2 * torch.randn(n, generator=g)).cuda(), (0.2 * torch.randn(n, generator=g)).cuda()
    want = _codes(x, w, b)
    for kind, rows in {"apart": _rows_apart(x, 1), "dense": x}.items():
        for m in (4, 403, len(x)):
            for name, p, q in zip(("codes", "gamma", "scale", "mean", "rstd"), _run_codes(rows[:m], w, b), want):
                bad = (p != q[:m]).view(m, -1).any(1).nonzero()[:, 0].tolist()
                assert not bad, (kind, m, name, len(bad), bad[:5])
            y, mean, _ = binding.layer_norm(rows[:m], None, None, EPS)
            flat = torch.arange(m, device="cuda") % 600 // 200 == 1
            assert torch.equal(mean[flat], rows[:m][flat][:, 0].float()) and not bool(y[flat].any()), (kind, m)


@pytest.mark.parametrize("dtype", TYPES)
def test_codes_of_rows_far_from_zero(dtype):
    """Offsets of 20 to 60 times the spread: rstd is still the binary64 one rounded once (its neighbour in some rows, where the
    variance came from the sum of squares)."""
    m, n = 400_000, 520
    g = torch.Generator(device="cuda").manual_seed(4)
    x = (torch.randn((m, n), device="cuda", generator=g) + 20 + 40 * torch.rand((m, 1), device="cuda", generator=g)).to(dtype)
    w, b = 1 + 0.2 * torch.randn(n, device="cuda", generator=g), 0.2 * torch.randn(n, device="cuda", generator=g)
    got = _run_codes(x, w, b)
    for lo in range(0, m, 50_000):
        for name, p, q in zip(("codes", "gamma", "scale", "mean", "rstd"), got, _codes(x[lo:lo + 50_000], w, b)):
            bad = (p[lo:lo + 50_000] != q).view(len(q), -1).any(1).nonzero()[:, 0].tolist()
            assert not bad, (name, lo, len(bad), bad[:5])


def _same(p, q):
    return bool(((p == q) | (torch.isnan(p) & torch.isnan(q))).all())


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("n", [128, 250, 264, 768, 2048, 4100, 16401])
def test_codes_of_values_that_are_not_finite(n, dtype):
    """The statistics are the formula's, whichever kernel takes the row: an infinity in x shows in the mean and makes the rest NaN,
    one in a parameter leaves mean and rstd alone."""
    many = _many()
    m = many if n < 16401 else 40
    x = torch.randn((m, n), device="cuda", generator=torch.Generator(device="cuda").manual_seed(n)).to(dtype)
    inf = float("inf")
    for at in (0, m // 2, m - 9):
        x[at, 7], x[at + 1, n - 1], x[at + 2, 0] = inf, -inf, float("nan")
        x[at + 3, 1], x[at + 3, n // 2] = inf, -inf
    bad = torch.tensor([r + k for r in (0, m // 2, m - 9) for k in range(4)], device="cuda")
    good = torch.ones(m, dtype=torch.bool, device="cuda")
    good[bad] = False
    w, b = torch.ones(n, device="cuda"), torch.zeros(n, device="cuda")
    want = _codes(x, w, b)
    for rows in (x, _rows_apart(x, 3), x[:5], _rows_apart(x[:5], 1)):
        q, gamma, scale, mean, rstd = _run_codes(rows, w, b)
        assert _same(mean, want[3][:len(rows)]) and _same(rstd, want[4][:len(rows)])
        assert _same(gamma, want[1][:len(rows)]) and _same(scale, want[2][:len(rows)])
        assert torch.equal(q[good[:len(rows)]], want[0][:len(rows)][good[:len(rows)]])
        assert bool(torch.isnan(gamma[bad[bad < len(rows)]]).all()) and bool(torch.isinf(mean[:2]).all())
    # parameters that are not finite, and values beyond binary32 behind finite ones
    for key, value in (("b", inf), ("w", float("nan")), ("w", 3e38)):
        w2, b2 = w.clone(), b.clone()
        (w2 if key == "w" else b2)[n - 2] = value
        x2 = x.clone()
        x2[bad] = 1.0
        x2[:, n - 2] = 50.0
        want = _codes(x2, w2, b2)
        for rows in (x2, _rows_apart(x2, 3), x2[:5], _rows_apart(x2[:5], 1)):
            q, gamma, scale, mean, rstd = _run_codes(rows, w2, b2)
            assert bool(torch.isfinite(mean).all()) and bool(torch.isfinite(rstd).all())
            assert _same(mean, want[3][:len(rows)]) and _same(rstd, want[4][:len(rows)])
            assert _same(gamma, want[1][:len(rows)]) and not bool(torch.isfinite(gamma).any())


@pytest.mark.parametrize("n", [129, 1283])
def test_backward_of_constant_rows_of_large_values(n):
    """xh is zero in all of the row and only there: what stands beside a row in its last piece of memory (mean rstd is 6e38) takes
    no part in its sums."""
    m = 40
    x = torch.full((m, n), 2e36, device="cuda")
    dy = torch.randn((m, n), device="cuda", generator=torch.Generator(device="cuda").manual_seed(n))
    mean, rstd = torch.full((m,), 2e36, device="cuda"), torch.full((m,), 316.25, device="cuda")
    dx, dw, db = binding.layer_norm_backward(dy, x, None, mean, rstd)
    g = dy.double()
    want = 316.25 * (g - g.mean(1, keepdim=True))
    assert bool(((dx.double() - want).abs() <= 316.25 * 256 * U * g.abs().amax(1, keepdim=True)).all())
    assert not bool(dw.any()) and bool(((db.double() - g.sum(0)).abs() <= 256 * U * g.abs().sum(0)).all())
