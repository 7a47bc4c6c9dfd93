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


def _near(got, want, slack, what):
    """|got - want| <= slack + half a step of got's type."""
    err = (got.double() - want).abs()
    info = torch.finfo(got.dtype)
    lim = slack + info.eps / 2 * 1.001 * want.abs() + info.tiny * info.eps
    bad = ~(err <= lim)
    assert not bool(bad.any()), (what, int(bad.sum()), [int(v) for v in bad.nonzero()[0]], float((err / lim).max()))


def _rows(seed, m, n, dtype, pitch=0):
    """Rows of a residual stream: scales and offsets of their own, every 16th one far from zero for its spread."""
    g = torch.Generator(device="cuda").manual_seed(seed)
    x = torch.randn((m, n), device="cuda", generator=g) * torch.exp(torch.randn((m, 1), device="cuda", generator=g))
    x += 0.3 * torch.randn((m, 1), device="cuda", generator=g)
    x[::16] += 100 * x[::16].std(1, keepdim=True) if n > 1 else 0.0
    x = x.to(dtype)
    w = 1 + 0.2 * torch.randn(n, device="cuda", generator=g)
    b = 0.2 * torch.randn(n, device="cuda", generator=g)
    return (_rows_apart(x, pitch) if pitch else x), w, b


# widths on both sides of where the kernels for many rows change, in 16-byte pieces: 32, 64 and 128 (registers), 512 and, for
# codes, 4096 values (shared memory); several rows of a warp in turn
WIDTHS = [8, 24, 96, 128, 132, 192, 256, 260, 264, 384, 512, 520, 768, 1024, 1032, 2048, 2056, 4096, 4104]


def _count(n):
    """Rows: three rounds of the warps that an SM holds at most, or enough for the kernels of many rows where that is much."""
    return 3 * 32 * torch.cuda.get_device_properties(0).multi_processor_count + 11 if n <= 1032 else _many() if n > 4096 else 8999


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("n", WIDTHS)
def test_forward_of_many_rows(n, dtype):
    m = _count(n)
    x, w, b = _rows(n, m, n, dtype)
    mu, rs = _statistics(x)
    top = (x.double().abs().amax(1, keepdim=True) + mu.abs()) * rs + 1
    slack = 256 * U * top * (w.double().abs() + 1)
    want = (x.double() - mu) * rs * w.double() + b.double()
    y, mean, rstd = binding.layer_norm(x, w, b, EPS)
    _near(y, want, slack, "y")
    _near(mean, mu[:, 0], 256 * U * x.double().abs().amax(1), "mean")
    _near(rstd, rs[:, 0], 256 * U * top[:, 0] * rs[:, 0], "rstd")
    # rows of a wider buffer, and in place: the same kernel, the same bits
    apart = _rows_apart(x, 16)
    assert torch.equal(binding.layer_norm(apart, w, b, EPS, out=(_rows_apart(x, 24), None, None))[0], y)
    assert torch.equal(binding.layer_norm(apart, w, b, EPS, out=(apart, None, None))[0], y)
    assert bool((torch.as_strided(apart, (m, 16), (n + 16, 1), n)[: m - 1] == 7.0).all())
    own = x.clone()
    binding.layer_norm(own, w, b, EPS, out=(own, None, None))
    assert torch.equal(own, y)
    kept = dtype if dtype != torch.float32 else torch.bfloat16          # parameters of a 16-bit type
    w2, b2 = w.to(kept), b.to(kept)
    _near(binding.layer_norm(x, w2, b2, EPS)[0], (x.double() - mu) * rs * w2.double() + b2.double(), slack * 1.01, "y")


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("n", WIDTHS)
def test_codes_of_many_rows(n, dtype):
    m = _count(n)
    x, w, b = _rows(n + 1, m, n, dtype)
    want = _codes(x, w, b)
    for rows in (x, _rows_apart(x, 16), _rows_apart(x, 1)):
        for name, p, q in zip(("codes", "gamma", "scale", "mean", "rstd"), _run_codes(rows, w, b), want):
            bad = (p != q).view(m, -1).any(1).nonzero()[:, 0].tolist()
            assert not bad, (name, len(bad), bad[:5])


# rows of a group of threads that go round its ring of copies several times; in 16-byte pieces 65 to 1024 (two a thread) and up
# to 2048 (four)
RINGS = [(9001, 520), (9001, 1024), (7001, 1536), (4001, 2048), (3001, 4096), (1501, 8192), (1201, 12288), (901, 16384)]


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("m,n", RINGS)
def test_backward_of_many_rows(m, n, dtype):
    if dtype == torch.float32:
        n //= 2
    x, w, _ = _rows(n + 2, m, n, dtype)
    dy = torch.randn((m, n), device="cuda", generator=torch.Generator(device="cuda").manual_seed(n)).to(dtype)
    mean, rstd = (t[:, 0].float() for t in _statistics(x))
    dx, dw, db = binding.layer_norm_backward(dy, x, w, mean, rstd)
    rd = rstd.double()[:, None]
    xh = (x.double() - mean.double()[:, None]) * rd
    gd = dy.double() * w.double()
    want = rd * (gd - gd.mean(1, keepdim=True) - xh * (gd * xh).mean(1, keepdim=True))
    top = ((x.double().abs() + mean.double().abs()[:, None]) * rd).amax(1, keepdim=True) + 1
    _near(dx, want, 256 * U * rd * gd.abs().amax(1, keepdim=True) * top * top, "dx")
    # a thread adds up to m / 148 rows behind each other, of sizes that add up to a 148th of the column's
    long = max(256.0, m / 148.0)
    _near(dw, (dy.double() * xh).sum(0), long * U * (dy.double().abs() * top).sum(0), "dweight")
    _near(db, dy.double().sum(0), long * U * dy.double().abs().sum(0), "dbias")
    # in place of either, from rows further apart, and again
    for place in ("dy", "x"):
        one, other = _rows_apart(dy, 8), _rows_apart(x, 24)
        into = one if place == "dy" else other
        got = binding.layer_norm_backward(one, other, w, mean, rstd, out=(into, torch.empty_like(dw), torch.empty_like(db)))
        assert torch.equal(into, dx) and torch.equal(got[1], dw) and torch.equal(got[2], db)
    only = binding.layer_norm_backward(dy, x, w, mean, rstd, out=(None, torch.empty_like(dw), None))
    assert torch.equal(only[1], dw)


def test_gradients_over_a_hundred_thousand_rows():
    """dweight in full where a group's column sums run over hundreds of rows."""
    m, n = 120_001, 2048
    x, w, _ = _rows(5, m, n, torch.bfloat16)
    dy = torch.empty_like(x).normal_(generator=torch.Generator(device="cuda").manual_seed(6))
    _, mean, rstd = binding.layer_norm(x, w, None, EPS)
    dx, dw, db = binding.layer_norm_backward(dy, x, w, mean, rstd)
    want = torch.zeros((4, n), dtype=torch.float64, device="cuda")
    for lo in range(0, m, 20_000):
        at = slice(lo, lo + 20_000)
        xd, dd, rd = x[at].double(), dy[at].double(), rstd[at].double()[:, None]
        xh = (xd - mean[at].double()[:, None]) * rd
        gd = dd * w.double()
        top = ((xd.abs() + mean[at].double().abs()[:, None]) * rd).amax(1, keepdim=True) + 1
        _near(dx[at], rd * (gd - gd.mean(1, keepdim=True) - xh * (gd * xh).mean(1, keepdim=True)),
              256 * U * rd * gd.abs().amax(1, keepdim=True) * top * top, "dx")
        want += torch.stack([(dd * xh).sum(0), (dd.abs() * top).sum(0), dd.sum(0), dd.abs().sum(0)])
    _near(dw, want[0], m / 148.0 * U * want[1], "dweight")
    _near(db, want[2], m / 148.0 * U * want[3], "dbias")


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("n", [40, 328, 392, 656, 1003, 2624, 16404])
def test_gradients_that_cancel(n, dtype):
    """Equal values of dy behind constant rows: the mean of g is each of them (a quotient, not a product with a rounded inverse), and
    dx is exactly zero."""
    m = 300
    x = torch.randint(1, 200, (m, 1), generator=torch.Generator().manual_seed(n)).to(dtype).cuda()
    dy = torch.flip(x, [0]).expand(m, n).contiguous()
    mean, rstd = x[:, 0].float(), torch.full((m,), 300.0, device="cuda")
    for rows in (x.expand(m, n).contiguous(), _rows_apart(x.expand(m, n), 1)):
        dx, dw, db = binding.layer_norm_backward(dy, rows, None, mean, rstd)
        assert not bool(dx.any()) and not bool(dw.any()) and torch.equal(db, dy.double().sum(0).float())
