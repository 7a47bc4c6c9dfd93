"""Layer norm on the GPU, forward, backward and straight to int8 codes, against the formulas in 64 bits.

Tolerances.  With u = 2^-24, a row's mean is a binary32 sum of at most a few dozen values per thread and a tree behind
it, so its error is within 64 u of the largest |x|; the same goes for the other sums.  A value of y passes five
roundings after that.  Everything is therefore compared with 256 u of the row's largest term (the products that cancel
included), plus half a step of the output's type (`torch.finfo(t).eps / 2` of the value)."""
import numpy as np
import pytest
import torch

from paper_2505_03254_b200 import binding, build
from gpu_util import Guarded

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


def _inputs(seed, m, n, dtype, ptype, pitch=None, offset=0.5):
    g = torch.Generator().manual_seed(seed)
    x = torch.randn((m, n), generator=g) * torch.exp(torch.randn((m, 1), generator=g)) + offset * torch.randn((m, 1), generator=g)
    w = 1 + 0.3 * torch.randn(n, generator=g)
    b = 0.3 * torch.randn(n, generator=g)
    x = x.to(dtype).cuda()
    if pitch:
        buf = torch.full((m, pitch), 7.0, dtype=dtype, device="cuda")
        buf[:, :n] = x
        x = buf[:, :n]
    return x, w.to(ptype).cuda(), b.to(ptype).cuda()


def _definition(x, w, b, eps=EPS):
    xd = x.double()
    mean = xd.mean(1, keepdim=True)
    rstd = 1 / torch.sqrt(((xd - mean) ** 2).mean(1, keepdim=True) + eps)
    xh = (xd - mean) * rstd
    w = 1.0 if w is None else w.double()
    b = 0.0 if b is None else b.double()
    return xh * w + b, mean, rstd, xh


def _near(got, want, slack, what):
    """|got - want| <= slack (64-bit, broadcastable) + half a step of got's type."""
    step = torch.finfo(got.dtype).eps / 2 if got.dtype != torch.float32 else U
    tiny = torch.finfo(got.dtype).tiny * torch.finfo(got.dtype).eps
    err = (got.double() - want).abs()
    lim = slack + step * want.abs() * 1.001 + tiny
    bad = ~(err <= lim)
    assert not bool(bad.any()), (what, int(bad.sum()), float((err / lim).max()))


def _slack(xd, mean, rstd, w):
    """256 u of the largest term that a value of the row is made of."""
    top = (xd.abs().amax(1, keepdim=True) + mean.abs()) * rstd + 1
    wd = 1.0 if w is None else w.double().abs() + 1
    return 256 * U * top * wd


# n: one value, a warp's row, more than a warp's, whole blocks, odd and even widths without whole pieces, the last
# widths that registers hold and the first ones that they do not
SHAPES = [(1, 1), (3, 2), (5, 7), (1, 64), (9, 96), (130, 192), (33, 384), (64, 1000), (17, 1283), (6, 2048), (4, 4096), (3, 4100),
          (2, 8192), (2, 16384), (2, 16392), (2, 16401), (2, 32768), (1, 32776), (1, 65536)]


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("m,n", SHAPES)
def test_forward(m, n, dtype):
    ptype = dtype if (m + n) % 2 else torch.float32
    x, w, b = _inputs(m * 7 + n, m, n, dtype, ptype)
    y, mean, rstd = binding.layer_norm(x, w, b, EPS)
    want, mu, rs, _ = _definition(x, w, b)
    slack = _slack(x.double(), mu, rs, w)
    _near(y, want, slack, "y")
    _near(mean, mu[:, 0], 256 * U * x.double().abs().amax(1), "mean")
    _near(rstd, rs[:, 0], 256 * U * (x.double().abs().amax(1) * rs[:, 0] + 1) * rs[:, 0], "rstd")


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("m,n", SHAPES)
def test_codes_are_those_of_the_definition(m, n, dtype):
    """Bit for bit: statistics in binary64 rounded once, then single binary32 operations."""
    ptype = dtype if (m + n) % 2 else torch.float32
    x, w, b = _inputs(m * 5 + n, m, n, dtype, ptype)
    mean, rstd = torch.empty(m, device="cuda"), torch.empty(m, device="cuda")
    q, gamma, scale = binding.layer_norm_i8(x, w, b, EPS, stats=(mean, rstd))
    _, mu, rs, _ = _definition(x, w, b)
    assert torch.equal(mean, mu[:, 0].float()) and torch.equal(rstd, rs[:, 0].float())
    y = (x.float() - mu.float()) * rs.float()
    y = y * w.float()
    y = y + b.float()
    top = y.abs().amax(1)
    want_scale = torch.full_like(top, 127.0) / top.clamp(min=1e-5)
    assert torch.equal(gamma, top) and torch.equal(scale, want_scale)
    assert torch.equal(q, torch.round(y * want_scale[:, None]).clamp(-128, 127).to(torch.int8))


BACKWARD = [(1, 1), (3, 2), (40, 7), (1, 64), (700, 96), (130, 192), (1500, 256), (33, 384), (64, 1000), (777, 1283), (300, 2048), (311, 4096),
            (160, 4100), (5, 6144), (7, 8184), (3, 8192), (5, 8200), (2, 16384), (2, 16392), (3, 16401), (2, 65536)]


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("m,n", BACKWARD)
def test_backward(m, n, dtype):
    ptype = dtype if (m + n) % 2 else torch.float32
    x, w, b = _inputs(m * 3 + n, m, n, dtype, ptype)
    g = torch.Generator().manual_seed(n)
    dy = torch.randn((m, n), generator=g).to(dtype).cuda()
    _, mu, rs, _ = _definition(x, w, b)
    mean, rstd = mu[:, 0].float(), rs[:, 0].float()
    dx, dw, db = binding.layer_norm_backward(dy, x, w, mean, rstd)
    xh = (x.double() - mean.double()[:, None]) * rstd.double()[:, None]
    gd = dy.double() * w.double()
    c1, c2 = gd.mean(1, keepdim=True), (gd * xh).mean(1, keepdim=True)
    want = rstd.double()[:, None] * (gd - c1 - xh * c2)
    top_xh = ((x.double().abs() + mean.double().abs()[:, None]) * rstd.double()[:, None]).amax(1, keepdim=True) + 1
    top_g = gd.abs().amax(1, keepdim=True)
    _near(dx, want, 256 * U * rstd.double()[:, None] * top_g * top_xh * top_xh, "dx")
    _near(dw, (dy.double() * xh).sum(0), 256 * U * (dy.double().abs() * top_xh).sum(0), "dweight")
    _near(db, dy.double().sum(0), 256 * U * dy.double().abs().sum(0), "dbias")
    # the same call gives the same bits
    again = binding.layer_norm_backward(dy, x, w, mean, rstd)
    assert all(torch.equal(p, q) for p, q in zip((dx, dw, db), again))


def test_backward_is_the_gradient_of_the_forward_pass():
    """Against differences of sum(y * c): the definition in 64 bits at x + h d and x - h d."""
    m, n = 6, 320
    x, w, b = _inputs(11, m, n, torch.float32, torch.float32)
    g = torch.Generator().manual_seed(12)
    c = torch.randn((m, n), generator=g).cuda()
    y, mean, rstd = binding.layer_norm(x, w, b, EPS)
    dx, dw, db = binding.layer_norm_backward(c, x, w, mean, rstd)

    def value(x_, w_, b_):
        return float((_definition(x_, w_, b_)[0] * c.double()).sum())

    h = 1e-4
    for which, grad in enumerate((dx, dw, db)):
        args = [x.double(), w.double(), b.double()]
        d = torch.randn(args[which].shape, generator=g).double().cuda()
        hi, lo = list(args), list(args)
        hi[which] = args[which] + h * d
        lo[which] = args[which] - h * d
        want = (value(*hi) - value(*lo)) / (2 * h)
        got = float((grad.double() * d).sum())
        # the difference's own error is O(h^2) of a value of order sqrt(m n) times the third derivative
        assert abs(got - want) <= 1e-5 * (float((grad.double().abs() * d.abs()).sum()) + 1), (which, got, want)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("n,pitch", [(96, 104), (1024, 1032), (1024, 1025), (100, 101), (4096, 4224)])
def test_row_pitches(n, pitch, dtype):
    """Rows that are a slice of a wider buffer: what lies between them is not written."""
    m = 37
    x, w, b = _inputs(n + pitch, m, n, dtype, torch.float32, pitch)
    size = torch.finfo(dtype).bits // 8
    out = Guarded(m * pitch * size, dtype=dtype, fill=3.0)
    y = out.view(m, pitch)[:, :n]
    _, mean, rstd = binding.layer_norm(x, w, b, EPS, out=(y, torch.empty(m, device="cuda"), torch.empty(m, device="cuda")))
    want, mu, rs, _ = _definition(x, w, b)
    _near(y, want, _slack(x.double(), mu, rs, w), "y")
    out.check("y")
    assert bool((out.view(m, pitch)[:, n:] == 3.0).all())
    # dense results from the same rows, and the backward pass
    # (within the same bound, not bit for bit: where a row starts decides which thread adds which of its values)
    _near(binding.layer_norm(x, w, b, EPS)[0], want, _slack(x.double(), mu, rs, w), "dense y")
    assert torch.equal(binding.layer_norm_i8(x, w, b, EPS)[0], binding.layer_norm_i8(x.contiguous(), w, b, EPS)[0])
    dy = torch.randn((m, n), device="cuda").to(dtype)
    res = Guarded(m * pitch * size, dtype=dtype, fill=3.0)
    dx = res.view(m, pitch)[:, :n]
    dw, db = torch.empty_like(w), torch.empty_like(b)
    binding.layer_norm_backward(dy, x, w, mean, rstd, out=(dx, dw, db))
    res.check("dx")
    assert bool((res.view(m, pitch)[:, n:] == 3.0).all())
    dense = binding.layer_norm_backward(dy, x.contiguous(), w, mean, rstd)
    slack = 64 * U * (dy.double().abs().sum(0) * 30)
    assert bool(((dense[0].double() - dx.double()).abs() <= torch.finfo(dtype).eps * dense[0].double().abs() + 1e-4).all())
    assert bool(((dense[1].double() - dw.double()).abs() <= slack).all()) and bool(((dense[2].double() - db.double()).abs() <= slack).all())


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("m,n", [(1, 5), (7, 3), (9, 17), (40, 95), (300, 97), (1201, 129), (500, 1003), (150, 2049), (40, 4093), (20, 8185), (20, 8200)])
@pytest.mark.parametrize("shift", [0, 2, 5])
def test_rows_that_start_anywhere(m, n, dtype, shift):
    """Dense rows of odd widths, from a base inside a 16-byte piece: nothing outside the rows is read into a result or written."""
    size = torch.finfo(dtype).bits // 8
    x0, w, b = _inputs(m + n + shift, m, n, dtype, torch.float32)
    flat = torch.full((m * n + 16,), float("nan"), dtype=dtype, device="cuda")
    x = flat[shift:shift + m * n].view(m, n)
    x.copy_(x0)
    want, mu, rs, _ = _definition(x, w, b)
    out = Guarded((m * n + 16) * size, dtype=dtype, fill=3.0)
    y = out.t[shift:shift + m * n].view(m, n)
    _, mean, rstd = binding.layer_norm(x, w, b, EPS, out=(y, torch.empty(m, device="cuda"), torch.empty(m, device="cuda")))
    out.check("y")
    assert bool((out.t[:shift] == 3.0).all()) and bool((out.t[shift + m * n:] == 3.0).all())
    _near(y, want, _slack(x.double(), mu, rs, w), "y")
    q, gamma, scale = binding.layer_norm_i8(x, w, b, EPS)
    wide = torch.zeros((m, (n + 15) // 16 * 16), dtype=dtype, device="cuda")
    wide[:, :n] = x
    ref = binding.layer_norm_i8(wide[:, :n], w, b, EPS)
    assert torch.equal(q, ref[0]) and torch.equal(gamma, ref[1]) and torch.equal(scale, ref[2])
    dflat = torch.full((m * n + 16,), float("nan"), dtype=dtype, device="cuda")
    dy = dflat[shift:shift + m * n].view(m, n)
    dy.copy_(torch.randn((m, n), device="cuda"))
    res = Guarded((m * n + 16) * size, dtype=dtype, fill=3.0)
    dx = res.t[shift:shift + m * n].view(m, n)
    dw, db = torch.empty_like(w), torch.empty_like(b)
    binding.layer_norm_backward(dy, x, w, mean, rstd, out=(dx, dw, db))
    res.check("dx")
    assert bool((res.t[:shift] == 3.0).all()) and bool((res.t[shift + m * n:] == 3.0).all())
    xh = (x.double() - mean.double()[:, None]) * rstd.double()[:, None]
    gd = dy.double() * w.double()
    top = xh.abs().amax(1, keepdim=True) + 1 + mean.double().abs()[:, None] * rstd.double()[:, None]
    want = rstd.double()[:, None] * (gd - gd.mean(1, keepdim=True) - xh * (gd * xh).mean(1, keepdim=True))
    _near(dx, want, 256 * U * rstd.double()[:, None] * gd.abs().amax(1, keepdim=True) * top * top, "dx")
    _near(dw, (dy.double() * xh).sum(0), 256 * U * (dy.double().abs() * top).sum(0), "dweight")
    _near(db, dy.double().sum(0), 256 * U * dy.double().abs().sum(0), "dbias")
    # tensors whose rows have different offsets
    if m > 1:
        plain = binding.layer_norm(x, w, b, EPS, out=(torch.empty((m, n + 1), dtype=dtype, device="cuda")[:, :n], None, None))[0]
        _near(plain, _definition(x, w, b)[0], _slack(x.double(), mu, rs, w), "y")
        other = binding.layer_norm_backward(dy.clone(), x, w, mean, rstd)
        _near(other[0], want, 256 * U * rstd.double()[:, None] * gd.abs().amax(1, keepdim=True) * top * top, "dx")


@pytest.mark.parametrize("shift", [1, 3])
def test_bases_off_sixteen_bytes(shift):
    """A view that starts inside a 16-byte piece is taken as it is."""
    m, n = 21, 256
    x, w, b = _inputs(5, m, n, torch.bfloat16, torch.bfloat16)
    flat = torch.zeros(m * n + 8, dtype=torch.bfloat16, device="cuda")
    xs = flat[shift:shift + m * n].view(m, n)
    xs.copy_(x)
    ws, bs = torch.zeros(n + 8, dtype=torch.bfloat16, device="cuda")[shift:shift + n], b
    ws.copy_(w)
    want = binding.layer_norm(x, w, b, EPS)
    got = binding.layer_norm(xs, ws, bs, EPS)
    _near(got[0], _definition(x, w, b)[0], _slack(x.double(), *_definition(x, w, b)[1:3], w), "y")
    assert torch.allclose(got[1], want[1], rtol=0, atol=1e-5)
    assert torch.equal(binding.layer_norm_i8(xs, ws, bs, EPS)[0], binding.layer_norm_i8(x, w, b, EPS)[0])
    codes = torch.empty(m * n + 8, dtype=torch.int8, device="cuda")[shift:shift + m * n].view(m, n)
    binding.layer_norm_i8(x, w, b, EPS, out=(codes, torch.empty(m, device="cuda"), torch.empty(m, device="cuda")))
    assert torch.equal(codes, binding.layer_norm_i8(x, w, b, EPS)[0])


@pytest.mark.parametrize("n", [256, 1283, 20000])
def test_in_place_and_without_parameters(n):
    m = 50
    x, w, b = _inputs(8, m, n, torch.float32, torch.float32)
    want = binding.layer_norm(x, w, b, EPS)
    y = x.clone()
    binding.layer_norm(y, w, b, EPS, out=(y, None, None))
    assert torch.equal(y, want[0])
    plain, mean, rstd = binding.layer_norm(x, None, None, EPS)
    ones, zeros = torch.ones_like(w), torch.zeros_like(b)
    assert torch.equal(plain, binding.layer_norm(x, ones, zeros, EPS)[0])
    assert torch.equal(binding.layer_norm_i8(x, None, None, EPS)[0], binding.layer_norm_i8(x, ones, zeros, EPS)[0])
    dy = torch.randn_like(x)
    dx, dw, db = binding.layer_norm_backward(dy, x, ones, mean, rstd)
    for inplace in (dy.clone(), x.clone()):
        d, xx = (inplace, x) if torch.equal(inplace, dy) else (dy, inplace)
        got = binding.layer_norm_backward(d, xx, None, mean, rstd, out=(inplace, torch.empty(n, device="cuda"), torch.empty(n, device="cuda")))
        assert torch.equal(inplace, dx) and torch.equal(got[1], dw) and torch.equal(got[2], db)
    # only what is wanted
    only = binding.layer_norm_backward(dy, x, None, mean, rstd, out=(torch.empty_like(x), None, None))
    assert torch.equal(only[0], dx)
    only = binding.layer_norm_backward(dy, x, None, mean, rstd, out=(None, torch.empty_like(dw), None))
    assert torch.equal(only[1], dw)
    only = binding.layer_norm_backward(dy, x, None, mean, rstd, out=(None, None, torch.empty_like(dw)))
    assert torch.equal(only[2], db)


def test_values_at_the_edges():
    """Constant rows, rows of zeros, an offset far above the spread, rows with an infinity or a NaN, huge values."""
    n = 512
    x = torch.randn((8, n), device="cuda")
    x[0] = 0.0
    x[1] = 5.0
    x[2] = x[2] + 4096.0
    x[3, 7] = float("inf")
    x[4, 9] = float("nan")
    x[5] *= 1e15
    y, mean, rstd = binding.layer_norm(x, None, None, EPS)
    assert bool((y[0] == 0).all()) and bool((y[1] == 0).all())
    assert torch.isnan(y[3]).all() and torch.isnan(y[4]).all()
    want, mu, rs, _ = _definition(x, None, None)
    keep = [0, 1, 2, 5, 6, 7]
    _near(y[keep], want[keep], _slack(x.double(), mu, rs, None)[keep], "y")
    q, gamma, scale = binding.layer_norm_i8(x, None, None, EPS)
    assert bool((q[0] == 0).all()) and float(gamma[0]) == 0.0 and float(scale[0]) == float(np.float32(127) / np.float32(1e-5))
    assert not torch.isfinite(gamma[3]) and not torch.isfinite(gamma[4])
    good = binding.layer_norm_i8(x[keep].contiguous(), None, None, EPS)
    assert torch.equal(q[keep], good[0]) and torch.equal(gamma[keep], good[1])
    # a bad row of dy or x stays in its row of dx, and shows in the column sums
    dy = torch.randn((8, n), device="cuda")
    dx, dw, db = binding.layer_norm_backward(dy, x, None, mean, rstd)
    ref = binding.layer_norm_backward(dy[keep].contiguous(), x[keep].contiguous(), None, mean[keep], rstd[keep])
    assert torch.equal(dx[keep], ref[0]) and torch.isnan(dx[3]).all() and torch.isnan(dw).any()
    assert torch.isfinite(db).all()


def test_no_rows():
    x = torch.empty((0, 128), device="cuda")
    w = torch.ones(128, device="cuda")
    y, mean, rstd = binding.layer_norm(x, w, w, EPS)
    assert y.shape == (0, 128) and mean.shape == (0,)
    assert binding.layer_norm_i8(x, w, w, EPS)[0].shape == (0, 128)
    dw, db = torch.full((128,), 5.0, device="cuda"), torch.full((128,), 5.0, device="cuda")
    binding.layer_norm_backward(x, x, w, mean, rstd, out=(torch.empty_like(x), dw, db))
    assert bool((dw == 0).all()) and bool((db == 0).all())


def test_more_dimensions_streams_and_graphs():
    x = torch.randn((4, 9, 320), device="cuda").bfloat16()
    w, b = torch.randn(320, device="cuda"), torch.randn(320, device="cuda")
    want = binding.layer_norm(x, w, b, EPS)
    codes = binding.layer_norm_i8(x, w, b, EPS)
    dy = torch.randn_like(x)
    grads = binding.layer_norm_backward(dy, x, w, want[1], want[2])
    assert want[0].shape == x.shape and codes[0].shape == x.shape and want[1].shape == (36,)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    got = binding.layer_norm(x, w, b, EPS, stream=side)
    got_g = binding.layer_norm_backward(dy, x, w, got[1], got[2], stream=side)
    side.synchronize()
    assert all(torch.equal(p, q) for p, q in zip(want + grads, got + got_g))
    # captured once, replayed on other inputs; two graphs of the same call have workspaces of their own
    graphs = []
    for _ in range(2):
        out = [torch.empty_like(t) for t in want + codes + grads]
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            binding.layer_norm(x, w, b, EPS, out=out[:3])
            binding.layer_norm_i8(x, w, b, EPS, out=out[3:6])
            binding.layer_norm_backward(dy, x, w, out[1], out[2], out=out[6:])
        graphs.append((g, out))
    x.copy_(torch.randn_like(x))
    for g, _ in graphs:
        g.replay()
    torch.cuda.synchronize()
    want = binding.layer_norm(x, w, b, EPS)
    fresh = want + binding.layer_norm_i8(x, w, b, EPS) + binding.layer_norm_backward(dy, x, w, want[1], want[2])
    for _, out in graphs:
        assert all(torch.equal(p, q) for p, q in zip(fresh, out))


def test_refusals():
    x = torch.randn((4, 64), device="cuda")
    w = torch.ones(64, device="cuda")
    stat = torch.empty(4, device="cuda")
    before = binding.launch_count()
    for bad in (x.cpu(), x.double(), x.t()[:32], x[:, ::2], x.expand(3, 4, 64)):
        with pytest.raises(ValueError):
            binding.layer_norm(bad, None, None, EPS, out=(torch.empty_like(x), None, None))
    for bad in (w[:32], w.double(), w.bfloat16().float().cpu(), torch.ones(128, device="cuda")[::2]):
        with pytest.raises(ValueError):
            binding.layer_norm(x, bad, None, EPS)
    with pytest.raises(ValueError):
        binding.layer_norm(x, w, w.bfloat16(), EPS)
    with pytest.raises(ValueError):
        binding.layer_norm(x, w, w, EPS, out=(torch.empty((4, 65), device="cuda"), None, None))
    with pytest.raises(ValueError):
        binding.layer_norm_backward(x.bfloat16(), x, w, stat, stat)
    with pytest.raises(ValueError):
        binding.layer_norm_backward(x, x, w, stat[:3], stat)
    for eps in (-1e-5, float("nan"), float("inf")):
        with pytest.raises(binding.PromError) as e:
            binding.layer_norm(x, w, w, eps)
        assert e.value.code == binding.PROM_ERR_RANGE
    with pytest.raises(binding.PromError) as e:
        binding.layer_norm(torch.zeros((1, 65537), device="cuda"))
    assert e.value.code == binding.PROM_ERR_SHAPE
    with pytest.raises(binding.PromError) as e:
        binding.layer_norm(x[:1].expand(4, 64), w, w, EPS)
    assert e.value.code == binding.PROM_ERR_SHAPE
    with pytest.raises(binding.PromError) as e:
        binding.layer_norm_backward(x, x, w, stat, stat, workspace=torch.empty(16, dtype=torch.uint8, device="cuda"))
    assert e.value.code == binding.PROM_ERR_WORKSPACE
    assert binding.launch_count() == before
