"""The ternary projection with low-rank adapters on the GPU against its formula in 64 bits.

Tolerances.  The integer sum is exact and at most 2^20, so the base term has three binary32 roundings.  The adapters'
inner products are binary32 sums of up to 4096 terms, added in parts of at most 128 and a tree of parts: an error within
256 u of the sum of the terms' sizes, u = 2^-24; where they pass through 16-bit values they are the sum of two (relative
error at most 2^-16) or, for float32 outputs, three (2^-24); the outer products are sums of at most 256 terms.  So with
T = sum_j |B| sum_k |A| |x| (and T1 = sum_j |B| |t_j|) a value is within
    8 u |base| + scale f (512 u T + 2^-16 T1 [16-bit outputs] + 512 u T1) + half a step of the output's type."""
import numpy as np
import pytest
import torch

from paper_2505_03254_b200 import binding, build
from gpu_util import Guarded

pytestmark = pytest.mark.gpu

U = 2.0 ** -24


@pytest.fixture(scope="module", autouse=True)
def _lib():
    build.build()
    binding.last_device_status()
    yield
    assert binding.last_device_status() == binding.PROM_OK


def _case(seed, batch, rows, cin, cout, n, rank, kind=torch.bfloat16, share=0.8, order="runs"):
    g = torch.Generator().manual_seed(seed)
    m = batch * rows
    x = torch.randint(-127, 128, (m, cin), generator=g).to(torch.int8)
    x[torch.rand(x.shape, generator=g) < 0.2] = 0
    w = torch.randint(-1, 2, (cout, cin), generator=g).to(torch.int8)
    c = dict(batch=batch, rows=rows, cout=cout, x=x.cuda(), w=w.cuda(), packed=binding.pack_ternary(w.cuda()),
             alpha=(torch.rand(cout, generator=g) * 0.05 + 0.01).cuda(),
             gamma=(torch.rand(batch, generator=g) * 6 + 0.5).cuda())
    if n:
        c["a"] = (torch.randn((n, rank, cin), generator=g) / cin ** 0.5).to(kind).cuda()
        c["b"] = (torch.randn((n, cout, rank), generator=g) / rank ** 0.5).to(kind).cuda()
        c["scale"] = (torch.rand(n, generator=g) * 2 - 0.5).cuda()
        which = torch.randint(0, n, (batch,), generator=g).to(torch.int32)
        if order == "runs":
            which = which.sort().values
        which[torch.rand(batch, generator=g) >= share] = -1
        c["which"] = which.cuda()
    return c


def _call(c, **kw):
    ad = [c.get(k) for k in ("a", "b", "scale", "which")]
    return binding.pw_proj_adapters(c["x"], c["batch"], c["packed"], c["cout"], c["alpha"], c["gamma"], *ad, **kw)


def _definition(c):
    """(value, slack without the output's rounding and the 16-bit pieces, the pieces' slack) in 64 bits."""
    f = (c["gamma"].double().clamp(min=float(np.float32(1e-5))) / 127).repeat_interleave(c["rows"])[:, None]
    x = c["x"].double()
    base = (x @ c["w"].double().T) * c["alpha"].double() * f
    slack, pieces = 8 * U * base.abs(), torch.zeros_like(base)
    if "a" in c:
        which = c["which"].repeat_interleave(c["rows"])
        for i in range(c["a"].shape[0]):
            at = (which == i).nonzero()[:, 0]
            if not len(at):
                continue
            a, b = c["a"][i].double(), c["b"][i].double()
            sc = float(c["scale"][i]) if c.get("scale") is not None else 1.0
            t = x[at] @ a.T
            base[at] += sc * f[at] * (t @ b.T)
            t0 = x[at].abs() @ a.abs().T
            slack[at] += 512 * U * abs(sc) * f[at] * ((t0 + t.abs()) @ b.abs().T)
            pieces[at] += 2.0 ** -16 * abs(sc) * f[at] * (t.abs() @ b.abs().T)
    return base, slack, pieces


def _check(got, c, what=""):
    want, slack, pieces = _definition(c)
    info = torch.finfo(got.dtype)
    lim = slack + 1e-30 + (info.eps / 2) * 1.001 * (want.abs() + slack) + info.tiny * info.eps
    if got.dtype != torch.float32:
        lim = lim + pieces
    err = (got.double() - want).abs()
    bad = ~(err <= lim)
    assert not bool(bad.any()), (what, int(bad.sum()), [int(v) for v in bad.nonzero()[0]], float((err / lim).max()))


SHAPES = [  # batch, rows, cin, cout, adapters, rank
    (1, 1, 16, 8, 1, 1), (1, 1, 2048, 2048, 8, 16), (3, 1, 48, 24, 2, 4), (8, 1, 4096, 256, 3, 16), (9, 1, 960, 1280, 4, 8),
    (32, 1, 1024, 512, 40, 16), (33, 1, 320, 104, 5, 12), (64, 1, 256, 384, 64, 32), (100, 1, 144, 200, 7, 64), (127, 1, 400, 8, 3, 5),
    (128, 1, 1536, 128, 16, 24), (129, 1, 208, 264, 4, 48), (205, 1, 960, 1280, 5, 8), (256, 1, 512, 640, 3, 100), (257, 1, 64, 520, 2, 256),
    (300, 1, 384, 1032, 300, 8), (600, 1, 2048, 256, 30, 16), (1000, 1, 16, 72, 12, 3), (5, 49, 576, 160, 3, 4), (4, 196, 384, 576, 12, 4),
    (2, 700, 96, 24, 1, 64), (1024, 1, 4096, 512, 16, 64), (2500, 1, 128, 256, 9, 16), (1100, 1, 256, 1024, 60, 16), (5000, 1, 48, 1280, 200, 8),
    (9000, 1, 512, 264, 2, 40), (40, 64, 160, 960, 6, 31)]


@pytest.mark.parametrize("shape", SHAPES)
@pytest.mark.parametrize("kind,out", [(torch.bfloat16, torch.bfloat16), (torch.float16, torch.float16), (torch.bfloat16, torch.float32),
                                      (torch.float16, torch.float32)])
def test_matches_the_formula(shape, kind, out):
    order = "runs" if sum(shape) % 2 else "mixed"
    c = _case(sum(shape), *shape, kind=kind, order=order)
    _check(_call(c, dtype=out), c, shape)


@pytest.mark.parametrize("mode", [1, 2])
@pytest.mark.parametrize("shape", [(1, 1, 16, 8, 1, 1), (7, 1, 3008, 72, 3, 16), (9, 1, 1040, 136, 4, 20), (31, 1, 4096, 264, 9, 8), (70, 1, 2064, 4096, 5, 12),
                                   (200, 1, 2048, 520, 40, 16), (300, 1, 976, 1288, 7, 64), (5, 70, 80, 328, 2, 33), (700, 1, 1536, 640, 90, 24)])
def test_both_sets_of_kernels(shape, mode):
    """Every shape runs on either; what the library's rule chooses is one of them."""
    binding.debug_adapters(mode)
    try:
        for kind, out in ((torch.bfloat16, torch.bfloat16), (torch.float16, torch.float32)):
            c = _case(sum(shape) + 1, *shape, kind=kind, order="mixed")
            y = _call(c, dtype=out)
            _check(y, c, shape)
            assert torch.equal(y, _call(c, dtype=out))
            c0 = {k: v for k, v in c.items() if k not in ("a", "b", "scale", "which")}
            _check(_call(c0, dtype=out), c0, shape)
    finally:
        binding.debug_adapters()


@pytest.mark.parametrize("batch", [1, 7, 40, 130, 700])
def test_without_adapters(batch):
    for out in (torch.float32, torch.bfloat16, torch.float16):
        c = _case(batch, batch, 1, 320, 1280, 0, 1)
        want = _call(c, dtype=out)
        _check(want, c)
        # an empty table, and samples that all have none, are the same call
        c2 = dict(c, a=torch.empty((0, 4, 320), dtype=torch.bfloat16, device="cuda"), b=torch.empty((0, 1280, 4), dtype=torch.bfloat16, device="cuda"),
                  scale=torch.empty(0, device="cuda"), which=torch.full((batch,), -1, dtype=torch.int32, device="cuda"))
        assert torch.equal(_call(c2, dtype=out), want)
        c3 = _case(batch, batch, 1, 320, 1280, 3, 8, share=0.0)
        for k in ("x", "packed", "alpha", "gamma"):
            c3[k] = c[k]
        assert torch.equal(_call(c3, dtype=out), want)


def test_the_base_term_is_exact():
    """Powers of two as factors: every output is the integer sum itself, scaled."""
    for batch in (4, 30, 200, 513):
        c = _case(3, batch, 1, 1040, 136, 0, 1)
        c["alpha"].fill_(0.25)
        c["gamma"].fill_(127.0)
        want = (c["x"].double() @ c["w"].double().T) * 0.25
        assert torch.equal(_call(c, dtype=torch.float32).double(), want)


@pytest.mark.parametrize("batch", [5, 60, 300, 700])
def test_outputs_in_a_wider_buffer(batch):
    for out, pitch in ((torch.bfloat16, 448), (torch.float32, 404), (torch.float16, 401)):
        c = _case(batch + 1, batch, 1, 272, 392, 6, 16)
        size = torch.finfo(out).bits // 8
        buf = Guarded(batch * pitch * size, dtype=out, fill=3.0)
        y = buf.view(batch, pitch)[:, :392]
        _call(c, y=y)
        buf.check("y")
        assert bool((buf.view(batch, pitch)[:, 392:] == 3.0).all())
        assert torch.equal(y, _call(c, dtype=out))
        # a base that is aligned to its type alone
        flat = torch.full((batch * 392 + 8,), 3.0, dtype=out, device="cuda")
        odd = flat[1:1 + batch * 392].view(batch, 392)
        _call(c, y=odd)
        assert torch.equal(odd, y) and float(flat[0]) == 3.0 and bool((flat[1 + batch * 392:] == 3.0).all())


@pytest.mark.parametrize("batch", [6, 90, 400])
def test_values_that_are_not_finite(batch):
    """An adapter's bad values stay with its own samples; an index outside the table counts as none."""
    c = _case(17, batch, 1, 256, 264, 4, 16, share=1.0, order="mixed")
    which = torch.arange(batch, dtype=torch.int32, device="cuda") % 4
    c["which"] = which
    good = _call(c)
    d = dict(c, a=c["a"].clone(), b=c["b"].clone())
    d["a"][1, 3, 5] = float("nan")
    d["x"] = c["x"].clone()
    d["x"][:, 5] = 1
    ref = _call(dict(d, a=c["a"]))
    got = _call(d)
    rows = (which == 1)
    assert torch.isnan(got[rows]).all() and torch.equal(got[~rows], ref[~rows])
    assert binding.last_device_status() == binding.PROM_OK
    e = dict(c, b=c["b"].clone())
    e["b"][2, 7, 0] = float("inf")
    e["b"][2, 9, 1] = float("nan")
    zeroed = c["b"].clone()
    zeroed[2, 7, 0] = 0
    zeroed[2, 9, 1] = 0
    got = _call(e)
    assert binding.last_device_status() == binding.PROM_ERR_BAD_WEIGHT
    assert torch.equal(got, _call(dict(c, b=zeroed)))
    f = dict(c, which=which.clone())
    f["which"][0], f["which"][batch - 1] = 4, -2
    none = which.clone()
    none[0] = none[batch - 1] = -1
    got = _call(f)
    assert binding.last_device_status() == binding.PROM_ERR_RANGE
    assert torch.equal(got, _call(dict(c, which=none)))
    gm = dict(c, gamma=c["gamma"].clone())
    gm["gamma"][1] = float("nan")
    gm["gamma"][2] = 0.0
    got = _call(gm)
    assert torch.isnan(got[1]).all() and torch.equal(got[3:], good[3:]) and torch.equal(got[0], good[0])
    _check(got[2:3], dict(gm, batch=1, x=gm["x"][2:3], gamma=gm["gamma"][2:3], which=which[2:3]))
    # large adapters: inner products beyond what float16 holds
    h = _case(18, batch, 1, 256, 264, 4, 16, kind=torch.float16, share=1.0)
    h["a"] = torch.full_like(h["a"], 60000.0)
    h["b"] = h["b"] * 1e-3
    h["scale"].fill_(1e-6)
    _check(_call(h, dtype=torch.float32), h)


def test_an_invalid_weight_code_is_reported():
    for batch in (4, 300):
        c = _case(4, batch, 1, 64, 32, 2, 8)
        c["packed"] = c["packed"].clone()
        c["packed"][3, 5] = 0b10
        _call(c)
        assert binding.last_device_status() == binding.PROM_ERR_BAD_WEIGHT


@pytest.mark.parametrize("batch", [1, 24, 150, 520])
def test_after_the_norm_in_a_graph_and_on_streams(batch):
    """Norm to codes, projection with adapters, norm of the result: live, on another stream, and captured and replayed on
    other inputs, twice in one graph."""
    n, cout = 512, 768
    c = _case(batch, batch, 1, n, cout, 5, 16)
    h = torch.randn((batch, n), device="cuda").bfloat16()
    w, b = torch.randn(n, device="cuda"), torch.randn(n, device="cuda")

    def chain(stream=None):
        q, gamma, _ = binding.layer_norm_i8(h, w, b, stream=stream)
        y = binding.pw_proj_adapters(q, batch, c["packed"], cout, c["alpha"], gamma, c["a"], c["b"], c["scale"], c["which"], stream=stream)
        return q, gamma, y, binding.layer_norm(y, stream=stream)[0]

    live = chain()
    _check(live[2], dict(c, x=live[0], gamma=live[1]))
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    other = chain(side)
    side.synchronize()
    assert all(torch.equal(p, q) for p, q in zip(live, other))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        first, second = chain(), chain()
    h.copy_(torch.randn_like(h))
    c["which"].copy_(torch.randint(-1, 5, (batch,), device="cuda").int())
    for _ in range(3):
        graph.replay()
    torch.cuda.synchronize()
    live = chain()
    assert all(torch.equal(p, q) for p, q in zip(live, first)) and all(torch.equal(p, q) for p, q in zip(live, second))


def test_two_streams_at_once():
    cases = [_case(i, 300 + 40 * i, 1, 512, 512, 6, 16) for i in range(2)]
    want = [_call(c) for c in cases]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in cases]
    got = [[], []]
    for _ in range(20):
        for i, (c, s) in enumerate(zip(cases, streams)):
            got[i].append(_call(c, stream=s))
    torch.cuda.synchronize()
    for i in range(2):
        assert all(torch.equal(y, want[i]) for y in got[i])


def test_random_shapes():
    rng = np.random.default_rng(5)
    for k in range(40):
        rows = int(rng.choice([1, 1, 1, 17, 49]))
        batch = max(1, int(np.exp(rng.uniform(0, np.log(1500)))) // rows)
        cin, cout = 16 * int(rng.integers(1, 80)), 8 * int(rng.integers(1, 90))
        n, rank = int(rng.integers(1, 20)), int(rng.choice([1, 2, 4, 7, 8, 16, 20, 32, 40, 64, 72]))
        c = _case(900 + k, batch, rows, cin, cout, n, rank, kind=[torch.bfloat16, torch.float16][k % 2], order=["runs", "mixed"][k // 2 % 2])
        if k % 5 == 0:
            c["scale"] = None
        _check(_call(c, dtype=[torch.bfloat16, torch.float32, torch.float16][k % 3]), c, (k, batch, rows, cin, cout, n, rank))


@pytest.mark.parametrize("batch,cin,cout", [(1000, 144, 4096), (1000, 2064, 2304), (5000, 48, 4096), (2600, 400, 1048)])
def test_tiles_with_and_without_adapters_in_turn(batch, cin, cout):
    """Several tiles per pair of CTAs, of widths with one and with two accumulators of the adapters: tiles of many adapters, of one
    and of none behind each other."""
    c = _case(batch, batch, 1, cin, cout, 30, 16, order="mixed")
    tile = torch.arange(batch, device="cuda") // 256
    c["which"] = torch.where(tile % 3 == 0, c["which"], torch.where(tile % 3 == 1, -1, 7)).int()
    binding.debug_adapters(2)
    try:
        for out in (torch.bfloat16, torch.float32):
            y = _call(c, dtype=out)
            _check(y, c, (batch, cin, cout))
            assert all(torch.equal(y, _call(c, dtype=out)) for _ in range(3))
            c0 = {k: v for k, v in c.items() if k not in ("a", "b", "scale", "which")}
            _check(_call(c0, dtype=out), c0, (batch, cin, cout))
    finally:
        binding.debug_adapters()


@pytest.mark.parametrize("mode", [1, 2])
@pytest.mark.parametrize("row", [0, 137, 260, 1031])
def test_an_invalid_weight_code_in_any_tile(row, mode):
    c = _case(6, 700, 1, 176, 1032, 2, 8)
    c["packed"] = c["packed"].clone()
    c["packed"][row, 43] = 0b10000000
    binding.debug_adapters(mode)
    try:
        _call(c)
    finally:
        binding.debug_adapters()
    assert binding.last_device_status() == binding.PROM_ERR_BAD_WEIGHT


def test_refusals():
    c = _case(1, 12, 1, 64, 32, 2, 8)
    before = binding.launch_count()
    for key, bads in {"x": [c["x"].cpu(), c["x"].float(), c["x"].t()], "packed": [c["packed"][:16], c["packed"].int()],
                      "alpha": [c["alpha"][:5], c["alpha"].double()], "gamma": [c["gamma"][:3], c["gamma"].half()],
                      "a": [c["a"].float(), c["a"][:, :, :32], c["a"].half()], "b": [c["b"].half(), c["b"][:1], c["b"][:, :, :4]],
                      "scale": [c["scale"][:1]], "which": [c["which"].long(), c["which"][:4]]}.items():
        for bad in bads:
            with pytest.raises((ValueError, TypeError)):
                _call(dict(c, **{key: bad}))
    for y in (torch.empty((12, 33), device="cuda"), torch.empty((11, 32), device="cuda"), torch.empty((12, 32), device="cuda").double(),
              torch.empty((12, 32))):
        with pytest.raises(ValueError):
            _call(c, y=y)
    with pytest.raises(ValueError):
        _call(dict(c, batch=5))
    with pytest.raises(binding.PromError) as e:
        _call(c, workspace=torch.empty(16, dtype=torch.uint8, device="cuda"))
    assert e.value.code == binding.PROM_ERR_WORKSPACE
    assert binding.launch_count() == before
    empty = _call(dict(c, batch=0, x=c["x"][:0], gamma=c["gamma"][:0], which=c["which"][:0]))
    assert empty.shape == (0, 32)
