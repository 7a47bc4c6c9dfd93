"""The projection with adapters where the number of rows chooses the kernels: the same rows in a call of a few, and in tiles; and calls that
meet the library's state: many adapters, the first call of a process inside a capture, threads."""
import os
import subprocess
import sys
import threading

import pytest
import torch

from paper_2505_03254_b200 import binding, build

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _lib():
    build.build()
    binding.last_device_status()
    yield
    assert binding.last_device_status() == binding.PROM_OK


@pytest.mark.parametrize("kind", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("out", [torch.bfloat16, torch.float16, torch.float32])
@pytest.mark.parametrize("rank", [1, 16])
def test_an_adapter_that_takes_the_projection_away(kind, out, rank):
    """A's first row is a row of the weights and B is -alpha, a power of two: y is exactly zero in that output.  The inner products
    are whole numbers below 2^19, which binary32 holds: nothing of them may be lost, however many rows there are."""
    m, cin, cout = 300, 4096, 264
    g = torch.Generator().manual_seed(rank)
    x = torch.randint(-127, 128, (m, cin), generator=g).to(torch.int8)
    w = torch.randint(-1, 2, (cout, cin), generator=g).to(torch.int8)
    x[: m // 2] = (x[: m // 2].abs() * w[5]).to(torch.int8)         # sums up to 127 x 4096
    a = torch.zeros((2, rank, cin))
    b = torch.zeros((2, cout, rank))
    a[:, 0], b[:, 5, 0] = w[5].float(), -0.25
    which = (torch.arange(m) % 2).int()
    args = [t.cuda() for t in (a.to(kind), b.to(kind))] + [None, which.cuda()]
    alpha, gamma = torch.full((cout,), 0.25, device="cuda"), torch.full((m,), 127.0, device="cuda")
    packed = binding.pack_ternary(w.cuda())
    want = (x.double() @ w.double().T * 0.25).cuda().to(out)
    want[:, 5] = 0
    for mode in (1, 2):
        binding.debug_adapters(mode)
        try:
            y = binding.pw_proj_adapters(x.cuda(), m, packed, cout, alpha, gamma, *args, dtype=out)
        finally:
            binding.debug_adapters()
        assert torch.equal(y, want), (mode, int((y != want).sum()), float(y[:, 5].abs().max()))


@pytest.mark.parametrize("mode", [1, 2])
@pytest.mark.parametrize("kind", [torch.bfloat16, torch.float16])
def test_every_value_of_a_code(kind, mode):
    """All 256 values of x in every place of a word, through the weights and through an adapter that picks one value a rank."""
    m, cin, cout, rank = 260, 256, 64, 64
    x = ((torch.arange(m)[:, None] * 3 + torch.arange(cin)[None, :]) % 256 - 128).to(torch.int8)
    assert int(x.min()) == -128 and int(x.max()) == 127
    a, b = torch.zeros((1, rank, cin)), torch.zeros((1, cout, rank))
    for j in range(rank):
        a[0, j, 4 * j + j % 4] = b[0, j, j] = 1.0
    w = torch.randint(-1, 2, (cout, cin), generator=torch.Generator().manual_seed(8)).to(torch.int8)
    ones = torch.ones(cout, device="cuda")
    which = (torch.arange(m) % 3 != 0).int() - 1
    want = x.double() @ w.double().T + (x.double() @ a[0].double().T) * (which[:, None] >= 0)
    binding.debug_adapters(mode)
    try:
        y = binding.pw_proj_adapters(x.cuda(), m, binding.pack_ternary(w.cuda()), cout, ones, torch.full((m,), 127.0, device="cuda"),
                                     a.to(kind).cuda(), b.to(kind).cuda(), None, which.cuda(), dtype=torch.float32)
    finally:
        binding.debug_adapters()
    assert torch.equal(y.double().cpu(), want)


@pytest.mark.parametrize("mode", [1, 2])
def test_as_many_adapters_as_there_may_be(mode):
    n, m, cin, cout = 1 << 20, 300, 16, 8
    g = torch.Generator().manual_seed(9)
    x = torch.randint(-128, 128, (m, cin), generator=g).to(torch.int8)
    w = torch.randint(-1, 2, (cout, cin), generator=g).to(torch.int8)
    which = torch.randint(0, n, (m,), generator=g).int()
    which[::7], which[3], which[200] = -1, n - 1, n - 1
    a = (torch.arange(n, dtype=torch.float32)[:, None, None] % 251 - 125).expand(n, 1, cin).bfloat16().cuda()
    b = torch.ones((n, cout, 1), dtype=torch.bfloat16, device="cuda")
    t = x.double().sum(1) * (which.double() % 251 - 125) * (which >= 0)
    binding.debug_adapters(mode)
    try:
        y = binding.pw_proj_adapters(x.cuda(), m, binding.pack_ternary(w.cuda()), cout, torch.ones(cout, device="cuda"),
                                     torch.full((m,), 127.0, device="cuda"), a, b, None, which.cuda(), dtype=torch.float32)
    finally:
        binding.debug_adapters()
    assert torch.equal(y.double().cpu(), x.double() @ w.double().T + t[:, None])


FIRST = """
import sys, torch
from paper_2505_03254_b200 import binding
m = int(sys.argv[1])
g = torch.Generator(device="cuda").manual_seed(1)
h = torch.randn((m, 512), device="cuda", generator=g).bfloat16()
w = torch.randint(-1, 2, (768, 512), device="cuda", generator=g).to(torch.int8)
a = (torch.randn((4, 16, 512), device="cuda", generator=g) / 22).bfloat16()
b = torch.randn((4, 768, 16), device="cuda", generator=g).bfloat16()
which, alpha, packed = torch.arange(m, device="cuda").int() % 5 - 1, torch.ones(768, device="cuda"), binding.pack_ternary(w)
def chain():
    q, gamma, _ = binding.layer_norm_i8(h)
    y = binding.pw_proj_adapters(q, m, packed, 768, alpha, gamma, a, b, None, which)
    n, mean, rstd = binding.layer_norm(y)
    return q, y, n, *binding.layer_norm_backward(n, y, None, mean, rstd)
graph = torch.cuda.CUDAGraph()
with torch.cuda.graph(graph):
    first = chain()
graph.replay()
torch.cuda.synchronize()
live = chain()
assert all(torch.equal(p, q) for p, q in zip(first, live)) and torch.isfinite(live[1].float()).all()
assert binding.last_device_status() == binding.PROM_OK
print("same")
"""


@pytest.mark.parametrize("m", [3, 1300])
def test_the_first_calls_of_a_process_are_captured(m):
    """What a kernel needs once (limits, occupancy, its code) is had while a graph is being captured."""
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    r = subprocess.run([sys.executable, "-c", FIRST, str(m)], cwd=root, capture_output=True, text=True, timeout=300)
    assert r.returncode == 0 and r.stdout.strip().endswith("same"), r.stderr[-2000:]


def test_two_threads_at_once():
    """The interpreter's lock is released inside a call: threads with streams of their own share nothing but the library."""
    m, results = 700, {}
    g = torch.Generator(device="cuda").manual_seed(3)
    h = torch.randn((2, m, 512), device="cuda", generator=g).bfloat16()
    w = torch.randint(-1, 2, (640, 512), device="cuda", generator=g).to(torch.int8)
    a = (torch.randn((4, 16, 512), device="cuda", generator=g) / 22).bfloat16()
    b = torch.randn((4, 640, 16), device="cuda", generator=g).bfloat16()
    which, alpha, packed = torch.arange(m, device="cuda").int() % 5 - 1, torch.ones(640, device="cuda"), binding.pack_ternary(w)

    def chain(x, stream=None):
        q, gamma, _ = binding.layer_norm_i8(x, stream=stream)
        y = binding.pw_proj_adapters(q, m, packed, 640, alpha, gamma, a, b, None, which, stream=stream)
        n, mean, rstd = binding.layer_norm(y, stream=stream)
        return y, n, *binding.layer_norm_backward(n, y, None, mean, rstd, stream=stream)

    want = [chain(x) for x in h]
    torch.cuda.synchronize()

    def work(i):
        stream = torch.cuda.Stream()
        results[i] = [chain(h[i], stream) for _ in range(60)]
        stream.synchronize()

    threads = [threading.Thread(target=work, args=(i,)) for i in range(2)]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    for i in range(2):
        assert len(results[i]) == 60 and all(torch.equal(p, q) for got in results[i] for p, q in zip(got, want[i]))
