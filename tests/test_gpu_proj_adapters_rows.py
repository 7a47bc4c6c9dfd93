"""The projection with adapters where the number of rows chooses the kernels: the same rows in a call of a few, and in tiles."""
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
