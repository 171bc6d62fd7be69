"""The ends of what a quantised decoder layer's calls accept, on the GPU."""
import numpy as np
import pytest
import torch

from decoder_reference import Cache, attention
from paper_2304_09049_amd import binding as dg

pytestmark = pytest.mark.gpu


def on_gpu(x):
    return torch.from_numpy(np.ascontiguousarray(x)).cuda()


@pytest.mark.parametrize("page_size,dim,bits", [(2097152, 256, 8), (4194304, 128, 8), (4194304, 256, 4), (8388608, 64, 4)])
def test_one_large_page(page_size, dim, bits):
    """A page whose codes' bits are more than 32-bit numbers count: tokens at both of its ends, among their neighbours' bytes, and attention over the first ones."""
    desc = dg.cache_desc(1, page_size, 1, dim, bits)
    cache = torch.zeros(dg.dg_cache_bytes(desc), dtype=torch.uint8, device="cuda")
    t = np.r_[0:33, page_size // 2 - 5:page_size // 2 + 9, page_size - 37:page_size]
    k, v = (torch.randn(len(t), 1, dim, generator=torch.Generator().manual_seed(i)).half() for i in range(2))
    dg.dg_cache_write(desc, cache, k.cuda(), v.cuda(), on_gpu(t.astype(np.int32)))
    small = Cache(1, len(t) // 16 * 16 + 16, 1, dim, bits)
    small.write(np.arange(len(t)), k.float().numpy(), v.float().numpy())
    want = small.read(np.arange(len(t)))
    for got, x in zip(dg.dg_cache_read(desc, cache, on_gpu(t.astype(np.int32))), want):
        assert np.array_equal(got.cpu().numpy(), x)
    # each code's byte and each scale where the header's formulas have them
    part, step, d = page_size * dim * bits // 8, dim * bits // 8, np.arange(0, dim, 8 // bits)
    key = (t[:, None] // 16) * 2 * bits * dim + (d // 16) * 32 * bits + (t[:, None] % 16) * 2 * bits + (d % 16) * bits // 8
    value = part + (t[:, None] // 4) * 4 * step + (d * bits // 8) * 4 + t[:, None] % 4
    for i, place in enumerate((key, value)):
        got = cache[on_gpu(place.reshape(-1)).long()].cpu().numpy().reshape(place.shape)
        assert np.array_equal(got, np.stack([small.bytes[small._places(n)[i]] for n in range(len(t))]))
        scale = cache.view(torch.float32)[on_gpu((2 * part + 4 * (i * page_size + t)) // 4).long()].cpu().numpy()
        assert np.array_equal(scale, np.stack([small._number(0, n, i) for n in range(len(t))]).copy().view(np.float32)[:, 0])
    q = torch.randn(3, 2, dim, generator=torch.Generator().manual_seed(2)).half()
    out = dg.dg_paged_attention(desc, cache, q.cuda(), on_gpu(np.array([0, 3], np.int32)), on_gpu(np.array([33], np.int32)),
                                torch.zeros(1, 1, dtype=torch.int32, device="cuda"), 3, 33)
    exact, off = attention(q.float().numpy(), want[0][:33], want[1][:33], 30, dim ** -0.5, True, 2.0 ** -11)
    assert (np.abs(out.float().cpu().numpy() - exact) <= off).all()
