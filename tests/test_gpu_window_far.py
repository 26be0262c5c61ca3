"""GPU parity of the append and of windowed attention in caches as large as a layer may be, just under 2^31 elements: pages
at the cache's end and on both sides of 2^31 and 2^32 bytes, in a layer behind another, against the definition in 64 bits
at sampled rows."""

import pytest
import torch

from _batch import PAGE, f64, i32, norm_rope, norm_rope_bound, within
from paper_2608_20397_amd import nexus as N
from test_gpu_window_long import _check

pytestmark = pytest.mark.gpu

B, F = torch.bfloat16, torch.float32


@pytest.mark.parametrize("hq,hkv,dim,dtype", [(8, 1, 64, B), (40, 8, 128, B), (4, 1, 128, B), (4, 2, 256, B), (2, 1, 256, B),
                                              (4, 1, 32, F), (4, 2, 128, F), (3, 1, 256, F)])
@pytest.mark.parametrize("vt", [False, True])
def test_pages_at_the_end_of_a_large_cache(hq, hkv, dim, dtype, vt):
    n_phys = (1 << 31) // (PAGE * hkv * dim) - 1
    n, rows, window, sinks = 700, 40, 300, 5
    g = torch.Generator(device="cuda").manual_seed(dim + hkv)
    shape = (2, n_phys, hkv, PAGE, dim)
    k = torch.empty(shape, dtype=dtype, device="cuda")
    v = torch.empty((2, hkv, dim, n_phys * PAGE) if vt else shape, dtype=dtype, device="cuda")
    cache = N.PagedKVCache(k, v, i32([0]), 1e6, N.V_TRANSPOSED if vt else N.V_ROWMAJOR)
    # pages of the sequence: the last ones, those around the halves and quarters of the layer, the first
    some = torch.cat([torch.arange(n_phys - 12, n_phys), n_phys // 2 + torch.arange(-6, 6),
                      n_phys // 4 + torch.arange(-6, 6), 3 * n_phys // 4 + torch.arange(-4, 4), torch.arange(6)])
    pages = some[torch.randperm(len(some), generator=torch.Generator().manual_seed(1))][:-(-n // PAGE)]
    maps = pages.to(torch.int32).cuda()[None].contiguous()
    slot = (pages[:, None] * PAGE + torch.arange(PAGE)).view(-1)[:n]
    # the tokens through the append, as a round writes them
    x = torch.randn((n, hq + 2 * hkv, dim), generator=g, device="cuda").to(dtype)
    q, kn, vn = x.split((hq, hkv, hkv), 1)
    got = N.norm_rope_append(cache, 1, q, kn, vn, i32(range(n)), i32(slot), eps=1e-6)
    ref, both = norm_rope(f64(q), None, 1e-6, range(n), 1e6, False)
    within(f64(got), ref, norm_rope_bound(ref, both, dtype, 1e-6), "queries")
    ref, both = norm_rope(f64(kn), None, 1e-6, range(n), 1e6, False)
    at = slot.cuda()
    within(f64(k[1, at // PAGE, :, at % PAGE]), ref, norm_rope_bound(ref, both, dtype, 1e-6), "keys")
    held = v[1].permute(2, 0, 1)[at] if vt else v[1, at // PAGE, :, at % PAGE]
    assert torch.equal(held, vn)
    # attention of the last rows, and of the last one as a decode step
    layer = N.PagedKVCache(k[1:], v[1:], i32([0]), 1e6, cache.v_layout)
    last = got[-rows:].contiguous()
    out = N.window_attn(last, cache, maps, i32([0, rows]), i32([n]), n, window, sinks, 1)
    step = N.window_decode_attn(last[-1:].contiguous(), cache, maps, i32([n]), n, window, sinks, 1)
    for row in (0, 7, rows - 1):
        for head in (0, hq - 1):
            _check(out, last, layer, maps[0], row, head, n - rows + row, window, sinks)
    for head in (0, hq - 1):
        _check(step, last[-1:], layer, maps[0], 0, head, n - 1, window, sinks)
