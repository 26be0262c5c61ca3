"""Page maps made under torch.inference_mode, which keep no version counter: the calls that check their map take
them, and see every change of them."""

import numpy as np
import pytest
import torch

import _kv8 as R
from paper_2608_20397_amd import nexus as N

pytestmark = pytest.mark.gpu


def test_maps_of_inference_mode():
    with torch.inference_mode():
        cache = R.make_cache(1, 8, 2, 64, 4, seed=5)
        k, v = (R.rows(s, 1, 40, 2, 64) for s in (1, 2))
        N.kv8_append(cache, k, v, 3, 3)
        a, b = N.kv8_read(cache, 3, 40, torch.float32)
        assert np.array_equal(R.f64(b), R.quantise(R.f64(v))[0])
        q = R.rows(3, 40, 4, 64, spread=0.0)
        N.kv8_append(cache, k[:, :3].contiguous(), v[:, :3].contiguous(), 0, 0)
        got = N.kv8_suffix_attn(q, cache, 0, 3)
        kk, vv = (R.f64(t)[0] for t in N.kv8_read(cache, 0, 43, torch.float32))
        R.assert_attention(R.f64(got), R.attention(R.f64(q), kk, vv, 4 + np.arange(40), 64 ** -0.5, 0), "suffix")
        cache.page_map[2] = 8                              # past the cache's pages
        for call in (lambda: N.kv8_append(cache, k, v, 3, 3), lambda: N.kv8_read(cache, 0, 1),
                     lambda: N.kv8_suffix_attn(q, cache, 0, 3)):
            with pytest.raises(N.NexusError) as e:
                call()
            assert e.value.status == N.ERANGE
        paged = N.PagedKVCache(*(torch.zeros(1, 8, 2, 16, 64, dtype=torch.bfloat16, device="cuda") for _ in range(2)),
                               torch.arange(4, dtype=torch.int32, device="cuda"), 1e4)
        assert paged.pt().n_logical_pages == 4
        paged.page_map[0] = 1                              # named twice
        with pytest.raises(N.NexusError):
            paged.pt()
