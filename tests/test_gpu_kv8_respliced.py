"""Rows of an 8-bit cache read back and spliced again: the same values, and the bytes that the definition gives
of them (the largest code 224 = 448 / 2 is written as 448 under half the scale, once)."""

import numpy as np
import pytest
import torch

import _kv8 as R
from paper_2608_20397_amd import nexus as N

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("D", [64, 128, 256])
def test_bytes_of_rows_spliced_again(D, dtype):
    n = 200
    g = np.random.default_rng([20397, 91, D])
    r = g.standard_normal((n, D)) * 50
    r[:, 3] = np.linspace(216, 240, n) * np.where(np.arange(n) % 2, 1, -1)    # amax on both sides of (224, 232]
    r *= np.exp2(g.integers(-20, 20, (n, 1)))
    r[0], r[1, 5] = 0, np.nan
    x = torch.from_numpy(r).to(dtype).view(1, n, 1, D).cuda()

    def spliced(k, v):
        cache = R.make_cache(1, 16, 1, D, 14, seed=D)
        N.kv8_splice(cache, N.Block(k, v, 7, 1e4), 5, 7)
        pm = cache.page_map.cpu().numpy()
        raw = {m: (R.tokens(getattr(cache, m).view(torch.uint8).cpu().numpy(), pm, 5, n)[0, :, 0],
                   R.tokens(getattr(cache, m + "_scale").cpu().numpy(), pm, 5, n)[0, :, 0].astype(int))
               for m in ("k", "v")}
        return cache, raw

    first, raw1 = spliced(x, x.clone())
    second, raw2 = spliced(*N.kv8_read(first, 5, n, dtype))
    third, raw3 = spliced(*N.kv8_read(second, 5, n, dtype))
    a, b = (N.kv8_read(c, 5, n, torch.float32) for c in (first, second))
    for i, m in enumerate(("k", "v")):
        assert np.array_equal(R.f64(a[i]), R.f64(b[i]), equal_nan=True)
        (c1, s1), (c2, s2), (c3, s3) = raw1[m], raw2[m], raw3[m]
        y = np.abs(R.TABLE[c1]).max(-1)
        moved = (y == 224) & (s1 < 255)
        assert 20 < moved.sum() < n - 20
        assert np.array_equal(s2, s1 - moved)
        assert np.array_equal(R.TABLE[c2], R.TABLE[c1] * np.where(moved, 2, 1)[:, None], equal_nan=True)
        assert np.array_equal(c2[~moved], c1[~moved])
        assert np.array_equal(c3, c2) and np.array_equal(s3, s2)
