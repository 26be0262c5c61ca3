"""Decode over the 8-bit cache with queries and keys of extreme magnitudes, against 64 bits: their products are
ordinary numbers though one of the factors is near a type's limits."""

import numpy as np
import pytest
import torch

import _kv8 as R
from paper_2608_20397_amd import nexus as N

pytestmark = pytest.mark.gpu

t = torch.from_numpy


# exponents of the query's and the keys' scale: the scores are of the order of one in each
@pytest.mark.parametrize("q_exp,k_exp", [(118, -88), (120, -60), (121, -10), (-90, 110), (0, 0), (60, -60)])
@pytest.mark.parametrize("D,Hq,H,cap", [(64, 8, 2, 0.0), (128, 5, 1, 0.0), (128, 5, 1, 20.0), (256, 4, 2, 0.0),
                                        (256, 4, 2, 20.0)])
def test_decode_of_extreme_queries_and_keys(D, Hq, H, cap, q_exp, k_exp):
    n, lens = 4, [1, 70, 1333, 1500]
    n_map = (max(lens) + 15) // 16
    cache = R.make_cache(1, n_map, H, D, n_map, seed=D)
    k, v = (R.rows(600 + s, 1, max(lens), H, D, dtype="f32", spread=0.5) for s in (0, 1))
    N.kv8_splice(cache, N.Block(k * 2.0 ** k_exp, v, 0, 1e4), 0, 0)
    g = np.random.default_rng([20397, 92, D])
    q = t(g.standard_normal((n, Hq, D)) * 2.0 ** q_exp).to(torch.bfloat16).cuda()
    scale = float(D ** -0.5 * 2.0 ** -(q_exp + k_exp))
    pm = cache.page_map.cpu().numpy()
    kk, vv = (R.tokens(R.values(cache, x)[0], pm, 0, max(lens))[0] for x in ("k", "v"))
    # the sequences' own lengths, and a bound from which on a launch reads shared pages together
    for bound in (max(lens), 2 ** 29 // (n * H * D * 2)):
        maps = torch.zeros(n, (bound + 15) // 16, dtype=torch.int32, device="cuda")
        maps[:, :n_map] = cache.page_map
        got = R.f64(N.kv8_decode_attn(q, cache, maps, t(np.array(lens, np.int32)).cuda(), bound, 0, softcap=cap,
                                      scale=scale))
        for b, m in enumerate(lens):
            ref = R.attention(R.f64(q)[b:b + 1], kk[:m], vv[:m], [m], scale, cap)
            R.assert_attention(got[b:b + 1], ref, f"D={D} q 2^{q_exp} k 2^{k_exp} length {m} of {bound}")
    # the suffix kernel, whose scores carry the keys' scales from the start, agrees on the longest
    suffix = R.f64(N.kv8_suffix_attn(q[3:], cache, 0, max(lens) - 1, softcap=cap, scale=scale))
    R.assert_attention(suffix, ref, "suffix")
