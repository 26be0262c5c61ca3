"""GPU parity of windowed attention, its keys in one piece and in several whose results are merged, where values are near
the largest and the smallest numbers of their type: a finite result is finite however the keys are cut, and keeps its
digits."""

import numpy as np
import pytest
import torch

from _batch import Paged, f64, i32, window_bound, within
from paper_2608_20397_amd import nexus as N

pytestmark = pytest.mark.gpu

B, F = torch.bfloat16, torch.float32
TOP = 3.3e38

FORMS = [(8, 2, 64, B, False, 0.0), (8, 2, 64, B, True, 20.0), (8, 2, 128, B, False, 0.0), (8, 2, 128, B, True, 0.0),
         (4, 2, 256, B, False, 0.0), (4, 2, 256, B, True, 50.0), (4, 2, 32, F, False, 0.0), (4, 2, 128, F, True, 0.0),
         (4, 2, 256, F, False, 20.0)]


def bound_of(ref, parts, dtype):
    """window_bound with what is lost below the smallest normal numbers in place of its floor: half a step of the result
    there (2^-134 in bf16, 2^-150 in fp32) and a step of 2^-149 for each of the sum's terms."""
    floor = (2.0 ** -134 if dtype == B else 2.0 ** -150) + (parts[2][:, None, None] + 64) * 2.0 ** -149
    return window_bound(ref, parts, dtype) - 1e-37 + floor


def run(pg, rows, n, hq, window=1 << 30, sinks=0, cap=0.0, split=None):
    q = torch.randn((rows, hq, pg.k.shape[3]), generator=torch.Generator().manual_seed(1)).to(pg.dtype)
    cache, maps = pg.device()
    if rows > 1:
        size = N.window_attn_workspace_bytes(cache, rows, hq, 1, n, window, sinks)
        got = N.window_attn(q.cuda(), cache, maps, i32([0, rows]), i32([n]), n, window, sinks, 0, softcap=cap)
    else:
        size = N.window_decode_attn_workspace_bytes(cache, 1, hq, n, window, sinks)
        got = N.window_decode_attn(q.cuda(), cache, maps, i32([n]), n, window, sinks, 0, softcap=cap)
    assert split is None or (size > 0) == split
    ref, parts = pg.exact(q, [0, rows], window, sinks, softcap=cap)
    return f64(got), ref, parts


@pytest.mark.parametrize("hq,hkv,dim,dtype,vt,cap", FORMS)
@pytest.mark.parametrize("rows", [1, 5])
@pytest.mark.parametrize("n", [20, 2100])
@pytest.mark.parametrize("size", [1e-36, 1e-30, 2e35, 1e36, 1e38])
def test_magnitudes(hq, hkv, dim, dtype, vt, cap, rows, n, size):
    pg = Paged([n], hkv, dim, dtype, vt, seed=3)
    pg.v = (pg.v.double() * size).clamp(-TOP, TOP).to(dtype)
    got, ref, parts = run(pg, rows, n, hq, cap=cap, split=n > 20)
    assert np.isfinite(ref).all()
    within(got, ref, bound_of(ref, parts, dtype), f"size {size} rows {rows} of {n}")


@pytest.mark.parametrize("hq,hkv,dim,dtype,vt,cap", FORMS)
@pytest.mark.parametrize("rows", [1, 5])
def test_pieces_of_unlike_magnitude(hq, hkv, dim, dtype, vt, cap, rows):
    """The first third of the keys' values near the top of the range, the last near its bottom: pieces whose powers of two
    lie 2^240 apart in one merge."""
    n = 2100
    pg = Paged([n], hkv, dim, dtype, vt, seed=4)
    for page, size in enumerate([1e37] * 44 + [1.0] * 44 + [1e-35] * 44):
        x = pg.v[pg.maps[0, page]].double() * size
        pg.v[pg.maps[0, page]] = x.to(dtype)
    got, ref, parts = run(pg, rows, n, hq, cap=cap, split=True)
    within(got, ref, bound_of(ref, parts, dtype), f"unlike pieces, rows {rows}")
    # ... of a window that only the last ones are in
    got, ref, parts = run(pg, rows, n, hq, window=600, cap=cap)
    within(got, ref, bound_of(ref, parts, dtype), f"the last pieces, rows {rows}")


@pytest.mark.parametrize("hq,hkv,dim,dtype,vt,cap", FORMS)
@pytest.mark.parametrize("rows", [1, 5])
def test_infinite_values_in_one_piece(hq, hkv, dim, dtype, vt, cap, rows):
    """An infinity in one piece beside large finite values in the others reaches its feature and no other."""
    n = 2100
    pg = Paged([n], hkv, dim, dtype, vt, seed=5)
    pg.v = (pg.v.double() * 1e36).to(dtype)
    pg.v[pg.maps[0, 7], 1, 3, 9] = float("inf")
    got, ref, parts = run(pg, rows, n, hq, cap=cap, split=True)
    assert np.isinf(ref[:, hq // 2:, 9]).all() and np.isfinite(np.delete(ref, 9, 2)).all()
    with np.errstate(all="ignore"):
        bound = bound_of(ref, parts, dtype)
    within(got, ref, bound, f"an infinity, rows {rows}")
