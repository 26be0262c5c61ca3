"""GPU parity of windowed attention where lengths, lists and launches are large: more pages than a workgroup lists at a
time, more sequences than a wave looks through, groups wider than a row tile, against the definition in 64 bits at
sampled rows."""

import math

import numpy as np
import pytest
import torch

from _batch import HALF, U, i32
from paper_2608_20397_amd import nexus as N

pytestmark = pytest.mark.gpu

B, F = torch.bfloat16, torch.float32


def _check(out, q, cache, maps, row, head, pos, window, sinks, cap=0.0):
    """One row and head against the definition, on the GPU in 64 bits."""
    dim, hkv = q.shape[2], cache.k.shape[2]
    h, dtype = head // (q.shape[1] // hkv), q.dtype
    key = torch.arange(pos + 1, device="cuda")
    key = key[(key > pos - window) | (key < sinks)]
    page, slot = maps[key // 16].long(), key % 16
    k = cache.k[0, page, h, slot].double()
    v = (cache.v[0, h][:, page * 16 + slot].T if cache.v_layout == N.V_TRANSPOSED else cache.v[0, page, h, slot]).double()
    x = q[row, head].double()
    s = k @ x / math.sqrt(dim)
    size = float((k.abs() @ x.abs()).max()) / math.sqrt(dim)
    if cap:
        s = cap * torch.tanh(s / cap)
    w = torch.softmax(s, 0)
    ref, mag = w @ v, w @ v.abs()
    fp32 = (2 * ((dim + 4) * size + 8 * cap) + len(key) + 64) * U
    weights = HALF[dtype] if dtype == B else 0.0
    bound = (weights + fp32) * (mag + ref.abs()) * 1.01 + HALF[dtype] * 1.01 * ref.abs()
    over = float(((out[row, head].double() - ref).abs() / bound).max())
    assert over <= 1, (row, head, over)


def _cache(n_phys, hkv, dim, dtype, vt, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    shape = (1, n_phys, hkv, 16, dim)
    k = torch.randn(shape, generator=g, device="cuda").to(dtype)
    v = torch.randn((1, hkv, dim, n_phys * 16) if vt else shape, generator=g, device="cuda").to(dtype)
    return N.PagedKVCache(k, v, i32([0]), 1e4, N.V_TRANSPOSED if vt else N.V_ROWMAJOR), g


@pytest.mark.parametrize("hkv,dim,rows,dtype,vt", [(32, 64, 2560, B, False), (32, 64, 2560, B, True),
                                                   (16, 128, 3968, B, False), (16, 256, 3840, B, True),
                                                   (16, 256, 3840, B, False), (4, 32, 2100, F, False)])
def test_more_pages_than_a_ring_holds(hkv, dim, rows, dtype, vt):
    """Runs of more than 32768 keys (2048 pages): so many row tiles that the keys are cut three times at most."""
    n = 140007
    n_pages = -(-n // 16)
    cache, g = _cache(n_pages, hkv, dim, dtype, vt, 1)
    maps = torch.randperm(n_pages, generator=g, device="cuda").to(torch.int32)
    q = torch.randn((rows, hkv, dim), generator=g, device="cuda").to(dtype)
    # (a split's partials: fp16 or fp32 rows and 16 bytes each)
    part = rows * hkv * (dim * (2 if dtype == B else 4) + 16)
    assert N.window_attn_workspace_bytes(cache, rows, hkv, 1, n, n, 0) <= 3 * part
    for window, sinks in ((n, 0), (130000, 77)):
        out = N.window_attn(q, cache, maps[None], i32([0, rows]), i32([n]), n, window, sinks, 0)
        for row in (0, 1, 127, 128, rows // 2 + 5, rows - 1):
            for head in (0, hkv - 1):
                _check(out, q, cache, maps, row, head, n - rows + row, window, sinks)


@pytest.mark.parametrize("hq,hkv,dim,dtype", [(8, 8, 64, B), (16, 8, 128, B), (8, 8, 32, F)])
def test_decode_lists_longer_than_lds(hq, hkv, dim, dtype):
    """Sequences over the same 50000 tokens: a workgroup's run is longer than its list in LDS."""
    n, n_seqs = 50000, 52
    n_pages = n // 16
    cache, g = _cache(n_pages, hkv, dim, dtype, False, 2)
    maps = torch.randperm(n_pages, generator=g, device="cuda").to(torch.int32)
    lens = [n - 37 * b for b in range(n_seqs)]
    q = torch.randn((n_seqs, hq, dim), generator=g, device="cuda").to(dtype)
    all_maps = maps[None].expand(n_seqs, -1).contiguous()
    for window, sinks in ((n, 0), (45000, 1000)):
        out = N.window_decode_attn(q, cache, all_maps, i32(lens), n, window, sinks, 0)
        for b in (0, 17, n_seqs - 1):
            for head in (0, hq - 1):
                _check(out, q, cache, maps, b, head, lens[b] - 1, window, sinks)


@pytest.mark.parametrize("dtype,dim", [(B, 64), (B, 256), (F, 16)])
def test_groups_wider_than_a_row_tile(dtype, dim):
    """300 query heads on one KV head: a token's rows go through several tiles."""
    n, rows, hq = 500, 5, 300
    cache, g = _cache(32, 1, dim, dtype, False, 3)
    maps = torch.randperm(32, generator=g, device="cuda").to(torch.int32)
    q = torch.randn((rows, hq, dim), generator=g, device="cuda").to(dtype)
    out = N.window_attn(q, cache, maps[None], i32([0, rows]), i32([n]), n, 100, 3, 0)
    dec = N.window_decode_attn(q[-1:].contiguous(), cache, maps[None], i32([n]), n, 100, 3, 0)
    for head in (0, 127, 128, 255, 256, 299):
        for row in range(rows):
            _check(out, q, cache, maps, row, head, n - rows + row, 100, 3)
        _check(dec, q[-1:], cache, maps, 0, head, n - 1, 100, 3)


def test_thousands_of_sequences():
    """More sequences than two looks of a wave find one in, some without rows."""
    n_seqs, hkv, dim = 5000, 2, 64
    rng = np.random.default_rng(4)
    fresh = rng.integers(0, 3, n_seqs)
    lens = fresh + rng.integers(0, 60, n_seqs)
    cache, g = _cache(600, hkv, dim, B, False, 5)
    maps = torch.randint(0, 600, (n_seqs, 4), generator=g, device="cuda", dtype=torch.int32)
    start = np.concatenate([[0], np.cumsum(fresh)])
    q = torch.randn((int(start[-1]), 4, dim), generator=g, device="cuda").to(B)
    out = N.window_attn(q, cache, maps, i32(start), i32(lens), 64, 20, 2, 0)
    for b in list(range(3)) + [63, 64, 65, 4095, 4096, 4097, n_seqs - 1] + rng.integers(0, n_seqs, 60).tolist():
        for i in range(fresh[b]):
            _check(out, q, cache, maps[b], int(start[b]) + i, 3, int(lens[b] - fresh[b]) + i, 20, 2)


@pytest.mark.parametrize("D,vt", [(64, False), (128, True), (256, True)])
def test_a_whole_sequence_of_nan_is_formed_again(D, vt):
    """Every value NaN: every row comes from the key-by-key way; the sequence beside it is untouched."""
    cache, g = _cache(40, 2, D, B, vt, 6)
    maps = torch.arange(40, device="cuda", dtype=torch.int32).view(2, 20)
    if vt:
        cache.v[..., :320] = float("nan")
    else:
        cache.v[:, :20] = float("nan")
    q = torch.randn((150, 4, D), generator=g, device="cuda").to(B)
    out = N.window_attn(q, cache, maps, i32([0, 100, 150]), i32([300, 311]), 320, 64, 4, 0)
    assert torch.isnan(out[:100]).all() and torch.isfinite(out[100:]).all()
    for row in (100, 131, 149):
        _check(out, q, cache, maps[1], row, 3, 311 - 150 + row, 64, 4)
