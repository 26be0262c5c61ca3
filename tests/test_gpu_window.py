"""GPU parity of windowed attention with sinks (many rows a sequence, and a decode step) against its definition in 64
bits: lengths from one token on, windows and sinks at page and tile borders, windows that leave pages, unseen places
that hold NaN, bf16 and fp32, every head_dim, both V layouts, soft caps, 1 to 32 query heads per KV head."""

import numpy as np
import pytest
import torch

from _batch import Paged, f64, i32, window_bound, within
from paper_2608_20397_amd import nexus as N

pytestmark = pytest.mark.gpu

B, F = torch.bfloat16, torch.float32


def run(batch, window, sinks, *, hq, hkv, dim, dtype=B, vt=False, cap=0.0, scale=0.0, seed=0, pad=0, max_len=None,
        std=1.0, layers=1, layer=0):
    """batch: (cached, fresh) of each sequence."""
    lens = [c + f for c, f in batch]
    q_start = np.concatenate([[0], np.cumsum([f for _, f in batch])])
    pg = Paged(lens, hkv, dim, dtype, vt, seed, layers=layers, layer=layer)
    pg.forget(q_start, window, sinks)
    g = torch.Generator().manual_seed(seed + 1)
    q = (std * torch.randn((int(q_start[-1]) + pad, hq, dim), generator=g)).to(dtype)
    cache, maps = pg.device()
    out = torch.full(q.shape, 7.0, dtype=dtype, device="cuda")
    got = N.window_attn(q.cuda(), cache, maps, i32(q_start), i32(lens), max_len or max(1, max(lens)), window, sinks,
                        layer, softcap=cap, scale=scale, out=out)
    torch.cuda.synchronize()
    ref, parts = pg.exact(q, q_start, window, sinks, softcap=cap, scale=scale, out=np.full(q.shape, 7.0))
    n = int(q_start[-1])
    what = f"{batch[:4]} window {window} sinks {sinks} heads {hq}/{hkv}/{dim} {dtype} vt {vt} cap {cap}"
    within(f64(got)[:n], ref[:n], window_bound(ref, parts, dtype)[:n], what)
    assert (f64(got)[n:] == 7.0).all(), "rows of no sequence changed"


BORDERS = [
    ([(0, 1)], 1, 0), ([(0, 1)], 64, 4), ([(5, 1)], 1, 0), ([(5, 1)], 2, 1), ([(40, 3)], 16, 0),
    ([(300, 1)], 64, 4), ([(300, 70)], 64, 4), ([(300, 70)], 1, 1), ([(0, 200)], 33, 17),
    ([(0, 200)], 1000, 0), ([(1000, 129)], 1000, 16), ([(1000, 2)], 256, 130), ([(511, 65)], 128, 64),
    ([(70, 1), (0, 0), (0, 33), (513, 2), (16, 16), (15, 1)], 48, 5),
    ([(0, 0), (200, 31), (0, 0), (0, 1), (0, 0)], 100, 0),
]


@pytest.mark.parametrize("batch,window,sinks", BORDERS)
def test_borders_bf16(batch, window, sinks):
    run(batch, window, sinks, hq=10, hkv=2, dim=128, pad=3)


@pytest.mark.parametrize("batch,window,sinks", BORDERS)
def test_borders_f32(batch, window, sinks):
    run(batch, window, sinks, hq=6, hkv=2, dim=32, dtype=F, pad=2)


FORMS = [
    (8, 8, 64, B, False, 0.0), (8, 2, 64, B, True, 0.0), (64, 2, 64, B, False, 0.0), (8, 2, 64, B, True, 30.0),
    (4, 4, 128, B, False, 20.0), (5, 1, 128, B, True, 0.0), (10, 2, 128, B, True, 50.0), (40, 8, 128, B, False, 0.0),
    (4, 2, 256, B, False, 0.0), (4, 2, 256, B, True, 50.0), (4, 2, 256, B, True, 0.0), (2, 1, 256, B, False, 50.0),
    (4, 1, 16, F, False, 0.0), (4, 2, 16, F, True, 0.0), (6, 2, 32, F, True, 20.0), (4, 1, 64, F, False, 0.0),
    (34, 2, 64, F, False, 0.0), (5, 1, 128, F, True, 0.0), (4, 2, 128, F, False, 10.0), (4, 2, 256, F, False, 0.0),
    (3, 1, 256, F, True, 50.0),
]


@pytest.mark.parametrize("hq,hkv,dim,dtype,vt,cap", FORMS)
def test_forms(hq, hkv, dim, dtype, vt, cap):
    kw = dict(hq=hq, hkv=hkv, dim=dim, dtype=dtype, vt=vt, cap=cap)
    run([(333, 75), (0, 37), (90, 1), (7, 0), (150, 18)], 97, 5, seed=3, pad=1, **kw)
    run([(100, 130), (0, 1)], 100000, 0, seed=4, **kw)


@pytest.mark.parametrize("dim,vt,cap", [(16, False, 0.0), (32, True, 10.0), (64, False, 0.0), (64, True, 0.0),
                                        (128, False, 20.0), (128, True, 0.0), (256, False, 0.0), (256, True, 50.0)])
def test_many_fp32_workgroups(dim, vt, cap):
    """More of them than run together: fewer waves each, two where lists are short, four where they are long."""
    few = [(20 + b % 31, 1 + b % 24) for b in range(60)]
    run(few, 40, 3, hq=8, hkv=8, dim=dim, dtype=F, vt=vt, cap=cap, seed=31, pad=2)
    run([(7 * b, 300 - 5 * b) for b in range(6)] + [(350, 3)], 290, 3, hq=8, hkv=8, dim=dim, dtype=F, vt=vt, cap=cap,
        seed=32)


@pytest.mark.parametrize("vt,cap", [(False, 0.0), (True, 0.0), (True, 20.0), (False, 20.0)])
def test_long_lists_of_many_fp32_workgroups(vt, cap):
    """Two blocks of pairs a workgroup: blocks that are full, begun, empty; windows whose edge lies in one block."""
    batch = [(500, 45)] + [(3 * b % 40, 1 + 7 * b % 48) for b in range(63)] + [(0, 540)]
    run(batch, 1000, 0, hq=8, hkv=8, dim=128, dtype=F, vt=vt, cap=cap, seed=35, pad=3)
    run(batch, 510, 5, hq=16, hkv=8, dim=128, dtype=F, vt=vt, cap=cap, seed=36)


def test_long_lists_with_values_that_are_not_finite():
    """... in keys and values that the second block sees and the first does not."""
    lens, q_start = [560] + [30] * 60, [0, 700] + [700 + 10 * b for b in range(1, 61)]
    pg = Paged(lens, 8, 128, F, True, seed=37)
    pg.v[pg.maps[0, 20], 3, 5, 17] = float("inf")
    pg.k[pg.maps[7, 1], 2, 8, 4] = float("nan")
    q = torch.randn((q_start[-1], 8, 128), generator=torch.Generator().manual_seed(38)).to(F)
    cache, maps = pg.device()
    got = N.window_attn(q.cuda(), cache, maps, i32(q_start), i32(lens), 560, 1000, 0, 0)
    ref, parts = pg.exact(q, q_start, 1000, 0)
    assert np.isinf(ref).any() and np.isnan(ref).any()
    with np.errstate(all="ignore"):
        bound = window_bound(ref, parts, F)
    within(f64(got), ref, bound, "not finite")


def test_many_fp32_workgroups_with_values_that_are_not_finite():
    lens = [40 + b for b in range(60)]
    q_start = [20 * b for b in range(61)]
    pg = Paged(lens, 8, 32, F, False, seed=33)
    for b in range(0, 60, 7):
        n = lens[b] - 5
        pg.v[pg.maps[b, n // 16], b % 8, n % 16, b % 32] = float("inf")
    q = torch.randn((1200, 8, 32), generator=torch.Generator().manual_seed(34)).to(F)
    cache, maps = pg.device()
    got = N.window_attn(q.cuda(), cache, maps, i32(q_start), i32(lens), 99, 30, 2, 0)
    ref, parts = pg.exact(q, q_start, 30, 2)
    assert np.isinf(ref).any() and not np.isnan(ref).any()
    with np.errstate(all="ignore"):
        bound = window_bound(ref, parts, F)
    within(f64(got), ref, bound, "not finite")


def test_peaked_scores_and_scale():
    """Scores of standard deviation about 11 (the running maximum moves), a scale of its own, another layer."""
    run([(200, 100)], 150, 3, hq=8, hkv=2, dim=128, std=11.0, seed=5)
    run([(200, 100)], 150, 3, hq=4, hkv=2, dim=64, dtype=F, std=6.0, seed=5)
    run([(200, 100)], 150, 3, hq=8, hkv=2, dim=128, scale=0.3, seed=6, layers=3, layer=2)


def test_many_sequences():
    """More sequences than a wave looks through at a time, and rows that start behind row 0."""
    rng = np.random.default_rng(8)
    batch = [(int(rng.integers(0, 90)), int(rng.integers(0, 4))) for _ in range(300)]
    run(batch, 40, 2, hq=4, hkv=1, dim=64, pad=5)
    run(batch[:150], 40, 2, hq=4, hkv=1, dim=32, dtype=F)


@pytest.mark.parametrize("dtype,dim", [(B, 128), (F, 64)])
def test_bound_above_the_lengths(dtype, dim):
    """max_seq_len far above what the sequences hold: many splits, most of them empty."""
    run([(30, 2)], 4096, 4, hq=4, hkv=2, dim=dim, dtype=dtype, max_len=16 * 2)
    lens, q_start = [32, 500], [0, 2, 5]
    pg = Paged(lens, 2, dim, dtype, seed=9, stride=600)
    cache, maps = pg.device()
    q = torch.randn((5, 4, dim), generator=torch.Generator().manual_seed(1)).to(dtype)
    got = N.window_attn(q.cuda(), cache, maps, i32(q_start), i32(lens), 9600, 7000, 4, 0)
    ref, parts = pg.exact(q, q_start, 7000, 4)
    within(f64(got), ref, window_bound(ref, parts, dtype), "empty splits")
    dec = N.window_decode_attn(q[:2].cuda(), cache, maps, i32(lens), 9600, 7000, 4, 0)
    ref, parts = pg.exact(q[:2], [0, 1, 2], 7000, 4)
    within(f64(dec), ref, window_bound(ref, parts, dtype), "empty splits, decode")


DECODE = [
    ([1], 1, 0), ([1, 0, 17], 16, 4), ([300, 16, 15, 33], 64, 4), ([1000, 999, 17, 0, 1], 100, 1),
    ([2049, 700], 1024, 130), ([900, 901, 902, 903, 904], 897, 3), ([5000], 4096, 4), ([260, 10], 1 << 20, 0),
    ([1100, 33], 1, 0), ([1100, 33], 2, 16),
]


@pytest.mark.parametrize("lens,window,sinks", DECODE)
@pytest.mark.parametrize("hq,hkv,dim,dtype,vt,cap", [(10, 2, 128, B, False, 0.0), (32, 1, 64, B, False, 0.0),
                                                     (4, 2, 64, B, True, 30.0), (4, 2, 256, B, True, 50.0),
                                                     (10, 2, 128, B, True, 0.0), (2, 2, 256, B, False, 0.0),
                                                     (6, 2, 32, F, False, 0.0), (20, 1, 64, F, True, 20.0)])
def test_decode(lens, window, sinks, hq, hkv, dim, dtype, vt, cap):
    pg = Paged(lens, hkv, dim, dtype, vt, seed=len(lens) + window)
    q_start = list(range(len(lens) + 1))
    rows = [0]
    for n in lens:
        rows.append(rows[-1] + (n > 0))
    pg.forget(rows, window, sinks)
    q = torch.randn((len(lens), hq, dim), generator=torch.Generator().manual_seed(2)).to(dtype)
    cache, maps = pg.device()
    got = N.window_decode_attn(q.cuda(), cache, maps, i32(lens), max(lens), window, sinks, 0, softcap=cap)
    torch.cuda.synchronize()
    ref, parts = pg.exact(q, q_start, window, sinks, softcap=cap)
    within(f64(got), ref, window_bound(ref, parts, dtype), f"decode {lens} {window} {sinks}")
    for b, n in enumerate(lens):
        if n == 0:
            assert (f64(got)[b] == 0).all()


@pytest.mark.parametrize("dtype,dim,vt", [(B, 64, False), (B, 128, False), (B, 128, True), (B, 256, True),
                                          (F, 64, False), (F, 32, True)])
def test_values_that_are_not_finite_stay_with_their_queries(dtype, dim, vt):
    """Infinities and NaN in keys and values at places that some rows of a tile see and others do not: ahead of a row,
    behind its window, in a page's middle; a sequence beside it has none of it."""
    batch, window, sinks, hq, hkv = [(100, 60), (30, 20)], 50, 3, 4, 2
    lens, q_start = [160, 50], [0, 60, 80]
    pg = Paged(lens, hkv, dim, dtype, vt, seed=11)
    at = lambda n: (pg.maps[0, n // 16], n % 16)  # noqa: E731
    for n, head, what, value in ((159, 0, pg.v, float("inf")), (130, 1, pg.v, float("nan")), (53, 0, pg.v, -float("inf")),
                                 (140, 0, pg.k, float("nan")), (70, 1, pg.v, float("inf")),
                                 (75, 1, pg.v, -float("inf"))):
        page, slot = at(n)
        what[page, head, slot, n % dim] = value
    q = torch.randn((80, hq, dim), generator=torch.Generator().manual_seed(3)).to(dtype)
    cache, maps = pg.device()
    got = N.window_attn(q.cuda(), cache, maps, i32(q_start), i32(lens), 160, window, sinks, 0)
    ref, parts = pg.exact(q, q_start, window, sinks)
    assert np.isnan(ref).any() and np.isinf(ref).any() and np.isfinite(ref[60:]).all()
    with np.errstate(all="ignore"):
        bound = window_bound(ref, parts, dtype)
    # (an element whose own feature is finite has a finite bound: the weights are)
    within(f64(got), ref, bound, "not finite")


@pytest.mark.parametrize("dtype,dim,vt", [(B, 64, False), (B, 64, True), (B, 128, False), (B, 256, True), (F, 64, False)])
@pytest.mark.parametrize("lens", [[37, 1, 20], [3000, 37, 20]])
def test_values_that_are_not_finite_in_a_decode_step(dtype, dim, vt, lens):
    """An infinite last value (whose page's other places are read as it), one in the sinks, a key of NaN: in features
    and sequences that see them, whole or split."""
    window, sinks, hq, hkv = 2048, 2, 6, 2
    pg = Paged(lens, hkv, dim, dtype, vt, seed=21)
    inf = float("inf")
    for b, n, head, what, value in ((0, lens[0] - 1, 0, pg.v, inf), (0, 1, 1, pg.v, -inf), (2, 7, 1, pg.k, float("nan"))):
        what[pg.maps[b, n // 16], head, n % 16, 5] = value
    q = torch.randn((3, hq, dim), generator=torch.Generator().manual_seed(6)).to(dtype)
    cache, maps = pg.device()
    got = N.window_decode_attn(q.cuda(), cache, maps, i32(lens), max(lens), window, sinks, 0)
    ref, parts = pg.exact(q, [0, 1, 2, 3], window, sinks)
    assert np.isposinf(ref[0, :3, 5]).all() and np.isneginf(ref[0, 3:, 5]).all() and np.isnan(ref[2, 3:]).all()
    with np.errstate(all="ignore"):
        bound = window_bound(ref, parts, dtype)
    within(f64(got), ref, bound, "not finite")


def test_a_window_past_32_bits_is_no_window():
    pg = Paged([300, 40], 2, 64, B, seed=22)
    cache, maps = pg.device()
    q, lens = torch.randn((2, 4, 64), generator=torch.Generator().manual_seed(7)).to(B).cuda(), i32([300, 40])
    want = N.window_decode_attn(q, cache, maps, lens, 300, 300, 0, 0)
    for window, sinks in (((1 << 32) + 5, 0), (1 << 62, 0), (5, (1 << 32) + 1)):
        got = N.window_decode_attn(q, cache, maps, lens, 300, window, sinks, 0)
        assert torch.equal(got.view(torch.int16), want.view(torch.int16))
        got = N.window_attn(q, cache, maps, i32([0, 1, 2]), lens, 300, window, sinks, 0)
        assert torch.equal(got.view(torch.int16), N.window_attn(q, cache, maps, i32([0, 1, 2]), lens, 300, 300, 0,
                                                                0).view(torch.int16))


def test_rows_before_the_sequence_are_zero():
    """A length below the rows it has (a refused sequence's is 0): rows before position 0 get zeros, the others see
    what there is."""
    for dtype, dim in ((B, 128), (F, 64)):
        pg = Paged([40, 5], 2, dim, dtype, seed=12)
        cache, maps = pg.device()
        q = torch.randn((30, 4, dim), generator=torch.Generator().manual_seed(4)).to(dtype)
        for lens in ([0, 5], [3, 5], [40, 0]):
            got = f64(N.window_attn(q.cuda(), cache, maps, i32([0, 20, 30]), i32(lens), 40, 16, 2, 0))
            pg.lens = lens
            ref, parts = pg.exact(q, [0, 20, 30], 16, 2)
            within(got, ref, window_bound(ref, parts, dtype), f"short lengths {lens}")
            for b, (lo, hi) in enumerate(((0, 20), (20, 30))):
                assert (got[lo:max(lo, hi - lens[b])] == 0).all()


def test_in_place_and_on_another_stream():
    pg = Paged([700, 90], 2, 128, B, seed=13)
    cache, maps = pg.device()
    q = torch.randn((120, 8, 128), generator=torch.Generator().manual_seed(5)).to(B).cuda()
    args = (cache, maps, i32([0, 80, 120]), i32([700, 90]), 700, 200, 4, 0)
    want = N.window_attn(q, *args)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        got = N.window_attn(q.clone(), *args)
    torch.cuda.current_stream().wait_stream(s)
    assert torch.equal(got.view(torch.int16), want.view(torch.int16))
    mine = q.clone()
    assert N.window_attn(mine, *args, out=mine) is mine
    assert torch.equal(mine.view(torch.int16), want.view(torch.int16))
