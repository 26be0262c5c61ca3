"""GPU parity of the append with head norms and rotation against its definition in 64 bits: bf16 and fp32, every
head_dim, both pairings and V layouts, with and without a norm and weights, packed and separate rows, positions far out,
rows without a slot, magnitudes whose squares leave fp32."""

import numpy as np
import pytest
import torch

from _batch import PAGE, f64, i32, norm_rope, norm_rope_bound, within
from paper_2608_20397_amd import nexus as N

pytestmark = pytest.mark.gpu

B, F = torch.bfloat16, torch.float32


def run(rows, *, hq, hkv, dim, dtype=B, vt=False, interleaved=False, eps=1e-6, weights=True, packed=True, base=1e6,
        pos0=0, hole=(), layers=1, layer=0, seed=0, size=1.0, in_place=False):
    g = torch.Generator().manual_seed(seed)
    n_phys = -(-rows // PAGE) + 2
    x = (size * torch.randn((rows, hq + 2 * hkv, dim), generator=g)).to(dtype)
    q, k, v = x.cuda().split((hq, hkv, hkv), 1)
    if not packed:
        q, k, v = q.contiguous(), k.contiguous(), v.contiguous()
    qw, kw = [(1 + 0.3 * torch.randn(dim, generator=g)) if weights and eps > 0 else None for _ in range(2)]
    slot = torch.randperm(n_phys * PAGE, generator=g)[:rows].numpy()
    for h in hole:
        slot[h] = -1 if h % 2 else n_phys * PAGE + h        # outside the cache either way
    pos = pos0 + np.arange(rows)
    shape = (layers, n_phys, hkv, PAGE, dim)
    ck = torch.full(shape, 3.0, dtype=dtype, device="cuda")
    cv = torch.full((layers, hkv, dim, n_phys * PAGE) if vt else shape, 5.0, dtype=dtype, device="cuda")
    cache = N.PagedKVCache(ck, cv, i32([0]), base, N.V_TRANSPOSED if vt else N.V_ROWMAJOR,
                           N.ROPE_INTERLEAVED if interleaved else N.ROPE_NEOX)
    out = q if in_place else torch.full((rows, hq, dim), 9.0, dtype=dtype, device="cuda")
    before = f64(q)
    dev = lambda w: None if w is None else w.cuda()  # noqa: E731
    got = N.norm_rope_append(cache, layer, q, k, v, i32(pos), i32(slot), q_weight=dev(qw), k_weight=dev(kw), eps=eps,
                             out=out)
    torch.cuda.synchronize()
    assert got is out
    what = f"{rows} rows {hq}/{hkv}/{dim} {dtype} vt {vt} il {interleaved} eps {eps} packed {packed} pos0 {pos0}"
    live = np.array([h not in hole for h in range(rows)], dtype=bool)
    np64 = lambda w: None if w is None else f64(w)  # noqa: E731
    ref, both = norm_rope(f64(x[:, :hq]), np64(qw), eps, pos, base, interleaved)
    within(f64(got)[live], ref[live], norm_rope_bound(ref, both, dtype, eps)[live], "q " + what)
    assert (f64(got)[~live] == (before[~live] if in_place else 9.0)).all()
    ref, both = norm_rope(f64(x[:, hq:hq + hkv]), np64(kw), eps, pos, base, interleaved)
    held = f64(ck[layer]).transpose(0, 2, 1, 3).reshape(-1, hkv, dim)
    within(held[slot[live]], ref[live], norm_rope_bound(ref, both, dtype, eps)[live], "k " + what)
    rest = np.ones(len(held), dtype=bool)
    rest[slot[live]] = False
    assert (held[rest] == 3.0).all()
    held = f64(cv[layer]).transpose(2, 0, 1) if vt else f64(cv[layer]).transpose(0, 2, 1, 3).reshape(-1, hkv, dim)
    assert (held[slot[live]] == f64(x[:, hq + hkv:])[live]).all() and (held[rest] == 5.0).all()
    for other in range(layers):
        if other != layer:
            assert (ck[other] == 3.0).all() and (cv[other] == 5.0).all()


FORMS = [(4, 2, 64, B), (40, 8, 128, B), (16, 8, 256, B), (1, 1, 16, B), (6, 2, 32, B), (4, 1, 64, F), (5, 5, 128, F),
         (3, 1, 256, F), (2, 2, 8, F), (64, 2, 64, B)]


@pytest.mark.parametrize("hq,hkv,dim,dtype", FORMS)
@pytest.mark.parametrize("vt", [False, True])
@pytest.mark.parametrize("interleaved", [False, True])
def test_forms(hq, hkv, dim, dtype, vt, interleaved):
    kw = dict(hq=hq, hkv=hkv, dim=dim, dtype=dtype, vt=vt, interleaved=interleaved)
    run(37, pos0=1000, hole=(0, 5, 36), seed=1, **kw)
    run(5, eps=0.0, packed=False, seed=2, **kw)


@pytest.mark.parametrize("rows", [1, 2, 3, 4, 5, 17, 64, 333])
def test_rows(rows):
    run(rows, hq=10, hkv=2, dim=128, pos0=17, seed=rows)
    run(rows, hq=4, hkv=1, dim=64, dtype=F, weights=False, packed=False, pos0=9, seed=rows)


def test_layers_bases_and_positions_far_out():
    run(20, hq=4, hkv=2, dim=64, layers=3, layer=1, base=500.0)
    for dtype in (B, F):
        # (fp64 angles: at 2^24 off by 3 roundings of 2^-53, 2^-27 radians, an eighth of a unit of the bound's steps)
        run(20, hq=4, hkv=2, dim=64, dtype=dtype, pos0=(1 << 24) - 3)


def test_in_place():
    run(19, hq=4, hkv=2, dim=128, packed=False, in_place=True, hole=(3,))
    run(19, hq=4, hkv=2, dim=32, dtype=F, packed=False, in_place=True)


@pytest.mark.parametrize("size,eps", [(1e25, 1e-6), (1e-3, 1e-6), (1e-25, 1e-30), (3e37, 1e-6), (1e18, 1e-6)])
def test_magnitudes(size, eps):
    """Squares past fp32's largest number and below its smallest."""
    for dtype in (B, F):
        run(9, hq=4, hkv=2, dim=64, dtype=dtype, eps=eps, size=size, seed=4)


def test_rows_of_zeros_and_not_finite_ones():
    """A head of zeros stays zeros; one with an element that is not finite is NaN or zero as the formula says, and no
    other head is touched."""
    x = torch.ones((3, 4, 64), dtype=B)
    x[0, 0] = 0
    x[1, 1, 5] = float("inf")
    x[2, 2, 7] = float("nan")
    q, k, v = x.cuda().split((2, 1, 1), 1)
    cache = N.PagedKVCache(torch.zeros((1, 1, 1, PAGE, 64), dtype=B, device="cuda"),
                           torch.zeros((1, 1, 1, PAGE, 64), dtype=B, device="cuda"), i32([0]), 1e4)
    got = f64(N.norm_rope_append(cache, 0, q, k, v, i32([0, 0, 0]), i32([0, 1, 2]), eps=1e-6))
    assert (got[0, 0] == 0).all() and (got[0, 1] != 0).all() and np.isfinite(got[[0, 2]]).all()
    # inf / inf and, through the rotation by 0 (sin 0 = 0 times it), its partner; the others finite / inf
    assert np.isnan(got[1, 1, [5, 37]]).all()
    assert (np.delete(got[1, 1], [5, 37]) == 0).all() and np.isfinite(got[1, 0]).all()
    held = f64(cache.k)[0, 0, 0]
    assert np.isnan(held[2]).all() and np.isfinite(held[:2]).all()


def test_refusals():
    q, k, v = torch.zeros((4, 6, 64), dtype=B, device="cuda").split((4, 1, 1), 1)
    cache = N.PagedKVCache(torch.zeros((1, 2, 1, PAGE, 64), dtype=B, device="cuda"),
                           torch.zeros((1, 2, 1, PAGE, 64), dtype=B, device="cuda"), i32([0]), 1e4)
    p = i32([0, 1, 2, 3])
    w = torch.ones(64, device="cuda")
    for call, status in [
            (lambda: N.norm_rope_append(cache, 0, q, k, v, p[:3], p), N.EINVAL),
            (lambda: N.norm_rope_append(cache, 0, q, k, v, p.long(), p), N.EINVAL),
            (lambda: N.norm_rope_append(cache, 0, q, k, v, p, p, q_weight=w), N.EINVAL),
            (lambda: N.norm_rope_append(cache, 0, q, k, v, p, p, q_weight=w[:32], eps=1e-6), N.EINVAL),
            (lambda: N.norm_rope_append(cache, 0, q, k, v, p, p, q_weight=w.to(B), eps=1e-6), N.EINVAL),
            (lambda: N.norm_rope_append(cache, 0, q.float(), k, v, p, p), N.EDTYPE),
            (lambda: N.norm_rope_append(cache, 0, q, k[:3], v, p, p), N.ESHAPE),
            (lambda: N.norm_rope_append(cache, 0, q[:, :, :32], k, v, p, p), N.ESHAPE),
            (lambda: N.norm_rope_append(cache, 0, q.transpose(0, 1), k, v, p, p), N.EINVAL),
            (lambda: N.norm_rope_append(cache, 0, q, k, v, p, p, out=q), N.EINVAL),
            (lambda: N.norm_rope_append(cache, 1, q, k, v, p, p), N.ERANGE)]:
        with pytest.raises(N.NexusError) as e:
            call()
        assert e.value.status == status
