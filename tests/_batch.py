"""The ragged-batch operators' definitions in 64 bits (numpy), for the tests: the layout of a round, norms with
rotation, windowed attention; and the bounds that the kernels' roundings allow."""

import numpy as np
import torch

from paper_2608_20397_amd import nexus as N

PAGE = 16
HALF = {torch.bfloat16: 2.0 ** -8, torch.float32: 2.0 ** -24}     # half a step, relative
U = 2.0 ** -24                                                     # of the fp32 arithmetic inside


def f64(x):
    return x.detach().cpu().to(torch.float64).numpy()


def i32(x):
    return torch.tensor(np.asarray(x), dtype=torch.int32, device="cuda")


# ---- pages


def lay_out(cached, fresh, free, n_free, maps, max_tokens):
    """(maps, q_start, seq_len, pos, slot, n_left), token by token."""
    maps, stride = np.array(maps), np.shape(maps)[1]
    n_free = min(max(n_free, 0), len(free))
    pos, slot = np.full(max_tokens, -1), np.full(max_tokens, -1)
    q_start, seq_len, left, wanted, row = [0], [], n_free, 0, 0
    for b, (c, f) in enumerate(zip(cached, fresh)):
        rows = max(f, 0)
        ok = c >= 0 and f >= 0 and c + f <= PAGE * stride and row + rows <= max_tokens
        need = -(-(c + f) // PAGE) - -(-c // PAGE) if ok else 0
        wanted += need
        if ok and need and wanted > n_free:
            ok = False
        if ok:
            for p in range(-(-c // PAGE), -(-(c + f) // PAGE)):
                left -= 1
                maps[b, p] = free[left]
            for t in range(f):
                pos[row + t] = c + t
                slot[row + t] = maps[b, (c + t) // PAGE] * PAGE + (c + t) % PAGE
        row = min(row + rows, max_tokens)
        q_start.append(row)
        seq_len.append(c + f if ok else 0)
    return maps, np.array(q_start), np.array(seq_len), pos, slot, left


# ---- norm and rotation


def norm_rope(x, weight, eps, pos, base, interleaved):
    """x [T][H][D] fp64 -> (result, size): size [T][H][D], the sum of the magnitudes of an element's pair."""
    D = x.shape[-1]
    if eps > 0:
        x = x / np.sqrt((x * x).mean(-1, keepdims=True) + eps)
        x = x if weight is None else x * weight
    ang = np.asarray(pos, dtype=np.longdouble)[:, None] * np.longdouble(base) ** (
        np.longdouble(-2.0) * np.arange(D // 2) / D)
    c, s = np.cos(ang).astype(np.float64)[:, None], np.sin(ang).astype(np.float64)[:, None]
    a, b = (x[..., 0::2], x[..., 1::2]) if interleaved else (x[..., :D // 2], x[..., D // 2:])
    size = np.abs(a) + np.abs(b)
    if not interleaved:
        return np.concatenate([a * c - b * s, b * c + a * s], -1), np.concatenate([size, size], -1)
    out, both = np.empty_like(x), np.empty_like(x)
    out[..., 0::2], out[..., 1::2] = a * c - b * s, b * c + a * s
    both[..., 0::2] = both[..., 1::2] = size
    return out, both


def norm_rope_bound(ref, size, dtype, eps):
    """One rounding to dtype, and fp32 before it: the sum of D squares (D roundings, halved by the root), the mean,
    the root and its reciprocal, two products; the compensated rotation, 2^-23 of the pair, and angles to 2^-40."""
    D = ref.shape[-1]
    steps = (D / 2 + 6 if eps > 0 else 0) + 4
    return HALF[dtype] * 1.001 * np.abs(ref) + steps * U * size + 1e-38


# ---- attention


def keys_of(cache_k, cache_v, row_map, n, transposed):
    """fp64 keys and values [n][H][D] of one sequence."""
    slots = np.asarray(row_map)[np.arange(n) // PAGE].astype(np.int64) * PAGE + np.arange(n) % PAGE
    k = cache_k.transpose(0, 2, 1, 3).reshape(-1, *cache_k.shape[1::2])[slots]
    v = cache_v[:, :, slots].transpose(2, 0, 1) if transposed else \
        cache_v.transpose(0, 2, 1, 3).reshape(-1, *cache_v.shape[1::2])[slots]
    return k, v


def window_attn(q, k_cache, v_cache, maps, q_start, seq_len, window, sinks, transposed, softcap=0.0, scale=0.0,
                out=None):
    """(result, bound parts) by the definition, a query at a time over the keys that it sees alone; rows of no
    sequence keep `out`.  Parts: abs [rows][H][D], the weighted mean of the values' magnitudes; err [rows][H], a bound
    on the score's error in natural units per unit of 2^-24; n [rows], keys seen."""
    rows, hq, D = q.shape
    hkv = k_cache.shape[1]
    scale = scale or 1.0 / np.sqrt(D)
    out = np.zeros(q.shape) if out is None else np.array(out)
    mag, err, cnt = np.zeros(q.shape), np.zeros((rows, hq)), np.zeros(rows, dtype=np.int64)
    for b, n in enumerate(seq_len):
        fresh = q_start[b + 1] - q_start[b]
        if fresh == 0:
            continue
        k, v = keys_of(k_cache, v_cache, maps[b], n, transposed)
        for i in range(fresh):
            r, p = q_start[b] + i, n - fresh + i
            if p < 0:
                out[r] = 0
                continue
            key = np.arange(p + 1)
            key = key[(key > p - window) | (key < sinks)]
            cnt[r] = len(key)
            for h in range(hq):
                kh, vh = k[key, h // (hq // hkv)], v[key, h // (hq // hkv)]
                with np.errstate(all="ignore"):
                    s = kh @ q[r, h] * scale
                    size = (np.abs(kh) @ np.abs(q[r, h]) * scale).max()
                    if softcap:
                        s = softcap * np.tanh(s / softcap)
                    w = np.exp(s - s.max())
                    w /= w.sum()
                    out[r, h] = w @ vh
                    mag[r, h] = w @ np.abs(vh)
                # a dot product of D terms, its scaling, a tanh (an exponential and a reciprocal, 8 units of the cap)
                err[r, h] = (D + 4) * size + 8 * softcap
    return out, (mag, err, cnt)


def window_bound(ref, parts, dtype):
    """A weight is off by the score's error (twice: the sum of weights too), by its exponential and, in bf16, by its
    rounding, 2^-8, against which the mean moves by at most mag + |out|; sums of n terms in fp32, the merges and one
    rounding of the result."""
    mag, err, cnt = parts
    fp32 = (2 * err[..., None] + cnt[:, None, None] + 64) * U
    weights = HALF[dtype] if dtype == torch.bfloat16 else 0.0
    return (weights + fp32) * (mag + np.abs(ref)) * 1.01 + HALF[dtype] * 1.01 * np.abs(ref) + 1e-37


def within(got, ref, bound, what):
    got = np.asarray(got)
    assert got.shape == ref.shape
    same = np.isnan(got) == np.isnan(ref)
    assert same.all(), f"{what}: NaN in {np.argwhere(~same)[:4].tolist()}"
    inf = np.isinf(ref)
    assert (got[inf] == ref[inf]).all(), f"{what}: infinities differ"
    ok = np.isnan(ref) | inf
    over = np.where(ok, 0, np.abs(np.where(ok, 0, got) - np.where(ok, 0, ref)) / np.where(ok, 1, bound))
    worst = float(over.max()) if over.size else 0.0
    print(f"{what}: {worst:.3f} of the bound", flush=True)
    assert worst <= 1, f"{what}: {worst:.3f} of the bound at {np.unravel_index(over.argmax(), over.shape)}"


class Paged:
    """A cache of sequences of the given lengths over shuffled pages; slots behind a sequence and pages of none hold
    NaN, and map entries behind a sequence's pages name such a page."""

    def __init__(self, lens, hkv, dim, dtype, transposed=False, seed=0, spare=3, interleaved=False, stride=None,
                 layers=1, layer=0):
        g = torch.Generator().manual_seed(seed)
        pages = [-(-n // PAGE) for n in lens]
        n_phys = sum(pages) + spare
        order = torch.randperm(n_phys, generator=g).tolist()
        stride = stride or max(1, max(pages))
        self.nowhere = order.pop()                     # (spare > 0: a page of NaN)
        self.maps = np.full((len(lens), stride), self.nowhere, dtype=np.int64)
        shape = (n_phys, hkv, PAGE, dim)
        self.k = torch.randn(shape, generator=g).to(dtype)
        self.v = torch.randn(shape, generator=g).to(dtype)
        unused = torch.ones((n_phys, PAGE), dtype=torch.bool)
        for b, n in enumerate(lens):
            for p in range(pages[b]):
                self.maps[b, p] = order.pop()
                unused[self.maps[b, p], :min(PAGE, n - PAGE * p)] = False
        self.free = order
        mask = unused[:, None, :, None].expand(shape)
        self.k[mask], self.v[mask] = float("nan"), float("nan")
        self.transposed, self.lens, self.dtype = transposed, lens, dtype
        self.interleaved, self.layers, self.layer = interleaved, layers, layer

    def forget(self, q_start, window, sinks):
        """What no row sees becomes NaN, and pages without a seen key leave the maps."""
        for b, n in enumerate(self.lens):
            first = n - (q_start[b + 1] - q_start[b])           # the first row's position
            key = np.arange(n)
            seen = ((key > first - window) | (key < sinks)) if first < n else key < 0
            for p in range(-(-n // PAGE)):
                here = seen[PAGE * p:PAGE * p + PAGE]
                if here.any():
                    page = self.maps[b, p]
                    gone = torch.tensor(np.flatnonzero(~here))
                    self.k[page][:, gone] = float("nan")
                    self.v[page][:, gone] = float("nan")
                else:
                    self.maps[b, p] = self.nowhere

    def v_as_held(self):
        return self.v.permute(1, 3, 0, 2).flatten(2).contiguous() if self.transposed else self.v

    def device(self, base=1e4):
        """(nexus cache, device maps); the other layers hold NaN."""
        def put(x):
            full = torch.full((self.layers, *x.shape), float("nan"), dtype=x.dtype)
            full[self.layer] = x
            return full.cuda()

        maps = i32(self.maps)
        return N.PagedKVCache(put(self.k), put(self.v_as_held()), maps[0], base,
                              N.V_TRANSPOSED if self.transposed else N.V_ROWMAJOR,
                              N.ROPE_INTERLEAVED if self.interleaved else N.ROPE_NEOX), maps

    def exact(self, q, q_start, window, sinks, **kw):
        return window_attn(f64(q), f64(self.k), f64(self.v_as_held()), self.maps, q_start, self.lens, window, sinks,
                           self.transposed, **kw)
