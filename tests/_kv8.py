"""The 8-bit cache's definition in 64 bits (numpy), for the tests: codes, scales, rotation, attention and
the bounds that the kernels' roundings allow."""

import numpy as np
import torch

from paper_2608_20397_amd import nexus as N

PAGE = 16


def _table():
    t = np.empty(256)
    for b in range(256):
        x, m = (b >> 3) & 15, b & 7
        v = (8 + m) * 2.0 ** (x - 10) if x else m * 2.0 ** -9
        t[b] = np.nan if b & 127 == 127 else -v if b & 128 else v
    return t


TABLE = _table()


def exponent(amax):
    """Least e with amax <= 448 * 2^e, held within [-100, 119]."""
    with np.errstate(divide="ignore"):
        e = np.ceil(np.log2(np.maximum(amax, 2.0 ** -300) / 448.0))
    e = np.where(448 * 2.0 ** (e - 1) >= amax, e - 1, e)
    e = np.where(448 * 2.0 ** e < amax, e + 1, e)
    return np.clip(e, -100, 119)


def to_code_value(y):
    """The nearest E4M3 value, ties to even, at most 448."""
    y = np.clip(y, -448, 448)
    b = np.floor(np.log2(np.maximum(np.abs(y), 2.0 ** -6)))
    grid = 2.0 ** (b - 3)
    return np.rint(y / grid) * grid          # (np.rint: ties to even)


def quantise(x):
    """Values and scale bytes of fp64 rows [..., D]."""
    bad = ~np.isfinite(x).all(-1)
    z = np.where(bad[..., None], 0.0, x)
    e = exponent(np.abs(z).max(-1))
    val = to_code_value(z / 2.0 ** e[..., None]) * 2.0 ** e[..., None]
    return np.where(bad[..., None], np.nan, val), np.where(bad, 255, e + 127).astype(np.int64)


def rotate(x, pos, base, interleaved):
    """x [L][T][H][D] fp64, token t turned by pos[t]."""
    D = x.shape[-1]
    ang = np.asarray(pos, dtype=np.float64)[:, None] * base ** (-2.0 * np.arange(D // 2) / D)
    c, s = np.cos(ang)[None, :, None], np.sin(ang)[None, :, None]
    a, b = (x[..., 0::2], x[..., 1::2]) if interleaved else (x[..., :D // 2], x[..., D // 2:])
    ra, rb = a * c - b * s, b * c + a * s
    if not interleaved:
        return np.concatenate([ra, rb], -1)
    out = np.empty_like(x)
    out[..., 0::2], out[..., 1::2] = ra, rb
    return out


def assert_written(got_val, got_byte, x, slack, what):
    """Rows got against the definition of x, whose elements the kernel may hold off by `slack` (0: exactly
    the definition; else an element may round either way where a border lies within slack of it)."""
    val, byte = quantise(x)
    if np.isscalar(slack) and slack == 0:
        assert np.array_equal(got_byte, byte), what
        assert np.array_equal(got_val, val, equal_nan=True), what
        return
    bad = byte == 255
    assert np.array_equal(got_byte == 255, bad), what
    amax = np.abs(np.where(bad[..., None], 0, x)).max(-1)
    s = np.broadcast_to(slack, x.shape).max(-1)
    lo, hi = exponent(np.maximum(amax - s, 0)) + 127, exponent(amax + s) + 127
    assert np.all(bad | ((got_byte >= lo) & (got_byte <= hi))), what
    scale = 2.0 ** (got_byte.astype(np.float64) - 127)[..., None]
    low = to_code_value((x - slack) / scale) * scale
    high = to_code_value((x + slack) / scale) * scale
    ok = bad[..., None] | ((got_val >= low) & (got_val <= high))
    assert ok.all(), (what, np.argwhere(~ok)[:3], got_val[~ok][:3], x[~ok][:3])
    # and only where a border is that near does it differ
    assert np.all(bad[..., None] | (got_val == val) | (low != high)), what


def rotation_slack(x):
    """rope_math.h: 2^-23 of the result and 2^-46 of the pair, here twice that."""
    return 2.0 ** -22 * np.abs(x) + 2.0 ** -44 * np.abs(x).max(-1, keepdims=True)


def make_cache(L, npp, H, D, n_map, base=1e4, style=N.ROPE_NEOX, seed=0, fill=0x7F):
    """A cache whose every slot holds NaN codes and the NaN scale, and a shuffled page map."""
    g = np.random.default_rng([20397, 77, seed])
    pm = torch.from_numpy(g.permutation(npp)[:n_map].astype(np.int32)).cuda()
    c = N.KV8Cache.empty(L, npp, H, D, pm, base, style)
    for t in (c.k, c.v):
        t.view(torch.uint8).fill_(fill)
    for t in (c.k_scale, c.v_scale):
        t.fill_(255)
    return c


def values(cache, name):
    """(values [L][pages][H][16][D], bytes) of the cache as fp64."""
    codes = getattr(cache, name).view(torch.uint8).cpu().numpy()
    byte = getattr(cache, name + "_scale").cpu().numpy().astype(np.int64)
    with np.errstate(invalid="ignore"):
        return TABLE[codes] * np.where(byte == 255, np.nan, 2.0 ** (byte - 127.0))[..., None], byte


def tokens(arr, pmap, offset, n):
    """Logical tokens of [L][pages][H][16](...) as [L][n][H](...)."""
    t = np.arange(offset, offset + n)
    return np.moveaxis(arr[:, pmap[t // PAGE], :, t % PAGE], 0, 1)


def rows(seed, *shape, dtype="bf16", spread=1.0):
    g = np.random.default_rng([20397, 78, seed])
    x = g.standard_normal(shape) * np.exp(spread * g.standard_normal(shape[:-1] + (1,)))
    return torch.from_numpy(x).to(torch.bfloat16 if dtype == "bf16" else torch.float32).cuda()


def f64(t):
    return t.float().cpu().numpy().astype(np.float64)


def attention(q, k, v, seen, scale, cap):
    """q [R][Hq][D], k, v [n][H][D] fp64; query r sees the first seen[r] keys.  (out, A, S): the result, the
    weighted mean of |v|, and the largest scale * sum |q k| of a row."""
    R, Hq, D = q.shape
    G = Hq // k.shape[1]
    out, mean, smax = np.zeros((R, Hq, D)), np.zeros((R, Hq, D)), np.zeros((R, Hq, 1))
    for h in range(Hq):
        kh, vh = k[:, h // G], v[:, h // G]
        s = q[:, h] @ kh.T * scale
        if cap:
            s = cap * np.tanh(s / cap)
        a = np.abs(q[:, h]) @ np.abs(kh).T * scale
        keep = np.arange(len(kh))[None] < np.asarray(seen)[:, None]
        s = np.where(keep, s, -np.inf)
        ok = keep.any(-1)
        p = np.exp(s - np.where(ok, s.max(-1, initial=-np.inf), 0)[:, None])
        p = p / np.where(ok, p.sum(-1), 1)[:, None]
        out[:, h], mean[:, h] = p @ vh, p @ np.abs(vh)
        smax[:, h, 0] = np.where(keep, a, 0).max(-1, initial=0)
    return out, mean, smax


def assert_attention(got, ref, what):
    """Element by element.  Rounding a probability to bf16 is off by 2^-8 at most, and the row sum adds the
    rounded ones, so sum p (v - o) moves by 2^-8 (A + |o|); a score is a sum of D products in fp32 plus the
    query's 2^-22 and the capped score's few 2^-22 of at most 50 log2 e; split partials are fp16 rows (2^-11);
    the result is rounded to bf16 once (2^-8)."""
    out, mean, smax = ref
    D = out.shape[-1]
    eps = 2.0 ** -8 + smax * (D + 16) * 2.0 ** -24 + 2.0 ** -13
    tol = eps * (mean + np.abs(out)) + 2.0 ** -8 * np.abs(out) + 2.0 ** -10 * mean.max(-1, keepdims=True)
    err = np.abs(got - out)
    assert np.all(err <= tol), (what, float((err / np.maximum(tol, 1e-300)).max()), np.argwhere(err > tol)[:3])
    rms = np.sqrt(np.mean((got - out) ** 2) / max(np.mean(out ** 2), 1e-300))
    assert rms <= 5e-3, (what, rms)
