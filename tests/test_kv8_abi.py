"""CPU tests of the 8-bit cache's C entry points and binding: what each call refuses, and with which status.
Every call here fails validation, so its placeholder pointers are never used."""

import ctypes as C

import pytest
import torch

from paper_2608_20397_amd import nexus as N

P = 0x10000          # a 16-byte aligned placeholder


def _cache(**kw):
    d = dict(k=P, v=P, k_scale=P, v_scale=P, n_layers=2, n_phys_pages=8, page_size=16, n_kv_heads=2,
             head_dim=128, rope_style=N.ROPE_NEOX, rope_base=1e4)
    d.update(kw)
    return N.CKv8Cache(*[d[n] for n, _ in N.CKv8Cache._fields_])


def _pt(n=8, m=P):
    return N.CPageTable(m, n)


def _block(**kw):
    d = dict(k=P, v=P, n_layers=2, n_tokens=10, n_kv_heads=2, head_dim=128, dtype=N.BF16, rope_style=N.ROPE_NEOX,
             base_pos=0, rope_base=1e4)
    d.update(kw)
    return N.CBlock(*[d[n] for n, _ in N.CBlock._fields_])


def append(c=None, pt=None, k=P, v=P, dtype=N.BF16, n=4, offset=0, pos0=0):
    return N.lib().nexus_kv8_append(C.byref(c or _cache()), C.byref(pt or _pt()), k, v, dtype, n, offset, pos0, 0)


def step(c=None, maps=P, stride=4, lens=P, n=3, max_len=64, k=P, v=P, dtype=N.BF16):
    return N.lib().nexus_kv8_append_step(C.byref(c or _cache()), maps, stride, lens, n, max_len, k, v, dtype, 0)


def splice(c=None, pt=None, b=None, offset=0, dst=0):
    return N.lib().nexus_kv8_splice(C.byref(c or _cache()), C.byref(pt or _pt()), C.byref(b or _block()), offset,
                                    dst, 0)


def read(c=None, pt=None, offset=0, n=4, dtype=N.F32, k=P, v=P):
    return N.lib().nexus_kv8_read(C.byref(c or _cache()), C.byref(pt or _pt()), offset, n, dtype, k, v, 0)


def suffix(c=None, pt=None, q=P, starts=(0,), lens=(4,), pasts=(3,), hq=4, layer=0, cap=0.0, scale=0.0, out=P, ws=0,
           nbytes=0):
    n = len(lens)
    return N.lib().nexus_kv8_suffix_attn_varlen(
        q, n, (C.c_int32 * n)(*starts), (C.c_int32 * n)(*lens), (C.c_int64 * n)(*pasts), hq,
        C.byref(c or _cache()), C.byref(pt or _pt()), layer, cap, scale, out, ws, nbytes, 0)


def decode(c=None, q=P, n=3, hq=4, maps=P, stride=4, lens=P, max_len=64, layer=0, cap=0.0, scale=0.0, out=P, ws=0,
           nbytes=0):
    return N.lib().nexus_kv8_decode_attn(q, n, hq, C.byref(c or _cache()), maps, stride, lens, max_len, layer, cap,
                                         scale, out, ws, nbytes, 0)


CALLS = [append, step, splice, read, suffix, decode]


@pytest.mark.parametrize("call", CALLS)
@pytest.mark.parametrize("field,value,status", [
    ("k", 0, N.EINVAL), ("v_scale", 0, N.EINVAL), ("v", P + 8, N.EINVAL), ("k_scale", P + 1, N.EINVAL),
    ("n_layers", 0, N.EINVAL), ("n_layers", 65536, N.ESHAPE), ("n_phys_pages", -1, N.EINVAL),
    ("n_phys_pages", 1 << 27, N.ESHAPE), ("page_size", 32, N.ESHAPE), ("n_kv_heads", 0, N.EINVAL),
    ("n_kv_heads", 1 << 21, N.ESHAPE), ("head_dim", 32, N.ESHAPE), ("head_dim", 96, N.ESHAPE),
    ("head_dim", 512, N.ESHAPE), ("rope_style", 2, N.EINVAL), ("rope_base", 1.0, N.EROPE),
    ("rope_base", float("nan"), N.EROPE), ("rope_base", float("inf"), N.EROPE),
])
def test_every_call_checks_the_cache(call, field, value, status):
    assert call(c=_cache(**{field: value})) == status


@pytest.mark.parametrize("call", [append, splice, read, suffix])
def test_every_call_checks_its_page_table(call):
    assert call(pt=_pt(m=0)) == N.EINVAL
    assert call(pt=_pt(n=0)) == N.EINVAL
    assert call(pt=_pt(n=9)) == N.ERANGE


@pytest.mark.parametrize("call", [append, read])
def test_rows_and_ranges(call):
    for bad in (dict(k=0), dict(v=0), dict(k=P + 2), dict(v=P + 8), dict(n=0), dict(n=-1)):
        assert call(**bad) == N.EINVAL, bad
    assert call(dtype=2) == N.EDTYPE
    for bad in (dict(offset=-1), dict(offset=125), dict(n=129), dict(offset=(1 << 63) - 1)):
        assert call(**bad) == N.ERANGE, bad
    assert call(c=_cache(n_kv_heads=1 << 15, n_phys_pages=1 << 20), n=1 << 10) == N.ESHAPE   # 2^32 elements a layer


def test_append_positions():
    assert append(pos0=-1) == N.ERANGE
    assert append(pos0=(1 << 63) - 1) == N.ERANGE


def test_step():
    for bad in (dict(maps=0), dict(lens=0), dict(stride=0), dict(n=0), dict(k=0), dict(v=P + 4)):
        assert step(**bad) == N.EINVAL, bad
    assert step(max_len=65) == N.ERANGE and step(max_len=-1) == N.ERANGE
    assert step(dtype=7) == N.EDTYPE
    assert step(max_len=0) == N.OK          # no length can name a slot: nothing enqueued


def test_splice_checks_the_block():
    for kw, st in ((dict(k=0), N.EINVAL), (dict(n_tokens=0), N.EINVAL), (dict(dtype=9), N.EDTYPE),
                   (dict(head_dim=64), N.ESHAPE), (dict(n_layers=1), N.ESHAPE), (dict(n_kv_heads=4), N.ESHAPE),
                   (dict(rope_base=1e6), N.EROPE), (dict(rope_style=N.ROPE_INTERLEAVED), N.EROPE),
                   (dict(base_pos=-1), N.ERANGE), (dict(v=P + 8), N.EINVAL)):
        assert splice(b=_block(**kw)) == st, kw
    assert splice(offset=119) == N.ERANGE and splice(offset=-1) == N.ERANGE and splice(dst=-1) == N.ERANGE


def test_suffix():
    for kw, st in ((dict(q=0), N.EINVAL), (dict(out=0), N.EINVAL), (dict(q=P + 2), N.EINVAL),
                   (dict(layer=2), N.ERANGE), (dict(layer=-1), N.ERANGE), (dict(hq=3), N.ESHAPE),
                   (dict(hq=0), N.ESHAPE), (dict(cap=-1.0), N.EINVAL), (dict(cap=float("inf")), N.EINVAL),
                   (dict(scale=float("nan")), N.EINVAL), (dict(lens=(0,)), N.EINVAL), (dict(starts=(-1,)), N.EINVAL),
                   (dict(pasts=(-1,)), N.ERANGE), (dict(pasts=(125,)), N.ERANGE),
                   (dict(pasts=((1 << 63) - 1,)), N.ERANGE), (dict(starts=(1 << 21,)), N.ERANGE),
                   (dict(starts=(), lens=(), pasts=()), N.EINVAL),
                   (dict(starts=(0, 3), lens=(4, 4), pasts=(0, 0)), N.EINVAL),          # rows overlap
                   (dict(starts=tuple(range(33)), lens=(1,) * 33, pasts=(0,) * 33), N.EINVAL)):
        assert suffix(**kw) == st, kw


def test_suffix_workspace():
    L = N.lib()
    c = _cache(n_phys_pages=4096, n_layers=1)
    need = L.nexus_kv8_suffix_attn_workspace(64, 4, C.byref(c), 20000)
    assert 0 < need < 1 << 40
    big = dict(c=c, pt=_pt(4096), lens=(64,), pasts=(20000,))
    assert suffix(**big) == N.EWORKSPACE
    assert suffix(**big, ws=P, nbytes=need - 1) == N.EWORKSPACE
    assert suffix(**big, ws=P + 8, nbytes=need) == N.EWORKSPACE
    bad = (1 << 64) - 1
    for args in ((0, 4, 10), (4, 3, 10), (4, 0, 10), (4, 4, -1), (1 << 30, 4, 10)):
        assert L.nexus_kv8_suffix_attn_workspace(args[0], args[1], C.byref(c), args[2]) == bad, args
    assert L.nexus_kv8_suffix_attn_workspace(4, 4, C.byref(_cache(head_dim=32)), 10) == bad


def test_decode():
    for kw, st in ((dict(q=0), N.EINVAL), (dict(out=P + 4), N.EINVAL), (dict(maps=0), N.EINVAL),
                   (dict(lens=0), N.EINVAL), (dict(stride=0), N.EINVAL), (dict(n=0), N.EINVAL),
                   (dict(hq=3), N.ESHAPE), (dict(layer=2), N.ERANGE), (dict(max_len=65), N.ERANGE),
                   (dict(max_len=-1), N.ERANGE), (dict(cap=-0.5), N.EINVAL), (dict(scale=-1.0), N.EINVAL),
                   (dict(n=65536), N.ESHAPE), (dict(n=60000, stride=1 << 20, max_len=16), N.ESHAPE)):
        assert decode(**kw) == st, kw
    L, c = N.lib(), _cache(n_phys_pages=4096)
    need = L.nexus_kv8_decode_attn_workspace(1, 4, C.byref(c), 20000)
    assert 0 < need < 1 << 40
    assert decode(c=c, n=1, stride=2000, max_len=20000) == N.EWORKSPACE
    assert decode(c=c, n=1, stride=2000, max_len=20000, ws=P, nbytes=need - 1) == N.EWORKSPACE
    bad = (1 << 64) - 1
    assert L.nexus_kv8_decode_attn_workspace(0, 4, C.byref(c), 10) == bad
    assert L.nexus_kv8_decode_attn_workspace(1, 5, C.byref(c), 10) == bad
    assert L.nexus_kv8_decode_attn_workspace(1, 4, C.byref(c), -1) == bad


def test_decode_length_limit_and_workspaces():
    """Lengths whose pages cannot be counted in 32 bits are refused; the workspace of large launches, with what
    shared pages take, stays far below the cache that it serves."""
    L, bad = N.lib(), (1 << 64) - 1
    c = _cache(n_phys_pages=1 << 20, n_layers=1, n_kv_heads=8)
    top = (1 << 31) - 17
    assert L.nexus_kv8_decode_attn_workspace(1, 8, C.byref(c), top) not in (0, bad)
    assert L.nexus_kv8_decode_attn_workspace(1, 8, C.byref(c), top + 1) == bad
    assert decode(c=c, n=1, hq=8, stride=1 << 27, max_len=top + 1) == N.ERANGE
    for n in (1, 2, 7, 31, 32, 33, 48, 64, 65, 300, 1000):
        for hq in (8, 40, 128):
            for length in (1, 513, 17473, 131072):
                need = L.nexus_kv8_decode_attn_workspace(n, hq, C.byref(c), length)
                codes = n * length * 8 * 128 * 2
                assert need != bad and need <= max(codes, 64 << 20), (n, hq, length, need)


def test_binding_refuses_host_tensors():
    rows = (1, 4, 2, 16)
    c = N.KV8Cache(torch.empty(*rows, 128, dtype=torch.float8_e4m3fn),
                   torch.empty(*rows, 128, dtype=torch.float8_e4m3fn), torch.empty(rows, dtype=torch.uint8),
                   torch.empty(rows, dtype=torch.uint8), torch.arange(4, dtype=torch.int32), 1e4)
    x = torch.zeros(1, 3, 2, 128, dtype=torch.bfloat16)
    i = torch.zeros(3, dtype=torch.int32)
    calls = [lambda: N.kv8_append(c, x, x, 0, 0), lambda: N.kv8_splice(c, N.Block(x, x, 0, 1e4), 0, 0),
             lambda: N.kv8_append_step(c, i.view(3, 1), i, 16, x, x), lambda: N.kv8_read(c, 0, 3),
             lambda: N.kv8_suffix_attn(x[0], c, 0, 0), lambda: N.kv8_decode_attn(x[0], c, i.view(3, 1), i, 16, 0),
             lambda: N.kv8_suffix_attn_varlen(x[0], [0], [3], [0], c, 0)]
    for call in calls:
        with pytest.raises(N.NexusError) as e:
            call()
        assert e.value.status == N.EINVAL
