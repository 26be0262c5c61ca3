"""CPU tests of the ragged-batch entry points and their binding: what each refuses, and with which status.  Every call
here fails validation, so its placeholder pointers are never used."""

import ctypes as C

import pytest
import torch

from paper_2608_20397_amd import nexus as N

P = 0x10000          # a 16-byte aligned placeholder
STEP = 1 << 24       # between placeholders whose ranges must not meet


def _cache(**kw):
    d = dict(k=P, v=P, n_layers=2, n_phys_pages=8, page_size=16, n_kv_heads=2, head_dim=128, dtype=N.BF16,
             v_layout=N.V_ROWMAJOR, rope_style=N.ROPE_NEOX, rope_base=1e4)
    d.update(kw)
    return N.CKvCache(*[d[n] for n, _ in N.CKvCache._fields_])


def pages(cached=STEP, fresh=2 * STEP, n=3, free=3 * STEP, n_free=4 * STEP, capacity=10, maps=5 * STEP, stride=4,
          max_tokens=8, q_start=6 * STEP, seq_len=7 * STEP, pos=8 * STEP, slot=9 * STEP, n_left=10 * STEP):
    return N.lib().nexus_batch_pages(cached, fresh, n, free, n_free, capacity, maps, stride, max_tokens, q_start,
                                     seq_len, pos, slot, n_left, 0)


def append(c=None, layer=0, q=STEP, qs=512, k=2 * STEP, ks=256, v=3 * STEP, vs=256, n=5, hq=4, qw=P, kw=P, eps=1e-6,
           pos=P, slot=P, out=4 * STEP):
    return N.lib().nexus_norm_rope_append(C.byref(c or _cache()), layer, q, qs, k, ks, v, vs, n, hq, qw, kw, eps, pos,
                                          slot, out, 0)


def rows(c=None, q=P, n_rows=6, hq=4, maps=P, stride=4, q_start=P, lens=P, n=3, max_len=64, window=16, sink=4,
         layer=0, cap=0.0, vl=N.V_ROWMAJOR, scale=0.0, out=P, ws=0, nbytes=0):
    return N.lib().nexus_window_attn(q, n_rows, hq, C.byref(c or _cache()), maps, stride, q_start, lens, n, max_len,
                                     window, sink, layer, cap, vl, scale, out, ws, nbytes, 0)


def decode(c=None, q=P, n=3, hq=4, maps=P, stride=4, lens=P, max_len=64, window=16, sink=4, layer=0, cap=0.0,
           vl=N.V_ROWMAJOR, scale=0.0, out=P, ws=0, nbytes=0):
    return N.lib().nexus_window_decode_attn(q, n, hq, C.byref(c or _cache()), maps, stride, lens, max_len, window,
                                            sink, layer, cap, vl, scale, out, ws, nbytes, 0)


@pytest.mark.parametrize("call", [append, rows, decode])
@pytest.mark.parametrize("field,value,status", [
    ("k", 0, N.EINVAL), ("v", 0, N.EINVAL), ("v", P + 8, N.EINVAL), ("k", P + 2, N.EINVAL), ("n_layers", 0, N.EINVAL),
    ("n_layers", 65536, N.ESHAPE), ("n_phys_pages", -1, N.EINVAL), ("n_phys_pages", 1 << 27, N.ESHAPE),
    ("page_size", 32, N.ESHAPE), ("n_kv_heads", 0, N.EINVAL), ("n_kv_heads", 3, N.ESHAPE), ("head_dim", 96, N.ESHAPE),
    ("head_dim", 512, N.ESHAPE), ("dtype", 2, N.EDTYPE), ("rope_style", 2, N.EINVAL), ("v_layout", 2, N.EINVAL),
    ("rope_base", 1.0, N.EROPE), ("rope_base", float("nan"), N.EROPE),
])
def test_every_call_checks_the_cache(call, field, value, status):
    assert call(c=_cache(**{field: value})) == status


@pytest.mark.parametrize("field", ["cached", "fresh", "free", "n_free", "maps", "q_start", "seq_len", "pos", "slot",
                                   "n_left"])
def test_pages_refuses_missing_arrays(field):
    assert pages(**{field: 0}) == N.EINVAL


@pytest.mark.parametrize("kw,status", [
    (dict(n=0), N.EINVAL), (dict(n=-1), N.EINVAL), (dict(n=8193), N.ESHAPE), (dict(capacity=-1), N.EINVAL),
    (dict(stride=0), N.EINVAL), (dict(max_tokens=0), N.EINVAL), (dict(stride=(1 << 25) + 1), N.ERANGE),
    (dict(max_tokens=(1 << 30) + 1, pos=1 << 40, slot=1 << 41), N.ERANGE),
    (dict(n=8192, stride=1 << 18), N.ESHAPE),
    # written arrays that meet what is read or each other: lengths in place, a count in place, one array twice
    (dict(seq_len=STEP), N.EINVAL), (dict(seq_len=2 * STEP + 8), N.EINVAL), (dict(n_left=4 * STEP), N.EINVAL),
    (dict(pos=9 * STEP), N.EINVAL), (dict(slot=8 * STEP + 28), N.EINVAL), (dict(q_start=7 * STEP - 12), N.EINVAL),
    (dict(maps=3 * STEP + 36), N.EINVAL), (dict(n_left=5 * STEP + 44), N.EINVAL),
])
def test_pages_refuses(kw, status):
    assert pages(**kw) == status


@pytest.mark.parametrize("field", ["q", "k", "v", "pos", "slot", "out"])
def test_append_refuses_missing_arrays(field):
    assert append(**{field: 0}) == N.EINVAL


@pytest.mark.parametrize("kw,status", [
    (dict(n=0), N.EINVAL), (dict(layer=-1), N.ERANGE), (dict(layer=2), N.ERANGE), (dict(hq=0), N.ESHAPE),
    (dict(hq=5), N.ESHAPE), (dict(q=STEP + 8), N.EINVAL), (dict(out=4 * STEP + 4), N.EINVAL),
    (dict(qs=508), N.EINVAL), (dict(qs=504), N.EINVAL), (dict(ks=248), N.EINVAL), (dict(vs=0), N.EINVAL),
    (dict(qs=-512), N.EINVAL), (dict(vs=1 << 41), N.EINVAL), (dict(eps=-1e-6), N.EINVAL),
    (dict(eps=float("nan")), N.EINVAL), (dict(eps=float("inf")), N.EINVAL), (dict(eps=0.0), N.EINVAL),
    (dict(eps=0.0, qw=0), N.EINVAL), (dict(n=1 << 24, hq=2), N.ESHAPE), (dict(n=(1 << 22) + 1, hq=2), N.ESHAPE),
    # queries written over rows that are read: over k, into v, over q with rows of another distance, shifted by a row
    (dict(out=2 * STEP), N.EINVAL), (dict(out=3 * STEP - 16), N.EINVAL), (dict(out=STEP, qs=1024), N.EINVAL),
    (dict(out=STEP + 1024), N.EINVAL),
    # rows that lie in the layer they are written to, queries written into it; (another layer's may be read)
    (dict(k=P), N.EINVAL), (dict(v=P + 256), N.EINVAL), (dict(q=P), N.EINVAL), (dict(out=P + 65520), N.EINVAL),
    (dict(k=P + 65536, layer=1), N.EINVAL),
])
def test_append_refuses(kw, status):
    assert append(**kw) == status


@pytest.mark.parametrize("call", [rows, decode])
@pytest.mark.parametrize("kw,status", [
    (dict(q=0), N.EINVAL), (dict(out=0), N.EINVAL), (dict(maps=0), N.EINVAL), (dict(lens=0), N.EINVAL),
    (dict(q=P + 4), N.EINVAL), (dict(out=P + 8), N.EINVAL), (dict(n=0), N.EINVAL), (dict(stride=0), N.EINVAL),
    (dict(window=0), N.EINVAL), (dict(window=-5), N.EINVAL), (dict(sink=-1), N.EINVAL), (dict(hq=3), N.ESHAPE),
    (dict(hq=0), N.ESHAPE), (dict(max_len=65), N.ERANGE), (dict(max_len=-1), N.ERANGE),
    (dict(max_len=(1 << 29) + 1, stride=1 << 26), N.ERANGE), (dict(layer=2), N.ERANGE), (dict(layer=-1), N.ERANGE),
    (dict(vl=N.V_TRANSPOSED), N.ELAYOUT), (dict(vl=7), N.EINVAL), (dict(cap=-1.0), N.EINVAL),
    (dict(cap=float("inf")), N.EINVAL), (dict(scale=float("nan")), N.EINVAL), (dict(scale=-0.5), N.EINVAL),
    (dict(n=65536), N.ESHAPE), (dict(n=40000, stride=1 << 16), N.ESHAPE),
    (dict(c=_cache(head_dim=32)), N.ESHAPE), (dict(c=_cache(head_dim=8, dtype=N.F32)), N.ESHAPE),
    (dict(c=_cache(head_dim=512, dtype=N.F32)), N.ESHAPE),
])
def test_window_refuses(call, kw, status):
    if call is rows and "n" in kw and kw["n"] > 0:
        kw = dict(kw, n_rows=kw["n"])
    assert call(**kw) == status


@pytest.mark.parametrize("call", [rows, decode])
def test_window_refuses_results_over_other_queries(call):
    row = 4 * 128 * 2
    for out in (P + row, P - row, P + 16):
        assert call(out=out) == N.EINVAL
    args = dict(n=1, max_len=4096, window=2048, stride=256)
    for at in (P, P + row - 16, 2 * STEP - 16):
        assert call(out=2 * STEP, ws=at, nbytes=1 << 24, **args) == N.EINVAL


def test_window_rows_refuses():
    assert rows(q_start=0) == N.EINVAL
    assert rows(n_rows=0) == N.EINVAL
    assert rows(n_rows=1 << 23) == N.ESHAPE


def test_window_workspace():
    L, c = N.lib(), _cache()
    big = (1 << 64) - 1
    args = dict(max_len=4096, window=2048, sink=4)
    one = L.nexus_window_decode_attn_workspace(1, 4, C.byref(c), *args.values())
    assert 0 < one < big
    assert decode(n=1, stride=256, ws=0, nbytes=0, **args) == N.EWORKSPACE
    assert decode(n=1, stride=256, ws=P, nbytes=one - 1, **args) == N.EWORKSPACE
    assert decode(n=1, stride=256, ws=P + 4, nbytes=one, **args) == N.EINVAL
    assert L.nexus_window_decode_attn_workspace(4096, 4, C.byref(c), *args.values()) == 0
    assert L.nexus_window_decode_attn_workspace(1, 3, C.byref(c), *args.values()) == big
    assert L.nexus_window_decode_attn_workspace(1, 4, C.byref(c), 4096, 0, 4) == big
    some = L.nexus_window_attn_workspace(8, 4, C.byref(c), 2, *args.values())
    assert 0 < some < big
    assert rows(n_rows=8, n=2, stride=256, ws=P, nbytes=some - 1, **args) == N.EWORKSPACE
    assert L.nexus_window_attn_workspace(100000, 4, C.byref(c), 2, *args.values()) == 0
    assert L.nexus_window_attn_workspace(8, 4, C.byref(c), 0, *args.values()) == big


def test_binding_refuses_host_tensors():
    """The kernels take every pointer for a device address: tensors of the host never reach them."""
    i = lambda *s: torch.zeros(s, dtype=torch.int32)  # noqa: E731
    x = lambda *s: torch.zeros(s, dtype=torch.bfloat16)  # noqa: E731
    with pytest.raises(N.NexusError) as e:
        N.batch_pages(i(2, 4), i(2), i(2), i(9), i(1), 8)
    assert e.value.status == N.EINVAL
    cache = N.PagedKVCache(x(1, 4, 2, 16, 64), x(1, 4, 2, 16, 64), i(4), 1e4)
    for call in (lambda: N.norm_rope_append(cache, 0, x(3, 4, 64), x(3, 2, 64), x(3, 2, 64), i(3), i(3)),
                 lambda: N.window_attn(x(3, 4, 64), cache, i(1, 4), i(2), i(1), 64, 16, 4, 0),
                 lambda: N.window_decode_attn(x(1, 4, 64), cache, i(1, 4), i(1), 64, 16, 4, 0)):
        with pytest.raises(N.NexusError) as e:
            call()
        assert e.value.status == N.EINVAL


def test_window_refuses_more_workgroups_than_a_grid_holds():
    """A grid dimension has fewer than 2^32 threads: 2^24 workgroups of 256, 2^23 of 512 (bf16 rows of head_dim 256).
    65000 sequences make that many with 130 to 258 KV heads."""
    big = (1 << 64) - 1
    for head_dim, dtype, hkv, fits in ((256, N.BF16, 129, True), (256, N.BF16, 130, False), (256, N.BF16, 200, False),
                                       (128, N.BF16, 258, True), (128, N.BF16, 259, False), (64, N.BF16, 200, True),
                                       (256, N.F32, 258, True), (256, N.F32, 259, False)):
        c = _cache(head_dim=head_dim, dtype=dtype, n_kv_heads=hkv, n_phys_pages=1)
        got = N.lib().nexus_window_attn_workspace(1, hkv, C.byref(c), 65000, 64, 16, 4)
        assert (got == 0) if fits else (got == big), (head_dim, dtype, hkv)
        if not fits:
            assert rows(c=c, n_rows=1, hq=hkv, n=65000, max_len=64) == N.ESHAPE


@pytest.mark.parametrize("at", range(4))
@pytest.mark.parametrize("value", [(1 << 32) + 8, 1 << 40, -(1 << 32) + 8, -(1 << 40) + 1])
def test_workspace_sizes_past_32_bits_are_refused(at, value):
    """... where an int32 argument would come round to sizes that are allowed; (a window has no such end)."""
    cache = N.PagedKVCache(*(torch.zeros((1, 4, 2, 16, 128), dtype=torch.bfloat16) for _ in range(2)),
                           torch.zeros(4, dtype=torch.int32), 1e4)
    args = [8, 4, 2, 64]                                   # rows, query heads, sequences, longest
    args[at] = value
    with pytest.raises(N.NexusError) as e:
        N.window_attn_workspace_bytes(cache, *args, 16, 4)
    assert e.value.status == N.EINVAL
    if at != 0:
        with pytest.raises(N.NexusError) as e:
            N.window_decode_attn_workspace_bytes(cache, args[2], args[1], args[3], 16, 4)
        assert e.value.status == N.EINVAL
    if value > 0:
        assert N.window_attn_workspace_bytes(cache, 8, 4, 2, 64, value, value) == 0
    else:
        for window, sinks in ((value, 4), (16, value)):
            with pytest.raises(N.NexusError):
                N.window_attn_workspace_bytes(cache, 8, 4, 2, 64, window, sinks)
