"""The forms that the 8-bit cache's kernels take in launches of their own kind: writers that go through two
layers with one table of angles, decode in workgroups of eight waves."""

import numpy as np
import pytest
import torch

import _kv8 as R
from paper_2608_20397_amd import nexus as N

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype,style", [("bf16", N.ROPE_NEOX), ("f32", N.ROPE_INTERLEAVED)])
def test_append_many_tokens_to_an_odd_number_of_layers(dtype, style):
    D, H, L, n, offset, pos0 = 64, 1, 7, 9601, 13, 4090
    n_map = (offset + n + 15) // 16
    cache = R.make_cache(L, n_map + 1, H, D, n_map, style=style, seed=1)
    k, v = (R.rows(s, L, n, H, D, dtype=dtype) for s in (61, 62))
    N.kv8_append(cache, k, v, offset, pos0)
    pm = cache.page_map.cpu().numpy()
    x = R.rotate(R.f64(k), pos0 + np.arange(n), 1e4, style == N.ROPE_INTERLEAVED)
    for name, src, slack in (("k", x, R.rotation_slack(x)), ("v", R.f64(v), 0)):
        val, byte = R.values(cache, name)
        R.assert_written(R.tokens(val, pm, offset, n), R.tokens(byte, pm, offset, n), src, slack, name)
        assert np.all(R.tokens(byte, pm, 0, offset) == 255)
        assert np.all(np.delete(byte, pm, axis=1) == 255)


def test_append_step_of_many_sequences():
    D, H, L, n = 64, 1, 7, 9601
    lens = (np.arange(n) % 17).astype(np.int32)              # every seventeenth has no token
    cache = R.make_cache(L, n + 1, H, D, 1, seed=2)
    maps = np.random.default_rng(8).permutation(n + 1)[:n].reshape(n, 1).astype(np.int32)
    k, v = (R.rows(s, L, n, H, D) for s in (63, 64))
    N.kv8_append_step(cache, torch.from_numpy(maps).cuda(), torch.from_numpy(lens).cuda(), 16, k, v)
    x = R.rotate(R.f64(k), np.maximum(lens - 1, 0), 1e4, False)
    b = np.flatnonzero(lens)
    at = np.zeros(cache.k_scale.shape, bool)
    at[:, maps[b, 0], :, lens[b] - 1] = True
    for name, src, slack in (("k", x, R.rotation_slack(x)), ("v", R.f64(v), 0)):
        val, byte = R.values(cache, name)
        pick = lambda a: np.moveaxis(a[:, maps[b, 0], :, lens[b] - 1], 0, 1)
        s = slack if np.isscalar(slack) else slack[:, b]
        R.assert_written(pick(val), pick(byte), src[:, b], s, name)
        assert np.all(byte[~at] == 255)


@pytest.mark.parametrize("D,Hq,H", [(64, 10, 2), (64, 32, 1), (128, 8, 4), (128, 7, 1)])
@pytest.mark.parametrize("lens", [[2003], [700, 0, 1], [513, 1024, 1500, 40, 17]])
def test_decode_of_few_sequences(D, Hq, H, lens):
    n, stride = len(lens), (max(lens) + 15) // 16
    cache = R.make_cache(1, n * stride, H, D, n * stride, seed=D + n)
    maps = cache.page_map.cpu().numpy().reshape(n, stride)
    k, v = (R.rows(s, 1, n * stride * 16, H, D, spread=0.5) for s in (65, 66))
    N.kv8_splice(cache, N.Block(k, v, 0, 1e4), 0, 0)
    for b, m in enumerate(lens):                             # nothing that no query may read
        for x in (cache.k, cache.v):
            x.view(torch.uint8)[0, maps[b, (m + 15) // 16:].tolist()] = 0x7F
            if m % 16:
                x.view(torch.uint8)[0, int(maps[b, m // 16]), :, m % 16:] = 0x7F
    g = np.random.default_rng([20397, 82, D, n])
    q = torch.from_numpy(g.standard_normal((n, Hq, D))).to(torch.bfloat16).cuda()
    got = R.f64(N.kv8_decode_attn(q, cache, torch.from_numpy(maps).cuda(),
                                  torch.from_numpy(np.array(lens, np.int32)).cuda(), max(lens), 0))
    kv = {x: R.values(cache, x)[0] for x in ("k", "v")}
    for b, m in enumerate(lens):
        if m == 0:
            assert np.all(got[b] == 0)
            continue
        kk, vv = (R.tokens(kv[x], maps[b], 0, m)[0] for x in ("k", "v"))
        R.assert_attention(got[b:b + 1], R.attention(R.f64(q)[b:b + 1], kk, vv, [m], D ** -0.5, 0.0),
                           f"D={D} length {m}")


@pytest.mark.parametrize("bound", [0, 300, 1 << 21])
def test_decode_reads_no_page_that_a_length_does_not_name(bound):
    """Map entries past a sequence's pages are anything at all; a bound of no tokens gives zeros; a bound far above
    the lengths takes the launches that look for shared pages."""
    D, H, Hq, n = 128, 2, 8, 4
    lens = [min(m, bound) for m in (290, 0, 17, 288)]
    stride = max(1, (bound + 15) // 16)
    cache = R.make_cache(1, 60, H, D, 60, seed=3)
    k, v = (R.rows(s, 1, 960, H, D, spread=0.5) for s in (67, 68))
    N.kv8_splice(cache, N.Block(k, v, 0, 1e4), 0, 0)
    own = np.random.default_rng(9).permutation(60).astype(np.int32)
    maps = np.full((n, stride), -2 ** 31, np.int32)
    maps[:, 1::2] = 2 ** 31 - 1
    for b, m in enumerate(lens):
        pages = (m + 15) // 16
        maps[b, :pages] = own[:pages] if b in (0, 3) else own[30 + b:30 + b + pages]
    q = torch.from_numpy(np.random.default_rng(10).standard_normal((n, Hq, D))).to(torch.bfloat16).cuda()
    got = R.f64(N.kv8_decode_attn(q, cache, torch.from_numpy(maps).cuda(),
                                  torch.from_numpy(np.array(lens, np.int32)).cuda(), bound, 0))
    kv = {x: R.values(cache, x)[0] for x in ("k", "v")}
    for b, m in enumerate(lens):
        if m == 0:
            assert np.all(got[b] == 0)
            continue
        kk, vv = (R.tokens(kv[x], maps[b], 0, m)[0] for x in ("k", "v"))
        R.assert_attention(got[b:b + 1], R.attention(R.f64(q)[b:b + 1], kk, vv, [m], D ** -0.5, 0.0), f"length {m}")


def test_calls_on_two_streams_at_once():
    """Suffix attention and decode of two caches, side by side with workspaces of their own, against one after
    the other; codes held as bytes."""
    D, H, Hq = 128, 8, 40
    jobs = []
    for seed in (70, 71):
        cache = R.make_cache(1, 300, H, D, 300, seed=seed)
        k, v = (R.rows(seed + s, 1, 4500, H, D, spread=0.5) for s in (0, 100))
        N.kv8_splice(cache, N.Block(k, v, 0, 1e4), 0, 0)
        cache = N.KV8Cache(cache.k.view(torch.uint8), cache.v.view(torch.uint8), cache.k_scale, cache.v_scale,
                           cache.page_map, 1e4)
        q = torch.from_numpy(np.random.default_rng(seed).standard_normal((150, Hq, D))).to(torch.bfloat16).cuda()
        maps = cache.page_map[:282].view(1, -1).repeat(3, 1).contiguous()
        lens = torch.tensor([4500, 4001, 77], dtype=torch.int32, device="cuda")
        cache.pt()                                    # (checks the map: a copy to the host)
        jobs.append((cache, q, maps, lens))

    def run(job):
        cache, q, maps, lens = job
        return [(N.kv8_suffix_attn(q, cache, 0, 4350), N.kv8_decode_attn(q[:3].contiguous(), cache, maps, lens, 4500, 0))
                for _ in range(4)]

    alone = [run(j) for j in jobs]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in jobs]
    both = []
    for s, j in zip(streams, jobs):
        with torch.cuda.stream(s):
            both.append(run(j))
    torch.cuda.synchronize()
    for a, b in zip(alone, both):
        for (s1, d1), (s2, d2) in zip(a, b):
            assert torch.equal(s1, s2) and torch.equal(d1, d2)
