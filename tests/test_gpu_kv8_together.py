"""The 8-bit cache's operators as a serving program uses them: a block spliced into a live cache, the user's
tokens appended, the suffix attended to, then tokens generated in a captured graph, and the block read back."""

import numpy as np
import pytest
import torch

import _kv8 as R
from paper_2608_20397_amd import nexus as N

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("D,Hq,H,cap", [(128, 10, 2, 0.0), (256, 4, 2, 50.0), (64, 8, 1, 0.0)])
def test_a_turn(D, Hq, H, cap):
    L, ctx, blk, user, steps, base = 2, 150, 70, 9, 6, 1e4
    total = ctx + blk + user + steps
    cache = R.make_cache(L, 40, H, D, (total + 15) // 16, base=base, seed=D)
    pm = cache.page_map.cpu().numpy()
    src = {n: (R.rows(s, L, m, H, D, spread=0.3), R.rows(s + 1, L, m, H, D, spread=0.3))
           for s, (n, m) in enumerate((("ctx", ctx), ("blk", blk), ("user", user), ("gen", steps)))}
    N.kv8_append(cache, *src["ctx"], 0, 0)
    # a block compiled at 40, spliced after the context
    bk = torch.from_numpy(R.rotate(R.f64(src["blk"][0]), 40 + np.arange(blk), base, False)).float().cuda()
    N.kv8_splice(cache, N.Block(bk, src["blk"][1].float(), 40, base), ctx, ctx)
    N.kv8_append(cache, *src["user"], ctx + blk, ctx + blk)
    n0 = ctx + blk + user

    # what the cache holds is what the definition says of the same tokens at their positions
    k_all = np.concatenate([R.f64(src[n][0]) for n in ("ctx", "blk", "user", "gen")], 1)
    k_all = R.rotate(k_all, np.arange(total), base, False)
    val, _ = R.quantise(k_all)
    held = R.tokens(R.values(cache, "k")[0], pm, 0, n0)
    # (the block's keys were turned twice and rounded to fp32 between: a border may lie that near)
    assert np.mean(held != val[:, :n0]) < 1e-3

    g = np.random.default_rng(D)
    q = torch.from_numpy(g.standard_normal((blk + user, Hq, D))).to(torch.bfloat16).cuda()
    for layer in range(L):
        got = N.kv8_suffix_attn(q, cache, layer, ctx, softcap=cap)
        k, v = (R.tokens(R.values(cache, x)[0], pm, 0, n0)[layer] for x in ("k", "v"))
        R.assert_attention(R.f64(got), R.attention(R.f64(q), k, v, ctx + 1 + np.arange(blk + user), D ** -0.5,
                                                   cap), "suffix")

    # generation: one captured step (length + 1, append, attention of every layer), replayed
    maps = cache.page_map.view(1, -1)
    lens = torch.full((1,), n0, dtype=torch.int32, device="cuda")
    step_k, step_v = (torch.empty(L, 1, H, D, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    qs = torch.empty(1, Hq, D, dtype=torch.bfloat16, device="cuda")
    outs = [torch.empty_like(qs) for _ in range(L)]
    ws = torch.empty(N.kv8_decode_attn_workspace_bytes(cache, 1, Hq, total) + 16, dtype=torch.uint8,
                     device="cuda")

    def step():
        lens.add_(1)
        N.kv8_append_step(cache, maps, lens, total, step_k, step_v)
        for layer in range(L):
            N.kv8_decode_attn(qs, cache, maps, lens, total, layer, softcap=cap, out=outs[layer], workspace=ws)

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    step_k.copy_(src["gen"][0][:, :1])
    step_v.copy_(src["gen"][1][:, :1])
    qs.copy_(q[:1])
    with torch.cuda.stream(side):
        step()                                  # warm up; the replays below start again from n0
    side.synchronize()
    lens.fill_(n0)
    with torch.cuda.graph(graph):
        step()
    for i in range(steps):
        step_k.copy_(src["gen"][0][:, i:i + 1])
        step_v.copy_(src["gen"][1][:, i:i + 1])
        qs.copy_(q[i:i + 1])
        graph.replay()
        torch.cuda.synchronize()
        n = n0 + i + 1
        assert int(lens) == n
        for layer in range(L):
            k, v = (R.tokens(R.values(cache, x)[0], pm, 0, n)[layer] for x in ("k", "v"))
            ref = R.attention(R.f64(qs), k, v, [n], D ** -0.5, cap)
            R.assert_attention(R.f64(outs[layer]), ref, f"step {i}")
            eager = N.kv8_decode_attn(qs, cache, maps, lens, total, layer, softcap=cap)
            assert torch.equal(eager, outs[layer])
    held = R.tokens(R.values(cache, "k")[0], pm, n0, steps)
    assert np.mean(held != val[:, n0:]) < 1e-3
    # the block, lifted out
    a, b = N.kv8_read(cache, ctx, blk, torch.float32)
    assert np.array_equal(R.f64(a), R.tokens(R.values(cache, "k")[0], pm, ctx, blk))
    assert np.array_equal(R.f64(b), R.quantise(R.f64(src["blk"][1]))[0])


def test_two_graphs_share_a_workspace():
    cache = R.make_cache(1, 300, 8, 128, 280, seed=1)
    k, v = (R.rows(s, 1, 4400, 8, 128, spread=0.3) for s in (20, 21))
    N.kv8_append(cache, k, v, 0, 0)
    q = R.rows(22, 100, 40, 128, spread=0.0)
    maps = cache.page_map.view(1, -1)
    lens = torch.full((1,), 4400, dtype=torch.int32, device="cuda")
    want = (N.kv8_suffix_attn(q, cache, 0, 4300), N.kv8_decode_attn(q[:1], cache, maps, lens, 4400, 0))
    size = max(N.kv8_suffix_attn_workspace_bytes(cache, 100, 40, 4300),
               N.kv8_decode_attn_workspace_bytes(cache, 1, 40, 4400))
    ws = torch.empty(size, dtype=torch.uint8, device="cuda")
    outs = [torch.empty_like(w) for w in want]
    calls = (lambda: N.kv8_suffix_attn(q, cache, 0, 4300, out=outs[0], workspace=ws),
             lambda: N.kv8_decode_attn(q[:1], cache, maps, lens, 4400, 0, out=outs[1], workspace=ws))
    graphs = []
    for call in calls:
        call()
        torch.cuda.synchronize()
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            call()
        graphs.append(g)
    for _ in range(3):
        for o in outs:
            o.zero_()
        for g in graphs + graphs[::-1]:
            g.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(o, w) for o, w in zip(outs, want))
