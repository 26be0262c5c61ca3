"""Rounds as a server runs them: the layout, the append and the attention of a ragged batch together, eager and captured;
against the same tokens' attention in 64 bits over dense keys and values, and beside the framework's other calls."""

import numpy as np
import pytest
import torch

from _batch import HALF, PAGE, U, f64, i32, lay_out, norm_rope, within
from paper_2608_20397_amd import nexus as N

pytestmark = pytest.mark.gpu

B, F = torch.bfloat16, torch.float32


class Server:
    """Sequences of one layer that grow by rounds; the reference keeps every token's rotated key and value."""

    def __init__(self, n_seqs, hq, hkv, dim, dtype, vt, seed, window=40, sinks=3, n_phys=60, stride=12, max_tokens=64,
                 eps=1e-5):
        self.g = torch.Generator().manual_seed(seed)
        self.hq, self.hkv, self.dim, self.dtype, self.vt = hq, hkv, dim, dtype, vt
        self.window, self.sinks, self.eps, self.max_tokens, self.stride = window, sinks, eps, max_tokens, stride
        shape = (1, n_phys, hkv, PAGE, dim)
        nan = lambda s: torch.full(s, float("nan"), dtype=dtype, device="cuda")  # noqa: E731
        self.maps = torch.full((n_seqs, stride), n_phys - 1, dtype=torch.int32, device="cuda")
        self.cache = N.PagedKVCache(nan(shape), nan((1, hkv, dim, n_phys * PAGE) if vt else shape), self.maps[0], 1e4,
                                    N.V_TRANSPOSED if vt else N.V_ROWMAJOR)
        self.weights = [1 + 0.2 * torch.randn(dim, generator=self.g) for _ in range(2)]
        self.free = i32(torch.randperm(n_phys - 1, generator=self.g))      # (the last page stays NaN)
        self.n_free = i32([n_phys - 1])
        self.cached, self.fresh = i32([0] * n_seqs), i32([0] * n_seqs)
        self.qkv = torch.zeros((max_tokens, hq + 2 * hkv, dim), dtype=dtype, device="cuda")
        self.rows = N.BatchRows.empty(n_seqs, max_tokens, "cuda")
        self.q = torch.zeros((max_tokens, hq, dim), dtype=dtype, device="cuda")
        self.out = torch.zeros_like(self.q)
        self.dev_weights = [w.cuda() for w in self.weights]
        need = N.window_attn_workspace_bytes(self.cache, max_tokens, hq, n_seqs, stride * PAGE, window, sinks)
        self.ws = torch.empty(max(need, 16), dtype=torch.uint8, device="cuda")
        self.tokens = [([], []) for _ in range(n_seqs)]      # rotated keys as held, values: fp64 [H][D]
        self.lens = [0] * n_seqs

    def launch(self):
        N.batch_pages(self.maps, self.cached, self.fresh, self.free, self.n_free, self.max_tokens, out=self.rows)
        q, k, v = self.qkv.split((self.hq, self.hkv, self.hkv), 1)
        N.norm_rope_append(self.cache, 0, q, k, v, self.rows.pos, self.rows.slot, q_weight=self.dev_weights[0],
                           k_weight=self.dev_weights[1], eps=self.eps, out=self.q)
        N.window_attn(self.q, self.cache, self.maps, self.rows.q_start, self.rows.seq_len, self.stride * PAGE,
                      self.window, self.sinks, 0, out=self.out, workspace=self.ws)

    def stage(self, fresh):
        """A round's inputs on the device."""
        self.new = torch.randn(self.qkv.shape, generator=self.g).to(self.dtype)
        self.qkv.copy_(self.new)
        self.fresh.copy_(i32(fresh))
        self.cached.copy_(i32(self.lens))
        self.out.fill_(7.0)

    def check(self, fresh, what):
        """The round's results, and the state that the next one starts from."""
        before = self.n_free.item()
        got, at = f64(self.out), 0
        held_q = f64(self.q)
        for b, f in enumerate(fresh):
            x = f64(self.new[at:at + f])
            pos = self.lens[b] + np.arange(f)
            ref_q, both = norm_rope(x[:, :self.hq], f64(self.weights[0]), self.eps, pos, 1e4, False)
            ref_k, both_k = norm_rope(x[:, self.hq:self.hq + self.hkv], f64(self.weights[1]), self.eps, pos, 1e4, False)
            steps = (self.dim / 2 + 10) * U
            within(held_q[at:at + f], ref_q, HALF[self.dtype] * 1.001 * np.abs(ref_q) + steps * both, "q " + what)
            keys, values = self.tokens[b]
            for i in range(f):
                slot = self.rows.slot[at + i].item()
                k = f64(self.cache.k[0, slot // PAGE, :, slot % PAGE])
                within(k, ref_k[i], HALF[self.dtype] * 1.001 * np.abs(ref_k[i]) + steps * both_k[i], "k " + what)
                keys.append(k)                       # as held: what follows reads these
                values.append(x[i, self.hq + self.hkv:])
            for i in range(f):
                p = int(pos[i])
                see = np.array([t for t in range(p + 1) if t > p - self.window or t < self.sinks])
                ks, vs = np.stack(keys)[see], np.stack(values)[see]
                for h in range(self.hq):
                    kh, vh, qh = ks[:, h * self.hkv // self.hq], vs[:, h * self.hkv // self.hq], held_q[at + i, h]
                    s = kh @ qh / np.sqrt(self.dim)
                    w = np.exp(s - s.max())
                    w /= w.sum()
                    ref, mag = w @ vh, w @ np.abs(vh)
                    size = (np.abs(kh) @ np.abs(qh)).max() / np.sqrt(self.dim)
                    fp32 = (2 * (self.dim + 4) * size + len(see) + 64) * U
                    wb = HALF[self.dtype] if self.dtype == B else 0.0
                    bound = (wb + fp32) * (mag + np.abs(ref)) * 1.01 + HALF[self.dtype] * 1.01 * np.abs(ref)
                    assert (np.abs(got[at + i, h] - ref) <= bound).all(), (what, b, p, h)
            at += f
            self.lens[b] += f
        assert (got[at:] == 7.0).all(), what
        assert self.rows.n_left.item() <= before
        self.n_free.copy_(self.rows.n_left)


ROUNDS = [[20, 0, 7, 33], [1, 1, 1, 1], [1, 40, 0, 1], [0, 0, 0, 0], [1, 1, 30, 1], [16, 1, 1, 15]]


@pytest.mark.parametrize("hq,hkv,dim,dtype,vt", [(4, 2, 64, B, False), (5, 1, 128, B, True), (2, 1, 256, B, True),
                                                 (4, 2, 32, F, False), (4, 4, 16, F, True)])
def test_rounds(hq, hkv, dim, dtype, vt):
    s = Server(4, hq, hkv, dim, dtype, vt, seed=dim)
    for r, fresh in enumerate(ROUNDS):
        s.stage(fresh)
        s.launch()
        torch.cuda.synchronize()
        s.check(fresh, f"round {r}")


def test_rounds_captured():
    """One capture of the three calls, replayed for rounds of other lengths, with eager work and synchronizations
    between; every replay against the definition, and a replay of the same round the same bits."""
    s = Server(4, 4, 2, 64, B, False, seed=99)
    s.stage(ROUNDS[0])
    s.launch()                                        # eager first: what capture must not do for the first time
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        s.launch()
    for r, fresh in enumerate(ROUNDS):
        s.stage(fresh)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        first = s.out.clone()
        s.out.fill_(7.0)
        (s.qkv.float() @ torch.ones(64, device="cuda")).sum().item()       # eager work of the program's own
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(first.view(torch.int16), s.out.view(torch.int16)), r
        s.check(fresh, f"replay {r}")


def test_two_graphs_share_a_workspace():
    """Graphs captured over one workspace and replayed in turn on one stream."""
    hq, hkv, dim, n = 8, 2, 128, 1000
    g = torch.Generator(device="cuda").manual_seed(1)
    k, v = (torch.randn((1, 70, hkv, PAGE, dim), generator=g, device="cuda").to(B) for _ in range(2))
    maps = torch.randperm(70, generator=g, device="cuda").to(torch.int32)[None, :63].contiguous()
    cache = N.PagedKVCache(k, v, maps[0], 1e4)
    q = torch.randn((40, hq, dim), generator=g, device="cuda").to(B)
    one = torch.randn((1, hq, dim), generator=g, device="cuda").to(B)
    lens, start = i32([n]), i32([0, 40])
    rows = lambda **kw: N.window_attn(q, cache, maps, start, lens, n, 700, 4, 0, **kw)  # noqa: E731
    step = lambda **kw: N.window_decode_attn(one, cache, maps, lens, n, 900, 4, 0, **kw)  # noqa: E731
    size = max(N.window_attn_workspace_bytes(cache, 40, hq, 1, n, 700, 4),
               N.window_decode_attn_workspace_bytes(cache, 1, hq, n, 900, 4))
    assert size > 0
    ws = torch.empty(size, dtype=torch.uint8, device="cuda")
    want, outs, graphs = [rows(), step()], [torch.empty_like(q), torch.empty_like(one)], []
    for call, out in ((rows, outs[0]), (step, outs[1])):
        call(out=out, workspace=ws)
        torch.cuda.synchronize()
        graphs.append(torch.cuda.CUDAGraph())
        with torch.cuda.graph(graphs[-1]):
            call(out=out, workspace=ws)
    for _ in range(4):
        for i in (0, 1, 1, 0):
            outs[i].fill_(float("nan"))
            ws.fill_(255)                             # (what a workspace holds does not matter: NaN everywhere)
            graphs[i].replay()
            torch.cuda.synchronize()
            assert torch.equal(outs[i].view(torch.int16), want[i].view(torch.int16))


def test_large_layout_captured():
    """A layout whose sums take more LDS than a launch gets unasked, captured and replayed."""
    n = 6000
    rng = np.random.default_rng(3)
    fresh, maps = rng.integers(0, 3, n), np.full((n, 4), -1)
    free = rng.permutation(9000)
    dmaps, dfresh, cached = i32(maps), i32(fresh), i32([0] * n)
    dfree, n_free = i32(free), i32([9000])
    rows = N.BatchRows.empty(n, 13000, "cuda")
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        N.batch_pages(dmaps, cached, dfresh, dfree, n_free, 13000, out=rows)
    for seed in (4, 5, 6):
        fresh = np.random.default_rng(seed).integers(0, 4 if seed < 6 else 2, n)
        dfresh.copy_(i32(fresh))
        dmaps.copy_(i32(maps))
        graph.replay()
        torch.cuda.synchronize()
        want = lay_out([0] * n, fresh.tolist(), free, 9000, maps, 13000)
        for got, ref in zip((dmaps, rows.q_start, rows.seq_len, rows.pos, rows.slot, rows.n_left), want):
            assert np.array_equal(got.cpu().numpy().reshape(-1), np.reshape(ref, -1))


def test_two_streams_at_once():
    """Rounds of two servers on two streams, overlapping, each as alone."""
    def results(streams):
        servers = [Server(4, 4, 2, 64, B, False, seed=s) for s in (1, 2)]
        torch.cuda.synchronize()
        outs = []
        for _ in range(6):
            for s, st in zip(servers, streams):
                with torch.cuda.stream(st):
                    s.stage([5, 1, 9, 0])
                    s.launch()
                    s.lens = [a + b for a, b in zip(s.lens, [5, 1, 9, 0])]
                    s.n_free.copy_(s.rows.n_left)
                    outs.append(s.out.clone())
        torch.cuda.synchronize()
        return outs

    cur = torch.cuda.current_stream()
    for a, b in zip(results([cur, cur]), results([torch.cuda.Stream(), torch.cuda.Stream()])):
        assert torch.equal(a.view(torch.int16), b.view(torch.int16))


def test_beside_the_calls_without_a_window():
    """A window that nothing outgrows gives what suffix_attn and decode_attn give, within their shared bounds."""
    hq, hkv, dim, n, rows = 8, 2, 128, 600, 70
    g = torch.Generator(device="cuda").manual_seed(7)
    k, v = (torch.randn((1, 50, hkv, PAGE, dim), generator=g, device="cuda").to(B) for _ in range(2))
    pm = torch.randperm(50, generator=g, device="cuda").to(torch.int32)[:38].contiguous()
    cache = N.PagedKVCache(k, v, pm, 1e4)
    q = torch.randn((rows, hq, dim), generator=g, device="cuda").to(B)
    a = N.window_attn(q, cache, pm[None], i32([0, rows]), i32([n]), n, n, 0, 0)
    b = N.suffix_attn(q, cache, 0, n - rows)
    # both within 3 roundings of 2^-8 of the mean of values of magnitude under 5
    assert (a.float() - b.float()).abs().max() <= 2 * 3 * 5 * 2.0 ** -8
    c = N.window_decode_attn(q[-1:].contiguous(), cache, pm[None], i32([n]), n, n, 0, 0)
    d = N.decode_attn(q[-1:].contiguous(), cache, pm[None], i32([n]), n, 0)
    assert (c.float() - d.float()).abs().max() <= 2 * 3 * 5 * 2.0 ** -8


def test_append_beside_rope_append():
    """Without a norm, rows in slots of a run are what rope_append writes there: fp32 keys the same bits, bf16 ones
    within a step, values as they are."""
    for dtype, vt in ((F, False), (B, False), (F, True), (B, True)):
        hkv, dim, n = 2, 64, 37
        x = torch.randn((n, 3 * hkv, dim), generator=torch.Generator().manual_seed(5)).to(dtype).cuda()
        q, k, v = x.split((hkv, hkv, hkv), 1)
        made = []
        for own in (True, False):
            shape = (1, 4, hkv, PAGE, dim)
            cache = N.PagedKVCache(torch.zeros(shape, dtype=dtype, device="cuda"),
                                   torch.zeros((1, hkv, dim, 64) if vt else shape, dtype=dtype, device="cuda"),
                                   i32([2, 0, 3, 1]), 1e6, N.V_TRANSPOSED if vt else N.V_ROWMAJOR)
            if own:
                t = np.arange(n) + 5
                slot = np.array([2, 0, 3, 1])[t // PAGE] * PAGE + t % PAGE
                N.norm_rope_append(cache, 0, q, k, v, i32(np.arange(n) + 900), i32(slot))
            else:
                N.rope_append(cache, k.contiguous()[None], v.contiguous()[None], 5, 900)
            made.append(cache)
        torch.cuda.synchronize()
        assert torch.equal(made[0].v, made[1].v)
        a, b = made[0].k.double(), made[1].k.double()
        assert ((a - b).abs() <= (0 if dtype == F else 2.0 ** -7) * b.abs()).all()


@pytest.mark.parametrize("fresh", [[70, 1, 0, 2], [0, 65, 1, 0]])
def test_a_round_whose_first_sequence_is_longer_than_the_launch(fresh):
    """Its rows and those behind it are refused: nothing is appended, attention writes zeros and reads no page, and the
    next round goes on from the state before."""
    s = Server(4, 4, 2, 64, B, False, seed=5)
    s.maps.fill_(-1)
    s.stage(fresh)
    s.launch()
    torch.cuda.synchronize()
    assert s.rows.seq_len.tolist() == [0] * 4 and s.rows.n_left.item() == s.n_free.item()
    assert (s.rows.pos == -1).all() and (s.rows.slot == -1).all() and (s.maps == -1).all()
    assert (s.out == 0).all() and torch.isnan(s.cache.k).all()
    s.stage([20, 1, 0, 3])
    s.launch()
    torch.cuda.synchronize()
    s.check([20, 1, 0, 3], "the round after")


def test_arguments_past_32_bits_are_refused():
    """... and not brought round to ones that are allowed."""
    s = Server(4, 4, 2, 64, B, False, seed=6)
    s.stage([5, 1, 9, 0])
    s.launch()
    torch.cuda.synchronize()
    s.check([5, 1, 9, 0], "a round")
    q, k, v = s.qkv.split((4, 2, 2), 1)
    top = s.stride * PAGE
    pages = lambda n: N.batch_pages(s.maps, s.cached, s.fresh, s.free, s.n_free, n)  # noqa: E731
    append = lambda layer: N.norm_rope_append(s.cache, layer, q, k, v, s.rows.pos, s.rows.slot)  # noqa: E731
    rows = lambda n=top, layer=0, window=40: N.window_attn(s.q, s.cache, s.maps, s.rows.q_start,  # noqa: E731
                                                           s.rows.seq_len, n, window, 3, layer)
    step = lambda n=top, layer=0, window=40: N.window_decode_attn(s.q[:4], s.cache, s.maps, s.rows.seq_len,  # noqa: E731
                                                                  n, window, 3, layer)
    far = 1 << 32
    for call, status in ((lambda: pages(far + 64), N.ERANGE), (lambda: pages(-far + 64), N.EINVAL),
                         (lambda: append(far), N.ERANGE), (lambda: append(-far), N.ERANGE),
                         (lambda: rows(n=far + top), N.ERANGE), (lambda: rows(layer=far), N.ERANGE),
                         (lambda: rows(window=-far + 40), N.EINVAL), (lambda: step(n=far + top), N.ERANGE),
                         (lambda: step(layer=-far), N.ERANGE), (lambda: step(window=-far + 40), N.EINVAL)):
        with pytest.raises(N.NexusError) as e:
            call()
        assert e.value.status == status
