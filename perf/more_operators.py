"""The operators of a serving round over a ragged batch of sequences with page maps of their own, as timed
cases: what each prepares, runs, returns and cannot do without.

A round takes some fresh tokens of every sequence: one of a sequence that generates, a chunk of a prompt that
is being read, none of one that waits.  Four operators carry it, the first once and the others in every layer:

    pages    the batch laid out on the device: rows of each sequence, its new length, pages out of a free list
             into its page map, position and cache slot of every row
    append   the rows' queries and keys normalised per head (root mean square, a weight per feature) and
             rotated to their positions, the keys written with the values to their slots
    attn     attention in a sliding window with the first tokens (sinks) in sight: the query at position p
             sees key k when k <= p and (k > p - window or k < sinks)
    decode   the same for one query a sequence

``own`` false: the plain forms, elementary torch operations in 32 bits (64 for rotations, whose angles grow
with the position).  ``own`` true: the calls of this package's entry points.
"""

import math
import random

import numpy as np
import torch

own = False

PAGE = 16
ALL = 1 << 30          # a window that no sequence outgrows
EPS = 1e-6

# Attention geometries: (query heads, KV heads, head_dim, rope base, transposed V, soft cap), those of perf/cases.py.
GEOMETRIES = {
    "qwen14b": (40, 8, 128, 1e6, False, 0.0),       # the attention shapes of the headline workload
    "gemma": (16, 8, 256, 1e4, True, 50.0),         # soft-capped, token-innermost V cache
    "d64": (32, 8, 64, 1e6, False, 0.0),            # a small model's heads
    "d64wide": (64, 2, 64, 1e6, False, 0.0),        # 32 query heads per KV head
    "d128vt": (40, 8, 128, 1e6, True, 0.0),         # transposed V without a cap
    "d256": (16, 8, 256, 1e4, False, 50.0),         # capped, row-major V
    "tiny": (4, 1, 64, 1e4, False, 0.0),            # the smallest configuration's heads
}


def listed():
    return [
        # the pages of a step in which 32 sequences generate: latency
        dict(name="pages_step", kind="pages", n_seqs=32, min_q=1, max_q=1, min_past=16385, max_past=17472,
             pad=0, short=False, lens=1),
        # prompts and generation mixed in one large round, more pages wanted than are free
        dict(name="pages_round", kind="pages", n_seqs=256, min_q=0, max_q=511, min_past=0, max_past=17000,
             pad=1000, short=True, lens=2),
        # one generated token of one layer, the smallest append
        dict(name="append_step", kind="append", geom="qwen14b", dtype="bf16", n_tokens=1, max_pos=17472, pad=0,
             norm=True, interleaved=False),
        # a chunk of prompts, one layer, rows of a packed projection
        dict(name="append_chunk", kind="append", geom="qwen14b", dtype="bf16", n_tokens=4096, max_pos=16384,
             pad=0, norm=True, interleaved=False),
        # an fp32 model of the other pairing, a token-innermost V cache, rows of padding
        dict(name="append_f32", kind="append", geom="d128vt", dtype="f32", n_tokens=1001, max_pos=9219, pad=23,
             norm=True, interleaved=True),
        # a chunk of a long prompt behind four sinks, the largest
        dict(name="window_chunk", kind="attn", geom="qwen14b", dtype="bf16", n_seqs=1, min_q=4096, max_q=4096,
             min_past=12288, max_past=12288, window=4096, sinks=4, pad=0, lens=3),
        # a round of sixteen sequences, some with a token or none, a small model's heads
        dict(name="window_round", kind="attn", geom="d64", dtype="bf16", n_seqs=16, min_q=0, max_q=517,
             min_past=0, max_past=6000, window=1024, sinks=1, pad=50, lens=4),
        # a layer of a soft-capped model with local attention: head_dim 256, transposed V
        dict(name="window_softcap", kind="attn", geom="gemma", dtype="bf16", n_seqs=2, min_q=512, max_q=1024,
             min_past=7000, max_past=8192, window=4096, sinks=0, pad=0, lens=5),
        # a short fp32 suffix, the precision a deployment is checked against
        dict(name="window_f32", kind="attn", geom="tiny", dtype="f32", n_seqs=3, min_q=1, max_q=77, min_past=0,
             max_past=900, window=256, sinks=4, pad=0, lens=6),
        # one sequence that generates, deep behind its sinks
        dict(name="decode_one", kind="decode", geom="qwen14b", dtype="bf16", n_seqs=1, min_len=17473,
             max_len=17473, window=4096, sinks=4),
        # a serving batch of ragged lengths
        dict(name="decode_batch", kind="decode", geom="qwen14b", dtype="bf16", n_seqs=32, min_len=16385,
             max_len=17473, window=4096, sinks=4),
        # many short sequences, 32 query heads on each KV head, some of length 0 or 1, a narrow window
        dict(name="decode_short", kind="decode", geom="d64wide", dtype="bf16", n_seqs=48, min_len=0, max_len=700,
             window=128, sinks=1),
    ]


def _log_int(rng, lo, hi):
    return min(hi, max(lo, int(math.exp(rng.uniform(math.log(lo), math.log(hi + 1))))))


def draw(rng):
    kind = rng.choice(["pages", "append", "append", "attn", "attn", "attn", "decode", "decode"])
    lens = rng.randrange(1 << 30)
    if kind == "pages":
        n_seqs = _log_int(rng, 1, 1024)
        max_q = _log_int(rng, 1, max(1, 131072 // n_seqs))
        max_past = _log_int(rng, 1, 32768) - 1
        return dict(kind=kind, n_seqs=n_seqs, min_q=rng.choice([0, 1, max_q]), max_q=max_q,
                    min_past=rng.choice([0, max_past]), max_past=max_past,
                    pad=rng.choice([0, rng.randrange(1, 500)]), short=rng.random() < 0.3, lens=lens)
    geom = rng.choice(sorted(GEOMETRIES))
    hq, hkv, dim, _, vt, _ = GEOMETRIES[geom]
    dtype = rng.choice(["bf16", "bf16", "bf16", "f32"])
    if kind == "append":
        wide = 2 if dtype == "f32" else 1
        # at most as many elements as the largest listed append
        n_tokens = _log_int(rng, 1, min(16384, 4096 * 40 * 128 // (hq * dim * wide)))
        return dict(kind=kind, geom=geom, dtype=dtype if not (vt and dim == 256) else "bf16", n_tokens=n_tokens,
                    max_pos=max(n_tokens, _log_int(rng, 1, 131072)), pad=rng.choice([0, 0, rng.randrange(1, 40)]),
                    norm=rng.random() < 0.8, interleaved=rng.random() < 0.3)
    window = rng.choice([ALL, _log_int(rng, 1, 8192), _log_int(rng, 16, 8192), _log_int(rng, 128, 8192)])
    sinks = rng.choice([0, 1, 4, 4, 16, rng.randrange(1, 200)])
    if kind == "decode":
        n_seqs = _log_int(rng, 1, 64)
        # at most as many keys as the largest listed batch sees
        max_len = _log_int(rng, 1, min(40000, 32 * 17000 * 8 * 128 // (n_seqs * hkv * dim)))
        if dtype == "f32" and max_len * n_seqs > 40000:
            dtype = "bf16"
        return dict(kind=kind, geom=geom, dtype=dtype, n_seqs=n_seqs, max_len=max_len,
                    min_len=rng.choice([0, 1, max(1, max_len * 9 // 10), max_len]),
                    window=min(window, 4096 * 32 * 8 * 128 // (n_seqs * hkv * dim)), sinks=sinks)
    n_seqs = rng.choice([1, 1, rng.randrange(2, 9), _log_int(rng, 2, 64)])
    while True:
        max_q = _log_int(rng, 1, 4096)
        max_past = rng.choice([0, _log_int(rng, 1, 20000)])
        padded = n_seqs * max_q * (max_past + max_q)
        if padded * hq * (8 if dtype == "f32" else 1) <= 4096 * 16384 * 40 and \
                n_seqs * (max_past + max_q) * hkv * dim <= 1 << 28:
            break
    return dict(kind=kind, geom=geom, dtype=dtype, n_seqs=n_seqs, min_q=rng.choice([0, 1, max_q]), max_q=max_q,
                min_past=rng.choice([0, max_past]), max_past=max_past, window=window, sinks=sinks,
                pad=rng.choice([0, 0, rng.randrange(1, 100)]), lens=lens)


# ---- inputs


def _gen(seed):
    return torch.Generator(device="cuda").manual_seed(20397 * 1000 + seed)


def _rows(g, *shape, dtype=torch.float32):
    """Rows as a model computes them: Gaussian features, tokens of different strength."""
    x = torch.randn(shape, generator=g, device="cuda")
    return x.mul_(torch.exp(0.4 * torch.randn(shape[:-1] + (1,), generator=g, device="cuda"))).to(dtype)


def _dtype(case):
    return torch.bfloat16 if case["dtype"] == "bf16" else torch.float32


def _batch(case):
    """Fresh and cached tokens of each sequence; the first has the most of both."""
    rng = random.Random(case["lens"])
    fresh = [rng.randint(case["min_q"], case["max_q"]) for _ in range(case["n_seqs"])]
    past = [rng.randint(case["min_past"], case["max_past"]) for _ in range(case["n_seqs"])]
    return [case["max_q"]] + fresh[1:], [case["max_past"]] + past[1:]


def _int32(x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


def _pages(tokens):
    return (tokens + PAGE - 1) // PAGE


def _prepare_pages(case, g):
    fresh, past = _batch(case)
    stride = _pages(case["max_past"] + case["max_q"])
    held = [_pages(p) for p in past]
    wanted = sum(_pages(p + f) - h for p, f, h in zip(past, fresh, held))
    n_free = wanted * 3 // 4 if case["short"] else wanted + 100
    order = torch.randperm(sum(held) + n_free + 7, generator=g, device="cuda").to(torch.int32)
    maps = torch.full((case["n_seqs"], stride), -1, dtype=torch.int32, device="cuda")
    mapped = torch.arange(stride, device="cuda") < _int32(held)[:, None]
    maps[mapped] = order[:sum(held)]
    # sequences in an order of their own each time
    perm = torch.randperm(case["n_seqs"], generator=g, device="cuda")
    return dict(cached=_int32(past)[perm], fresh=_int32(fresh)[perm], maps=maps[perm].contiguous(),
                free=order[sum(held):].contiguous(), n_free=_int32([n_free]),
                max_tokens=max(1, sum(fresh) + case["pad"]))


def _prepare_append(case, g):
    hq, hkv, dim, base, vt, _ = GEOMETRIES[case["geom"]]
    dt, n = _dtype(case), case["n_tokens"]
    rows = n + case["pad"]
    n_phys = _pages(n) + 3
    qkv = _rows(g, rows, hq + 2 * hkv, dim, dtype=dt)
    # runs of up to 16 tokens of one page, pages in any order, the run's first position anywhere
    page = torch.randperm(n_phys, generator=g, device="cuda")[:_pages(n)]
    slot = (page[:, None] * PAGE + torch.arange(PAGE, device="cuda")).view(-1)[:n]
    first = torch.randint(0, case["max_pos"] - n + 1, (1,), generator=g, device="cuda")
    pos = first + torch.arange(n, device="cuda")
    fill = torch.full((case["pad"],), -1, device="cuda")
    shape = (1, n_phys, hkv, PAGE, dim)
    weights = [1 + 0.2 * torch.randn((2, dim), generator=g, device="cuda")] if case["norm"] else [[None, None]]
    return dict(q=qkv[:, :hq], k_new=qkv[:, hq:hq + hkv], v_new=qkv[:, hq + hkv:],
                slot=torch.cat([slot, fill]).to(torch.int32), pos=torch.cat([pos, fill]).to(torch.int32),
                q_out=torch.zeros((rows, hq, dim), dtype=dt, device="cuda"), q_weight=weights[0][0],
                k_weight=weights[0][1], k=torch.zeros(shape, dtype=dt, device="cuda"),
                v=torch.zeros((1, hkv, dim, n_phys * PAGE) if vt else shape, dtype=dt, device="cuda"),
                maps=torch.arange(n_phys, dtype=torch.int32, device="cuda")[None])


def _cache(case, g, n_seqs, n_pages):
    _, hkv, dim, _, vt, _ = GEOMETRIES[case["geom"]]
    n_phys = n_seqs * n_pages
    shape = (1, n_phys, hkv, PAGE, dim)
    maps = torch.randperm(n_phys, generator=g, device="cuda").to(torch.int32).view(n_seqs, n_pages)
    v = _rows(g, *shape, dtype=_dtype(case))
    if vt:
        v = v.permute(0, 2, 4, 1, 3).reshape(1, hkv, dim, n_phys * PAGE).contiguous()
    return dict(k=_rows(g, *shape, dtype=_dtype(case)), v=v, maps=maps)


def _prepare_attn(case, g):
    hq, _, dim, _, _, _ = GEOMETRIES[case["geom"]]
    fresh, past = _batch(case)
    s = _cache(case, g, case["n_seqs"], _pages(max(p + f for p, f in zip(past, fresh))))
    rows = sum(fresh) + case["pad"]
    s["q"] = torch.randn((rows, hq, dim), generator=g, device="cuda").to(_dtype(case))
    s["q_start"] = _int32(np.concatenate([[0], np.cumsum(fresh)]).tolist())
    s["seq_len"] = _int32([p + f for p, f in zip(past, fresh)])
    s["max_len"] = max(p + f for p, f in zip(past, fresh))
    s["max_q"] = max(fresh)
    s["out"] = torch.zeros((rows, hq, dim), dtype=_dtype(case), device="cuda")   # rows of padding stay as they are
    return s


def _prepare_decode(case, g):
    hq, _, dim, _, _, _ = GEOMETRIES[case["geom"]]
    n = case["n_seqs"]
    s = _cache(case, g, n, _pages(max(1, case["max_len"])))
    lens = torch.randint(case["min_len"], case["max_len"] + 1, (n,), generator=g, device="cuda", dtype=torch.int32)
    s["seq_len"] = torch.cat([_int32([case["max_len"]]), lens[1:]])
    s["max_len"] = case["max_len"]
    s["q"] = torch.randn((n, hq, dim), generator=g, device="cuda").to(_dtype(case))
    return s


def prepare(case, seed):
    make = {"pages": _prepare_pages, "append": _prepare_append, "attn": _prepare_attn, "decode": _prepare_decode}
    s = make[case["kind"]](case, _gen(seed))
    s["case"] = case
    if own and case["kind"] != "pages":
        from paper_2608_20397_amd import nexus

        _, _, _, base, vt, _ = GEOMETRIES[case["geom"]]
        s["cache"] = nexus.PagedKVCache(
            s["k"], s["v"], s["maps"][0], base, nexus.V_TRANSPOSED if vt else nexus.V_ROWMAJOR,
            nexus.ROPE_INTERLEAVED if case.get("interleaved") else nexus.ROPE_NEOX)
    return s


# ---- one pass


def _own(s):
    from paper_2608_20397_amd import nexus

    c = s["case"]
    if c["kind"] == "pages":
        rows = nexus.batch_pages(s["maps"], s["cached"], s["fresh"], s["free"], s["n_free"], s["max_tokens"])
        return (s["maps"], rows.q_start, rows.seq_len, rows.pos, rows.slot, rows.n_left)
    if c["kind"] == "append":
        nexus.norm_rope_append(s["cache"], 0, s["q"], s["k_new"], s["v_new"], s["pos"], s["slot"],
                               q_weight=s["q_weight"], k_weight=s["k_weight"], eps=EPS if c["norm"] else 0.0,
                               out=s["q_out"])
        return (s["q_out"], s["k"], s["v"])
    cap = GEOMETRIES[c["geom"]][5]
    if c["kind"] == "attn":
        return nexus.window_attn(s["q"], s["cache"], s["maps"], s["q_start"], s["seq_len"], s["max_len"],
                                 c["window"], c["sinks"], 0, softcap=cap, out=s["out"])
    return nexus.window_decode_attn(s["q"], s["cache"], s["maps"], s["seq_len"], s["max_len"], c["window"],
                                    c["sinks"], 0, softcap=cap)


def _lay_out(s):
    cached, fresh, maps, n = s["cached"].long(), s["fresh"].long(), s["maps"], s["max_tokens"]
    n_free, stride = s["n_free"].long(), s["maps"].shape[1]
    end = torch.cumsum(fresh.clamp(0, n), 0)
    first, last = (cached + PAGE - 1) // PAGE, (cached + fresh + PAGE - 1) // PAGE
    valid = (cached >= 0) & (fresh >= 0) & (cached + fresh <= PAGE * stride) & ((end <= n) | (fresh == 0))
    need = torch.where(valid, last - first, 0)
    upto = torch.cumsum(need, 0)
    ok = valid & ((need == 0) | (upto <= n_free))
    before = upto - need
    q_start = torch.cat([torch.zeros_like(end[:1]), end]).clamp(max=n)
    # the maps' new entries
    p = torch.arange(stride, device="cuda")
    new = ok[:, None] & (p >= first[:, None]) & (p < last[:, None])
    at = n_free - 1 - before[:, None] - p + first[:, None]
    maps.copy_(torch.where(new, s["free"][at.clamp(0, s["free"].numel() - 1)], maps))
    # the rows
    t = torch.arange(n, device="cuda")
    b = torch.searchsorted(q_start[1:].contiguous(), t, right=True)
    live = b < cached.numel()
    b = b.clamp(max=cached.numel() - 1)
    live &= ok[b]
    pos = torch.where(live, cached[b] + t - q_start[b], 0)
    slot = maps[b, pos // PAGE].long() * PAGE + pos % PAGE
    i32 = torch.int32
    return (maps, q_start.to(i32), torch.where(ok, cached + fresh, 0).to(i32), torch.where(live, pos, -1).to(i32),
            torch.where(live, slot, -1).to(i32), (n_free - torch.where(ok, need, 0).sum()).to(i32))


def _rotate(x, pos, base, interleaved):
    """Feature pair i of row t turned by pos[t] * base^(-2i/D), in 64 bits: x [T][H][D]."""
    dim = x.shape[-1]
    theta = base ** (-2.0 * torch.arange(dim // 2, dtype=torch.float64, device=x.device) / dim)
    ang = (pos.double()[:, None] * theta)[:, None, :]
    cos, sin, x = torch.cos(ang), torch.sin(ang), x.double()
    if interleaved:
        a, b = x[..., 0::2], x[..., 1::2]
        return torch.stack([a * cos - b * sin, b * cos + a * sin], -1).flatten(-2)
    a, b = x[..., :dim // 2], x[..., dim // 2:]
    return torch.cat([a * cos - b * sin, b * cos + a * sin], -1)


def _append(s):
    c = s["case"]
    _, _, _, base, vt, _ = GEOMETRIES[c["geom"]]
    live, dt = s["slot"] >= 0, _dtype(c)
    rows = []
    for x, w in ((s["q"], s["q_weight"]), (s["k_new"], s["k_weight"])):
        x = x.float()
        if c["norm"]:
            x = x * torch.rsqrt((x * x).mean(-1, keepdim=True) + EPS) * w
        rows.append(_rotate(x, s["pos"], base, c["interleaved"]).to(dt))
    s["q_out"].copy_(torch.where(live[:, None, None], rows[0], s["q_out"]))
    n = c["n_tokens"]                              # rows of padding come last
    slot = s["slot"][:n].long()
    s["k"][0, slot // PAGE, :, slot % PAGE] = rows[1][:n]
    if vt:
        s["v"][0, :, :, slot] = s["v_new"][:n].permute(1, 2, 0)
    else:
        s["v"][0, slot // PAGE, :, slot % PAGE] = s["v_new"][:n]
    return (s["q_out"], s["k"], s["v"])


def _keys(s, name, slots):
    """Cache rows of the given slots, fp32 [..., H, D]."""
    x = s[name][0]
    if x.dim() == 3:                               # transposed: [H, D, slots]
        return x.permute(2, 0, 1)[slots].float()
    return x[slots // PAGE, :, slots % PAGE].float()


def _softmax_pv(scores, keep, v, cap):
    if cap > 0:
        scores = cap * torch.tanh(scores / cap)
    scores = scores.masked_fill(~keep, float("-inf"))
    top = scores.amax(-1, keepdim=True)
    p = torch.exp(scores - torch.where(top == float("-inf"), 0.0, top))
    total = p.sum(-1, keepdim=True)
    return torch.matmul(p, v) / torch.where(total == 0, 1.0, total)


def _sees(pos, key, c):
    return (key <= pos) & ((key > pos - c["window"]) | (key < c["sinks"]))


def _attn(s):
    c = s["case"]
    hq, hkv, dim, _, _, cap = GEOMETRIES[c["geom"]]
    n_seqs, n, top_q = c["n_seqs"], s["max_len"], s["max_q"]
    start, lens = s["q_start"].long(), s["seq_len"].long()
    fresh = start[1:] - start[:-1]
    t = torch.arange(n, device="cuda")
    slots = s["maps"][:, t // PAGE].long() * PAGE + t % PAGE                             # [B, n]
    k = _keys(s, "k", slots).permute(0, 2, 3, 1).contiguous()                            # [B, H, D, n]
    v = _keys(s, "v", slots).transpose(1, 2).contiguous()                                # [B, H, n, D]
    # the queries by sequence, padded to the longest
    i = torch.arange(top_q, device="cuda")
    row = (start[:-1, None] + i).clamp(max=s["q"].shape[0] - 1)
    q = s["q"][row].float().view(n_seqs, top_q, hkv, hq // hkv, dim).permute(0, 2, 3, 1, 4)
    scores = torch.matmul(q.reshape(n_seqs, hkv, -1, dim), k) * (1.0 / math.sqrt(dim))
    pos = (lens - fresh)[:, None] + i
    keep = _sees(pos[..., None], t, c)[:, None, None]
    o = _softmax_pv(scores.view(n_seqs, hkv, hq // hkv, top_q, n), keep, v[:, :, None], cap)
    o = o.permute(0, 3, 1, 2, 4).reshape(n_seqs, top_q, hq, dim).to(_dtype(c))
    # back to the rows; rows of padding stay as they are
    r = torch.arange(s["q"].shape[0], device="cuda")
    b = torch.searchsorted(start[1:].contiguous(), r, right=True)
    live = b < n_seqs
    b = b.clamp(max=n_seqs - 1)
    o = o[b, torch.where(live, r - start[b], 0)]
    return s["out"].copy_(torch.where(live[:, None, None], o, s["out"]))


def _decode(s):
    c = s["case"]
    hq, hkv, dim, _, _, cap = GEOMETRIES[c["geom"]]
    n_seqs, pos = c["n_seqs"], s["seq_len"].long()[:, None] - 1
    sinks, width = min(c["sinks"], s["max_len"]), min(c["window"], s["max_len"])
    # the sinks that the window does not hold, then the window
    first = torch.arange(sinks, device="cuda").expand(n_seqs, -1)
    last = pos - torch.arange(width, device="cuda")
    key = torch.cat([first, last], 1)                                                    # [B, n]
    keep = torch.cat([first <= pos - c["window"], last >= 0], 1)
    at = key.clamp(0, max(s["max_len"] - 1, 0))
    slots = torch.gather(s["maps"].long(), 1, at // PAGE) * PAGE + at % PAGE
    k = _keys(s, "k", slots).permute(0, 2, 3, 1).contiguous()
    v = _keys(s, "v", slots).transpose(1, 2).contiguous()
    q = s["q"].float().view(n_seqs, hkv, hq // hkv, dim)
    scores = torch.matmul(q, k) * (1.0 / math.sqrt(dim))
    return _softmax_pv(scores, keep[:, None, None], v, cap).reshape(n_seqs, hq, dim).to(_dtype(c))


def run(state):
    if own:
        return _own(state)
    return {"pages": _lay_out, "append": _append, "attn": _attn, "decode": _decode}[state["case"]["kind"]](state)


# ---- what a pass cannot do without


def work(case):
    kind = case["kind"]
    if kind == "pages":
        fresh, past = _batch(case)
        new = sum(_pages(p + f) - _pages(p) for p, f in zip(past, fresh)) * (0.75 if case["short"] else 1)
        rows = sum(fresh) + case["pad"]
        # lengths read, starts and new lengths written; each new page read and written; two words a row
        return {"bytes": 4 * (4 * case["n_seqs"] + 2 * new + 2 * rows + 3), "flops": 0}
    hq, hkv, dim, _, _, _ = GEOMETRIES[case["geom"]]
    wide = 2 if case["dtype"] == "bf16" else 4
    if kind == "append":
        n = case["n_tokens"]
        # a square, two products and a rotation (three operations) an element of q and k
        return {"bytes": n * (2 * (hq + 2 * hkv) * dim * wide + 8), "flops": n * (hq + hkv) * dim * 7}
    w, sinks = case["window"], case["sinks"]
    if kind == "decode":
        # lengths lie evenly between their bounds, the first at the upper one
        lens = np.linspace(case["min_len"], case["max_len"], 1001)
        seen = lambda n: np.minimum(n, w) + np.minimum(sinks, np.maximum(n - w, 0))  # noqa: E731
        keys = float(seen(case["max_len"]) + (case["n_seqs"] - 1) * seen(lens).mean())
        rows, cached = case["n_seqs"], keys
    else:
        fresh, past = _batch(case)
        pos = np.concatenate([p + np.arange(f) for p, f in zip(past, fresh)] or [[]]) + 1
        keys = float((np.minimum(pos, w) + np.minimum(sinks, np.maximum(pos - w, 0))).sum())
        rows = sum(fresh)
        cached = 0
        for p, f in zip(past, fresh):
            low = max(0, p - w + 1)
            cached += (p + f - low + min(sinks, low)) if f else 0
    return {"bytes": cached * hkv * 2 * dim * wide + 2 * rows * hq * dim * wide, "flops": 4 * dim * hq * keys}


# ---- the definition in 64 bits, written apart from the plain forms


def _exact_append(s):
    c = s["case"]
    hq, hkv, dim, base, vt, _ = GEOMETRIES[c["geom"]]
    n = c["n_tokens"]
    exponent = torch.arange(dim // 2, device="cuda").double() * (-2.0 / dim)
    theta = torch.pow(torch.tensor(base, dtype=torch.float64, device="cuda"), exponent)
    z = torch.polar(torch.ones((n, dim // 2), dtype=torch.float64, device="cuda"),
                    s["pos"][:n, None].double() * theta)[:, None]
    turned = []
    for x, w in ((s["q"], s["q_weight"]), (s["k_new"], s["k_weight"])):
        x = x[:n].double()
        if c["norm"]:
            x = x / torch.sqrt(torch.linalg.vector_norm(x, dim=-1, keepdim=True) ** 2 / dim + EPS) * w.double()
        if not c["interleaved"]:
            x = x.unflatten(-1, (2, dim // 2)).transpose(-1, -2).flatten(-2)
        x = torch.view_as_real(torch.view_as_complex(x.unflatten(-1, (dim // 2, 2)).contiguous()) * z)
        turned.append(x.flatten(-2) if c["interleaved"] else x.transpose(-1, -2).flatten(-2))
    q = torch.zeros(s["q_out"].shape, dtype=torch.float64, device="cuda")
    q[:n] = turned[0]
    k = torch.zeros((s["k"].shape[1] * PAGE, hkv, dim), dtype=torch.float64, device="cuda")
    v = torch.zeros_like(k)
    k[s["slot"][:n].long()] = turned[1]
    v[s["slot"][:n].long()] = s["v_new"][:n].double()
    paged = lambda x: x.view(-1, PAGE, hkv, dim).transpose(1, 2)[None]  # noqa: E731
    return (q, paged(k).contiguous(), v.permute(1, 2, 0)[None].contiguous() if vt else paged(v).contiguous())


def _exact_sequence(s, out, rows, q, b, positions):
    """Rows `rows` of out: queries q [n, Hq, D] of sequence b at the given positions (a list)."""
    c = s["case"]
    hq, hkv, dim, _, vt, cap = GEOMETRIES[c["geom"]]
    n, group = positions[-1] + 1, hq // hkv
    pages = s["maps"][b, :_pages(n)].long()
    where = torch.tensor(positions, device="cuda")
    for h in range(hkv):
        k = s["k"][0, pages, h].flatten(0, 1)[:n].double()
        if vt:
            v = s["v"][0, h].unflatten(-1, (-1, PAGE))[:, pages].flatten(1)[:, :n].double().T
        else:
            v = s["v"][0, pages, h].flatten(0, 1)[:n].double()
        for i in range(0, len(positions), 512):
            at = where[i:i + 512]
            low, high = int(at[0]) - c["window"] + 1, int(at[-1]) + 1
            keys = torch.arange(n, device="cuda")
            keys = keys[(keys < high) & ((keys >= low) | (keys < c["sinks"]))]
            x = torch.einsum("rgd,kd->grk", q[i:i + 512, h * group:(h + 1) * group].double(), k[keys])
            x = x / math.sqrt(dim)
            if cap:
                x = torch.tanh(x / cap) * cap
            behind = at[:, None] - keys
            hidden = (behind < 0) | ((behind >= c["window"]) & (keys >= c["sinks"]))
            x[:, hidden] = -math.inf
            out[rows[i:i + 512], h * group:(h + 1) * group] = (torch.softmax(x, -1) @ v[keys]).transpose(0, 1)


def exact(case, seed):
    if case["kind"] == "pages":
        return None
    s = prepare(case, seed)
    if case["kind"] == "append":
        return _exact_append(s)
    out = torch.zeros(s["q"].shape, dtype=torch.float64, device="cuda")
    lens = s["seq_len"].tolist()
    starts = s["q_start"].tolist() if case["kind"] == "attn" else range(len(lens) + 1)
    for b, n in enumerate(lens):
        fresh = starts[b + 1] - starts[b]
        if fresh and n:
            rows = torch.arange(starts[b], starts[b + 1], device="cuda")
            _exact_sequence(s, out, rows, s["q"][starts[b]:starts[b + 1]], b, list(range(n - fresh, n)))
    return out
