"""Performance cases of the FULL-layer decode calls that go with a shared or a
bounded KV cache (``paper_2607_13095_amd.hswa``), each with its plain form in
elementary torch operations:

  shared  ``decode_shared``: decode of a batch in which runs of consecutive
          sequences share a long prefix (the same pages of the pool)
  scored  ``decode_scored``: decode that also adds every key's attention
          weight, summed over the query heads of its KV head and over the
          call's queries, to a running score
  evict   ``kv_evict``: per KV head, keeps the highest-scored keys (and the
          first and last ones) and moves them, in their order, to new pages

A case is a dict of plain values:

  op       "shared", "scored", "evict"
  hq, hkv  query and KV heads (head dim 128); pg: page size
  ns       sequences of the batch; nq: queries per sequence
  lens     seed of the lengths (the inputs' own seed is prepare()'s)
  shared:  groups of consecutive sequences (sizes drawn; a single sequence is a
           group of its own), each with a prefix of slo .. shi tokens, followed
           by lo .. hi tokens of each sequence's own
  scored:  lo .. hi cached tokens per sequence
  evict:   lo .. hi cached tokens per sequence, of which klo .. khi stay,
           among them the first `sinks` and the last `recent`

q, k and v are N(0, 1) in bf16, positions already encoded; pages are placed by
a random permutation of the pool. Whole pages of a shared prefix are shared, the
tokens of its last, partly filled page are copied to each sequence's own page.
"""

import math
import random

import torch

own = False

D = 128
SCALE = 1.0 / math.sqrt(D)


def _case(name, op, hq, hkv, pg, ns, lo, hi, nq=1, groups=1, slo=0, shi=0, klo=0, khi=0, sinks=0, recent=0, lens=1):
    c = {"op": op, "hq": hq, "hkv": hkv, "pg": pg, "ns": ns, "lo": lo, "hi": hi, "nq": nq, "groups": groups,
         "slo": slo, "shi": shi, "klo": klo, "khi": khi, "sinks": sinks, "recent": recent, "lens": lens}
    return {"name": name, **c} if name else c


def listed():
    return [
        # Two users of one system prompt: the smallest call, where latency counts.
        _case("shared_b2_1k", "shared", 64, 8, 64, 2, 50, 200, slo=1000, shi=1000),
        # A serving batch over one long document or tool description.
        _case("shared_b32_8k", "shared", 64, 8, 64, 32, 100, 1500, slo=8192, shi=8192),
        # Several prompts of unlike popularity in one batch, small pages, lengths that fit nothing.
        _case("shared_groups5_pg16", "shared", 32, 8, 16, 24, 30, 900, groups=5, slo=500, shi=6000),
        # Verification of 1 + 3 predicted tokens of every sequence.
        _case("shared_multi4_b16", "shared", 64, 8, 64, 16, 100, 1000, nq=4, slo=16000, shi=16000),
        # Many samples of one very long context: matrix work decides.
        _case("shared_b64_64k", "shared", 64, 8, 64, 64, 200, 2000, slo=65536, shi=65536),
        # One user's step on a bounded cache.
        _case("scored_b1_4k", "scored", 64, 8, 64, 1, 4000, 4200),
        # A serving batch of mixed contexts.
        _case("scored_b16_16k", "scored", 64, 8, 64, 16, 2000, 16384),
        # The last 16 queries of each prompt score its keys before the cache is cut.
        _case("scored_window16_pg16", "scored", 32, 8, 16, 4, 3000, 9000, nq=16),
        # Long contexts: memory decides.
        _case("scored_b16_64k", "scored", 64, 8, 64, 16, 60000, 65536),
        # One conversation cut to a quarter.
        _case("evict_b1_4k", "evict", 64, 8, 64, 1, 4000, 4200, klo=1024, khi=1024, sinks=4, recent=128),
        # The eviction of a serving batch.
        _case("evict_b16_16k", "evict", 64, 8, 64, 16, 6000, 16384, klo=2048, khi=4096, sinks=4, recent=256),
        # Long prompts on small pages.
        _case("evict_pg16_b8_64k", "evict", 32, 8, 16, 8, 50000, 65536, klo=8000, khi=16384, sinks=0, recent=1000),
    ]


MAX_BYTES = 4.3e9   # of a drawn decode or eviction (the largest listed scored one takes 4.2e9)
MAX_FLOPS = 1.3e11  # of a drawn shared decode (the largest listed one takes 1.4e11)


def _log_int(rng, lo, hi):
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi + 1)))))))


def draw(rng):
    while True:
        op = rng.choice(["shared", "scored", "evict"])
        hq, hkv = rng.choice([(64, 8), (64, 8), (32, 8), (16, 2), (8, 1), (16, 16)])
        pg = rng.choice([16, 32, 64, 64, 128])
        lens = rng.randrange(1 << 20)
        if op == "shared":
            ns = _log_int(rng, 2, 96)
            shi = _log_int(rng, 600, 65536)
            hi = _log_int(rng, 20, 4000)
            c = _case("", op, hq, hkv, pg, ns, max(1, hi // rng.choice([1, 3, 20])), hi, nq=rng.choice([1, 1, 2, 4]),
                      groups=rng.choice([1, 1, rng.randint(1, max(1, ns // 2))]), slo=max(1, shi // rng.choice([1, 4])),
                      shi=shi, lens=lens)
        elif op == "scored":
            hi = _log_int(rng, 300, 65536)
            c = _case("", op, hq, hkv, pg, _log_int(rng, 1, 48), max(1, hi // rng.choice([1, 3, 20])), hi,
                      nq=rng.choice([1, 1, 1, rng.randint(2, 4), rng.randint(5, 32)]), lens=lens)
        else:
            hi = _log_int(rng, 300, 65536)
            khi = _log_int(rng, max(1, hi // 20), hi)
            c = _case("", op, hq, hkv, pg, _log_int(rng, 1, 32), max(1, hi // rng.choice([1, 3, 20])), hi,
                      klo=max(1, khi // rng.choice([1, 3])), khi=khi, sinks=rng.choice([0, 4]),
                      recent=rng.randint(0, max(1, khi // 4)), lens=lens)
        w = work(c)
        if w["bytes"] > MAX_BYTES or w["flops"] > MAX_FLOPS:
            continue
        if c["ns"] * (c["hi"] + c["shi"]) * c["hkv"] > 3.6e7:  # what the plain form lays out in 32 bits
            continue
        if c["ns"] * c["nq"] * c["hq"] * (c["hi"] + c["shi"]) > 6e8:
            continue
        return c


# ---- lengths and work ----------------------------------------------------

def _sizes(case):
    """Group of every sequence, shared tokens of every group, context of every
    sequence (shared and own tokens), keys each one keeps."""
    r = random.Random(case["lens"])
    ns, ng = case["ns"], case["groups"]
    cuts = [0] + sorted(r.sample(range(1, ns), ng - 1)) + [ns] if ng > 1 else [0, ns]
    shared = [r.randint(case["slo"], case["shi"]) for _ in range(ng)] if case["op"] == "shared" else [0] * ng
    group = [max(i for i in range(ng) if cuts[i] <= b) for b in range(ns)]
    # (the queries of a call are the last nq of the sequence's own tokens)
    ctx = [shared[group[b]] + max(case["nq"], r.randint(case["lo"], case["hi"])) for b in range(ns)]
    keep = [min(c, r.randint(case["klo"], case["khi"])) for c in ctx]
    return cuts, group, shared, ctx, keep


def work(case):
    cuts, group, shared, ctx, keep = _sizes(case)
    ns, nq, hq, hkv = case["ns"], case["nq"], case["hq"], case["hkv"]
    kv = hkv * 2 * D * 2  # K and V of a position
    if case["op"] == "evict":
        # every score is read; kept keys are read and written, with their number and score
        return {"bytes": sum(ctx) * hkv * 4 + sum(keep) * (2 * kv + hkv * 8), "flops": 0}
    seen = sum(nq * c - nq * (nq - 1) // 2 for c in ctx)  # (query, key) pairs of a head
    positions = sum(shared) + sum(c - shared[g] for c, g in zip(ctx, group))
    data = positions * kv + ns * nq * hq * D * 2 * 2
    if case["op"] == "scored":
        data += positions * hkv * 8  # the score, read and written
    return {"bytes": data, "flops": 4 * D * hq * seen}


# ---- inputs ----------------------------------------------------------------

def _normal(n, heads, seed, i, tag):
    """n rows of heads x D N(0, 1) values in bf16, drawn on the GPU."""
    g = torch.Generator(device="cuda")
    g.manual_seed((seed * 1000003 + i * 131 + tag) & 0x7FFFFFFFFFFF)
    return torch.randn((n, heads, D), generator=g, device="cuda", dtype=torch.float32).to(torch.bfloat16)


def _history(case, seed, kind, i, n):
    """K, V of n positions: the shared prefix of group i, or sequence i's own."""
    t = 10 if kind == "prefix" else 20
    return _normal(n, case["hkv"], seed, i, t), _normal(n, case["hkv"], seed, i, t + 1)


def _scores(case, seed, b, n):
    """Running scores of n positions: positive, spread over several orders of
    magnitude, one in sixteen never attended to (an exact zero, so that ties
    are decided too)."""
    g = torch.Generator(device="cuda")
    g.manual_seed((seed * 1000003 + b * 131 + 30) & 0x7FFFFFFFFFFF)
    x = torch.randn((case["hkv"], n), generator=g, device="cuda", dtype=torch.float32)
    z = torch.rand((case["hkv"], n), generator=g, device="cuda", dtype=torch.float32)
    return torch.where(z < 1.0 / 16, torch.zeros_like(x), 1e-4 * torch.exp(1.5 * x))


def _i32(x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


def _k_pages(x, pg):
    """[pages * pg, Hkv, D] in order -> pages of the K pool [pages, Hkv, PG/B, 2, D/32, 4, B/2, 8]."""
    bk, h = min(pg, 32), x.shape[1]
    x = x.view(-1, pg // bk, bk // 8, 2, 4, h, D // 32, 4, 8)  # key 8 a + 4 half + c of a block
    return x.permute(0, 5, 1, 3, 6, 7, 2, 4, 8).reshape(-1, h, pg // bk, 2, D // 32, 4, bk // 2, 8)


def _v_pages(x, pg):
    """[pages * pg, Hkv, D] in order -> pages of the V pool [pages, Hkv, PG/B, D, B]."""
    bk, h = min(pg, 32), x.shape[1]
    return x.view(-1, pg // bk, bk, h, D).permute(0, 3, 1, 4, 2)


def _pad(x, n):
    return torch.cat([x, x.new_zeros((n - x.shape[0],) + tuple(x.shape[1:]))])


def prepare(case, seed):
    cuts, group, shared, ctx, keep = _sizes(case)
    ns, nq, hq, hkv, pg = case["ns"], case["nq"], case["hq"], case["hkv"], case["pg"]
    r = random.Random(seed * 7 + 1)
    common = [s // pg for s in shared]  # whole pages of the prefixes
    mine = [-(-c // pg) - common[g] for c, g in zip(ctx, group)]
    pages = sum(common) + sum(mine)
    spare = sum(-(-k // pg) for k in keep) if case["op"] == "evict" else 0
    perm = list(range(pages + spare + 2))
    r.shuffle(perm)
    bk = min(pg, 32)
    k_pool = torch.zeros((len(perm), hkv, pg // bk, 2, D // 32, 4, bk // 2, 8), dtype=torch.bfloat16, device="cuda")
    v_pool = torch.zeros((len(perm), hkv, pg // bk, D, bk), dtype=torch.bfloat16, device="cuda")

    def fill(ids, k, v):
        if ids:
            at = torch.tensor(ids, device="cuda")
            k_pool[at] = _k_pages(_pad(k, len(ids) * pg), pg)
            v_pool[at] = _v_pages(_pad(v, len(ids) * pg), pg)

    stride = -(-max(ctx) // pg)
    table = [[-1] * stride for _ in range(ns)]
    used = 0
    for g in range(case["groups"]):
        whole = common[g] * pg
        pk, pv = _history(case, seed, "prefix", g, shared[g])
        ids = perm[used:used + common[g]]
        used += common[g]
        fill(ids, pk[:whole], pv[:whole])
        for b in range(cuts[g], cuts[g + 1]):
            own_ids = perm[used:used + mine[b]]
            used += mine[b]
            table[b][:common[g] + mine[b]] = ids + own_ids
            k, v = _history(case, seed, "own", b, ctx[b] - shared[g])
            fill(own_ids, torch.cat([pk[whole:], k]), torch.cat([pv[whole:], v]))
    s = {"case": case, "k_pool": k_pool, "v_pool": v_pool, "table": _i32(table), "ctx": _i32(ctx), "max_ctx": max(ctx)}
    if case["op"] == "evict":
        s["scores"] = torch.zeros((ns, hkv, max(ctx)), device="cuda")
        for b in range(ns):
            s["scores"][b, :, :ctx[b]] = _scores(case, seed, b, ctx[b])
        new_stride = -(-max(keep) // pg)
        new_table = [[-1] * new_stride for _ in range(ns)]
        for b in range(ns):
            n = -(-keep[b] // pg)
            new_table[b][:n] = perm[used:used + n]
            used += n
        s["new_table"], s["keep"], s["max_keep"] = _i32(new_table), _i32(keep), max(keep)
        # the pages that the kept keys go to lie in the same pools, as a server's would
        s["kept"] = torch.full((ns, hkv, max(keep)), -1, dtype=torch.int32, device="cuda")
        s["new_scores"] = torch.zeros((ns, hkv, max(keep)), device="cuda")
        s["new_lens"] = torch.zeros(ns, dtype=torch.int32, device="cuda")
    else:
        s["q"] = torch.stack([_normal(nq, hq, seed, b, 40) for b in range(ns)])
        s["out"] = torch.empty_like(s["q"])
    if case["op"] == "scored":
        s["scores"] = torch.zeros((ns, hkv, max(ctx)), device="cuda")
        for b in range(ns):
            s["scores"][b, :, :ctx[b]] = _scores(case, seed, b, ctx[b])
        s["new_scores"] = torch.zeros_like(s["scores"])
    if case["op"] == "shared":
        s["cu_groups"], s["shared"], s["max_shared"] = _i32(cuts), _i32(shared), max(shared)
    if own:  # the handles and the workspace that a server keeps
        from paper_2607_13095_amd import hswa

        s["layer"], s["shape"] = hswa.Layer.full(), hswa.Shape(hq, hkv, D, pg)
        s["cache"] = hswa.Cache(k_pool, v_pool, s["table"])
        need = 0
        if case["op"] == "evict":
            s["new_cache"] = hswa.Cache(k_pool, v_pool, s["new_table"])
        elif case["op"] == "scored":
            need = hswa.decode_scored_workspace_bytes(s["shape"], ns, nq, s["max_ctx"])
        else:
            need = hswa.decode_shared_workspace_bytes(s["shape"], ns, nq, s["max_ctx"], case["groups"], s["max_shared"])
        s["ws"] = torch.empty(max(1, need), dtype=torch.uint8, device="cuda")
    return s


# ---- one pass ----------------------------------------------------------------

def run(s):
    op = s["case"]["op"]
    if own:
        from paper_2607_13095_amd import hswa

        if op == "shared":
            hswa.decode_shared(s["layer"], s["shape"], s["cache"], s["q"], s["ctx"], s["max_ctx"], s["cu_groups"],
                               s["shared"], s["max_shared"], s["out"], workspace=s["ws"])
            return s["out"]
        if op == "scored":
            hswa.decode_scored(s["layer"], s["shape"], s["cache"], s["q"], s["ctx"], s["max_ctx"], s["scores"],
                               s["new_scores"], s["out"], workspace=s["ws"])
            return s["out"], s["new_scores"]
        hswa.kv_evict(s["layer"], s["shape"], s["cache"], s["new_cache"], s["scores"], s["ctx"], s["keep"],
                      s["max_ctx"], s["kept"], s["new_lens"], num_recent=s["case"]["recent"],
                      num_sinks=s["case"]["sinks"], scores_out=s["new_scores"])
        return _evicted(s)
    if op == "evict":
        _plain_evict(s)
        return _evicted(s)
    k, v = _gathered(s)
    out, weights = _plain_attention(s, k, v)
    if op == "shared":
        return out
    j = torch.arange(weights.shape[-1], device="cuda")
    held = (j[None, :] < s["ctx"][:, None])[:, None, :]
    return out, torch.where(held, s["scores"] + weights, s["new_scores"])


def _evicted(s):
    return s["kept"], s["new_scores"], s["new_lens"], s["k_pool"], s["v_pool"]


def _gathered(s):
    """K, V of every sequence in order, [ns, Hkv, positions, D] in 32 bits."""
    at = s["table"].clamp(min=0).long()
    h, pg = s["case"]["hkv"], s["case"]["pg"]
    ns, n, bk = at.shape[0], at.shape[1], min(pg, 32)
    k = s["k_pool"][at].view(ns, n, h, pg // bk, 2, D // 32, 4, bk // 8, 4, 8)
    k = k.permute(0, 2, 1, 3, 7, 4, 8, 5, 6, 9).reshape(ns, h, n * pg, D).float()
    v = s["v_pool"][at].permute(0, 2, 1, 3, 5, 4).reshape(ns, h, n * pg, D).float()
    return k[:, :, :s["max_ctx"]], v[:, :, :s["max_ctx"]]


def _plain_attention(s, k, v):
    """Output rows, and each key's weight summed over queries and heads of its KV head."""
    c = s["case"]
    ns, nq, hq, h = c["ns"], c["nq"], c["hq"], c["hkv"]
    q = s["q"].float().view(ns, nq, h, hq // h, D).permute(0, 2, 1, 3, 4).reshape(ns, h, nq * (hq // h), D)
    a = (torch.matmul(q, k.transpose(2, 3)) * SCALE).view(ns, h, nq, hq // h, -1)
    j = torch.arange(a.shape[-1], device="cuda")
    last = s["ctx"][:, None] - nq + torch.arange(nq, device="cuda")  # each query's own position
    seen = (j <= last[:, :, None])[:, None, :, None, :]
    a = torch.where(seen, a, torch.full_like(a, -math.inf))
    a = torch.exp(a - a.amax(-1, keepdim=True))
    a = a / a.sum(-1, keepdim=True)
    out = torch.matmul(a.reshape(ns, h, nq * (hq // h), -1), v).view(ns, h, nq, hq // h, D)
    return out.permute(0, 2, 1, 3, 4).reshape(ns, nq, hq, D).to(torch.bfloat16), a.sum((2, 3))


def _plain_evict(s):
    c, ctx, keep = s["case"], s["ctx"].long(), s["keep"].long()
    ns, h, n = s["scores"].shape
    j = torch.arange(n, device="cuda")
    held = j < ctx[:, None]
    fixed = held & ((j < c["sinks"]) | (j >= (ctx - c["recent"])[:, None]))
    # fixed ones first, then by score, ties to the lowest position; where there is no room for
    # all fixed ones the last ones go before the first
    value = torch.where(fixed[:, None], torch.full_like(s["scores"], math.inf), s["scores"])
    value = torch.where(held[:, None], value, torch.full_like(value, -math.inf))
    late = torch.where((j >= (ctx - c["recent"])[:, None]) & held, n - j, n + 1)  # the latest first
    first = torch.argsort(late[:, None].expand(ns, h, n), dim=-1, stable=True)
    order = first.gather(-1, torch.argsort(value.gather(-1, first), dim=-1, descending=True, stable=True))
    kept = torch.zeros_like(order, dtype=torch.bool).scatter(-1, order, (j < keep[:, None])[:, None].expand(ns, h, n))
    kept = torch.where(kept, j, n).sort(-1).values[..., :s["max_keep"]]  # positions in order, then n
    there = kept < n
    src = kept.clamp(max=n - 1)
    s["kept"].copy_(torch.where(there, kept, s["kept"]))
    s["new_scores"].copy_(torch.where(there, s["scores"].gather(-1, src), s["new_scores"]))
    s["new_lens"].copy_(keep)
    b, g, i = torch.nonzero(there, as_tuple=True)
    src, i = src[b, g, i], i
    k, v = _pool_places(s, s["table"], b, src), _pool_places(s, s["new_table"], b, i)
    s["k_pool"][v[0], g, v[1], v[3], :, :, v[4]] = s["k_pool"][k[0], g, k[1], k[3], :, :, k[4]]
    s["v_pool"][v[0], g, v[1], :, v[2]] = s["v_pool"][k[0], g, k[1], :, k[2]]


def _pool_places(s, table, b, j):
    """Page, block, key of the block, and half and row of the K block, of positions j."""
    pg = s["case"]["pg"]
    bk = min(pg, 32)
    o = j % bk
    return table.long()[b, j // pg], j % pg // bk, o, o // 4 % 2, o // 8 * 4 + o % 4


# ---- the same in 64 bits, from the definition ------------------------------

def exact(case, seed):
    cuts, group, shared, ctx, keep = _sizes(case)
    nq, hq, h = case["nq"], case["hq"], case["hkv"]
    if case["op"] == "evict":
        return None  # kept positions are whole numbers, the rest are copies
    outs, sums, prefix = [], [], {}
    for b in range(case["ns"]):
        if group[b] not in prefix:
            prefix = {group[b]: _history(case, seed, "prefix", group[b], shared[group[b]])}
        k, v = [torch.cat([x, y]).double() for x, y in
                zip(prefix[group[b]], _history(case, seed, "own", b, ctx[b] - shared[group[b]]))]
        q = _normal(nq, hq, seed, b, 40).double()
        out = torch.empty((nq, hq, D), dtype=torch.float64, device="cuda")
        total = torch.zeros((h, max(ctx)), dtype=torch.float64, device="cuda")
        if case["op"] == "scored":
            total[:, :ctx[b]] = _scores(case, seed, b, ctx[b]).double()
        for i in range(nq):
            n = ctx[b] - nq + i + 1  # keys this query sees
            for g in range(h):
                heads = slice(g * (hq // h), (g + 1) * (hq // h))
                w = torch.softmax((q[i, heads] @ k[:n, g].T) / math.sqrt(D), dim=-1)
                out[i, heads] = w @ v[:n, g]
                total[g, :n] += w.sum(0)
        outs.append(out)
        sums.append(total)
    if case["op"] == "shared":
        return torch.stack(outs)
    return torch.stack(outs), torch.stack(sums)
