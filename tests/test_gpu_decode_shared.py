"""GPU parity of decode over shared prefixes (hswa_decode_shared) against the
fp64 oracle: groups of any size over prefixes of any length, pages that are
shared or copied, sequences that do not fit their group, offsets that make no
sense, and agreement with hswa_decode_multi where nothing is shared."""

import numpy as np
import pytest
import torch

import synth
from oracle import attention as OA
from paper_2607_13095_amd import hswa
from tests.hswa_testlib import SeqHistory, append_history, assert_close, i32, make_layer, to_dev, to_f64

pytestmark = pytest.mark.gpu

D = 128
WIDE = 150000  # a bound on the contexts under which two sequences of one KV head may gain


class Shared:
    """A FULL layer whose rows name the same pages for the whole pages of their
    group's prefix, and pages of their own from there on."""

    def __init__(self, groups, nq, hq, hkv, pg, seed, scale=None, max_ctx=WIDE):
        # groups: (shared tokens, [own tokens of each sequence])
        self.nq, self.hq, self.hkv, self.pg = nq, hq, hkv, pg
        self.shape = hswa.Shape(hq, hkv, D, pg, scale=scale)
        self.sizes = [len(own) for _, own in groups]
        self.shared = [s for s, _ in groups]
        whole = [s // pg * pg for s in self.shared]
        own = [(i, n) for i, (_, ns) in enumerate(groups) for n in ns]
        self.ctx = [self.shared[i] + n for i, n in own]
        self.ns = len(own)
        # stored runs of pages: each prefix's whole pages, then each sequence's from there on
        lens = whole + [c - whole[i] for (i, _), c in zip(own, self.ctx)]
        self.layer, self.kv = make_layer("full", 0, self.shape, lens, seed)
        hist = SeqHistory(lens, hkv, D, *seed)
        tail = [synth.normal_bf16((s - w, hkv, D), *seed, i, t) for t in (901, 902)
                for i, (s, w) in enumerate(zip(self.shared, whole))]
        ng = len(groups)
        for b, (i, _) in enumerate(own):  # the prefix's last, partly filled page: a copy for each sequence
            n = self.shared[i] - whole[i]
            hist.k[ng + b][:n], hist.v[ng + b][:n] = tail[i], tail[ng + i]
        if sum(lens):
            append_history(self.layer, self.shape, self.kv, hist, [0] * len(lens), lens)
        self.k = [np.concatenate([hist.k[i], hist.k[ng + b]]) for b, (i, _) in enumerate(own)]
        self.v = [np.concatenate([hist.v[i], hist.v[ng + b]]) for b, (i, _) in enumerate(own)]
        self.max_ctx = max_ctx
        self.table = np.full((self.ns, max(1, -(-self.max_ctx // pg))), -1, np.int32)
        for b, (i, _) in enumerate(own):
            ids = list(self.kv.table_host[i][: whole[i] // pg]) + list(
                self.kv.table_host[ng + b][: -(-lens[ng + b] // pg)])
            self.table[b, : len(ids)] = ids[: self.table.shape[1]]
        self.cu = np.concatenate([[0], np.cumsum(self.sizes)])
        self.qbits = synth.normal_bf16((self.ns, nq, hq, D), *seed, synth.TAG_QDEC)
        self.q = to_dev(self.qbits)

    def run(self, cu=None, shared=None, ctx=None, table=None, max_shared=WIDE, **kw):
        cu = i32(self.cu if cu is None else cu)
        shared = self.shared if shared is None else shared
        self.lens = list(self.ctx if ctx is None else ctx)
        cache = hswa.Cache(self.kv.k_pool, self.kv.v_pool, i32(self.table if table is None else table))
        top = max_shared
        need = hswa.decode_shared_workspace_bytes(self.shape, self.ns, self.nq, self.max_ctx, len(shared), top)
        plain = hswa.decode_multi_workspace_bytes(self.shape, self.ns, self.nq, self.max_ctx)
        self.by_prefix = need != plain
        self.ws = torch.full((max(1, need),), 255, dtype=torch.uint8, device="cuda")
        self.out = torch.full_like(self.q, 7.0)
        self.args = (self.layer, self.shape, cache, self.q, i32(self.lens), self.max_ctx, cu, i32(shared), top, self.out)
        hswa.decode_shared(*self.args, workspace=self.ws, **kw)
        torch.cuda.synchronize()
        return to_f64(self.out)

    def check(self, got, what, held=None, by_prefix=True):
        assert self.by_prefix == by_prefix, what
        for b, n in enumerate(self.lens):
            n = min(n, self.max_ctx)
            ref = np.zeros((self.nq, self.hq, D))
            pos = np.arange(n - self.nq, n)
            ok = pos >= 0
            if n >= 1:
                q, k, v = [OA.bf16_bits_to_f64(x) for x in (self.qbits[b][ok], self.k[b][:n], self.v[b][:n])]
                if held is not None:
                    keep = held[b][:n]
                    pos = np.cumsum(keep)[pos[ok]] - 1  # (places among the keys that are held)
                    k, v = k[keep], v[keep]
                    ref[ok] = OA.masked_attention(q, k, v, pos, None, self.shape.scale)
                else:
                    ref[ok] = OA.masked_attention(q, k, v, pos[ok], None, self.shape.scale)
            assert_close(got[b], ref, f"{what}: sequence {b} of {n}")


@pytest.mark.parametrize("nq", [1, 3])
@pytest.mark.parametrize("pg", [16, 32, 64, 128, 256])
def test_decode_shared(gpu_lib, pg, nq):
    """Groups of one and of many, prefixes below, at and above tiles and pages."""
    print(f"[shared] pg={pg} nq={nq}", flush=True)
    groups = [(63, [5, 70]), (64, [3, 4, 200]), (65, [40]), (1000, [3, 31, 32, 33, 500]), (640, [700] * 3),
              (0, [9, 100]), (129, [64, 63])]
    s = Shared(groups, nq, 16, 2, pg, (1500, pg, nq))
    s.check(s.run(), f"pg={pg} nq={nq}")


@pytest.mark.parametrize("hq,hkv,n,nq", [(8, 8, 5, 1), (64, 8, 2, 1), (64, 8, 17, 1), (32, 1, 9, 1), (16, 1, 40, 1),
                                         (128, 1, 3, 1), (64, 8, 5, 8), (8, 4, 150, 2), (4, 2, 4, 64)])
def test_decode_shared_columns(gpu_lib, hq, hkv, n, nq):
    """From 5 columns of a KV head to over 256: few waves at work, one and two
    column groups, several workgroups' columns with an odd rest."""
    print(f"[shared-columns] hq={hq} hkv={hkv} n={n} nq={nq}", flush=True)
    r = np.random.default_rng(n)
    s = Shared([(700, [int(x) for x in r.integers(nq, 90 + nq, n)])], nq, hq, hkv, 64, (1501, hq, n, nq))
    s.check(s.run(), f"{n} sequences, {hq} / {hkv} heads, nq={nq}")


def test_decode_shared_long(gpu_lib):
    """Prefixes of many spans, unlike ones in one batch, beside a long sequence
    of no group (its own keys are cut into spans too)."""
    groups = [(20000, [10, 3000, 700]), (5000, [1, 1, 1, 1]), (0, [9000]), (333, [100] * 10)]
    s = Shared(groups, 1, 8, 1, 64, (1502,))
    s.check(s.run(), "long")
    s = Shared([(40000, [20, 30])], 2, 16, 2, 16, (1503,))
    s.check(s.run(), "long, small pages")


@pytest.mark.parametrize("scale", [1.0, 4.0])
def test_decode_shared_peaked(gpu_lib, scale):
    """Scores far apart: the running maximum rises again and again, and one of
    the two parts of a row carries nearly no weight."""
    s = Shared([(1500, [10, 400, 33]), (200, [1, 2])], 2, 16, 2, 64, (1504,), scale=scale)
    s.check(s.run(), f"scale {scale}")


def test_decode_shared_members_that_do_not_fit(gpu_lib):
    """A sequence without a context (the first of a group among them: a padded
    batch), one shorter than the prefix, one shorter than the queries, contexts
    above max_context_len; a group of empty ones."""
    s = Shared([(500, [20, 30, 40]), (300, [10, 20]), (700, [5, 6, 7, 8]), (100, [5, 5])], 2, 16, 2, 64, (1505,))
    c = list(s.ctx)
    for change in ({0: 0}, {0: 0, 1: 0}, {1: 100}, {4: 1}, {2: 500, 5: 0, 8: 650}, {9: 0, 10: 0}, {6: 64, 7: 1},
                   dict.fromkeys(range(s.ns), 0)):
        ctx = [change.get(b, n) for b, n in enumerate(c)]
        s.check(s.run(ctx=ctx), f"contexts {change}")


def test_decode_shared_clamped(gpu_lib):
    """Contexts above max_context_len and prefixes above max_shared_len count as
    those bounds."""
    r = np.random.default_rng(5)
    own = [[int(x) for x in r.integers(1, 120, n)] for n in (14, 10)]
    s = Shared([(600, own[0]), (300, own[1])], 1, 16, 16, 64, (1513,), max_ctx=650)
    assert max(s.ctx) > 650
    s.check(s.run(), "contexts")
    s = Shared([(200, [int(x) for x in r.integers(1, 30, 40)])], 1, 32, 32, 32, (1514,))
    s.check(s.run(max_shared=128), "prefixes")


def test_decode_shared_lengths_and_offsets_out_of_line(gpu_lib):
    """shared_lens above the contexts and below 0; offsets that do not cover the batch, decrease or leave it: rows stay right
    wherever the promise of equal keys holds."""
    s = Shared([(600, [20, 30, 40]), (300, [10, 20])], 1, 16, 2, 64, (1506,))
    s.check(s.run(shared=[600, -5]), "a negative length")
    s.check(s.run(shared=[600, -5], cu=[3, 5, 5]), "nothing shared")
    s.check(s.run(shared=[600, 300], cu=[0, 3, 3]), "an empty group")
    s.check(s.run(shared=[600, 300], cu=[1, 3, 5]), "a sequence of no group")
    s.check(s.run(shared=[600, 300], cu=[0, 2, 2]), "the rest of no group")
    s.check(s.run(shared=[600, 300], cu=[0, 3, 1 << 30]), "past the batch")
    s.check(s.run(shared=[600, 300], cu=[-9, 3, 5]), "before the batch")
    s.check(s.run(shared=[600, 300], cu=[0, 3, 1]), "decreasing")
    s.check(s.run(shared=[0, 300, 64, 5], cu=[0, 3, 5, 2, 4]), "decreasing, more of them")


def test_decode_shared_many_groups(gpu_lib):
    """More groups than a workgroup has threads: the plan takes them in turns."""
    n = 1100
    s = Shared([(64, [1 + (i % 3), 2]) for i in range(n)], 1, 2, 1, 16, (1507,))
    s.check(s.run(), "many groups")


@pytest.mark.parametrize("n,ng", [(64, 63), (65, 1), (66, 64), (100, 63), (130, 64), (256, 255), (257, 256), (257, 20)])
def test_decode_shared_batches(gpu_lib, n, ng):
    """Batches and group counts about the sizes at which the plan is found
    another way; members without a context; offsets that decrease."""
    print(f"[shared-batches] n={n} ng={ng}", flush=True)
    r = np.random.default_rng(n + ng)
    cuts = [0] + sorted(int(x) for x in r.choice(np.arange(1, n), ng - 1, replace=False)) + [n]
    groups = [(int(r.integers(60, 400)), [int(x) for x in r.integers(1, 90, b - a)]) for a, b in zip(cuts, cuts[1:])]
    s = Shared(groups, 1, 8, 1, 64, (1520, n, ng))
    s.check(s.run(), f"{n} sequences in {ng} groups")
    ctx = [0 if r.random() < 0.2 else c for c in s.ctx]
    s.check(s.run(ctx=ctx), f"{n} sequences in {ng} groups, some without a context")
    if ng >= 20:
        cu = [int(x) for x in s.cu]
        cu[10], cu[11] = cu[11], cu[9]  # (group 9 would reach into group 10's: it shares what both have)
        shared = list(s.shared)
        shared[9] = 0
        s.check(s.run(cu=cu, shared=shared, ctx=ctx), f"{n} sequences in {ng} groups, decreasing")


def test_decode_shared_copied_prefix(gpu_lib):
    """Rows that hold copies of the prefix in pages of their own."""
    lens = [900, 1000, 905]
    shape = hswa.Shape(16, 2, D, 64)
    layer, kv = make_layer("full", 0, shape, lens[:2] + [WIDE], (1508,))
    hist = SeqHistory(lens, 2, D, 1508)
    for b in (1, 2):
        hist.k[b][:850], hist.v[b][:850] = hist.k[0][:850], hist.v[0][:850]
    append_history(layer, shape, kv, hist, [0] * 3, lens)
    qbits = synth.normal_bf16((3, 16, D), 1508, synth.TAG_QDEC)
    out = torch.empty((3, 16, D), dtype=torch.bfloat16, device="cuda")
    need = hswa.decode_shared_workspace_bytes(shape, 3, 1, WIDE, 1, WIDE)
    assert need > hswa.decode_workspace_bytes(shape, 3, WIDE)
    ws = torch.empty(need, dtype=torch.uint8, device="cuda")
    hswa.decode_shared(layer, shape, kv.cache, to_dev(qbits), i32(lens), WIDE, i32([0, 3]), i32([850]), WIDE, out,
                       workspace=ws)
    torch.cuda.synchronize()
    for b, n in enumerate(lens):
        ref = OA.decode(OA.bf16_bits_to_f64(qbits[b]), OA.bf16_bits_to_f64(hist.k[b]), OA.bf16_bits_to_f64(hist.v[b]),
                        None)
        assert_close(to_f64(out)[b], ref, f"copied prefix, sequence {b}")


@pytest.mark.parametrize("pg", [16, 32, 64])
def test_decode_shared_bad_pages(gpu_lib, pg):
    """Keys on page ids outside the pool are left out, in a prefix (by every
    sequence of the group) and behind it; a prefix with no page at all."""
    s = Shared([(512, [100, 200, 10])], 1, 16, 2, pg, (1509, pg))
    for lost in ([1], [0, 3], list(range(512 // pg))):
        table = s.table.copy()
        table[:, lost] = -1
        table[1, 600 // pg] = 1 << 30
        held = [np.repeat(table[b] >= 0, pg) & np.repeat(table[b] < s.kv.num_pages, pg) for b in range(3)]
        s.check(s.run(table=table), f"pg={pg}, pages {lost}", held=held)


def test_decode_shared_without_gain_is_decode_multi(gpu_lib):
    """No group, one sequence a group, prefixes below a tile, few positions: the
    same bits as hswa_decode_multi, with its workspace; an SWA layer too."""
    s = Shared([(400, [500, 2000, 30])], 2, 16, 2, 64, (1510,), max_ctx=2400)
    ws = torch.empty(max(1, hswa.decode_multi_workspace_bytes(s.shape, 3, 2, s.max_ctx)), dtype=torch.uint8,
                     device="cuda")
    got = s.run(max_shared=400)
    s.check(got, "few positions", by_prefix=False)
    out = torch.empty_like(s.q)
    hswa.decode_multi(*s.args[:6], out, workspace=ws)
    torch.cuda.synchronize()
    assert np.array_equal(to_f64(out), got)
    for cu, sl, top in (([0], [], WIDE), ([0, 1, 2, 3], [400] * 3, WIDE), ([0, 3], [400], 63)):
        out.fill_(7.0)
        hswa.decode_shared(*s.args[:6], i32(cu), i32(sl), top, out, workspace=ws)
        torch.cuda.synchronize()
        assert np.array_equal(to_f64(out), got), cu
    layer, kv = make_layer("swa", 128, s.shape, s.ctx, (1511,))
    hist = SeqHistory(s.ctx, 2, D, 1511)
    append_history(layer, s.shape, kv, hist, [0] * 3, s.ctx)
    hswa.decode_shared(layer, s.shape, kv.cache, s.q, i32(s.ctx), s.max_ctx, i32([0, 3]), i32([400]), WIDE, out)
    ref = torch.empty_like(out)
    hswa.decode_multi(layer, s.shape, kv.cache, s.q, i32(s.ctx), s.max_ctx, ref)
    torch.cuda.synchronize()
    assert torch.equal(out.view(torch.int16), ref.view(torch.int16))


def test_decode_shared_captured(gpu_lib):
    """Replays with other lengths and groups, eager work and another stream's
    call between; the same bits as the eager call."""
    s = Shared([(1000, [20, 30, 400]), (256, [10, 20]), (0, [300])], 1, 32, 4, 64, (1512,))
    s.check(s.run(), "eager")
    layer, shape, cache, q, ctx, mc, cu, sh, top, out = s.args
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        hswa.decode_shared(*s.args, workspace=s.ws)
    args, ws = s.args, s.ws
    side = torch.cuda.Stream()
    for rep, (c, gr, sl) in enumerate([(s.ctx, s.cu, s.shared), ([1010, 0] + s.ctx[2:], s.cu, [900, 256, 0]),
                                       (s.ctx, [0, 3, 3, 6], [1000, 7, 100]), (s.ctx, s.cu, s.shared)]):
        if rep == 2:
            sl = [1000, 0, 0]
        ctx.copy_(i32(c))
        cu.copy_(i32(gr))
        sh.copy_(i32(sl))
        out.fill_(7.0)
        ws.fill_(rep)
        torch.cuda.synchronize()
        g.replay()
        torch.cuda.synchronize()
        got = to_f64(out)
        side.wait_stream(torch.cuda.current_stream())
        eager = s.run(ctx=c, cu=gr, shared=sl, max_shared=top, stream=side)
        side.synchronize()
        eager = to_f64(s.out)
        assert np.array_equal(got, eager), rep
        s.check(got, f"replay {rep}")
        s.args, s.ws = args, ws
