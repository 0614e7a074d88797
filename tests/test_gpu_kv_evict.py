"""GPU parity of eviction by accumulated attention weight (hswa_kv_evict): kept
positions, their scores, the new lengths and every bit of the pools (the slots
that the call has no business with among them) against the oracle's selection
applied to the history; and decode over the evicted cache."""

import numpy as np
import pytest
import torch

import synth
from oracle import attention as OA
from oracle import eviction as OE
from oracle import layout as OL
from paper_2607_13095_amd import hswa
from paper_2607_13095_amd.kvcache import LayerKV, pages_for
from tests.hswa_testlib import SeqHistory, append_history, assert_close, i32, to_bits, to_dev, to_f64

pytestmark = pytest.mark.gpu

D = 128


class Evict:
    """A FULL layer's filled cache, and a table of spare pages for what stays."""

    def __init__(self, lens, max_keep, hkv, pg, seed, group=2, max_ctx=None):
        self.lens, self.hkv, self.pg, self.max_keep = lens, hkv, pg, max_keep
        self.ns, self.max_ctx = len(lens), max_ctx or max(max(lens), 1)
        self.shape = hswa.Shape(group * hkv, hkv, D, pg)
        self.layer = hswa.Layer.full()
        each = -(-max_keep // pg)
        spare = self.ns * each
        total = pages_for(self.layer, pg, lens) + spare + 2
        perm = synth.page_permutation(total, *seed)
        self.kv = LayerKV(self.layer, self.shape, lens, perm=perm, extra_pages=spare + 2,
                          stride=max(1, -(-self.max_ctx // pg)))
        self.hist = SeqHistory(lens, hkv, D, *seed)
        if sum(lens):
            append_history(self.layer, self.shape, self.kv, self.hist, [0] * self.ns, lens)
        self.new_table = perm[total - spare:].reshape(self.ns, each).astype(np.int32)
        self.dst = hswa.Cache(self.kv.k_pool, self.kv.v_pool, i32(self.new_table))

    def run(self, scores, budgets, recent, sinks, **kw):
        self.before = to_bits(self.kv.k_pool), to_bits(self.kv.v_pool)
        self.kept = torch.full((self.ns, self.hkv, self.max_keep), -7, dtype=torch.int32, device="cuda")
        self.lens_out = torch.full((self.ns,), -7, dtype=torch.int32, device="cuda")
        self.scores_out = torch.full((self.ns, self.hkv, self.max_keep + 3), -7.0, device="cuda")
        self.budgets = i32(budgets)
        hswa.kv_evict(self.layer, self.shape, self.kv.cache, self.dst, scores, i32(self.lens), self.budgets,
                      self.max_ctx, self.kept, self.lens_out, num_recent=recent, num_sinks=sinks,
                      scores_out=self.scores_out, **kw)
        torch.cuda.synchronize()

    def check(self, scores, budgets, recent, sinks):
        s = scores.cpu().numpy()
        kp, vp = [x.copy() for x in self.before]
        kept, got = self.kept.cpu().numpy(), self.scores_out.cpu().numpy()
        for b, n in enumerate(self.lens):
            for g in range(self.hkv):
                ref = OE.kept_positions(s[b, g], n, min(budgets[b], self.max_keep), recent, sinks)
                assert int(self.lens_out[b]) == ref.size
                assert np.array_equal(kept[b, g, :ref.size], ref), (b, g)
                assert np.all(kept[b, g, ref.size:] == -7)
                assert np.array_equal(got[b, g, :ref.size], s[b, g, ref], equal_nan=True)
                assert np.all(got[b, g, ref.size:] == -7)
                for i, j in enumerate(ref):
                    page, off = int(self.new_table[b, i // self.pg]), i % self.pg
                    at = OL.k_slot(kp.shape, page, off)
                    kp[at[:1] + (g,) + at[2:]] = self.hist.k[b][j, g].reshape(D // 32, 4, 8)
                    v = vp.shape[4]
                    vp[page, g, off // v, :, off % v] = self.hist.v[b][j, g]
        assert np.array_equal(to_bits(self.kv.k_pool), kp)
        assert np.array_equal(to_bits(self.kv.v_pool), vp)


def _scores(ns, hkv, n, seed, kind="spread"):
    r = np.random.default_rng(seed)
    x = np.exp(1.5 * r.standard_normal((ns, hkv, n))).astype(np.float32)
    if kind == "ties":  # few values, many zeros of both signs
        x = np.round(np.minimum(x, 3)).astype(np.float32)
        x[r.random(x.shape) < 0.3] = -0.0
    elif kind == "equal":
        x[:] = 0.25
    elif kind == "odd":  # infinities, NaN, negative, denormal
        for v in (np.inf, -np.inf, np.nan, -1.0, 1e-42, -1e-42):
            x[r.random(x.shape) < 0.1] = v
    return torch.from_numpy(x).cuda()


@pytest.mark.parametrize("kind", ["spread", "ties", "equal", "odd"])
@pytest.mark.parametrize("pg", [16, 32, 64, 256])
def test_kv_evict(gpu_lib, pg, kind):
    print(f"[evict] pg={pg} {kind}", flush=True)
    lens = [0, 1, 2, 31, 65, 200, 777, 1500]
    budgets = [5, 1, 1, 8, 64, 33, 300, 300]
    e = Evict(lens, 300, 2, pg, (1300, pg))
    s = _scores(len(lens), 2, max(lens) + 5, (1, pg), kind)
    e.run(s, budgets, 8, 4)
    e.check(s, budgets, 8, 4)


@pytest.mark.parametrize("pg", [16, 32, 256])
@pytest.mark.parametrize("longest,max_keep,kind", [(1500, 600, "ties"), (5000, 600, "spread"), (5000, 200, "odd"),
                                                   (16384, 70, "ties"), (17000, 70, "spread"), (40000, 70, "ties"),
                                                   (9000, 600, "spread"), (20000, 600, "odd"), (32768, 70, "equal")])
def test_kv_evict_sizes(gpu_lib, longest, max_keep, kind, pg):
    """Contexts up to and past 8K, 16K and 32K, with few slots in all and many (more
    than 256 runs of 32)."""
    print(f"[evict-sizes] pg={pg} longest={longest} max_keep={max_keep} {kind}", flush=True)
    lens = [0, 33, 777, 1024, 600, 1025, 63, longest]
    budgets = [9, 33, 32, max_keep, 500, 61, 64, max_keep]
    e = Evict(lens, max_keep, 2, pg, (1320, pg, longest))
    s = _scores(len(lens), 2, longest, (5, pg), kind)
    e.run(s, budgets, 20, 3)
    e.check(s, budgets, 20, 3)


@pytest.mark.parametrize("recent,sinks,budgets", [(0, 0, [0, 1, 31, 32, 33, 500]), (0, 3, [2, 3, 4, -5, 90, 90]),
                                                  (40, 0, [39, 40, 41, 80, 90, 0]), (1000, 1000, [7, 50, 90, 90, 1, 2]),
                                                  (30, 20, [10, 30, 45, 50, 51, 90])])
def test_kv_evict_fixed_keys(gpu_lib, recent, sinks, budgets):
    """Budgets below, at and above what the first and last keys take; above the
    context, above kept_stride, negative."""
    print(f"[evict-fixed] recent={recent} sinks={sinks}", flush=True)
    lens = [100, 100, 333, 90, 91, 64]
    e = Evict(lens, 96, 3, 16, (1301, recent, sinks), group=1)
    s = _scores(6, 3, 333, (2, recent))
    e.run(s, budgets, recent, sinks)
    e.check(s, budgets, recent, sinks)


@pytest.mark.parametrize("n,keep,kind", [(16384, 2048, "spread"), (70000, 20000, "ties"), (131072, 100, "spread"),
                                         (66000, 65999, "odd")])
def test_kv_evict_long(gpu_lib, n, keep, kind):
    """Long contexts: the kept positions, and attention over what stays."""
    print(f"[evict-long] n={n} keep={keep} {kind}", flush=True)
    e = Evict([n, n // 3], keep, 1, 64, (1302, n), group=8)
    s = _scores(2, 1, n, (3, n), kind)
    budgets = [keep, keep]
    e.run(s, budgets, 64, 4)
    q = synth.normal_bf16((2, 8, D), 1302, n, synth.TAG_QDEC)
    out = torch.empty((2, 8, D), dtype=torch.bfloat16, device="cuda")
    ws = torch.empty(max(1, hswa.decode_workspace_bytes(e.shape, 2, keep)), dtype=torch.uint8, device="cuda")
    hswa.decode(e.layer, e.shape, e.dst, to_dev(q), e.lens_out, keep, out, workspace=ws)
    torch.cuda.synchronize()
    for b, m in enumerate(e.lens):
        ref = OE.kept_positions(s[b, 0].cpu().numpy(), m, keep, 64, 4)
        assert int(e.lens_out[b]) == ref.size
        assert np.array_equal(e.kept[b, 0, :ref.size].cpu().numpy(), ref)
        o = OA.decode(OA.bf16_bits_to_f64(q[b]), OA.bf16_bits_to_f64(e.hist.k[b][ref]),
                      OA.bf16_bits_to_f64(e.hist.v[b][ref]), None)
        assert_close(to_f64(out)[b], o, f"decode over the kept keys, n={m}")


def test_kv_evict_bad_pages(gpu_lib):
    """Page ids outside the pool and -1: what is read there is zero, what would
    be stored there is not, and nothing else changes."""
    e = Evict([300, 300], 128, 2, 64, (1303,))
    table, new = e.kv.block_table.clone(), i32(e.new_table)
    table[0, 1], table[1, 2] = -1, 10 ** 6
    new[0, 0], new[1, 1] = 1 << 30, -3
    src, dst = hswa.Cache(e.kv.k_pool, e.kv.v_pool, table), hswa.Cache(e.kv.k_pool, e.kv.v_pool, new)
    s = _scores(2, 2, 300, (4,))
    kept = torch.empty((2, 2, 128), dtype=torch.int32, device="cuda")
    lens = torch.empty(2, dtype=torch.int32, device="cuda")
    kp, vp = to_bits(e.kv.k_pool), to_bits(e.kv.v_pool)
    hswa.kv_evict(e.layer, e.shape, src, dst, s, i32([300, 300]), i32([128, 100]), 300, kept, lens)
    torch.cuda.synchronize()
    for b, n in enumerate([128, 100]):
        for g in range(2):
            ref = OE.kept_positions(s[b, g].cpu().numpy(), 300, n, 0, 0)
            assert np.array_equal(kept[b, g, :n].cpu().numpy(), ref)
            for i, j in enumerate(ref):
                page, off = int(new[b, i // 64]), i % 64
                if not 0 <= page < e.kv.num_pages:
                    continue
                held = 0 <= int(table[b, j // 64]) < e.kv.num_pages
                at = OL.k_slot(kp.shape, page, off)
                kp[at[:1] + (g,) + at[2:]] = e.hist.k[b][j, g].reshape(4, 4, 8) if held else 0
                vp[page, g, off // 32, :, off % 32] = e.hist.v[b][j, g] if held else 0
    assert np.array_equal(to_bits(e.kv.k_pool), kp) and np.array_equal(to_bits(e.kv.v_pool), vp)


def test_kv_evict_captured(gpu_lib):
    """Captured once, replayed with other scores and budgets, eager work between."""
    lens = [900, 333]
    e = Evict(lens, 128, 2, 32, (1304,))
    s = _scores(2, 2, 900, (5, 0))
    e.run(s, [128, 100], 16, 2)
    g = torch.cuda.CUDAGraph()
    lens_dev = i32(lens)
    torch.cuda.synchronize()
    with torch.cuda.graph(g):
        hswa.kv_evict(e.layer, e.shape, e.kv.cache, e.dst, s, lens_dev, e.budgets, 900, e.kept, e.lens_out,
                      num_recent=16, num_sinks=2, scores_out=e.scores_out)
    for rep in range(3):
        s.copy_(_scores(2, 2, 900, (5, rep)))
        budgets = [128 - rep, 40 * rep]
        e.budgets.copy_(i32(budgets))
        e.kept.fill_(-7)
        e.scores_out.fill_(-7)
        e.before = to_bits(e.kv.k_pool), to_bits(e.kv.v_pool)
        g.replay()
        torch.cuda.synchronize()
        e.check(s, budgets, 16, 2)


def test_kv_evict_other_stream_and_shared_source(gpu_lib):
    """On a stream of the caller's; two sequences that name the same source
    pages (a shared prefix) keep different keys of it, and it stays as it was."""
    e = Evict([400, 400], 64, 2, 64, (1305,))
    table = e.kv.block_table.clone()
    table[1] = table[0]
    src = hswa.Cache(e.kv.k_pool, e.kv.v_pool, table)
    s = _scores(2, 2, 400, (6,))
    kept = torch.empty((2, 2, 64), dtype=torch.int32, device="cuda")
    lens, ctx, bud = torch.empty(2, dtype=torch.int32, device="cuda"), i32([400, 400]), i32([64, 50])
    pages = table[0].long()
    kp = e.kv.k_pool[pages].clone()
    st = torch.cuda.Stream()
    st.wait_stream(torch.cuda.current_stream())
    hswa.kv_evict(e.layer, e.shape, src, e.dst, s, ctx, bud, 400, kept, lens, num_recent=5, stream=st)
    st.synchronize()
    assert torch.equal(e.kv.k_pool[pages].view(torch.int16), kp.view(torch.int16))
    e.hist.k[1], e.hist.v[1] = e.hist.k[0], e.hist.v[0]
    for b, n in enumerate([64, 50]):
        for g in range(2):
            ref = OE.kept_positions(s[b, g].cpu().numpy(), 400, n, 5, 0)
            assert np.array_equal(kept[b, g, :n].cpu().numpy(), ref)
            for i, j in enumerate(ref):
                at = OL.k_slot(e.kv.k_pool.shape, int(e.new_table[b, i // 64]), i % 64)
                got = to_bits(e.kv.k_pool[at[:1] + (g,) + at[2:]])
                assert np.array_equal(got.reshape(-1), e.hist.k[b][j, g])
