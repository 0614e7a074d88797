"""The calls on shared and bounded caches beside each other: two of each at once on
two streams with every round's outputs compared; contexts that an eviction clamps;
a budgeted cache whose pages come from the allocator and go back to it."""

import numpy as np
import pytest
import torch

import synth
from oracle import attention as OA
from oracle import eviction as OE
from paper_2607_13095_amd import hswa
from paper_2607_13095_amd.kvcache import prefix_groups
from tests.hswa_testlib import assert_close, i32, to_dev, to_f64
from tests.test_gpu_decode_shared import Shared
from tests.test_gpu_kv_evict import Evict, _scores

pytestmark = pytest.mark.gpu

D = 128
WIDE = 150000


def _differ(a, b):
    return (a.view(torch.int32 if a.dtype != torch.bfloat16 else torch.int16)
            != b.view(torch.int32 if b.dtype != torch.bfloat16 else torch.int16)).any()


def test_every_round_of_two_at_once(gpu_lib):
    """Shared decode, scored decode with kept and with re-formed scores, and an
    eviction to pools of its own, on each of two streams at the same time: every
    round's outputs are filled with junk before and compared after, on that stream."""
    lens, hkv, pg = [900, 905, 1000, 64, 333], 2, 64
    e = Evict(lens, 128, hkv, pg, (1710,), group=8)
    shape, layer, src = e.shape, e.layer, e.kv.cache
    table = torch.full((5, WIDE // pg + 1), -1, dtype=torch.int32, device="cuda")
    table[:, :e.kv.block_table.shape[1]] = e.kv.block_table
    table[1, :13] = table[0, :13]  # 832 positions of sequence 0's pages
    wide = hswa.Cache(e.kv.k_pool, e.kv.v_pool, table)
    ctx, cu, sh, budgets = i32(lens), i32([0, 2, 5]), i32([832, 0]), i32([128, 100, 64, 64, 1])
    scores = _scores(5, hkv, 1000, (1710,))

    class Calls:
        def __init__(self):
            self.q = [to_dev(synth.normal_bf16((5, n, 16, D), 1710, n, synth.TAG_QDEC)) for n in (1, 1, 9)]
            self.out = [torch.empty_like(q) for q in self.q]
            self.sc = [torch.empty((5, hkv, 1000), device="cuda") for _ in range(2)]
            self.kept = torch.empty((5, hkv, 128), dtype=torch.int32, device="cuda")
            self.kept_sc = torch.empty((5, hkv, 128), device="cuda")
            self.lens = torch.empty(5, dtype=torch.int32, device="cuda")
            self.k, self.v = torch.empty_like(e.kv.k_pool), torch.empty_like(e.kv.v_pool)
            self.dst = hswa.Cache(self.k, self.v, i32(e.new_table))
            need = [hswa.decode_shared_workspace_bytes(shape, 5, 1, WIDE, 2, WIDE),
                    hswa.decode_scored_workspace_bytes(shape, 5, 1, 1000),
                    hswa.decode_scored_workspace_bytes(shape, 5, 9, 1000)]
            assert need[0] > hswa.decode_workspace_bytes(shape, 5, WIDE)
            self.ws = torch.empty(max(need), dtype=torch.uint8, device="cuda")
            self.bad = torch.zeros(1, dtype=torch.bool, device="cuda")

        def outputs(self):
            return [*self.out, *self.sc, self.kept, self.kept_sc, self.lens, self.k, self.v]

        def run(self, stream):
            for x in self.outputs():
                x.fill_(-7)
            self.ws.fill_(0x5A)
            hswa.decode_shared(layer, shape, wide, self.q[0], ctx, WIDE, cu, sh, WIDE, self.out[0], workspace=self.ws,
                               stream=stream)
            for i in (0, 1):
                hswa.decode_scored(layer, shape, src, self.q[1 + i], ctx, 1000, scores, self.sc[i], self.out[1 + i],
                                   workspace=self.ws, stream=stream)
            hswa.kv_evict(layer, shape, src, self.dst, scores, ctx, budgets, 1000, self.kept, self.lens, num_recent=8,
                          num_sinks=2, scores_out=self.kept_sc, stream=stream)

        def compare(self, want):
            for x, y in zip(self.outputs(), want):
                self.bad |= _differ(x, y)

    both, streams = [Calls(), Calls()], [torch.cuda.Stream(), torch.cuda.Stream()]
    both[0].run(None)
    torch.cuda.synchronize()
    want = [x.clone() for x in both[0].outputs()]
    assert not any(bool(torch.isnan(x.float()).any()) for x in want[:5])
    for b, n in enumerate([128, 100, 64, 64, 1]):  # (the eviction's own bits stand in test_gpu_kv_evict.py)
        ref = OE.kept_positions(scores[b, 0].cpu().numpy(), lens[b], n, 8, 2)
        assert np.array_equal(want[5][b, 0, :ref.size].cpu().numpy(), ref)
    for s in streams:
        s.wait_stream(torch.cuda.current_stream())
    for _ in range(20):
        for c, s in zip(both, streams):
            with torch.cuda.stream(s):
                c.run(s)
                c.compare(want)
    torch.cuda.synchronize()
    assert not bool(both[0].bad) and not bool(both[1].bad)


@pytest.mark.parametrize("max_ctx", [256, 257])
@pytest.mark.parametrize("nq", [1, 3])
def test_shared_decode_about_one_pass(gpu_lib, max_ctx, nq):
    """Contexts of up to 256 keys are hswa_decode_multi's, bit for bit and without a
    workspace; one key more is shared."""
    r = np.random.default_rng(max_ctx + nq)
    s = Shared([(190, [int(x) for x in r.integers(nq, 67, 90)]), (64, [int(x) for x in r.integers(nq, 100, 70)])], nq, 16,
               8, 64, (1713, nq), max_ctx=max_ctx)
    got = s.run(max_shared=190)
    assert (s.ws.numel() > 1) == (max_ctx > 256)
    s.check(got, f"contexts of {max_ctx}", by_prefix=max_ctx > 256)
    if max_ctx == 256:
        out = torch.full_like(s.q, 7.0)
        hswa.decode_multi(*s.args[:6], out)
        torch.cuda.synchronize()
        assert np.array_equal(to_f64(out), got)


@pytest.mark.parametrize("max_ctx,max_keep", [(500, 96), (500, 600), (9000, 3000), (33000, 96)])
def test_evict_contexts_out_of_line(gpu_lib, max_ctx, max_keep):
    """Contexts above max_context_len count as that, those below zero as none; in
    one launch, in two, by passes over the scores."""
    print(f"[together] evict max_ctx={max_ctx} max_keep={max_keep}", flush=True)
    lens, budgets = [max_ctx, 300, 0, max_ctx, 0], [90, 100, 7, max_keep + 5, 1]
    e = Evict(lens, max_keep, 2, 64, (1711, max_ctx), max_ctx=max_ctx)
    s = _scores(5, 2, max_ctx + 9, (1711, max_keep))
    e.lens = [max_ctx + 1, 300, -5, (1 << 31) - 1, -(1 << 31)]
    e.run(s, budgets, 8, 4)
    e.lens = lens
    e.check(s, budgets, 8, 4)


def test_budgeted_cache_of_the_allocator(gpu_lib):
    """Two sequences decode on a FULL layer whose pages are the allocator's. Once a
    context passes its budget, it is cut to a spare slot's pages and its old slot is
    freed, so that pages change owners again and again; every step is compared with
    attention over the positions that each KV head still holds."""
    pg, hq, hkv, stride, limit, keep = 16, 16, 2, 24, 320, 200
    pages = 60  # (three full rows would be 72: freed pages have to be used again)
    alloc = hswa.Allocator(pg, 16, pages, pages, 3, stride)
    shape, layer = hswa.Shape(hq, hkv, D, pg), hswa.Layer.full()
    k_pool = torch.full(hswa.k_pool_shape(pages, hkv, pg), float("nan"), dtype=torch.bfloat16, device="cuda")
    v_pool = torch.full(hswa.v_pool_shape(pages, hkv, pg), float("nan"), dtype=torch.bfloat16, device="cuda")
    ws = torch.empty(hswa.decode_scored_workspace_bytes(shape, 1, 1, stride * pg), dtype=torch.uint8, device="cuda")
    seqs = []

    def row(slot):
        return hswa.Cache(k_pool, v_pool, i32(alloc.tables()[0][slot:slot + 1]))

    def append(s, n, tag):
        start, at = len(s["held"][0]), len(s["k"])
        assert alloc.extend(s["slot"], start + n) == 0
        k, v = [synth.normal_bf16((n, hkv, D), 1712, s["id"], tag, t) for t in (synth.TAG_K, synth.TAG_V)]
        hswa.kv_append(layer, shape, row(s["slot"]), to_dev(k), to_dev(v), i32([0, n]), i32([start]))
        alloc.step_end(s["slot"], n == 1)
        s["k"], s["v"] = np.concatenate([s["k"], k]), np.concatenate([s["v"], v])
        s["held"] = [np.concatenate([h, at + np.arange(n)]) for h in s["held"]]

    for i, n in enumerate((290, 131)):
        s = {"id": i, "slot": i, "k": np.zeros((0, hkv, D), np.uint16), "v": np.zeros((0, hkv, D), np.uint16),
             "held": [np.zeros(0, np.int64)] * hkv, "scores": torch.zeros((1, hkv, stride * pg), device="cuda")}
        assert alloc.admit(i, n, n) == 0
        append(s, n, 1000)
        seqs.append(s)
    spare, cuts, owners = 2, 0, {}
    for step in range(160):
        for s in seqs:
            for _ in range(1 + 2 * s["id"]):  # (the second grows faster)
                append(s, 1, len(s["k"]))
            n = len(s["held"][0])
            q = synth.normal_bf16((1, 1, hq, D), 1712, s["id"], step, synth.TAG_QDEC)
            out = torch.full((1, 1, hq, D), 7.0, dtype=torch.bfloat16, device="cuda")
            hswa.decode_scored(layer, shape, row(s["slot"]), to_dev(q), i32([n]), n, s["scores"], s["scores"], out,
                               workspace=ws)
            if n >= limit:
                assert alloc.admit(spare, keep, keep) == 0 and alloc.extend(spare, keep) == 0
                kept = torch.full((1, hkv, keep), -1, dtype=torch.int32, device="cuda")
                lens, scores = torch.zeros(1, dtype=torch.int32, device="cuda"), torch.zeros_like(s["scores"])
                hswa.kv_evict(layer, shape, row(s["slot"]), row(spare), s["scores"], i32([n]), i32([keep]), n, kept, lens,
                              num_recent=32, num_sinks=4, scores_out=scores)
            torch.cuda.synchronize()
            ref = np.zeros((1, hq, D))
            for g in range(hkv):
                k, v = [OA.bf16_bits_to_f64(x[s["held"][g]][:, g:g + 1]) for x in (s["k"], s["v"])]
                qg = OA.bf16_bits_to_f64(q[0])[:, g * 8:(g + 1) * 8]
                ref[:, g * 8:(g + 1) * 8] = OA.masked_attention(qg, k, v, [n - 1], None, shape.scale)
            assert_close(to_f64(out)[0], ref, f"step {step}, sequence {s['id']}, {n} keys")
            if n >= limit:
                at = [OE.kept_positions(s["scores"][0, g].cpu().numpy(), n, keep, 32, 4) for g in range(hkv)]
                assert int(lens) == keep and all(np.array_equal(kept[0, g].cpu().numpy(), at[g]) for g in range(hkv))
                s["held"] = [h[a] for h, a in zip(s["held"], at)]
                for p in alloc.tables()[0][s["slot"]]:
                    if p >= 0:
                        owners.setdefault(int(p), set()).add((s["id"], cuts))
                alloc.free(s["slot"])
                s["slot"], spare, s["scores"] = spare, s["slot"], scores
                cuts += 1
    assert cuts >= 4 and any(len({i for i, _ in o}) == 2 for o in owners.values())  # pages went from one to the other
    cu, shared = prefix_groups(alloc.tables()[0][[s["slot"] for s in seqs]], [len(s["held"][0]) for s in seqs], pg)
    assert not shared.any()
    alloc.close()
