"""The calls on shared and bounded caches in one run, as a server makes them:
samples of one prompt decode over its shared pages (groups found from the block
table), the prompt's last queries and every step score the keys, the cache is
cut to a budget on new pages, and decoding and scoring go on over what stayed.
Every output is compared with fp64 attention over the positions that each KV
head still holds."""

import numpy as np
import pytest
import torch

import synth
from oracle import attention as OA
from oracle import eviction as OE
from paper_2607_13095_amd import hswa
from paper_2607_13095_amd.kvcache import prefix_groups
from tests.hswa_testlib import assert_close, i32, to_dev, to_f64

pytestmark = pytest.mark.gpu

D, HQ, HKV, PG = 128, 16, 2, 64
G = HQ // HKV
WIDE = 150000
U = 2.0 ** -24


class Server:
    def __init__(self, prompt, samples, seed):
        self.ns, self.seed = samples, seed
        self.shape, self.layer = hswa.Shape(HQ, HKV, D, PG), hswa.Layer.full()
        self.pages = 96
        self.k_pool = torch.full(hswa.k_pool_shape(self.pages, HKV, PG), float("nan"), dtype=torch.bfloat16, device="cuda")
        self.v_pool = torch.full(hswa.v_pool_shape(self.pages, HKV, PG), float("nan"), dtype=torch.bfloat16, device="cuda")
        self.free = list(synth.page_permutation(self.pages, *seed))
        self.stride = WIDE // PG + 1
        self.table = np.full((samples, self.stride), -1, np.int32)
        self.k = [np.zeros((0, HKV, D), np.uint16) for _ in range(samples)]  # every token ever appended
        self.v = [x.copy() for x in self.k]
        self.held = [[np.zeros(0, np.int64)] * HKV for _ in range(samples)]  # positions each KV head holds, in order
        self.step = 0
        # the prompt, once, and its table row for every sample; the last page, partly filled, is copied
        k, v = self.new(prompt, 0)
        n = -(-prompt // PG)
        self.table[:, :n] = [self.free.pop() for _ in range(n)]
        self.append(0, k, v, 0)
        for b in range(1, samples):
            self.k[b], self.v[b], self.held[b] = self.k[0], self.v[0], list(self.held[0])
            if prompt % PG:
                page = self.free.pop()
                self.k_pool[page], self.v_pool[page] = self.k_pool[int(self.table[0, n - 1])], self.v_pool[int(self.table[0, n - 1])]
                self.table[b, n - 1] = page

    def new(self, n, tag):
        self.step += 1
        return (synth.normal_bf16((n, HKV, D), *self.seed, self.step, tag, synth.TAG_K),
                synth.normal_bf16((n, HKV, D), *self.seed, self.step, tag, synth.TAG_V))

    def cache(self):
        return hswa.Cache(self.k_pool, self.v_pool, i32(self.table))

    def lens(self):
        return [len(h[0]) for h in self.held]

    def append(self, b, k, v, tag):
        start = self.lens()[b]
        for lp in range(start // PG, -(-(start + len(k)) // PG)):
            if self.table[b, lp] < 0:
                self.table[b, lp] = self.free.pop()
        one = hswa.Cache(self.k_pool, self.v_pool, i32(self.table[b:b + 1]))
        hswa.kv_append(self.layer, self.shape, one, to_dev(k), to_dev(v), i32([0, len(k)]), i32([start]))
        at = len(self.k[b]) + np.arange(len(k))
        self.k[b], self.v[b] = np.concatenate([self.k[b], k]), np.concatenate([self.v[b], v])
        self.held[b] = [np.concatenate([h, at]) for h in self.held[b]]

    def tokens(self):
        for b in range(self.ns):
            self.append(b, *self.new(1, b), b)

    def queries(self, nq):
        self.step += 1
        return synth.normal_bf16((self.ns, nq, HQ, D), *self.seed, self.step, synth.TAG_QDEC)

    def refs(self, qbits, b):
        """Rows, and each held key's weight, of sequence b."""
        nq = qbits.shape[1]
        out, w = np.zeros((nq, HQ, D)), []
        for g in range(HKV):
            k, v = [OA.bf16_bits_to_f64(x[b][self.held[b][g]][:, g:g + 1]) for x in (self.k, self.v)]
            q = OA.bf16_bits_to_f64(qbits[b][:, g * G:(g + 1) * G])
            pos = np.arange(len(k) - nq, len(k))
            out[:, g * G:(g + 1) * G] = OA.masked_attention(q, k, v, pos, None, self.shape.scale)
            w.append(OE.attention_weights(q, k, pos, self.shape.scale)[0])
        return out, np.stack(w)


def _decode_shared(s):
    qbits = s.queries(1)
    lens = s.lens()
    cu, shared = prefix_groups(s.table, lens, PG)
    out = torch.full((s.ns, 1, HQ, D), 7.0, dtype=torch.bfloat16, device="cuda")
    need = hswa.decode_shared_workspace_bytes(s.shape, s.ns, 1, WIDE, len(shared), WIDE)
    ws = torch.empty(need, dtype=torch.uint8, device="cuda")
    hswa.decode_shared(s.layer, s.shape, s.cache(), to_dev(qbits), i32(lens), WIDE, i32(cu), i32(shared), WIDE, out,
                       workspace=ws)
    torch.cuda.synchronize()
    for b in range(s.ns):
        assert_close(to_f64(out)[b], s.refs(qbits, b)[0], f"shared decode, sequence {b}")
    return cu, shared


def _decode_scored(s, nq, scores, totals):
    """One scored call, in place; totals: the reference sums [b][Hkv, held]."""
    qbits, lens = s.queries(nq), s.lens()
    out = torch.full((s.ns, nq, HQ, D), 7.0, dtype=torch.bfloat16, device="cuda")
    ws = torch.empty(hswa.decode_scored_workspace_bytes(s.shape, s.ns, nq, max(lens)), dtype=torch.uint8, device="cuda")
    hswa.decode_scored(s.layer, s.shape, s.cache(), to_dev(qbits), i32(lens), max(lens), scores, scores, out, workspace=ws)
    torch.cuda.synchronize()
    for b in range(s.ns):
        ref, w = s.refs(qbits, b)
        assert_close(to_f64(out)[b], ref, f"scored decode, sequence {b}")
        grown = np.zeros((HKV, lens[b]))
        grown[:, :totals[b].shape[1]] = totals[b]
        totals[b] = grown + w
        got = scores.cpu().numpy()[b, :, :lens[b]].astype(np.float64)
        # weights within 2^-11 (a score of 128 products under 1/sqrt(128), twice: see test_gpu_decode_scored.py), sums in fp32
        assert np.all(np.abs(got - totals[b]) <= 2.0 ** -11 * totals[b] + 64 * U * totals[b])


@pytest.mark.parametrize("prompt", [640, 777])
def test_serve_with_a_bounded_cache(gpu_lib, prompt):
    print(f"[bounded cache] prompt of {prompt}", flush=True)
    s = Server(prompt, 4, (1600, prompt))
    room = prompt + 64
    scores = torch.zeros((s.ns, HKV, room), device="cuda")
    totals = [np.zeros((HKV, 0)) for _ in range(s.ns)]
    cu, shared = prefix_groups(s.table, s.lens(), PG)
    assert cu.tolist() == [0, 4] and shared.tolist() == [prompt // PG * PG]
    _decode_scored(s, 8, scores, totals)  # the prompt's last 8 queries: all its keys
    for _ in range(3):
        s.tokens()
        cu, shared = _decode_shared(s)
        assert len(shared) == 1 and shared[0] >= 64
        _decode_scored(s, 1, scores, totals)
    # cut every sample to a budget of its own, on new pages; the prompt's pages stay as they were
    budgets, most = [200, 128, 77, 10 ** 6], 1024
    old, lens = s.table.copy(), s.lens()
    before = s.k_pool[torch.from_numpy(old[0][:prompt // PG].astype(np.int64)).cuda()].clone()
    new = np.full_like(s.table, -1)
    for b in range(s.ns):
        n = min(budgets[b], lens[b], most)
        new[b, :-(-n // PG)] = [s.free.pop() for _ in range(-(-n // PG))]
    src = s.cache()
    s.table = new
    kept = torch.full((s.ns, HKV, most), -1, dtype=torch.int32, device="cuda")
    new_lens = torch.zeros(s.ns, dtype=torch.int32, device="cuda")
    new_scores = torch.zeros((s.ns, HKV, most), device="cuda")
    hswa.kv_evict(s.layer, s.shape, src, s.cache(), scores, i32(lens), i32(budgets), max(lens), kept, new_lens,
                  num_recent=32, num_sinks=4, scores_out=new_scores)
    torch.cuda.synchronize()
    for b in range(s.ns):
        for g in range(HKV):
            ref = OE.kept_positions(scores[b, g].cpu().numpy(), lens[b], budgets[b], 32, 4)
            assert np.array_equal(kept[b, g, :ref.size].cpu().numpy(), ref) and int(new_lens[b]) == ref.size
            s.held[b][g] = s.held[b][g][ref]
        totals[b] = np.stack([totals[b][g][kept[b, g, :int(new_lens[b])].cpu().numpy()] for g in range(HKV)])
    after = s.k_pool[torch.from_numpy(old[0][:prompt // PG].astype(np.int64)).cuda()]
    assert torch.equal(before.view(torch.int16), after.view(torch.int16))
    for _ in range(3):  # decoding goes on over what stayed
        s.tokens()
        cu, shared = prefix_groups(s.table, s.lens(), PG)
        assert np.all(shared == 0)
        _decode_scored(s, 1, new_scores, totals)
    _decode_scored(s, 3, new_scores, totals)
    _decode_shared(s)  # no prefix is left: as hswa_decode_multi
