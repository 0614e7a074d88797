"""GPU parity of decode with attention scores (hswa_decode_scored) against the
fp64 oracle: output rows as decode's, and every key's weight summed over the
queries and the query heads of its KV head.

Tolerance of a weight. The products of bf16 values are exact in fp32 and a
score is a sum of 128 of them, so it is off by at most 128 u S, S the sum of
their magnitudes, u = 2^-24; times the scale that is the error of an exponent.
It enters once in the key's own exponential and once, at most as large, in the
row's sum: a factor within 1 +- 2 * 128 u S scale. The exponent's multiply-add
and subtraction round values below 2^8 twice or so (2^-15 u-steps: 4 * 2^8 u),
and the exponential, the sums over pieces and the logarithm a few u more; 2^-14
covers them for scores below 2^8 in exp2 units."""

import numpy as np
import pytest
import torch

import synth
from oracle import attention as OA
from oracle import eviction as OE
from paper_2607_13095_amd import hswa
from tests.hswa_testlib import SeqHistory, append_history, assert_close, i32, make_layer, to_dev, to_f64

pytestmark = pytest.mark.gpu

D = 128
U = 2.0 ** -24


class Scored:
    def __init__(self, lens, nq, hq, hkv, pg, seed, scale=None, max_ctx=None, stride=None):
        self.lens, self.nq, self.hq, self.hkv, self.ns = lens, nq, hq, hkv, len(lens)
        self.max_ctx = max_ctx or max(max(lens), 1)
        self.shape = hswa.Shape(hq, hkv, D, pg, scale=scale)
        self.layer, self.kv = make_layer("full", 0, self.shape, [max(n, 1) for n in lens[:-1]] + [self.max_ctx], seed)
        self.hist = SeqHistory(lens, hkv, D, *seed)
        if sum(lens):
            append_history(self.layer, self.shape, self.kv, self.hist, [0] * self.ns, lens)
        self.qbits = synth.normal_bf16((self.ns, nq, hq, D), *seed, synth.TAG_QDEC)
        self.q, self.ctx = to_dev(self.qbits), i32(lens)
        n = stride or self.max_ctx + 3
        self.start = torch.from_numpy(np.random.default_rng(7).random((self.ns, hkv, n)).astype(np.float32)).cuda()
        self.scores = torch.full_like(self.start, -7.0)
        self.out = torch.full_like(self.q, 7.0)
        need = hswa.decode_scored_workspace_bytes(self.shape, self.ns, nq, self.max_ctx)
        self.ws = torch.full((need,), 255, dtype=torch.uint8, device="cuda")

    def run(self, scores_in="start", **kw):
        s = self.start if isinstance(scores_in, str) else scores_in
        hswa.decode_scored(self.layer, self.shape, self.kv.cache, self.q, self.ctx, self.max_ctx, s, self.scores,
                           self.out, workspace=self.ws, **kw)
        torch.cuda.synchronize()

    def refs(self):
        for b, n in enumerate(self.lens):
            q, k, v = [OA.bf16_bits_to_f64(x) for x in (self.qbits[b], self.hist.k[b][:n], self.hist.v[b][:n])]
            pos = np.arange(n - self.nq, n)
            out = np.zeros((self.nq, self.hq, D))
            if n:
                out[pos >= 0] = OA.masked_attention(q[pos >= 0], k, v, pos[pos >= 0], None, self.shape.scale)
            w = OE.attention_weights(q, k, pos, self.shape.scale) if n else np.zeros((self.hkv, 0))
            spread = max([np.abs(q).reshape(-1, D) @ np.abs(k[j]).T for j in range(n)], key=np.max).max() if n else 0.0
            yield b, n, out, w, 2 * 128 * U * spread * self.shape.scale + 2.0 ** -14

    def check(self, base="start", what=""):
        got = self.scores.cpu().numpy().astype(np.float64)
        start = self.start.cpu().numpy().astype(np.float64) if base == "start" else np.zeros_like(got)
        for b, n, out, w, rel in self.refs():
            assert_close(to_f64(self.out)[b], out, f"{what} rows of sequence {b}")
            ref = start[b, :, :n] + w
            err = np.abs(got[b, :, :n] - ref)
            assert np.all(err <= rel * w + 2 * U * np.abs(ref)), (what, b, float((err / (rel * w + 2 * U * ref)).max()))
            assert np.all(got[b, :, n:] == -7.0), (what, b)


@pytest.mark.parametrize("nq", [1, 2, 5, 16])
@pytest.mark.parametrize("pg", [16, 32, 64, 256])
def test_decode_scored(gpu_lib, pg, nq):
    print(f"[scored] pg={pg} nq={nq}", flush=True)
    s = Scored([0, 1, 15, 33, 129, 700, 1500], nq, 16, 2, pg, (1400, pg, nq))
    s.run()
    s.check(what=f"pg={pg} nq={nq}")


@pytest.mark.parametrize("hq,hkv,nq", [(8, 8, 1), (16, 1, 1), (64, 8, 4), (32, 1, 3), (128, 1, 1), (4, 2, 64)])
def test_decode_scored_groups(gpu_lib, hq, hkv, nq):
    print(f"[scored-groups] hq={hq} hkv={hkv} nq={nq}", flush=True)
    s = Scored([70, 513, 1030], nq, hq, hkv, 64, (1401, hq, nq))
    s.run()
    s.check(what=f"hq={hq} hkv={hkv} nq={nq}")


@pytest.mark.parametrize("lens,nq", [([9000], 1), ([40000, 300], 1), ([5000, 2600], 8), ([2048, 4097, 1, 6144], 3)])
def test_decode_scored_long(gpu_lib, lens, nq):
    """Contexts cut into many spans, one at a time and unlike ones together."""
    print(f"[scored-long] {lens} nq={nq}", flush=True)
    s = Scored(lens, nq, 8, 1, 64, (1402, len(lens), nq))
    s.run()
    s.check(what=f"{lens}")


@pytest.mark.parametrize("scale", [1.0, 4.0])
def test_decode_scored_peaked(gpu_lib, scale):
    """Scores far apart: one key takes nearly all, most weights are 0 in fp32.
    (Exponents reach 2^9 here: their roundings are 2^-13 relative at most, and
    the tolerance's constant grows with them.)"""
    s = Scored([5, 300, 3001], 2, 16, 2, 64, (1403,), scale=scale)
    s.run()
    got = s.scores.cpu().numpy().astype(np.float64)
    start = s.start.cpu().numpy().astype(np.float64)
    for b, n, out, w, rel in s.refs():
        assert_close(to_f64(s.out)[b], out, "rows")
        ref = start[b, :, :n] + w
        assert np.all(np.abs(got[b, :, :n] - ref) <= (rel + scale * 2.0 ** -12) * w + 2 * U * ref)


def test_decode_scored_in_place_steps(gpu_lib):
    """Three steps on one score tensor, in place, from no scores at all; the sum
    of a step's weights is the number of its (query, head) rows."""
    s = Scored([1200, 77], 1, 16, 2, 64, (1404,))
    s.run(scores_in=None)
    s.check(base="none", what="first")
    first = s.scores.clone()
    for step in range(2):
        s.run(scores_in=s.scores)
    w = s.scores.cpu().numpy().astype(np.float64)
    f = first.cpu().numpy().astype(np.float64)
    for b, n in enumerate(s.lens):
        assert np.all(np.abs(w[b, :, :n] - 3 * f[b, :, :n]) <= 4 * U * 3 * f[b, :, :n])
        assert np.allclose(f[b, :, :n].sum(-1), 8, rtol=2.0 ** -12)
    assert np.all(w[1, :, 77:] == -7.0)


def test_decode_scored_same_bits_again(gpu_lib):
    s = Scored([3000, 10, 900], 4, 32, 4, 16, (1405,))
    s.run()
    a, o = s.scores.clone(), s.out.clone()
    s.ws.fill_(0)
    s.run()
    assert torch.equal(a, s.scores) and torch.equal(o.view(torch.int16), s.out.view(torch.int16))


def test_decode_scored_bad_pages(gpu_lib):
    """Keys on page ids outside the pool are left out and add nothing."""
    s = Scored([640], 2, 16, 2, 64, (1406,))
    s.kv.block_table[0, 3], s.kv.block_table[0, 7] = -1, s.kv.num_pages
    s.run()
    gone = np.zeros(640, bool)
    gone[192:256] = gone[448:512] = True
    got = s.scores.cpu().numpy().astype(np.float64)[0, :, :640]
    start = s.start.cpu().numpy().astype(np.float64)[0, :, :640]
    assert np.array_equal(got[:, gone], start[:, gone])
    k, v = [OA.bf16_bits_to_f64(x[0][:640][~gone]) for x in (s.hist.k, s.hist.v)]
    q = OA.bf16_bits_to_f64(s.qbits[0])
    n = int((~gone).sum())
    out = OA.masked_attention(q, k, v, np.arange(n - 2, n), None, s.shape.scale)
    assert_close(to_f64(s.out)[0], out, "rows without the lost keys")
    w = OE.attention_weights(q, k, np.arange(n - 2, n), s.shape.scale)
    assert np.allclose(got[:, ~gone] - start[:, ~gone], w, rtol=2e-3, atol=4 * U)


def test_decode_scored_wide_table_and_stride(gpu_lib):
    """max_context_len far above every context, lengths above it clamped, score
    rows of a longer stride; on a stream of the caller's."""
    s = Scored([100, 517], 1, 16, 2, 64, (1407,), max_ctx=20000, stride=20011)
    st = torch.cuda.Stream()
    st.wait_stream(torch.cuda.current_stream())
    s.run(stream=st)
    s.check(what="wide")


def test_decode_scored_captured(gpu_lib):
    s = Scored([2500, 31, 800], 2, 32, 4, 64, (1408,))
    s.run()
    s.check(what="eager")
    want, rows = s.scores.clone(), s.out.clone()
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        hswa.decode_scored(s.layer, s.shape, s.kv.cache, s.q, s.ctx, s.max_ctx, s.start, s.scores, s.out,
                           workspace=s.ws)
    for rep in range(3):
        s.scores.fill_(-7.0)
        s.out.fill_(7.0)
        s.ws.fill_(rep)
        torch.cuda.synchronize()
        g.replay()
        torch.cuda.synchronize()
        assert torch.equal(want, s.scores) and torch.equal(rows.view(torch.int16), s.out.view(torch.int16))
        s.run()


@pytest.mark.parametrize("stride", [1204, 1201])
def test_decode_scored_unaligned_scores(gpu_lib, stride):
    """Score tensors at every address that fp32 has, in place too: the same bits."""
    s = Scored([1201, 3, 642], 1, 16, 2, 32, (1409,), stride=stride)
    s.run()
    s.check(what="aligned")
    want, n = s.scores.clone(), s.scores.numel()
    for off in (1, 2, 3):
        buf = torch.full((n + 8,), -7.0, device="cuda")
        s.scores = buf[off:off + n].view(s.start.shape)
        s.run()
        assert torch.equal(s.scores, want), off
        s.scores.copy_(s.start)
        s.run(scores_in=s.scores)
        for b, c in enumerate(s.lens):
            assert torch.equal(s.scores[b, :, :c], want[b, :, :c]), off
            assert torch.equal(s.scores[b, :, c:], s.start[b, :, c:]), off
        assert bool((buf[:off] == -7.0).all()) and bool((buf[off + n:] == -7.0).all())
