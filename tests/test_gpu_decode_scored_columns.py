"""GPU parity of decode with attention scores (hswa_decode_scored), beyond
test_gpu_decode_scored.py: more than 16 (query, head) columns of a KV head, whose
scores are formed anew from K, in both of that kernel's forms (128 and 512 keys a
workgroup); batches past 64 and 256 sequences on both ways; contexts above
max_context_len and below zero. Tolerances are those derived there."""

import numpy as np
import pytest
import torch

from oracle import attention as OA
from oracle import eviction as OE
from paper_2607_13095_amd import hswa
from tests.hswa_testlib import assert_close, i32, to_f64
from tests.test_gpu_cache_calls_edges import Far
from tests.test_gpu_decode_scored import U, Scored

pytestmark = pytest.mark.gpu

WIDE = 25000  # 8 KV heads x 49 runs of 512 keys: enough workgroups for the form of 512 keys, whatever the contexts


@pytest.mark.parametrize("pg", [16, 32, 64])
@pytest.mark.parametrize("ns", [47, 48])
def test_about_the_switch_of_forms(gpu_lib, ns, pg):
    """8 KV heads x 47 and 48 sequences of up to 512 keys: 376 and 384 runs of 512,
    on both sides of the switch, with contexts about chunks and the queries' number."""
    print(f"[scored-columns] ns={ns} pg={pg}", flush=True)
    r = np.random.default_rng(ns + pg)
    lens = [0, 1, 8, 9, 10, 31, 32, 33, 127, 128, 129, 511, 512]
    lens += [int(x) for x in r.integers(1, 513, ns - len(lens))]
    s = Scored(lens, 9, 16, 8, pg, (1410, ns, pg), max_ctx=512)
    s.run()
    s.check(what=f"{ns} sequences, pg={pg}")


@pytest.mark.parametrize("pg", [16, 64])
@pytest.mark.parametrize("longest", [3584, 4200])
def test_several_runs_of_keys(gpu_lib, longest, pg):
    """Contexts of up to 7 runs of 512 keys (336 in all: the small form) and of up to
    9 (432: the large one), ragged at their ends."""
    print(f"[scored-columns] longest={longest} pg={pg}", flush=True)
    s = Scored([longest, 513, 1023, 1, 2049, longest - 37], 9, 16, 8, pg, (1411, longest, pg))
    s.run()
    s.check(what=f"up to {longest}, pg={pg}")


@pytest.mark.parametrize("max_ctx", [None, WIDE])
@pytest.mark.parametrize("scale", [1.0, 4.0])
def test_peaked(gpu_lib, scale, max_ctx):
    """(The tolerance's constant grows with the exponents, as with kept scores.)"""
    s = Scored([5, 300, 2001], 9, 16, 8, 64, (1412,), scale=scale, max_ctx=max_ctx)
    s.run()
    got, start = [x.cpu().numpy().astype(np.float64) for x in (s.scores, s.start)]
    for b, n, out, w, rel in s.refs():
        assert_close(to_f64(s.out)[b], out, "rows")
        ref = start[b, :, :n] + w
        assert np.all(np.abs(got[b, :, :n] - ref) <= (rel + scale * 2.0 ** -12) * w + 2 * U * ref)
        assert np.all(got[b, :, n:] == -7.0)


@pytest.mark.parametrize("max_ctx", [None, WIDE])
@pytest.mark.parametrize("pg", [16, 32, 64])
def test_bad_pages(gpu_lib, pg, max_ctx):
    """Keys on page ids outside the pool are left out and add nothing: single
    pages (half a chunk with 16 keys), neighbours, the last one."""
    print(f"[scored-columns] bad pages, pg={pg} max_ctx={max_ctx}", flush=True)
    s = Scored([645], 9, 16, 8, pg, (1413, pg), max_ctx=max_ctx)
    lost = [1, 4, 5, 644 // pg]
    gone = np.zeros(645, bool)
    for i, lp in enumerate(lost):
        s.kv.block_table[0, lp] = (-1, s.kv.num_pages, 1 << 30, -7)[i]
        gone[lp * pg:(lp + 1) * pg] = True
    s.run()
    got, start = [x.cpu().numpy().astype(np.float64)[0] for x in (s.scores, s.start)]
    assert np.array_equal(got[:, :645][:, gone], start[:, :645][:, gone]) and np.all(got[:, 645:] == -7.0)
    # what each query still sees: the held ones of its keys, in their order
    k, v = [OA.bf16_bits_to_f64(x[0][:645][~gone]) for x in (s.hist.k, s.hist.v)]
    q = OA.bf16_bits_to_f64(s.qbits[0])
    pos = np.cumsum(~gone)[np.arange(645 - 9, 645)] - 1
    assert_close(to_f64(s.out)[0], OA.masked_attention(q, k, v, pos, None, s.shape.scale), "rows without the lost keys")
    w = OE.attention_weights(q, k, pos, s.shape.scale)
    spread = (np.abs(q).reshape(-1, 128) @ np.abs(k).reshape(-1, 128).T).max()
    rel = 2 * 128 * U * spread * s.shape.scale + 2.0 ** -14
    ref = start[:, :645][:, ~gone] + w
    assert np.all(np.abs(got[:, :645][:, ~gone] - ref) <= rel * w + 2 * U * ref)


@pytest.mark.parametrize("max_ctx", [None, WIDE])
def test_in_place_steps(gpu_lib, max_ctx):
    """Three steps on one score tensor, in place, from no scores at all; a step's
    weights sum to the number of its (query, head) rows of a KV head."""
    s = Scored([1200, 77], 9, 16, 8, 64, (1414,), max_ctx=max_ctx)
    s.run(scores_in=None)
    s.check(base="none", what="first")
    f = s.scores.cpu().numpy().astype(np.float64)
    for _ in range(2):
        s.run(scores_in=s.scores)
    w = s.scores.cpu().numpy().astype(np.float64)
    for b, n in enumerate(s.lens):
        assert np.all(np.abs(w[b, :, :n] - 3 * f[b, :, :n]) <= 4 * U * 3 * f[b, :, :n])
        assert np.allclose(f[b, :, :n].sum(-1), 18, rtol=2.0 ** -12)
        assert np.all(w[b, :, n:] == -7.0)


@pytest.mark.parametrize("max_ctx", [None, WIDE])
def test_unaligned_scores_and_another_stream(gpu_lib, max_ctx):
    s = Scored([1201, 3, 642], 9, 16, 8, 32, (1415,), max_ctx=max_ctx)
    s.run()
    s.check(what="aligned")
    want, n = s.scores.clone(), s.scores.numel()
    side = torch.cuda.Stream()
    for off in (1, 2, 3):
        buf = torch.full((n + 8,), -7.0, device="cuda")
        s.scores = buf[off:off + n].view(s.start.shape)
        side.wait_stream(torch.cuda.current_stream())
        s.run(stream=side)
        assert torch.equal(s.scores, want), off
        assert bool((buf[:off] == -7.0).all()) and bool((buf[off + n:] == -7.0).all())


@pytest.mark.parametrize("max_ctx", [None, WIDE])
def test_captured(gpu_lib, max_ctx):
    """Replays with other contexts and queries, eager work between: the eager bits."""
    s = Scored([2500, 31, 800], 9, 16, 8, 64, (1416,), max_ctx=max_ctx)
    s.run()
    s.check(what="eager")
    ctx, ws = s.ctx, s.ws
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        hswa.decode_scored(s.layer, s.shape, s.kv.cache, s.q, ctx, s.max_ctx, s.start, s.scores, s.out, workspace=ws)
    for rep, lens in enumerate(([2500, 31, 800], [1, 31, 799], [2499, 0, 5], [2500, 31, 800])):
        ctx.copy_(i32(lens))
        s.q.copy_(s.q.flip(0))
        s.run()
        want, rows = s.scores.clone(), s.out.clone()
        s.scores.fill_(-7.0)
        s.out.fill_(7.0)
        ws.fill_(rep)
        torch.cuda.synchronize()
        g.replay()
        torch.cuda.synchronize()
        for b, n in enumerate(lens):
            assert torch.equal(want[b, :, :n], s.scores[b, :, :n]) and bool((s.scores[b, :, n:] == -7.0).all()), rep
        assert torch.equal(rows.view(torch.int16), s.out.view(torch.int16)), rep
        s.scores.fill_(-7.0)


@pytest.mark.parametrize("nq", [1, 3])
@pytest.mark.parametrize("ns", [63, 64, 65, 130, 255, 256, 257, 300])
def test_batches(gpu_lib, ns, nq):
    """8 and 24 columns of a KV head: the batch sizes at which the loops over
    sequences take a second turn and the plan is found another way."""
    print(f"[scored-columns] batch of {ns}, nq={nq}", flush=True)
    r = np.random.default_rng(ns)
    lens = [int(x) for x in r.integers(1, 150, ns)]
    for b in (0, ns // 2, ns - 1):
        lens[b] = 0
    lens[ns // 3], lens[1] = 700, 1000
    s = Scored(lens, nq, 16, 2, 64, (1417, ns, nq))
    s.run()
    s.check(what=f"{ns} sequences, nq={nq}")


@pytest.mark.parametrize("nq,hkv", [(1, 2), (9, 8)])
def test_contexts_out_of_line(gpu_lib, nq, hkv):
    """Contexts above max_context_len count as that, those below zero as none."""
    s = Scored([500, 300, 0, 500], nq, 16, hkv, 64, (1418, nq), max_ctx=500)
    s.ctx = i32([501, 300, -5, (1 << 31) - 1])
    s.run()
    s.check(what="clamped")
    s.scores.fill_(-7.0)
    s.ctx = i32([-(1 << 31), -1, 0, 0])
    s.run()
    assert bool((s.scores == -7.0).all()) and bool((s.out == 0).all())


@pytest.mark.parametrize("pg", [16, 64])
def test_weights_on_pools_past_4_gib(gpu_lib, pg):
    """16 queries (32 columns) whose K is read a second time past 4 GiB."""
    print(f"[scored-columns] far pages, pg={pg}", flush=True)
    f = Far(pg)
    nq = 16
    q = f.q.expand(2, nq, 2 * f.hkv, 128).contiguous()
    for max_ctx in (420, WIDE):
        scores, out = torch.full((2, f.hkv, max_ctx), -7.0, device="cuda"), torch.empty_like(q)
        ws = torch.empty(hswa.decode_scored_workspace_bytes(f.shape, 2, nq, max_ctx), dtype=torch.uint8, device="cuda")
        hswa.decode_scored(f.layer, f.shape, f.cache, q, f.ctx, max_ctx, None, scores, out, workspace=ws)
        torch.cuda.synchronize()
        for b, n in enumerate(f.lens):
            qs = np.repeat(OA.bf16_bits_to_f64(f.qbits[b]), nq, axis=0)
            k, v = [OA.bf16_bits_to_f64(x[b]) for x in (f.hk, f.hv)]
            pos = np.arange(n - nq, n)
            w = OE.attention_weights(qs, k, pos, 128 ** -0.5)
            spread = (np.abs(qs).reshape(-1, 128) @ np.abs(k).reshape(-1, 128).T).max()
            rel = 2 * 128 * U * spread * 128 ** -0.5 + 2.0 ** -14
            got = scores[b].cpu().numpy().astype(np.float64)
            assert np.all(np.abs(got[:, :n] - w) <= rel * w + 2 * U * w), (b, max_ctx)
            assert np.all(got[:, n:] == -7.0)
            assert_close(to_f64(out)[b], OA.masked_attention(qs, k, v, pos, None), f"rows {b}")
