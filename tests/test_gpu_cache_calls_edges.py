"""The calls on shared and bounded caches where other calls and large memory are
near: pools past 4 GiB, two calls at once on two streams, the binding's check of
the device, everything around the outputs left as it was."""

import numpy as np
import pytest
import torch

import synth
from oracle import attention as OA
from oracle import eviction as OE
from paper_2607_13095_amd import hswa
from tests.hswa_testlib import assert_close, i32, to_dev, to_f64

pytestmark = pytest.mark.gpu

D = 128
WIDE = 150000


class Far:
    """Two sequences that share 300 tokens on the last pages of pools of 5 GiB."""

    def __init__(self, pg=64, hkv=8):
        self.shape, self.layer = hswa.Shape(2 * hkv, hkv, D, pg), hswa.Layer.full()
        self.hkv, self.pg = hkv, pg
        pages = (5 << 30) // (hkv * pg * D * 2)
        self.k = torch.empty(hswa.k_pool_shape(pages, hkv, pg), dtype=torch.bfloat16, device="cuda")
        self.v = torch.empty(hswa.v_pool_shape(pages, hkv, pg), dtype=torch.bfloat16, device="cuda")
        self.lens = [420, 377]
        n = -(-300 // pg)
        self.table = np.full((2, WIDE // pg + 1), -1, np.int32)
        self.new = np.full_like(self.table, -1)
        at = pages - 1
        for t in (self.table, self.new):
            for b in range(2):
                for i in range(-(-self.lens[b] // pg)):
                    t[b, i], at = at, at - 1
        self.hk = [synth.normal_bf16((c, hkv, D), 1700, b, synth.TAG_K) for b, c in enumerate(self.lens)]
        self.hv = [synth.normal_bf16((c, hkv, D), 1700, b, synth.TAG_V) for b, c in enumerate(self.lens)]
        self.hk[1][:300], self.hv[1][:300] = self.hk[0][:300], self.hv[0][:300]
        self.cache = hswa.Cache(self.k, self.v, i32(self.table))
        self.dst = hswa.Cache(self.k, self.v, i32(self.new))
        hswa.kv_append(self.layer, self.shape, self.cache, to_dev(np.concatenate(self.hk)),
                       to_dev(np.concatenate(self.hv)), i32([0, 420, 797]), i32([0, 0]))
        self.table[1, :n - 1] = self.table[0, :n - 1]
        self.cache = hswa.Cache(self.k, self.v, i32(self.table))
        self.qbits = synth.normal_bf16((2, 1, 2 * hkv, D), 1700, synth.TAG_QDEC)
        self.q, self.ctx = to_dev(self.qbits), i32(self.lens)

    def ref(self, b, keep=None):
        k, v = [OA.bf16_bits_to_f64(x[b]) for x in (self.hk, self.hv)]
        q = OA.bf16_bits_to_f64(self.qbits[b])
        if keep is None:
            return OA.masked_attention(q, k, v, [len(k) - 1], None), OE.attention_weights(q, k, [len(k) - 1], D ** -0.5)
        out = np.zeros((1, 2 * self.hkv, D))
        for g in range(self.hkv):
            out[:, 2 * g:2 * g + 2] = OA.masked_attention(q[:, 2 * g:2 * g + 2], k[keep[g], g:g + 1], v[keep[g], g:g + 1],
                                                          [len(keep[g]) - 1], None)
        return out, None


@pytest.mark.parametrize("pg", [16, 64])
def test_pools_past_4_gib(gpu_lib, pg):
    print(f"[far pages] pg={pg}", flush=True)
    f = Far(pg)
    out = torch.empty_like(f.q)
    need = hswa.decode_shared_workspace_bytes(f.shape, 2, 1, WIDE, 1, WIDE)
    ws = torch.empty(need, dtype=torch.uint8, device="cuda")
    hswa.decode_shared(f.layer, f.shape, f.cache, f.q, f.ctx, WIDE, i32([0, 2]), i32([300]), WIDE, out, workspace=ws)
    torch.cuda.synchronize()
    for b in range(2):
        assert_close(to_f64(out)[b], f.ref(b)[0], f"shared {b}")
    for nq in (1, 16):  # scores kept, and formed anew
        scores = torch.zeros((2, f.hkv, 500), device="cuda")
        q = f.q.expand(2, nq, 2 * f.hkv, D).contiguous()
        o = torch.empty_like(q)
        ws = torch.empty(hswa.decode_scored_workspace_bytes(f.shape, 2, nq, 420), dtype=torch.uint8, device="cuda")
        hswa.decode_scored(f.layer, f.shape, f.cache, q, f.ctx, 420, None, scores, o, workspace=ws)
        torch.cuda.synchronize()
        for b in range(2):
            assert_close(to_f64(o)[b, -1:], f.ref(b)[0], f"scored {b}")
            if nq == 1:
                got = scores[b, :, :f.lens[b]].cpu().numpy().astype(np.float64)
                assert np.allclose(got, f.ref(b)[1], rtol=2.0 ** -11, atol=0)
    kept = torch.empty((2, f.hkv, 100), dtype=torch.int32, device="cuda")
    lens = torch.empty(2, dtype=torch.int32, device="cuda")
    hswa.kv_evict(f.layer, f.shape, f.cache, f.dst, scores, f.ctx, i32([100, 64]), 420, kept, lens)
    ws = torch.empty(max(1, hswa.decode_workspace_bytes(f.shape, 2, 100)), dtype=torch.uint8, device="cuda")
    hswa.decode(f.layer, f.shape, f.dst, f.q, lens, 100, out, workspace=ws)
    torch.cuda.synchronize()
    for b, n in enumerate([100, 64]):
        keep = [OE.kept_positions(scores[b, g].cpu().numpy(), f.lens[b], n, 0, 0) for g in range(f.hkv)]
        assert all(np.array_equal(kept[b, g, :n].cpu().numpy(), keep[g]) for g in range(f.hkv))
        assert_close(to_f64(out)[b], f.ref(b, keep)[0], f"decode over the kept keys {b}")


def test_two_calls_at_once(gpu_lib):
    """Each call on two streams at the same time, with workspaces of their own,
    many times over: always the bits of a call alone."""
    f = Far()
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    need = max(hswa.decode_shared_workspace_bytes(f.shape, 2, 1, WIDE, 1, WIDE),
               hswa.decode_scored_workspace_bytes(f.shape, 2, 1, 420), 1)
    ws = [torch.empty(need, dtype=torch.uint8, device="cuda") for _ in streams]
    cu, sh = i32([0, 2]), i32([300])
    outs = [[torch.empty_like(f.q) for _ in range(2)] for _ in streams]
    scores = [torch.zeros((2, f.hkv, 420), device="cuda") for _ in streams]

    def calls(i, stream):
        hswa.decode_shared(f.layer, f.shape, f.cache, f.q, f.ctx, WIDE, cu, sh, WIDE, outs[i][0], workspace=ws[i],
                           stream=stream)
        hswa.decode_scored(f.layer, f.shape, f.cache, f.q, f.ctx, 420, None, scores[i], outs[i][1], workspace=ws[i],
                           stream=stream)

    calls(0, None)
    torch.cuda.synchronize()
    want = [o.clone() for o in outs[0]], scores[0].clone()
    for s in streams:
        s.wait_stream(torch.cuda.current_stream())
    for _ in range(20):
        for i, s in enumerate(streams):
            calls(i, s)
    torch.cuda.synchronize()
    for i in range(2):
        assert all(torch.equal(a.view(torch.int16), b.view(torch.int16)) for a, b in zip(outs[i], want[0]))
        assert torch.equal(scores[i], want[1])


def test_nothing_written_around_the_outputs(gpu_lib):
    """Outputs and workspace inside larger tensors: what lies around them stays."""
    f = Far()
    need = hswa.decode_shared_workspace_bytes(f.shape, 2, 1, WIDE, 1, WIDE)
    need2 = hswa.decode_scored_workspace_bytes(f.shape, 2, 3, 420)
    need3 = hswa.decode_scored_workspace_bytes(f.shape, 2, 20, 420)
    pad = 4096
    ws = torch.full((max(need, need2, need3) + 2 * pad,), 0xA5, dtype=torch.uint8, device="cuda")
    for which, n, nq in (("shared", need, 1), ("scored", need2, 3), ("scored", need3, 20)):
        ws.fill_(0xA5)
        q = f.q.expand(2, nq, 2 * f.hkv, D).contiguous()
        out = torch.full((q.numel() + 256,), 7.0, dtype=torch.bfloat16, device="cuda")
        o = out[128:128 + q.numel()].view(q.shape)
        scores = torch.full((2 * f.hkv * 420 + 64,), -3.0, device="cuda")
        s = scores[32:32 + 2 * f.hkv * 420].view(2, f.hkv, 420)
        w = ws[pad:pad + n]
        if which == "shared":
            hswa.decode_shared(f.layer, f.shape, f.cache, q, f.ctx, WIDE, i32([0, 2]), i32([300]), WIDE, o, workspace=w)
        else:
            hswa.decode_scored(f.layer, f.shape, f.cache, q, f.ctx, 420, None, s, o, workspace=w)
        torch.cuda.synchronize()
        assert torch.all(ws[:pad] == 0xA5) and torch.all(ws[pad + n:] == 0xA5), which
        assert torch.all(out[:128] == 7.0) and torch.all(out[128 + q.numel():] == 7.0), which
        assert torch.all(scores[:32] == -3.0) and torch.all(scores[32 + 2 * f.hkv * 420:] == -3.0), which


def test_tensors_of_another_device_are_refused(gpu_lib, monkeypatch):
    """The binding runs a call on the current device's stream: tensors that live
    elsewhere are refused (one GPU here: the current one is said to be another)."""
    f = Far()
    out = torch.empty_like(f.q)
    scores = torch.zeros((2, f.hkv, 420), device="cuda")
    kept = torch.empty((2, f.hkv, 8), dtype=torch.int32, device="cuda")
    lens = torch.empty(2, dtype=torch.int32, device="cuda")
    monkeypatch.setattr(torch.cuda, "current_device", lambda: 1)
    with pytest.raises(ValueError):
        hswa.decode_shared(f.layer, f.shape, f.cache, f.q, f.ctx, 420, i32([0, 2]), i32([300]), 300, out)
    with pytest.raises(ValueError):
        hswa.decode_scored(f.layer, f.shape, f.cache, f.q, f.ctx, 420, None, scores, out)
    with pytest.raises(ValueError):
        hswa.kv_evict(f.layer, f.shape, f.cache, f.dst, scores, f.ctx, f.ctx, 420, kept, lens)
