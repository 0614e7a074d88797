"""Workspace sizes of the shared and scored decode for batches past their limit
of rows, and the C ABI's code for the calls on shared and bounded caches under
the address and undefined-behaviour sanitizers (no GPU is touched)."""

import os
import subprocess
import sys

import pytest

from paper_2607_13095_amd import build_lib, hswa

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
FILES = ("test_cache_calls_abi.py", "test_cache_calls_integers.py", "test_cache_calls_sizes.py")
ROWS = 1 << 25  # (sequence, query, head) rows that a call takes


@pytest.mark.parametrize("hq,hkv,nq", [(64, 8, 1), (64, 8, 3), (96, 96, 1), (128, 1, 64), (4096, 4096, 1)])
def test_sizes_at_the_limit_of_rows(hq, hkv, nq):
    """A size up to the last batch that the call takes, 0 from the next one on
    (products of the largest arguments leave 64 bits)."""
    sh, last = hswa.Shape(hq, hkv), ROWS // (hq * nq)
    assert hswa.decode_scored_workspace_bytes(sh, last, nq, 1 << 30) > 0
    assert hswa.decode_shared_workspace_bytes(sh, last, nq, 1 << 30, 1, 1 << 30) > 0
    for ns in (last + 1, 2 * last, (1 << 31) - 1):
        assert hswa.decode_scored_workspace_bytes(sh, ns, nq, 100) == 0
        assert hswa.decode_scored_workspace_bytes(sh, ns, nq, 1 << 30) == 0
        assert hswa.decode_shared_workspace_bytes(sh, ns, nq, 1 << 30, 1, 1 << 30) == 0


@pytest.mark.parametrize("hq,hkv,ns,nq,ng", [(64, 8, 300, 1, 1), (64, 8, 300, 4, 30), (32, 32, 336, 8, 1), (16, 16, 150, 2, 3)])
def test_contexts_of_one_pass_are_not_shared(hq, hkv, ns, nq, ng):
    """Contexts of up to 256 keys: hswa_decode_multi, which takes them in one pass
    without a workspace, was 1.06 to 6.4 times as fast as the way by prefix."""
    sh = hswa.Shape(hq, hkv)
    for max_ctx, top in ((65, 64), (256, 128), (256, 256), (256, 1 << 30)):
        assert hswa.decode_multi_workspace_bytes(sh, ns, nq, max_ctx) == 0
        assert hswa.decode_shared_workspace_bytes(sh, ns, nq, max_ctx, ng, top) == 0
    assert hswa.decode_shared_workspace_bytes(sh, ns, nq, 257, ng, 256) > hswa.decode_multi_workspace_bytes(
        sh, ns, nq, 257)


@pytest.mark.skipif("HSWA_LIB" in os.environ or not os.path.exists(build_lib.CXX), reason="runs the sanitizer build itself")
def test_under_sanitizers(tmp_path):
    lib = build_lib.build_host_sanitized(str(tmp_path))
    files = [os.path.join("tests", f) for f in FILES]
    r = subprocess.run([sys.executable, "-m", "pytest", "-q", "-x", "-m", "not gpu", "-p", "no:cacheprovider", *files],
                       cwd=ROOT, env=build_lib.sanitizer_env(lib), capture_output=True, text=True, timeout=600)
    tail = (r.stdout + r.stderr)[-4000:]
    assert r.returncode == 0, tail
    assert "ERROR: AddressSanitizer" not in r.stderr and "runtime error" not in r.stderr, tail
