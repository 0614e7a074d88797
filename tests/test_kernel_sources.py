"""Rules that the kernel sources keep to (read as text, no GPU)."""

import os
import re

from paper_2607_13095_amd import build_lib

BARRIER = "__builtin_amdgcn_wave_barrier"


def _code(name):
    with open(os.path.join(build_lib.CSRC, name)) as f:
        return re.sub(r"//[^\n]*|/\*.*?\*/", "", f.read(), flags=re.S)


def test_lanes_exchange_lds_data_behind_fences():
    """The wave barrier orders no memory: a lane's load after it may be given what
    that lane itself stored before it, whatever other lanes have made of it since.
    It stands in one place, between a release and an acquire fence."""
    sources = {f: _code(f) for f in sorted(os.listdir(build_lib.CSRC)) if f.endswith((".hip", ".h"))}
    where = [f for f, s in sources.items() for _ in range(s.count(BARRIER))]
    assert where == ["hswa_common.h"], where
    body = re.search(r"void wave_exchange\(\)\s*\{(.*?)\}", sources["hswa_common.h"], re.S).group(1)
    calls = re.findall(r"(\w+)\(([^()]*)\);", body)
    assert calls == [("__builtin_amdgcn_fence", '__ATOMIC_RELEASE, "wavefront"'), (BARRIER, ""),
                     ("__builtin_amdgcn_fence", '__ATOMIC_ACQUIRE, "wavefront"')], calls
