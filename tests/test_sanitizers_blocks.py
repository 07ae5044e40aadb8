"""The host code of the attention over selected blocks under ASan and UBSan (no
GPU): all of the library's sources with host-side instrumentation, driven by
tests/sanitize/blocks_checks.cpp."""
from __future__ import annotations

import os
from concurrent.futures import ThreadPoolExecutor

from test_sanitizers import CSRC, ENV_NO_LEAKS, HERE, OUT, ROOT, SOURCES, _hipcc, _run


def test_blocks_host_code_under_asan_ubsan():
    hipcc = _hipcc()
    out = OUT + "_blocks"
    os.makedirs(out, exist_ok=True)
    san = ["-Xarch_host", "-fsanitize=address", "-Xarch_host", "-fsanitize=undefined",
           "-Xarch_host", "-fno-sanitize-recover=all", "-Xarch_host", "-fno-omit-frame-pointer"]
    common = ["-O1", "-g", "-std=c++17", "-fPIC", "--offload-arch=gfx950",
              "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops",
              f"-I{os.path.join(ROOT, 'include')}", f"-I{CSRC}"]
    more = ("ckv_paged.hip", "ckv_paged.cpp", "ckv_blocks.hip", "ckv_blocks.cpp")
    sources = [os.path.join(CSRC, s) for s in SOURCES + more]
    sources.append(os.path.join(HERE, "sanitize", "blocks_checks.cpp"))
    objs = [os.path.join(out, os.path.basename(s) + ".asan.o") for s in sources]
    with ThreadPoolExecutor(max_workers=4) as ex:
        list(ex.map(lambda so: _run([hipcc, "-x", "hip", *common, *san, "-c", so[0], "-o", so[1]]),
                    zip(sources, objs)))
    exe = os.path.join(out, "blocks_checks")
    _run([hipcc, "--offload-arch=gfx950", *san, *objs, "-o", exe])
    r = _run([exe], env=dict(os.environ, **ENV_NO_LEAKS), timeout=300)
    assert "blocks checks ok" in r.stdout
