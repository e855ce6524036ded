"""AddressSanitizer and UndefinedBehaviorSanitizer runs of the host code of rotary positions and differential attention (no
GPU needed): their sources, sanitizers on the host side only, linked with tests/sanitize/dense_driver.cpp."""
import os
import tempfile
from concurrent.futures import ThreadPoolExecutor

import pytest

from tests.test_sanitizers import CLANGXX, ENV, HIPCC, ROOT, SAN_HOST, _run


@pytest.mark.skipif(not (os.path.exists(HIPCC) and os.path.exists(CLANGXX)), reason="ROCm compilers missing")
def test_dense_host_validation_under_asan_and_ubsan():
    csrc = os.path.join(ROOT, "paper_2201_02767_amd", "csrc")
    srcs = [os.path.join(csrc, n) for n in ("diff_api.hip", "diff_attn.hip", "diff_attn_bwd.hip", "rotary.hip")]
    with tempfile.TemporaryDirectory() as d:
        def compile_one(src):
            obj = os.path.join(d, os.path.basename(src) + ".o")
            _run([HIPCC, "--offload-arch=gfx950", "-O1", "-g", "-std=c++17", "-fPIC",
                  "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops", *SAN_HOST,
                  f"-I{os.path.join(ROOT, 'include')}", "-c", src, "-o", obj])
            return obj
        with ThreadPoolExecutor(max_workers=8) as ex:
            objs = list(ex.map(compile_one, srcs + [os.path.join(ROOT, "tests", "sanitize", "dense_driver.cpp")]))
        exe = os.path.join(d, "dense_san")
        _run([CLANGXX, "-fsanitize=address,undefined", "-o", exe, *objs, "-L/opt/rocm/lib", "-lamdhip64",
              "-Wl,-rpath,/opt/rocm/lib"])
        r = _run([exe], env=ENV, timeout=300)
        assert "0 failures" in r.stdout
