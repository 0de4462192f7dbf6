"""Host side of the attention and page calls under AddressSanitizer and UndefinedBehaviourSanitizer, without a
device: tests/native/serving_driver.cpp replaces the HIP launch entry points, sweeps sizes and checks every launch
against what its kernels assume."""
import os
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def test_serving_host_code_clean_under_asan_ubsan(tmp_path):
    from paper_2606_08635_amd import build as B

    if not os.path.exists(B.HIPCC):
        pytest.skip("hipcc not found")
    api = "serving/serving_api.cpp"
    objs = [os.path.join(B.BUILD_DIR, os.path.splitext(s)[0] + ".o") for s in B.SOURCES if s != api]
    if not all(os.path.exists(o) for o in objs):
        B.build()
    # host-side instrumentation only: every sanitizer flag is scoped to the host pass
    host = []
    for f in ("-fsanitize=address", "-fsanitize=undefined", "-fno-sanitize-recover=all", "-fno-omit-frame-pointer", "-g"):
        host += ["-Xarch_host", f]
    own = []
    for src in (os.path.join(B.CSRC, api), os.path.join(ROOT, "tests", "native", "serving_driver.cpp")):
        own.append(str(tmp_path / (os.path.basename(src) + ".o")))
        r = subprocess.run([B.HIPCC, *B.FLAGS, *host, "-c", src, "-o", own[-1]], capture_output=True, text=True, timeout=600)
        assert r.returncode == 0, r.stderr[-3000:]
    exe = str(tmp_path / "serving")
    r = subprocess.run([B.HIPCC, "--offload-arch=gfx950", *host, "-o", exe, *own, *objs], capture_output=True, text=True,
                       timeout=600)
    assert r.returncode == 0, r.stderr[-3000:]
    # the HIP runtime keeps allocations alive at exit: leak checking off for this binary
    r = subprocess.run([exe], capture_output=True, text=True, timeout=600, env=dict(os.environ, ASAN_OPTIONS="detect_leaks=0"))
    assert r.returncode == 0 and r.stdout.startswith("ok"), r.stdout[-2000:] + r.stderr[-4000:]
