"""AddressSanitizer + UndefinedBehaviorSanitizer pass over the host side of rotary positions and the paged cache (CPU only, no kernel
runs): csrc/thrift_api.hip compiled with the sanitizers on its host code, linked with tests/sanitize_paged_driver.cpp."""
import os
import shutil
import subprocess

import pytest

from paper_2605_23081_amd.build import CSRC, INCLUDE, SOURCES

CLANGXX = "/opt/rocm/lib/llvm/bin/clang++"


def test_host_code_is_clean_under_asan_and_ubsan(tmp_path):
    if shutil.which("hipcc") is None or not os.path.exists(CLANGXX):
        pytest.skip("no ROCm toolchain")
    objects = [os.path.join(CSRC, s.replace(".hip", ".o")) for s in SOURCES if s != "thrift_api.hip"]
    if not all(os.path.exists(o) for o in objects):
        from paper_2605_23081_amd import build
        build.build()
    inc = ["-I", INCLUDE, "-I", CSRC]
    on_host = ["-Xarch_host", "-fsanitize=address", "-Xarch_host", "-fsanitize=undefined", "-Xarch_host", "-fno-sanitize-recover=all"]
    api, driver, exe = (str(tmp_path / n) for n in ("api.o", "driver.o", "run"))
    here = os.path.dirname(os.path.abspath(__file__))
    for cmd in (["hipcc", "--offload-arch=gfx950", "-O1", "-g", "-std=c++17", "-fPIC", "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops", *on_host, *inc,
                 "-c", os.path.join(CSRC, "thrift_api.hip"), "-o", api],
                [CLANGXX, "-O1", "-g", "-std=c++17", "-fsanitize=address,undefined", "-fno-sanitize-recover=all", *inc,
                 "-c", os.path.join(here, "sanitize_paged_driver.cpp"), "-o", driver],
                ["hipcc", "--offload-arch=gfx950", driver, api, *objects, "-o", exe, "-fno-gpu-sanitize", "-fsanitize=address,undefined"]):
        done = subprocess.run(cmd, capture_output=True, text=True)
        if done.returncode != 0 and ("asan" in done.stderr.lower() or "ubsan" in done.stderr.lower()) and "cannot find" in done.stderr.lower():
            pytest.skip("no sanitizer runtime for this toolchain")
        assert done.returncode == 0, done.stderr[-3000:]
    run = subprocess.run([exe], capture_output=True, text=True, timeout=300)
    assert run.returncode == 0, (run.stdout[-2000:], run.stderr[-4000:])
    assert "paged abi sanitizer pass: ok" in run.stdout
