"""The argument checks of the state-to-state calls under AddressSanitizer and UndefinedBehaviorSanitizer: api.hip is built for the host
with stand-in launchers as in test_sanitizers.py, and the tests whose calls all end on the host are run on that build."""
import os
import subprocess

import pytest

from test_sanitizers import CSRC, ROOT, _preload, _run


def test_decode_argument_checks_under_sanitizers(tmp_path):
    hipcc = "/opt/rocm/bin/hipcc"
    rt = subprocess.run([hipcc, "-print-file-name=libclang_rt.asan-x86_64.so"], capture_output=True, text=True).stdout.strip()
    if not os.path.isabs(rt) or not os.path.exists(rt):
        import glob
        cand = glob.glob("/opt/rocm/lib/llvm/lib/clang/*/lib/linux/libclang_rt.asan-x86_64.so")
        if not cand:
            pytest.skip("clang's AddressSanitizer runtime is not installed")
        rt = cand[0]
    host_san = ["-Xarch_host", "-fsanitize=address", "-Xarch_host", "-fsanitize=undefined", "-Xarch_host", "-fno-sanitize-recover=all"]
    objs = []
    for src in (os.path.join(CSRC, "api.hip"), os.path.join(ROOT, "tests", "host_stubs", "launch_stubs.cpp")):
        obj = str(tmp_path / (os.path.basename(src) + ".o"))
        r = subprocess.run([hipcc, "--offload-arch=gfx950", "-O1", "-g", "-std=c++17", "-fPIC", "-I", os.path.join(ROOT, "include"), "-I", CSRC] + host_san +
                           (["-x", "hip"] if src.endswith(".cpp") else []) + ["-c", src, "-o", obj], capture_output=True, text=True)
        assert r.returncode == 0, r.stderr[-3000:]
        objs.append(obj)
    lib = str(tmp_path / "libssmv_hostsan.so")
    r = subprocess.run([hipcc, "--offload-arch=gfx950", "-shared", "-fPIC", "-fno-gpu-sanitize", "-fsanitize=address", "-fsanitize=undefined",
                        "-shared-libsan"] + objs + ["-o", lib], capture_output=True, text=True)
    assert r.returncode == 0, r.stderr[-3000:]
    env = _preload(os.environ, os.path.realpath(rt))
    env["SSMV_LIBRARY"] = lib
    _run(env, ["tests/test_decode_abi.py"])
