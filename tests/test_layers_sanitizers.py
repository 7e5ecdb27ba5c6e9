"""The argument checks of the layer operators under AddressSanitizer and UndefinedBehaviorSanitizer: the two argument-checking files are built for the host with stand-in
launchers as in test_sanitizers.py, and the tests whose calls all end on the host are run on that build.  And no launcher that they call is a weak symbol."""
import glob
import os
import shutil
import subprocess

import pytest

from paper_2408_15237_amd import build
from test_launchers_are_linked import _nm
from test_sanitizers import CSRC, ROOT, _preload, _run


def test_layer_argument_checks_under_sanitizers(tmp_path):
    hipcc = "/opt/rocm/bin/hipcc"
    rt = subprocess.run([hipcc, "-print-file-name=libclang_rt.asan-x86_64.so"], capture_output=True, text=True).stdout.strip()
    if not os.path.isabs(rt) or not os.path.exists(rt):
        cand = glob.glob("/opt/rocm/lib/llvm/lib/clang/*/lib/linux/libclang_rt.asan-x86_64.so")
        if not cand:
            pytest.skip("clang's AddressSanitizer runtime is not installed")
        rt = cand[0]
    host_san = ["-Xarch_host", "-fsanitize=address", "-Xarch_host", "-fsanitize=undefined", "-Xarch_host", "-fno-sanitize-recover=all"]
    objs = []
    stubs = os.path.join(ROOT, "tests", "host_stubs")
    for src in (os.path.join(CSRC, "api.hip"), os.path.join(CSRC, "layers_api.hip"), os.path.join(stubs, "launch_stubs.cpp"), os.path.join(stubs, "layer_launch_stubs.cpp")):
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
    _run(env, ["tests/test_layers_abi.py"])


def test_no_layer_launcher_is_weak(tmp_path):
    hipcc = build._hipcc()
    if not shutil.which(hipcc):
        pytest.skip("no hipcc")
    obj = str(tmp_path / "layers_api.o")
    subprocess.run([hipcc] + [f for f in build.FLAGS if not f.startswith("-O")] + ["-O0", "--offload-host-only", "-c", os.path.join(build.CSRC, "layers_api.hip"), "-o", obj],
                   check=True, capture_output=True)
    called = {name: kind for kind, name in _nm(obj, "--undefined-only") if "ssmv" in name and "launch_" in name}
    assert len(called) == 5 and set(called.values()) == {"U"}
    assert set(called) <= {name for kind, name in _nm(build.LIB, "--defined-only") if kind in "TW"}
