"""A library without one of its kernel files must not load: every launcher that the argument checks (csrc/api.hip) call is an ordinary
undefined symbol of them, none a weak one, which would be address 0 where its file is missing from the build."""
import os
import re
import shutil
import subprocess

import pytest

from paper_2408_15237_amd import build


def _nm(path, *flags):
    out = subprocess.run(["nm", *flags, path], check=True, capture_output=True, text=True).stdout
    return [(m[1], m[2]) for m in re.finditer(r"^\S*\s+([A-Za-z]) (\S+)$", out, flags=re.M)]


def test_no_launcher_is_weak(tmp_path):
    hipcc = build._hipcc()
    if not shutil.which(hipcc):
        pytest.skip("no hipcc")
    obj = str(tmp_path / "api.o")
    subprocess.run([hipcc] + [f for f in build.FLAGS if not f.startswith("-O")] + ["-O0", "--offload-host-only", "-c", os.path.join(build.CSRC, "api.hip"), "-o", obj],
                   check=True, capture_output=True)
    called = {name: kind for kind, name in _nm(obj, "--undefined-only") if "ssmv" in name and "launch_" in name}
    assert len(called) >= 15 and any("launch_beam_select" in n for n in called)
    assert {n: k for n, k in called.items() if k != "U"} == {}
    defined = {name for kind, name in _nm(build.LIB, "--defined-only") if kind in "TW"}
    assert set(called) <= defined
