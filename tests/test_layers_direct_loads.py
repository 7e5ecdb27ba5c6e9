"""The gated recurrence's backward kernel loads its next tile straight into LDS with inline assembly (csrc/gated_common.h), inside which the
compiler resolves no hazards: a vector memory access may read a scalar that a vector instruction wrote only five wait states later, and a load
into LDS may follow a write of M0 only one wait state later.  A probe whose base comes from a vector instruction is compiled for the device
(no GPU needed) and both distances are counted."""
import re
import shutil
import subprocess

import pytest

from paper_2408_15237_amd import build

PROBE = """
#include "gated_common.h"
using namespace ssmv;
extern "C" __global__ void probe(const char *const *bases, uint32_t *out)
{
    __shared__ uint32_t lds[64];
    const size_t a = (size_t)bases[threadIdx.x];
    const size_t base = ((size_t)__builtin_amdgcn_readfirstlane((int)(a >> 32)) << 32) | (unsigned)__builtin_amdgcn_readfirstlane((int)a);
    load_to_lds((const char *)base, threadIdx.x * 4u, lds);
    wait_but<0>();
    out[threadIdx.x] = lds[threadIdx.x];
}
"""


def _scalars(operand):
    m = re.match(r"s(?:(\d+)|\[(\d+):(\d+)\])$", operand)
    return range(0) if not m else range(int(m[1]), int(m[1]) + 1) if m[1] else range(int(m[2]), int(m[3]) + 1)


def test_wait_states_ahead_of_a_load_into_lds(tmp_path):
    hipcc = build._hipcc()
    if not shutil.which(hipcc):
        pytest.skip("no hipcc")
    src, asm = tmp_path / "probe.hip", tmp_path / "probe.s"
    src.write_text(PROBE)
    subprocess.run([hipcc] + build.FLAGS + ["--offload-device-only", "-S", str(src), "-o", str(asm)], check=True, capture_output=True)
    now, by_vector, m0, base_waits, m0_waits, vector_bases = 0, {}, None, [], [], 0
    for line in asm.read_text().splitlines():
        m = re.match(r"\s+([a-z]\w+)\s*(.*)", line.split(";")[0])
        if not m:
            continue
        op, args = m[1], [a.split()[0] for a in m[2].split(",") if a.split()]
        if op.startswith("global_load_lds"):
            base_waits.append(min((now - by_vector[r] for a in args for r in _scalars(a) if r in by_vector), default=5))
            m0_waits.append(now - m0)
        now += int(args[0], 0) + 1 if op == "s_nop" else 1
        if op.startswith("v_") and args:
            by_vector.update((r, now) for r in _scalars(args[0]))
            vector_bases += op.startswith("v_readfirstlane")
        elif op.startswith("s_") and args:        # waits for the vector instruction itself; what it writes may be read at any time
            for r in _scalars(args[0]):
                by_vector.pop(r, None)
            if args[0] == "m0":
                m0 = now
    assert vector_bases, "the probe's base did not come from a vector instruction"
    assert len(base_waits) == 1 and base_waits[0] >= 5 and m0_waits[0] >= 1, (base_waits, m0_waits)
