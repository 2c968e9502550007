"""Loads into LDS that are written out (lds_loads.h), in the code that comes of them: a base that a vector instruction has brought into scalar registers is not read too early."""
import os
import re
import subprocess

import pytest

from paper_2211_13939_amd import build

SOURCE = """
#include "lds_loads.h"
extern "C" __global__ void probe(const uint64_t* from, float* out)
{
    extern __shared__ float lds[];
    const uint64_t x = from[threadIdx.x];
    const uint32_t low = __builtin_amdgcn_readfirstlane((uint32_t)x), high = __builtin_amdgcn_readfirstlane((uint32_t)(x >> 32));
    tts::to_lds_from<WIDTH>(reinterpret_cast<const void*>((uint64_t)high << 32 | low), threadIdx.x * WIDTH, 0);
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
    out[threadIdx.x] = lds[threadIdx.x];
}
"""


def _states_since_a_vector_write(lines, base):
    """Wait states between the last vector instruction that writes one of the base's registers and the load; None: a scalar one wrote it last."""
    states, lo, hi = 0, *map(int, re.match(r"s\[(\d+):(\d+)\]", base).groups())
    for line in reversed(lines):
        op, _, rest = line.partition(" ")
        to = re.match(r"\s*s(?:\[(\d+):(\d+)\]|(\d+)\b)", rest)
        if to:
            a, b = (int(to[3]),) * 2 if to[3] else (int(to[1]), int(to[2]))
            if a <= hi and b >= lo:
                return states if op.startswith("v_") else None
        states += int(rest, 0) + 1 if op == "s_nop" else 1
    raise AssertionError("nobody wrote the base")


@pytest.mark.parametrize("width,name", [(16, "global_load_lds_dwordx4"), (4, "global_load_lds_dword")])
def test_a_base_from_vector_instructions(tmp_path, width, name):
    if not os.path.exists(build.HIPCC):
        pytest.skip("no hipcc")
    src = tmp_path / "probe.hip"
    src.write_text(SOURCE)
    flags = [f for f in build.FLAGS if f not in ("-shared", "-fPIC", "-Wall")]
    subprocess.run([build.HIPCC, *flags, f"-DWIDTH={width}", "-I", build.CSRC, "--cuda-device-only", "-S", "-x", "hip", str(src), "-o", str(tmp_path / "probe.s")], check=True, capture_output=True)
    text = (tmp_path / "probe.s").read_text()
    lines = [re.sub(r"\s+", " ", line.split(";")[0]).strip() for line in text[text.index("probe:"):].splitlines()]
    lines = [line for line in lines if line and not line.startswith(".") and not line.endswith(":")]
    at = next(i for i, line in enumerate(lines) if line.startswith(name + " "))
    assert any(line.startswith("v_readfirstlane_b32") for line in lines[:at])
    states = _states_since_a_vector_write(lines[:at], lines[at].split(", ")[1])
    assert states is None or states >= 5
