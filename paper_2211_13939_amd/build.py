"""Build the C-ABI library (HIP kernels + host code) for gfx950 into
paper_2211_13939_amd/libtts_pool.so.  Run on the CPU machine; hipcc cross-compiles."""
import os
import re
import subprocess
import sys

HERE = os.path.dirname(os.path.abspath(__file__))
CSRC = os.path.join(HERE, "csrc")
OUT = os.path.join(HERE, "libtts_pool.so")
SOURCES = ["kernels.hip", "segment.hip", "segment32.hip", "tts_pool.cpp", "postnet.hip", "postnet.cpp", "vocoder.hip", "vocoder.cpp", "encoder.hip", "encoder.cpp",
           "norm.hip", "norm.cpp", "linear8.hip", "linear8.cpp", "cross.hip", "cross.cpp", "rotary.hip", "rotary.cpp", "cache.cpp", "paged.hip", "paged.cpp"]
HIPCC = os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")
FLAGS = ["-O3", "-std=c++17", "--offload-arch=gfx950", "-fPIC", "-shared",
         "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops",
         # the first 16 dwords of a kernel's arguments arrive in scalar registers with the wave (gfx950 preloads them):
         # the first loads of a kernel no longer wait for a cold read of the argument block
         "-mllvm", "-amdgpu-kernarg-preload-count=16",
         # accumulators of the matrix instructions in ordinary vector registers.  Left to its heuristics the compiler keeps them in the
         # accumulation half of the file in the vocoder's up-samplings and its last layer, with 544 moves in and out (none with the
         # option): a two-byte call of 128 windows of 48 frames 512 -> 509 us, of 256 1049 -> 1040; up to 64 windows, in fp32 and in the
         # other files, whose kernels hold no such moves either way, the times are the same
         "-mllvm", "-amdgpu-mfma-vgpr-form=1",
         "-Wall", "-Wno-unused-result",
         # (what spilled() reads)
         "-Rpass-analysis=kernel-resource-usage"]
# Kernels that keep sums in registers through a loop whose loads the compiler does not see.  A form of k_paged_many whose sums were copied from turn to turn, with registers in scratch memory
# besides, gave wrong results now and then; why is not known.  A compiler that spills here again, or a change that has it do so, is to be noticed.
WHOLE = ("k_paged_many", "k_cross_many")


def sources():
    return [os.path.join(CSRC, s) for s in SOURCES]


def spilled(remarks: str) -> list:
    """Of the compiler's remarks on resources: the kernels of WHOLE that have vector registers in scratch memory, or any of it."""
    got, name = [], ""
    for what, value in re.findall(r"remark: +(Function Name|VGPRs Spill|ScratchSize \[bytes/lane\]): (\S+)", remarks):
        if what == "Function Name":
            name = value
        elif value != "0" and any(kernel in name for kernel in WHOLE) and name not in got:
            got.append(name)
    return got


def messages(stderr: str) -> str:
    """What the compiler said beside those remarks (each of which it shows a line of the source under)."""
    kept, on = [], True
    for line in stderr.splitlines():
        if line[:1].strip():
            on = "remark: " not in line and not re.match(r"\d+ remarks? generated", line)
        if on:
            kept.append(line)
    return "\n".join(kept)


def build(verbose: bool = False) -> str:
    cmd = [HIPCC] + FLAGS + ["-x", "hip"] + sources() + ["-o", OUT]
    if verbose:
        print(" ".join(cmd), flush=True)
    done = subprocess.run(cmd, stderr=subprocess.PIPE, text=True)
    said = messages(done.stderr)
    if said:
        print(said, file=sys.stderr, flush=True)
    done.check_returncode()
    bad = spilled(done.stderr)
    if bad:
        os.remove(OUT)
        raise RuntimeError(f"kernels that must not spill do: {', '.join(bad)}")
    return OUT


if __name__ == "__main__":
    print(build(verbose=True))
    sys.exit(0)
