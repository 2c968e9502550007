"""What the build does with the compiler's remarks on resources: kernels that have to keep their registers end it when they do not, and other messages still come through."""
import subprocess

import pytest

from paper_2211_13939_amd import build


def _remarks(name, spill, scratch):
    tail = "[-Rpass-analysis=kernel-resource-usage]"
    lines = [f"Function Name: {name}", "    TotalSGPRs: 50", "    VGPRs: 31", f"    ScratchSize [bytes/lane]: {scratch}", "    Dynamic Stack: False", "    SGPRs Spill: 3", f"    VGPRs Spill: {spill}"]
    return "".join(f"x/paged.hip:126:1: remark: {line} {tail}\n" + ("  126 | {\n      | ^\n" if i == 0 else "") for i, line in enumerate(lines))


MANY, CROSS, FEW = "_ZN3tts12_GLOBAL__N_112k_paged_manyILi64EEEvT_", "_ZN3tts12_GLOBAL__N_112k_cross_manyILi128EEEvT_", "_ZN3tts12_GLOBAL__N_111k_paged_fewIfEEvT_"


def test_kernels_that_spill():
    assert build.spilled(_remarks(MANY, 0, 0) + _remarks(FEW, 9, 40) + _remarks(CROSS, 0, 0)) == []
    assert build.spilled(_remarks(FEW, 0, 0) + _remarks(MANY, 2, 12) + _remarks(CROSS, 0, 8)) == [MANY, CROSS]
    assert "-Rpass-analysis=kernel-resource-usage" in build.FLAGS


def test_other_messages():
    warning = "x/paged.hip:7:3: warning: unused variable 'y' [-Wunused-variable]\n    7 |   int y;\n      |       ^\n"
    assert build.messages(_remarks(MANY, 0, 0) + warning + _remarks(FEW, 0, 0) + "21 remarks generated when compiling for gfx950.\n") == warning.rstrip("\n")
    assert build.messages("") == ""


@pytest.mark.parametrize("spill,code", [(0, 0), (4, 0), (0, 1)])
def test_a_build(tmp_path, monkeypatch, spill, code):
    out = tmp_path / "lib.so"

    def run(cmd, **_):
        out.write_text("")
        return subprocess.CompletedProcess(cmd, code, stderr=_remarks(MANY, spill, 4 * spill))

    monkeypatch.setattr(build, "OUT", str(out))
    monkeypatch.setattr(build.subprocess, "run", run)
    if code:
        with pytest.raises(subprocess.CalledProcessError):
            build.build()
    elif spill:
        with pytest.raises(RuntimeError, match="k_paged_many"):
            build.build()
        assert not out.exists()
    else:
        assert build.build() == str(out)
