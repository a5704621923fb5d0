"""The build refuses kernels whose registers are not those that their launch is planned with.  No GPU, no compiler: a fake of its report."""
import os
import sys

import pytest

from paper_1903_04488_b200 import build as B

REPORT = """ptxas info    : 0 bytes gmem
ptxas info    : Compiling entry function '_Z9k_productILi1EEv6Common' for 'sm_100a'
ptxas info    : Function properties for _Z9k_productILi1EEv6Common
    0 bytes stack frame, 0 bytes spill stores, 0 bytes spill loads
ptxas info    : Used %d registers, used 1 barriers
ptxas info    : Compiling entry function '_Z7k_otherv' for 'sm_100a'
ptxas info    : Used 40 registers, used 0 barriers
ptxas info    : Compiling entry function '_Z9k_productILi2EEv6Common' for 'sm_100a'
ptxas info    : Used 168 registers, used 1 barriers, 16 bytes cumulative stack size
"""


def test_the_report_is_read():
    assert B.check_registers(REPORT % 168, 168) == 2
    with pytest.raises(B.RegisterError, match="ILi1EE.*160 registers.*168"):
        B.check_registers(REPORT % 160, 168)
    with pytest.raises(B.RegisterError):
        B.check_registers(REPORT % 168, 160)
    with pytest.raises(B.RegisterError):
        B.check_registers("", 168)


def test_sources_that_hand_registers_over_state_their_plan():
    plans = {}
    for src in B.sources():
        with open(src) as f:
            text = f.read()
        plans[os.path.basename(src)] = B.planned_registers(text)
        assert ("setmaxnreg" in text) == (plans[os.path.basename(src)] is not None), src
    # 384 threads; what the warps keep between them is what the launch has: 224 + 224 + 56 in three groups of four warps
    assert plans["muon.cu"] * 3 == 224 + 224 + 56


@pytest.mark.parametrize("registers", [168, 160])
def test_an_object_that_is_not_as_planned_is_not_kept(tmp_path, registers):
    src, obj, report = tmp_path / "a.cu", tmp_path / "a.o", tmp_path / "report"
    src.write_text("// setmaxnreg\nconstexpr int LAUNCH_REGISTERS = 168;\n")
    report.write_text(REPORT % registers)
    fake = [sys.executable, "-c", f"import sys; open({str(obj)!r}, 'w').close(); sys.stderr.write(open({str(report)!r}).read()); assert '-v' in sys.argv"]
    if registers == 168:
        assert B.compile_one(fake, str(src), str(obj)) == 0 and obj.exists()
    else:
        with pytest.raises(B.RegisterError):
            B.compile_one(fake, str(src), str(obj))
        assert not obj.exists()
