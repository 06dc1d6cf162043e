"""The build's check of the register split of the block-scaled product's kernel."""
import os
import sys

import pytest

from paper_2602_19362_b200 import build

REPORT = """ptxas info    : Compiling entry function '_ZN4oapl12other_kernelILi1EEEv' for 'sm_100a'
ptxas info    : Used 40 registers, used 1 barriers
ptxas info    : Compiling entry function '_ZN4oapl20scaled_matmul_kernelILi2ELb0EEEv14CUtensorMap_st' for 'sm_100a'
ptxas info    : Function properties for _ZN4oapl20scaled_matmul_kernelILi2ELb0EEEv14CUtensorMap_st
    56 bytes stack frame, 72 bytes spill stores, 132 bytes spill loads
ptxas info    : Used %d registers, used 1 barriers
ptxas info    : Compiling entry function '_ZN4oapl20scaled_matmul_kernelILi1ELb0EEEv14CUtensorMap_st' for 'sm_100a'
ptxas info    : Used %d registers, used 1 barriers
"""


def test_registers_of_the_split_are_checked():
    build.check_registers(REPORT % (168, 168), 168)
    for a, b in [(160, 168), (168, 160), (176, 176)]:
        with pytest.raises(RuntimeError, match="counts on kSmRegs = 168"):
            build.check_registers(REPORT % (a, b), 168)
    with pytest.raises(RuntimeError):
        build.check_registers("", 168)


def test_the_constant_is_the_sources():
    assert build._split_constant() == 168


def test_a_build_that_fails_the_check_leaves_the_library_alone(tmp_path, monkeypatch):
    # a stand-in for the compiler: writes the output, reports other registers
    cc = tmp_path / "nvcc"
    cc.write_text(f"#!{sys.executable}\nimport sys\nopen(sys.argv[sys.argv.index('-o') + 1], 'w').write('new')\n"
                  f"sys.stderr.write({REPORT % (160, 160)!r})\n")
    cc.chmod(0o755)
    lib = tmp_path / "liboapl.so"
    lib.write_text("old")
    monkeypatch.setenv("NVCC", str(cc))
    monkeypatch.setattr(build, "LIB", str(lib))
    monkeypatch.setattr(build, "HERE", str(tmp_path))
    with pytest.raises(RuntimeError, match="kSmRegs"):
        build.build(force=True)
    assert lib.read_text() == "old" and sorted(os.listdir(tmp_path)) == ["liboapl.so", "nvcc"]
    cc.write_text(cc.read_text().replace("160", "168"))
    build.build(force=True)
    assert lib.read_text() == "new" and sorted(os.listdir(tmp_path)) == ["liboapl.so", "nvcc"]
