"""The operators around the passes from plain C (tests/c_abi/check_operators.c): the header's prototypes under a C
compiler, results against the formulas, and the refusals that need a handle."""
import os
import subprocess

import pytest

HERE = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(HERE)
ROCM = os.environ.get("ROCM_PATH", "/opt/rocm")


def _build(to):
    lib_dir = os.path.join(ROOT, "paper_1412_7580_amd")
    subprocess.check_call(
        ["gcc", "-std=c99", "-O2", "-Wall", "-Werror", "-Wno-unused-result", "-D_GNU_SOURCE", "-I" + os.path.join(ROOT, "include"),
         "-I" + os.path.join(ROCM, "include"), os.path.join(HERE, "c_abi", "check_operators.c"), "-o", to, "-L" + lib_dir, "-lfftconv",
         "-L" + os.path.join(ROCM, "lib"), "-lamdhip64", "-lm", "-Wl,-rpath," + lib_dir, "-Wl,-rpath," + os.path.join(ROCM, "lib")])
    return to


def test_the_program_compiles_and_links(tmp_path):
    if not os.path.exists(os.path.join(ROOT, "paper_1412_7580_amd", "libfftconv.so")):
        pytest.skip("libfftconv.so not built")
    assert os.path.exists(_build(str(tmp_path / "check_operators")))


@pytest.mark.gpu
def test_operators_from_plain_c(tmp_path):
    run = subprocess.run([_build(str(tmp_path / "check_operators"))], capture_output=True, text=True, timeout=100)
    print(run.stdout, run.stderr)
    assert run.returncode == 0 and "all checks passed" in run.stdout
    assert run.stdout.count("  ok\n") == 26
