"""Properties of the 8-bit kernels that a run does not show: the choice of a product's form over sizes, and what the build's compiler
and flags make of the kernels."""
import os
import subprocess

import pytest

from test_device_code import ROOT, _compile, _ends_with_load_in_flight

CSRC = os.path.join(ROOT, "paper_2410_17375_amd", "csrc")


def test_choice_of_a_products_form(tmp_path):
    exe = str(tmp_path / "q8_plan_test")
    src = os.path.join(ROOT, "tests", "cpu", "q8_plan_test.cpp")
    r = subprocess.run(["g++", "-std=c++17", "-O2", src, "-o", exe], capture_output=True, text=True)
    assert r.returncode == 0, r.stderr
    r = subprocess.run([exe], capture_output=True, text=True, timeout=120)
    assert r.returncode == 0, r.stdout


def test_room_for_attentions_sums(tmp_path):
    exe = str(tmp_path / "q8_tiles_test")
    src = os.path.join(ROOT, "tests", "cpu", "q8_tiles_test.cpp")
    r = subprocess.run(["g++", "-std=c++17", "-O2", src, "-o", exe], capture_output=True, text=True)
    assert r.returncode == 0, r.stderr
    r = subprocess.run([exe], capture_output=True, text=True, timeout=120)
    assert r.returncode == 0, r.stdout


@pytest.mark.parametrize("source", ["amusd_q8.hip", "amusd_q8_gemm.hip", "amusd_q8_attention.hip"])
def test_kernels_keep_to(tmp_path, source):
    kernels = _compile(os.path.join(CSRC, source), tmp_path / "q8.s")
    assert kernels
    for name, body in kernels.items():
        assert not _ends_with_load_in_flight(body), name
        assert not any(line.split()[0] in ("v_pk_add_f32", "v_pk_mul_f32", "v_pk_fma_f32") for line in body), name
        # no array in memory; attention of many rows with heads of 64 lays two registers aside for a chunk
        assert sum(line.startswith("scratch_") for line in body) <= (4 if "k_q8_att_wholeILi64" in name else 0), name
