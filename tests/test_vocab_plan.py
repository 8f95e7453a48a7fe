"""How calls of the vocabulary's loss are laid out (csrc/dfx_vocab_plan.h, compiled for the host alone), looked at on the CPU."""
import os
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module")
def exe(tmp_path_factory):
    out = str(tmp_path_factory.mktemp("plan") / "vocab_plan_check")
    subprocess.run(["g++", "-std=c++17", "-O2", "-Wall", "-Werror", os.path.join(ROOT, "tests", "rules", "vocab_plan_check.cpp"), "-o", out], check=True, timeout=120)
    return out


def test_what_a_call_touches_lies_in_its_place(exe):
    """Nothing of a call lies on anything else of it: of few 32-bit rows and a vocabulary above 78592 the third plane of dz lay on the kept logits."""
    out = subprocess.run([exe], capture_output=True, text=True, timeout=300)
    assert out.returncode == 0 and out.stdout.strip() == "ok", out.stdout
