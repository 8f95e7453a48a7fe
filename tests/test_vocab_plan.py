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


# Calls with gradients that take the wide tiles: (rows, dim, vocab, piece), and what they are to take with 32-bit and with 16-bit inputs.  logits: all by wide tiles, or ending in quarters
WIDE = [
    ((1290, 704, 9001, 0), dict(logits="all", steps=11, dx_wide=1, dw_wide=1, splits=2, pieces=1), dict(logits="all", steps=11, dx_wide=1, dw_wide=1, splits=2, pieces=1)),
    ((1290, 1000, 6001, 0), dict(logits="all", steps=16, dx_wide=1, dw_wide=1, splits=2, pieces=1), dict(logits="all", steps=16, dx_wide=1, dw_wide=1, splits=2, pieces=1)),
    ((1000, 520, 9001, 0), dict(logits="all", steps=9, dx_wide=1, dw_wide=1, splits=2, pieces=1), dict(logits="all", steps=9, dx_wide=0, dw_wide=1, splits=2, pieces=1)),
    ((700, 2050, 4001, 3584), dict(dx_wide=1, dw_wide=1, splits=2, pieces=2), dict(dx_wide=1, dw_wide=1, splits=2, pieces=2)),
    ((2570, 320, 6001, 0), dict(logits="part", steps=5, dx_wide=1, splits=2, pieces=1), dict(logits="part", steps=5, dx_wide=1, splits=2, pieces=1, keep=0)),
    ((2049, 200, 4101, 512), dict(logits="all", steps=4, dx_wide=1, pieces=9), dict(logits="all", steps=4, dx_wide=1, pieces=9)),
]


@pytest.mark.parametrize("kind", [0, 1, 2])
@pytest.mark.parametrize("case", WIDE, ids=lambda c: "x".join(map(str, c[0])))
def test_what_the_wide_cases_take(exe, case, kind):
    """The GPU tests of the wide tiles' products are of these: a change of the rules that leaves one to other products shows here."""
    (rows, dim, vocab, piece), want = case[0], case[2 if kind else 1]
    for aligned in (0, 1):
        got = dict((k, int(n)) for k, n in (f.split("=") for f in subprocess.run([exe] + [str(n) for n in (rows, dim, vocab, kind, piece, aligned)], capture_output=True, text=True, timeout=60).stdout.split()))
        assert got["few"] == 0
        for k, n in want.items():
            if k == "logits":
                assert got["wide"] >= vocab if n == "all" else 0 < got["wide"] < vocab
            elif k == "splits":
                assert got[k] >= n
            else:
                assert got[k] == n, (k, got)
