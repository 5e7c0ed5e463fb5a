"""Which kernel instance a product takes, from the library's own estimate
compiled for the host: the sizes of the instance tests reach every instance, so
that none ships untested after a change of the estimate."""
import os
import shutil
import subprocess

import pytest

from tests.mx4_cases import CASES, INSTANCES

CXX = shutil.which("g++") or shutil.which("c++")
pytestmark = pytest.mark.skipif(CXX is None, reason="needs a C++ compiler")


@pytest.fixture(scope="module")
def pick(tmp_path_factory):
    exe = str(tmp_path_factory.mktemp("pick") / "pick")
    main = os.path.join(os.path.dirname(os.path.abspath(__file__)), "mx4_pick_main.cpp")
    subprocess.run([CXX, "-O1", "-std=c++17", "-Wall", "-Werror", main, "-o", exe], check=True)

    def run(cases, cus=256):
        text = "".join("%d %d %d %d %d %d %d %d\n" % (n, m, max(g, 1), d_in, d_out, g > 0, gathered, cus)
                       for g, n, m, d_in, d_out, gathered in cases)
        out = subprocess.run([exe], input=text, text=True, capture_output=True, check=True).stdout.split("\n")
        return [(f, int(s), int(w)) for f, s, w in (x.split() for x in out if x)]
    return run


def test_every_case_takes_its_instance(pick):
    got = pick([case for _, case in CASES])
    wrong = [(case, key, p) for (key, case), p in zip(CASES, got) if p != key]
    assert not wrong, wrong


def test_every_instance_has_cases():
    shapes = {"split": 5, "line": 7, "tile": 3}
    assert set(INSTANCES) == {(f, s, w) for f, n in shapes.items() for s in range(n) for w in (0, 1)}
    for (form, shape, _), cases in INSTANCES.items():
        assert any(c[0] > 0 for c in cases)
        # 16 x 64 outputs with short rows: by expert only
        assert any(c[0] == 0 for c in cases) or (form, shape) == ("split", 2)


def test_general_rows_at_both_alignments():
    # scale rows that begin at dwords (whole 128 elements) and at any byte
    for (form, shape, whole), cases in INSTANCES.items():
        if form == "line" and not whole:
            assert {c[3] % 128 == 0 for c in cases} == {True, False}, (form, shape)


def test_a_form_for_the_smallest_and_largest_sizes(pick):
    most = 1 << 30
    cases = [(0, 1, 1, 32, 1, 0), (0, most, most, 131072, most, 0), (4096, 1, 1, 32, 1, 1),
             (4096, most, most, 131072, most, 1), (4096, 1, 1, 131072, most, 1), (1, most, most, 512, 1, 0),
             (0, 1, 1, 480, most, 0), (0, 1, 1, 512, 1, 0)]
    for cus in (8, 256, 304):
        for (g, n, m, d_in, *_, gathered), (form, _, whole) in zip(cases, pick(cases, cus)):
            assert (form == "split") == (d_in < 512)
            assert whole == (d_in % {"split": 128, "line": 256, "tile": 512}[form] == 0)
            # large tiles address gathered rows by 32 bits
            assert not (form == "tile" and gathered and n * (d_in // 2) >= 2 ** 32)
