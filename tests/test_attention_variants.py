"""Which variant of differential attention the shapes of attention_cases take, so that a changed rule cannot leave a kernel
without its test; and the workspaces of random shapes: big enough, apart.  The host code under the address and
undefined-behaviour sanitizers, its launches replaced (tests/sanitize/attention_driver.cpp); no GPU."""
import os
import random
import shutil
import subprocess

import pytest

import attention_cases as cases

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
pytestmark = pytest.mark.skipif(shutil.which("g++") is None or not os.path.isdir("/opt/rocm/include"),
                                reason="needs g++ and the ROCm headers")


@pytest.fixture(scope="module")
def ask(tmp_path_factory):
    exe = tmp_path_factory.mktemp("driver") / "attention_driver"
    subprocess.run(["g++", "-std=c++17", "-O1", "-g", "-fsanitize=address,undefined", "-fno-sanitize-recover=all",
                    "-D__HIP_PLATFORM_AMD__", "-I/opt/rocm/include", f"-I{ROOT}/include",
                    os.path.join(ROOT, "tests", "sanitize", "attention_driver.cpp"),
                    os.path.join(ROOT, "paper_2607_12505_amd", "csrc", "nmspmm_attention.cpp"), "-o", str(exe)],
                   check=True, capture_output=True, timeout=300)

    def run(what, shapes):
        """[[numbers of a line]] of (shape, lengths given)."""
        text = "".join(f"{what} {' '.join(map(str, s))} {int(given)}\n" for s, given in shapes)
        done = subprocess.run([str(exe)], input=text, capture_output=True, text=True, timeout=300)
        assert done.returncode == 0, (done.stdout + done.stderr)[-2000:]
        return [[int(x) for x in line.split()] for line in done.stdout.splitlines()]
    return run


def width_class(d, dv):
    return 0 if d <= 32 and dv <= 64 else 1 if d <= 64 and dv <= 128 else 2 if dv <= 128 else 3


def test_many_rows(ask):
    got = ask("forward", [(s, False) for s in cases.MANY_ROWS + cases.MANY_ROWS_WIDE])
    assert got == [[1, 1]] * len(got)
    got = ask("forward", [(s, True) for s in (*cases.PADDED, *cases.PACKED, cases.STEP)])
    assert got == [[1, 1]] * len(got)
    assert {width_class(*s[5:]) for s in cases.MANY_ROWS} == {0, 1}
    assert {width_class(*s[5:]) for s in cases.MANY_ROWS_WIDE} == {2, 3}


def test_parts_of_the_keys(ask):
    got = ask("forward", [(s, given) for s, given, _ in cases.PARTS])
    assert got == [[0, n] for _, _, n in cases.PARTS]
    assert {width_class(*s[5:]) for s, _, _ in cases.PARTS} == {0, 1, 2, 3}


def test_parts_of_the_rows(ask):
    assert ask("backward", [(s, False) for s, _ in cases.ROW_PARTS]) == [[n] for _, n in cases.ROW_PARTS]
    assert {width_class(*s[5:]) for s, _ in cases.ROW_PARTS} == {0, 1, 2, 3}


def test_workspaces_of_random_shapes(ask):
    r = random.Random(5)
    shapes = []
    for _ in range(4000):
        hk = r.choice((1, 1, 2, 3, 8))
        shapes.append(((r.choice((1, 2, 5, 64, 300)), int(2 ** r.uniform(0, 14)), int(2 ** r.uniform(0, 17)), hk * r.choice((1, 2, 5)),
                        hk, r.randint(1, 128), r.randint(1, 256)), r.random() < 0.3))
    assert len(ask("forward", shapes)) == len(ask("backward", shapes)) == len(shapes)
