"""Which kernels' shapes the tests of log probabilities from hidden states reach,
by the library's own rules, compiled for the host (CPU)."""
import os
import subprocess

import pytest

from tests import linear_shapes as S
from tests.test_gpu_linear import SIZES as SMALL

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module")
def layouts(tmp_path_factory):
    program = str(tmp_path_factory.mktemp("layout") / "layout")
    subprocess.run(["g++", "-std=c++17", "-D__HIP_PLATFORM_AMD__", "-I/opt/rocm/include", "-I" + os.path.join(ROOT, "include"),
                    "-I" + os.path.join(ROOT, "paper_2401_04829_amd", "csrc"),
                    os.path.join(ROOT, "tests", "linear_layout.cpp"), "-o", program], check=True)

    def layouts_of(sizes):
        lines = "\n".join(" ".join(map(str, s)) for s in sizes)
        out = subprocess.run([program], input=lines, text=True, capture_output=True, check=True).stdout
        return [set(line.split()) for line in out.strip().split("\n")]
    return layouts_of


def _split(words):
    """Words of one shape, and of two segments by the second's."""
    return ({w for w in words if "+" not in w} | {w.split("+")[0] for w in words}, {w for w in words if "+" in w})


@pytest.mark.parametrize("element", [2, 4])
def test_sizes_reach_every_shape(layouts, element):
    """Aligned operands reach every shape that the rules can choose, and a second
    segment of each product; those that go through registers theirs."""
    sizes = {True: [], False: []}
    for e, rows, vocab, width in S.SIZES:
        if e == element:
            sizes[S.direct(e, width)].append((e, rows, vocab, width, int(S.direct(e, width))))
    for rows, vocab, width in SMALL:                          # there all of them at odd addresses too
        sizes[False].append((element, rows, vocab, width, 0))
        if S.direct(element, width):
            sizes[True].append((element, rows, vocab, width, 1))
    sums = ["", "s"] if element == 2 else [""]                # dh's second parts as rows, or as a second sum
    want = {True: {f"{k}{s}" for k in ("logits", "d") for s in (0, 1, 2, 3, 5)} | {f"dw{s}" for s in range(4)}
            | {f"dwparts{s}" for s in range(4)} | {f"dh{s}{t}" for s in (0, 1, 3, 4) for t in sums},
            False: {f"{k}{s}" for k in ("logits", "d") for s in (1, 3, 5)} | {f"{k}{s}" for k in ("dw", "dwparts") for s in (1, 3)}
            | {f"dh{s}{t}" for s in (1, 3) for t in sums}}
    for kind in (True, False):
        got, two = _split(set().union(*layouts(sizes[kind])))
        assert want[kind] <= got, want[kind] - got
        assert got - want[kind] <= {"pieces"}
        assert (len({w[:w.index("0")] for w in two}) == 3 and len(two) >= 5) if kind else not two, two
    assert "pieces" in set().union(*layouts(sizes[True]))


def test_the_long_sum_is_one(layouts):
    words, = layouts([(*S.LONG_SUM, 1)])
    assert "dw3" in words and not any(w.startswith("dwparts") for w in words)
