"""The unit in which ec_sample sums weights, by the vocabulary: what a thread's column can hold at most, whatever the launch rule."""
import ctypes
import pathlib
import re
import subprocess

import pytest

SRC = pathlib.Path(__file__).parent.parent / "paper_2603_18489_b200" / "csrc" / "ec_sample.cu"
THREADS, SEGMENT_TOKENS = 512, 1016


@pytest.fixture(scope="module")
def unit_bits(tmp_path_factory):
    """unit_bits_of of the source itself, compiled for the host."""
    src = SRC.read_text()
    names = re.findall(r"^constexpr int k(?:Threads|WeightBits|MaxUnitBits|Segment)\b[^;]*;", src, re.M)
    body = re.search(r"__host__ __device__ (constexpr int unit_bits_of\(int vocab\) \{.*?\n\})", src, re.S).group(1)
    tmp = tmp_path_factory.mktemp("units")
    (tmp / "u.cpp").write_text("\n".join(names) + "\n" + body + '\nextern "C" int bits(int v) { return unit_bits_of(v); }\n'
                               'extern "C" int tokens() { return kSegment / kThreads; }\nextern "C" int weight() { return kWeightBits; }\n')
    subprocess.run(["g++", "-std=c++17", "-shared", "-fPIC", "-o", str(tmp / "u.so"), str(tmp / "u.cpp")], check=True)
    return ctypes.CDLL(str(tmp / "u.so"))


def test_a_row_of_largest_weights_fits_a_thread_s_column(unit_bits):
    """A column: the sum below 2^53, the count above it.  A thread takes eight tokens of every 4096 of its CTA's segment; with one CTA
    the whole row is a segment, up to the most that a CTA takes.  All of weight 1 they have to stay BELOW 2^53: 2^53 itself is
    one of the count."""
    assert unit_bits.tokens() == SEGMENT_TOKENS and unit_bits.weight() == 53
    bad = [v for v in sorted({1, 7, *(m * 4096 + d for m in range(1, 257) for d in (-1, 0, 1))}) if 1 <= v <= 1 << 20
           and min((v + 4095) // 4096 * 8, SEGMENT_TOKENS) << unit_bits.bits(v) >= 1 << 53]
    assert not bad


def test_units_as_documented(unit_bits):
    assert [unit_bits.bits(v) for v in (1, 28672, 28673, 126464, 1 << 20)] == [47, 47, 46, 45, 43]
