"""CPU test of how contractions are cut into accumulators: the header that the product kernel's roles share, compiled for the host."""
import ctypes
import os
import random
import subprocess

import pytest

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2605_17862_b200", "csrc")
SOURCE = """
#include "accumulators.cuh"
extern "C" int accumulator_end(int done, int small, int blocks, int chunk) { return fopd::accumulator_end(done, small, blocks, chunk); }
extern "C" int long_chunk() { return fopd::kLongChunk; }
"""


@pytest.fixture(scope="module")
def cut(tmp_path_factory):
    at = tmp_path_factory.mktemp("accumulators")
    (at / "cut.cpp").write_text(SOURCE)
    subprocess.check_call(["g++", "-O1", "-std=c++17", "-shared", "-fPIC", "-I", CSRC, str(at / "cut.cpp"), "-o", str(at / "cut.so")])
    return ctypes.CDLL(str(at / "cut.so"))


# blocks of 64 of the largest contractions that the entry points take: 2^27 rows, 2^20 dimensions, 2^24 rows of a matrix
LONGEST = (2 ** 21, 2 ** 14, 2 ** 18)


def test_no_accumulator_is_longer_than_sixteen_thousand_terms(cut):
    rng = random.Random(1)
    sizes = [0, 1, 2, 7, 8, 9, 255, 256, 257, 511, 512, 513, *LONGEST] + [int(2 ** rng.uniform(0, 21)) for _ in range(40)]
    assert cut.long_chunk() == 256
    for k_blocks in sizes:
        for passes in (1, 2, 3):
            for chunk in (1, 2, 8, 16, 255, 256):
                small, blocks = (passes - 1) * k_blocks, passes * k_blocks
                if blocks > 300_000 and chunk < 16:
                    continue  # (millions of calls that say the same)
                done = 0
                while done < blocks:
                    end = cut.accumulator_end(done, small, blocks, chunk)
                    most = 256 if done < small else chunk
                    assert done < end <= min(done + most, small if done < small else blocks)
                    done = end
                assert cut.accumulator_end(0, 0, 0, chunk) == 0
