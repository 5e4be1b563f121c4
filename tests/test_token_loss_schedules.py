"""CPU: the functions that cut a contraction into parts, compiled for the host from the kernels' own header."""
import os
import subprocess

import pytest

from paper_2605_26646_b200 import build

PROGRAM = r"""
#include <cstdio>
#include <cstdlib>
#include <cstring>
#include "internal.h"
using namespace unity;

// the choice that a warp makes with one candidate per lane
static SplitShape choose(const SplitParams& p, int m_tiles) {
    SplitShape s, best = {0, 0};
    long long least = 0x7fffffffffffffffll;
    for (int c = 1; c <= kMaxKSplits; ++c) {
        if (!split_allowed(p, m_tiles, c)) continue;
        const long long cost = split_candidate(p, m_tiles, c, s);
        if (cost < least) { least = cost; best = s; }
    }
    return best;
}

int main(int argc, char** argv) {
    if (argc > 1 && !strcmp(argv[1], "empty")) {
        // a model without a token, and one whose last block does not exist (its rows end with a full one)
        for (int k_iters : {0, -1, -3}) {
            const SplitParams p{kMaxKSplits, 4, k_iters, 74, kTileM, kSplitWavesDw};
            const SplitShape s = choose(p, 1);
            printf("%d %d\n", s.splits, s.per_split);
            if (s.splits != 1 || s.per_split != 1) return 1;
        }
        return 0;
    }
    if (argc > 1 && !strcmp(argv[1], "parts")) {
        // dW of a full block whose last rows hold no token (rows are padded to 256): every part that is used has a slab, and
        // the parts that are used hold all slabs.  Also for plans that this choice does not make: every allowed count of parts.
        long long cases = 0;
        for (int rows = kTileM; rows <= 18432; rows += kTileM)
            for (int tiles = 1; tiles <= 74; ++tiles) {
                const SplitParams p{kMaxKSplits, tiles, rows / kTileK, 74, kTileM, kSplitWavesDw};
                const SplitShape chosen = choose(p, 1);
                for (int c = 0; c <= kMaxKSplits; ++c) {
                    SplitShape s = chosen;
                    if (c > 0 && !split_allowed(p, 1, c)) continue;
                    if (c > 0) split_candidate(p, 1, c, s);
                    for (int valid = rows - kTileM + 1; valid <= rows; valid += 5) {
                        const int slabs = (valid + kTileK - 1) / kTileK, n = parts_in_use(s.splits, s.per_split, slabs);
                        ++cases;
                        if (n < 1 || (n - 1) * s.per_split >= slabs || n * s.per_split < slabs) {
                            printf("rows %d valid %d tiles %d: %d of %d parts of %d\n", rows, valid, tiles, n, s.splits, s.per_split);
                            return 1;
                        }
                    }
                }
            }
        printf("%lld\n", cases);
        return 0;
    }
    return 2;
}
"""


@pytest.fixture(scope="module")
def program(tmp_path_factory):
    where = tmp_path_factory.mktemp("schedules")
    source = where / "schedules.cu"
    source.write_text(PROGRAM)
    out = str(where / "schedules")
    subprocess.run([build._nvcc(), "-std=c++17", "-O1", "-gencode", "arch=compute_100a,code=sm_100a", "-I", build.CSRC,
                    "-I", os.path.join(build.PKG_DIR, "..", "include"), "-o", out, str(source)], check=True, capture_output=True)
    return out


def test_contractions_without_rows_have_one_part(program):
    """No division by a part's length of zero."""
    run = subprocess.run([program, "empty"], capture_output=True, text=True)
    assert run.returncode == 0, (run.returncode, run.stdout)


def test_no_part_of_a_contraction_over_rows_is_empty(program):
    run = subprocess.run([program, "parts"], capture_output=True, text=True)
    assert run.returncode == 0, run.stdout
    assert int(run.stdout) > 1_000_000
