"""Index arithmetic of rows seen as vectors (``RowSpan``), run on the CPU: the vectors of a row cover its columns once, whole vectors
lie within the row, and the aligned loads around a vector of a shared row (the gain) stay within that row."""
import subprocess
from pathlib import Path

import pytest

from paper_1708_08917_b200.build import CSRC, FLAGS, NVCC

PROGRAM = r"""
#include <cstdio>

#include "circ_rows.cuh"

template <int VEC, bool ALIGNED>
static int check(long row, int dim, long stride) {
    const circ::RowSpan<VEC, ALIGNED> span(row, dim, stride);
    int next = 0, bad = 0;
    for (int v = 0; span.any(v); ++v) {
        bad += v >= circ::RowSpan<VEC, ALIGNED>::most(dim);
        bad += (long)span.at(v) - span.col(v) != row * stride || span.at(v) % VEC != 0;
        const int lo = span.lo(v), hi = span.hi(v);
        bad += lo < 0 || hi > VEC || lo >= hi || span.col(v) + lo != next;
        next = span.col(v) + hi;
        if (span.whole(v)) bad += lo != 0 || hi != VEC;
        if (span.turns(v)) {
            const int first = span.col(v) - (span.col(v) & 3);
            bad += first < 0 || first + VEC + 4 - 1 >= dim;        // the last float that the loads touch
        }
    }
    bad += next != dim;
    if (bad) printf("VEC %d aligned %d row %ld dim %d stride %ld: %d faults\n", VEC, ALIGNED, row, dim, stride, bad);
    return bad;
}

int main() {
    int bad = 0;
    for (int dim = 1; dim <= 4100; ++dim)
        for (long row = 0; row < 9; ++row) {
            bad += check<4, false>(row, dim, dim) + check<8, false>(row, dim, dim) + check<4, false>(row, dim, dim + 3) + check<8, false>(row, dim, dim + 5);
            if (dim % 8 == 0) bad += check<4, true>(row, dim, dim) + check<8, true>(row, dim, dim);
            if (bad) return 1;
        }
    for (long row : {0L, 131071L, 2147483646L})
        for (int dim : {16777215, 16777213}) bad += check<8, false>(row, dim, dim);        // offsets beyond 32 bits
    return bad != 0;
}
"""


def test_vectors_of_a_row_stay_within_it(tmp_path: Path):
    if not Path(NVCC).exists():
        pytest.skip("no compiler")
    (tmp_path / "spans.cu").write_text(PROGRAM)
    subprocess.run([NVCC, *FLAGS[:2], "-O1", "-std=c++17", "--expt-relaxed-constexpr", "-I", str(CSRC), "-I", str(CSRC.parent.parent / "include"),
                    "-o", str(tmp_path / "spans"), str(tmp_path / "spans.cu")], check=True, capture_output=True)
    out = subprocess.run([str(tmp_path / "spans")], capture_output=True, text=True, timeout=300)
    assert out.returncode == 0, out.stdout
