"""Arguments of the classification head and of the log probabilities, without a GPU: what the binding has to refuse
because a kernel would read it wrongly or beyond its end, and what it must not refuse."""
import os
import subprocess

import pytest
import torch

import paper_1707_04585_amd as rv
from paper_1707_04585_amd.binding import rvn_head_desc, rvn_head_ptrs
from test_abi_host import BASE, fake, status_of
from test_operators_host import ALIAS, FAR, NULL, matrix

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
C, CLASSES = 8, 5
SHAPES = dict(gamma=(C,), beta=(C,), w=(CLASSES, C), b=(CLASSES,))


def head_arrays(**other):
    return {k: other.get(k, torch.zeros(SHAPES[k])) for k in SHAPES}


def head_calls(desc):
    """Calls of the head with the arrays given in each place that takes such a set; every other argument is in order."""
    x, dx, logits = fake(BASE, c=C), fake(BASE + 0x100000, c=C), matrix(BASE + 0x400000, 2, CLASSES)
    raw, far = rvn_head_ptrs(16, 16, 16, 16), (FAR, 1 << 20)
    return [lambda P: rv.revnet_head_fwd(desc, x, P, logits, far),
            lambda P: rv.revnet_head_bwd(desc, x, far, logits, P, dx, raw, 0, (FAR + (1 << 21), 1 << 20)),
            lambda P: rv.revnet_head_bwd(desc, x, far, logits, raw, dx, P, 0, (FAR + (1 << 21), 1 << 20))]


@pytest.mark.parametrize("bad", [
    dict(gamma=torch.zeros(C, dtype=torch.float64)), dict(beta=torch.zeros(C, dtype=torch.int32)),
    dict(w=torch.zeros(CLASSES, C, dtype=torch.bfloat16)), dict(b=torch.zeros(CLASSES, dtype=torch.float16)),
    dict(w=torch.zeros(C, CLASSES).t()),
], ids=lambda b: next(iter(b)))
def test_head_arrays_of_another_type_or_with_gaps_are_refused_when_packed(bad):
    with pytest.raises(ValueError):
        rv.pack_head(head_arrays(**bad))


@pytest.mark.parametrize("packed", [False, True])
@pytest.mark.parametrize("desc", [rv.HeadDesc(C, CLASSES), rvn_head_desc(C, CLASSES, 1e-5)], ids=["HeadDesc", "rvn_head_desc"])
@pytest.mark.parametrize("bad", [
    dict(gamma=torch.zeros(C - 1)), dict(beta=torch.zeros(C + 1)), dict(w=torch.zeros(CLASSES - 1, C)), dict(w=torch.zeros(CLASSES, C - 1)),
    dict(w=torch.zeros(C, CLASSES)), dict(b=torch.zeros(1)),
], ids=lambda b: "%s%s" % next((k, list(v.shape)) for k, v in b.items()))
def test_head_arrays_of_another_size_are_refused(bad, desc, packed):
    arrays = head_arrays(**bad)
    if packed:
        arrays = rv.pack_head(arrays)
    for call in head_calls(desc):
        with pytest.raises(ValueError):
            call(arrays)


def test_head_arrays_that_fit_reach_the_library():
    """Arrays in order, packed or not, and raw pointers get past the binding: what is refused next is refused by the library."""
    desc, x, far = rv.HeadDesc(C, CLASSES), fake(BASE, c=C), (FAR, 1 << 20)
    wide = {k: v.view(1, -1, 1, 1) if v.dim() == 1 else v.view(CLASSES, C, 1, 1) for k, v in head_arrays().items()}
    for P in (head_arrays(), rv.pack_head(head_arrays()), wide, rv.pack_head(dict(gamma=16, beta=16, w=16, b=16)), rvn_head_ptrs(16, 16, 16, 16)):
        assert status_of(rv.revnet_head_fwd, desc, x, P, None, far)[0] == NULL
    missing = rv.pack_head(dict(head_arrays(), b=None))
    assert status_of(rv.revnet_head_fwd, desc, x, missing, matrix(BASE + 0x400000, 2, CLASSES), far)[0] == NULL


def test_overlap_of_matrices_is_exact_where_their_rows_are_equally_far_apart(tmp_path):
    """Every small pair against the bytes themselves; rows of different pitch may be called overlapping, never the reverse."""
    src = tmp_path / "overlap.cpp"
    src.write_text("""
#include <vector>
#include "matrix_overlap.h"
using rvn::RowBlock;
static bool shares(const RowBlock &a, const RowBlock &b) {
    std::vector<char> taken(4096, 0);
    for (int64_t i = 0; i < a.rows; ++i)
        for (int64_t x = 0; x < a.row; ++x) taken[a.at + i * a.pitch + x] = 1;
    for (int64_t i = 0; i < b.rows; ++i)
        for (int64_t x = 0; x < b.row; ++x)
            if (taken[b.at + i * b.pitch + x]) return true;
    return false;
}
int main() {
    for (int64_t pa = 1; pa <= 6; ++pa)
        for (int64_t pb = 1; pb <= 6; ++pb)
            for (int64_t ra = 1; ra <= pa; ++ra)
                for (int64_t rb = 1; rb <= pb; ++rb)
                    for (int64_t na = 1; na <= 4; ++na)
                        for (int64_t nb = 1; nb <= 4; ++nb)
                            for (int64_t off = -30; off <= 30; ++off) {
                                const RowBlock a{1000, ra, pa, na}, b{1000 + off, rb, pb, nb};
                                const bool got = rvn::row_blocks_overlap(a, b), want = shares(a, b);
                                if (want && !got) return 1;
                                if (got && !want && (pa == pb || na == 1 || nb == 1)) return 2;
                            }
    // far apart in one huge matrix: nothing is counted row by row, and nothing passes 64 bits
    const int64_t rows = 0x7fffffffLL, pitch = 1LL << 31;
    if (rvn::row_blocks_overlap({0, 100, pitch, rows}, {100, pitch - 100, pitch, rows})) return 3;
    if (!rvn::row_blocks_overlap({0, 101, pitch, rows}, {100, pitch - 100, pitch, rows})) return 4;
    return 0;
}
""")
    exe = tmp_path / "overlap"
    subprocess.run(["g++", "-std=c++17", "-O1", "-I", os.path.join(ROOT, "paper_1707_04585_amd", "csrc"), str(src), "-o", str(exe)], check=True)
    assert subprocess.run([str(exe)]).returncode == 0


def test_gradient_over_part_of_the_logits_is_refused():
    call = lambda l, g: status_of(rv.revnet_logprob_bwd, l, 16, 16, 16, None, None, 1.0, g)[0]  # noqa: E731
    l = matrix(BASE, 3, 7, ld=14)
    assert call(l, matrix(BASE + 4 * 6, 3, 7, ld=14)) == ALIAS          # the block begins in the other's last column
    assert call(l, matrix(BASE + 4 * 8, 3, 7, ld=14)) == ALIAS          # it ends in the next row's first
    assert call(l, matrix(BASE + 4 * 7, 3, 7, ld=13)) == ALIAS          # rows of another pitch
    assert call(matrix(BASE, 1, 7), matrix(BASE + 24, 1, 7)) == ALIAS
