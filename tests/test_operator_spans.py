"""Which buffers of a training operator's call count as overlapping (no GPU: what is accepted here ends at the missing
workspace, which is looked at next)."""
import pytest

from tests.test_operators import BF16, EINVAL, EOVERLAP, F32, fp8, linear, matrix, place

ROWS, K, N, LD = 300, 256, 50, 600  # x and y in one matrix of 600 binary32 columns


def at(column, **kw):
    return matrix(0, ROWS, N, ld=LD, at=place(0) + 4 * column, **kw)


@pytest.mark.parametrize("first", [0, 7, 200])
def test_column_slices_of_one_matrix_do_not_overlap(first):
    x, w = matrix(0, ROWS, K, ld=LD, at=place(0) + 4 * first), fp8(1, N, K)
    behind = first + K
    for column in (behind, behind + 1, LD - N + min(first, 7)):
        if column + N <= LD + first:
            assert linear(x, w, at(column)) == EINVAL, column           # to the next row's first column of x
    for column in (first, behind - 1, first + 100, LD + first - N + 1, LD + first - 1):
        assert linear(x, w, at(column)) == EOVERLAP, column
    if first >= N:
        assert linear(x, w, at(0)) == linear(x, w, at(first - N)) == EINVAL
        assert linear(x, w, at(first - N + 1)) == EOVERLAP
    # bytes count, not elements; and rows that are not as far apart meet somewhere
    half = place(0) + 4 * behind
    assert linear(x, w, matrix(0, ROWS, N, ld=2 * LD, at=half, dtype=BF16)) == EINVAL
    assert linear(x, w, matrix(0, ROWS, N, ld=2 * LD, at=half - 2, dtype=BF16)) == EOVERLAP
    for ld in (LD - 1, LD + 1, 2 * LD):
        assert linear(x, w, matrix(0, ROWS, N, ld=ld, at=place(0) + 4 * behind, dtype=F32)) == EOVERLAP


def test_one_row_among_others():
    """A weight of one row in the gap behind the rows of x, and reaching over its end."""
    x, y = matrix(0, ROWS, 128, ld=LD), matrix(3, ROWS, 1)
    gap = place(0) + 4 * 128
    def w(start):
        return fp8(1, 1, 128, at=start, scale=place(2))
    assert linear(x, w(gap), y) == EINVAL and linear(x, w(place(0)), y) == EINVAL  # (inputs may share memory)
    y = matrix(0, ROWS, 1, ld=LD, at=gap)
    assert linear(x, w(gap + 16), y) == EINVAL
    assert linear(x, w(gap - 16), y) == EOVERLAP                        # over the first element of y
