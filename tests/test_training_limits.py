"""CPU-side checks of the limits that the operators around the encoder's blocks state."""
from test_training_host import lib  # noqa: F401


def test_loss_workspace_of_many_rows(lib):  # noqa: F811
    """g takes 2^27 values at most, whatever the rows: the rest is of the size of the inputs and
    their gradients (h packed, h weighed, in two planes at least, sums of dh in fp32, two numbers a
    row; and 16 sums of a piece of dtable's 256 rows)."""
    for rows in ((1 << 19) + 256, 1 << 20, 1 << 24):
        for dtype, planes in ((0, 3), (1, 1), (2, 1)):
            for n in (64, 61):
                size = lib.sieve_loss_workspace(rows, 50, n, dtype, 1)
                inputs = rows * (64 * (2 * planes + 2 * max(planes, 2) + 4) + 8)
                assert 0 < size < inputs + (1 << 28) + (1 << 21), (rows, dtype)


def test_loss_workspace_holds_no_sums_that_are_not_needed(lib):  # noqa: F811
    """Where a product writes its gradient itself: h, the table and h weighed, each in 16 bits, g,
    and two numbers a row."""
    rows, n = 2048, 768
    size = lib.sieve_loss_workspace(rows, rows, n, 1, 1)
    assert 0 < size <= 3 * 2 * rows * n + 2 * rows * rows + 8 * rows + (1 << 13)
    # dh's sums in three splits, none of dtable's
    rows, vocab = 8192, 32768
    size = lib.sieve_loss_workspace(rows, vocab, n, 2, 1)
    assert 0 < size <= 2 * (2 * rows + vocab // 2) * n + (1 << 28) + 3 * 4 * rows * n + 8 * rows + \
        (1 << 13)
