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
