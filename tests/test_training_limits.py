"""CPU-side checks of the limits that the operators around the encoder's blocks state."""
import os
import subprocess

from test_training_host import lib  # noqa: F401

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


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


SHAPES = r'''
#include <stdio.h>
#include <stdlib.h>
#include "loss_plan.h"
using namespace sieve::loss;
// rows vocab n dtype -> the tiles of the forward pass, of g and of the products, the planes of
// weighed h, the pieces of the vocabulary in the backward pass
int main(int argc, char** argv) {
  const int64_t rows = atoll(argv[1]), vocab = atoll(argv[2]);
  const int n = atoi(argv[3]), dtype = atoi(argv[4]);
  const char* names[] = {"small", "deep", "large", "triple"};
  const Layout f = layout_of(rows, vocab, n, dtype, false);
  const Layout b = layout_of(rows, vocab, n, dtype, true);
  const bool as_is = dtype != 0 && n % 8 == 0;
  const Size forward = size_of(std::min(as_is ? int64_t(1) << 20 : f.piece, vocab),
                               std::min(rows, kRowChunk), f.k, f.planes);
  const Size g = size_of(std::min(b.piece, vocab), b.chunk, b.k, b.planes);
  printf("%s %s %s %d %lld\n", names[forward], names[g], names[b.spread.size], b.weighed_planes,
         (long long)((vocab + b.piece - 1) / b.piece));
}
'''


def test_loss_shapes_are_what_the_gpu_tests_ask_for(tmp_path):
    """The sizes of tests/test_gpu_loss_shapes.py take the shapes that they are there for."""
    from test_gpu_loss_shapes import SHAPES as sizes
    src, exe = tmp_path / "shapes.cpp", tmp_path / "shapes"
    src.write_text(SHAPES)
    subprocess.run(["g++", "-std=c++17", "-O2", "-Wall", "-Werror", "-I",
                    os.path.join(ROOT, "paper_2608_03199_amd", "csrc"), "-I",
                    os.path.join(ROOT, "include"), str(src), "-o", str(exe)], check=True)
    codes = {"f32": 0, "f16": 1, "bf16": 2}
    for size in sizes:
        for dtype in size[3]:
            out = subprocess.run([str(exe), *map(str, size[:3]), str(codes[dtype])],
                                 capture_output=True, text=True, check=True).stdout.split()
            assert out == [str(x) for x in size[4:]], (size, out)
