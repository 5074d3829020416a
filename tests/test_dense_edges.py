"""The host side of the dense operators where its rules meet: what test_dense_refusals leaves out."""

import ctypes as C
import os
import shutil
import subprocess

import pytest

from tests.test_dense_refusals import CSRC, HERE, INVAL, OK, ROOT, TABLE, at, backward, ctx, lib  # noqa: F401

ROW = 100 * 4
# the word of *status in every other piece of memory of a backward pass on table rows
PLACES = {"dy_first": at(1), "dy_second": at(1) + 4, "dy_last": at(1) + 10 * ROW - 4, "mean": at(2) + 8, "rstd": at(3), "weight": at(4) + 4, "dx": at(6) + ROW,
          "dweight": at(7) + 4, "dbias": at(8), "workspace": at(9) + 64, "ids": at(10) + 8}


@pytest.mark.parametrize("name", PLACES)
def test_backward_refuses_a_status_word_in_other_memory(lib, ctx, name):  # noqa: F811
    before = lib.stub_launches()
    assert lib.legend_layer_norm_backward(ctx, backward(**dict(TABLE, table=0, status=PLACES[name]))) == INVAL
    assert lib.legend_last_error() and lib.stub_launches() == before


def test_backward_takes_a_status_word_beside_its_memory(lib, ctx):  # noqa: F811
    for place in (at(1) - 4, at(1) + 10 * ROW, at(2) + 40, at(10) + 80, at(6) - 4):
        assert lib.legend_layer_norm_backward(ctx, backward(**dict(TABLE, table=0, status=place))) == OK, lib.legend_last_error()


@pytest.mark.skipif(shutil.which("g++") is None, reason="needs g++")
def test_a_step_of_any_size_that_is_accepted_fits_one_launch(tmp_path):
    """A launch holds fewer than 2^32 threads; an optimiser has up to 2^28 units (2^24 tensors of one element have as many units)."""
    native, so = os.path.join(HERE, "native"), tmp_path / "grid.so"
    subprocess.run(["g++", "-std=c++17", "-Wall", "-shared", "-fPIC", "-I", os.path.join(native, "dense"), "-I", CSRC, "-I", os.path.join(ROOT, "include"),
                    os.path.join(native, "dense_grid_stub.cpp"), "-o", str(so)], check=True, timeout=120)
    grid = C.CDLL(str(so)).stub_adam_grid
    grid.restype, grid.argtypes = C.c_int64, [C.c_int64, C.c_int]
    for units in (0, 1, 1_279, 1_280, 1_281, 1 << 20, (1 << 24) - 1, 1 << 24, (1 << 24) + 1, 1 << 28):
        for large in (0, 1):
            assert 1 <= grid(units, large) <= max(units, 1) and grid(units, large) * 256 < 1 << 32
    assert [grid(u, 1) for u in (1 << 20, (1 << 24) - 1, 1 << 24, 1 << 28)] == [1 << 20, (1 << 24) - 1, (1 << 24) - 1, (1 << 24) - 1]
    assert [grid(u, 0) for u in (1_279, 1_280, 1 << 20)] == [1_279, 1_280, 1_280]
