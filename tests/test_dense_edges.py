"""The host side of the dense operators where its rules meet: what test_dense_refusals leaves out."""

import pytest

from tests.test_dense_refusals import INVAL, OK, TABLE, at, backward, ctx, forward, lib  # noqa: F401

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
