"""Layer norm where its numbers run out: rows whose squares leave fp32, and table rows that a call may not read beside a weight
that is not finite.  Tolerances as in test_gpu_layer_norm: the squares are then summed in units of a power of two, which rounds nothing."""

import numpy as np
import pytest

from tests.test_gpu_layer_norm import TableCase, Case, backward, check_backward, check_forward, ctx, forward, table_call, tables  # noqa: F401

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("yt", [0, 1], ids=["f", "b"])
@pytest.mark.parametrize("dim", [2, 3, 8, 100, 777, 2_000, 4_096, 5_000, 16_384, 20_000, 20_001, 1 << 20], ids=str)
def test_rows_whose_squares_leave_fp32(ctx, dim, yt):  # noqa: F811
    """Rows up to the documented 1e37 / dim, between rows of ordinary numbers, which keep their bits."""
    rng = np.random.default_rng(dim)
    ordinary = rng.standard_normal((7, dim))
    x = ordinary.copy()
    top = 1e37 / dim
    for r, size in ((1, 0.15 * top), (2, 1e19 if 1e20 < top else 0.01 * top), (4, 3e17)):      # (normal numbers stay within 6 of these)
        x[r] *= size
    x[5] = 0.9 * top                                        # but for its first number
    x[5, 0] = -0.9 * top
    clean = Case(7, dim, 0, yt, x=ordinary)
    clean_y, clean_mean, clean_rstd = (t.clone() for t in forward(ctx, clean))
    case = Case(7, dim, 0, yt, x=x)
    y, mean, rstd = forward(ctx, case)
    check_forward(case, y, mean, rstd)
    for r in (0, 3, 6):
        assert bool((y[r] == clean_y[r]).all()) and mean[r] == clean_mean[r] and rstd[r] == clean_rstd[r]
    check_backward(case, backward(ctx, case, mean, rstd), case.x64, case.dy64, mean, rstd)


@pytest.mark.parametrize("value", [float("inf"), float("nan")], ids=["inf", "nan"])
@pytest.mark.parametrize("rows", [60, 3_000], ids=str)
def test_rows_that_may_not_be_read_are_zeros_whatever_the_weight(tables, rows, value):  # noqa: F811
    import torch
    from paper_2505_09258_amd import binding as L
    c, node, _ = tables
    V, d = node.shape
    part = -(-V // 5)
    rng = np.random.default_rng(rows)
    ids = rng.integers(0, part, rows)
    wrong = rng.random(rows) < 0.3
    ids[wrong] = rng.choice([-1, V, 1 << 40, part, 3 * part + 1], int(wrong.sum()))       # out of range, or in partitions 1 and 3, which are not resident
    case = TableCase(node[np.where(wrong, 0, ids)])
    case.w[17] = value
    dids, bad = torch.from_numpy(ids).cuda(), torch.from_numpy(wrong).cuda()
    y, dx = case.blank(0), case.blank(0)
    mean, rstd = (torch.full((rows,), -77.0, device="cuda") for _ in range(2))
    dw, db = (torch.full((d,), -77.0, device="cuda") for _ in range(2))
    size = L.legend_layer_norm_workspace(rows, d)
    space = torch.full((size // 4,), float("nan"), device="cuda")
    assert table_call(c, case, L.TABLE_NODE_EMB, dids, L.legend_layer_norm_forward, mean, rstd, y=y[1].data_ptr()) == 3
    assert table_call(c, case, L.TABLE_NODE_EMB, dids, L.legend_layer_norm_backward, mean, rstd, dy=case.dy[1].data_ptr(), dx=dx[1].data_ptr(),
                      dweight=dw.data_ptr(), dbias=db.data_ptr(), workspace=space.data_ptr(), workspace_bytes=size) == 3
    for t in (y[1], dx[1], mean, rstd):
        assert not bool(t[bad].any())
    # the weight has no part in the sums over the rows that were read
    sub = TableCase(node[ids[~wrong]])
    check_backward(sub, {"dweight": dw, "dbias": db}, sub.x64, case.dy64[~wrong], mean[~bad], rstd[~bad])
