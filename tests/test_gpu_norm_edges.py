"""Layer norm at the edges of what it takes.  Tolerances as in test_gpu_layer_norm."""

import numpy as np
import pytest

from tests.test_gpu_layer_norm import TableCase, check_backward, table_call, tables  # noqa: F401

pytestmark = pytest.mark.gpu


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
