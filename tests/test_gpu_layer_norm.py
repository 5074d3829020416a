"""Layer norm, forward and backward, against the 64-bit oracle.

Tolerances count roundings.  E = 2^-24 is half a step of fp32.  A sum over a row is taken by at least 8 threads of a short row
(at most 256 numbers) and 64 of a longer one, each adding at most ceil(d / 64) + 16 terms in turn, and joined in a tree of at
most 10: its error is at most n E sum|terms| with n = ceil(d / 64) + 26.
  mean: the first sweep is off by k = n E mean|x|; the second takes that off up to n E (mean|c| + k); E |mean| for its rounding
  var: (n + 3) E relative and the square of the mean's error, rstd half of that + 3 E
  xh:   the mean's error times rstd (mean|c| rstd <= 1), and (n + 6) E |xh|:  (2 n + 6) E (|xh| + 1)
  (what k adds, n E k, times rstd, beside it)
  y:    that times |w|, two roundings, and half a step of y's type;  half adds 2^-25, half of its smallest number
  dx:   with u = dy w (1 rounding) and xh (2): sums n + 3 roundings each, then four operations, then the type's half step
  dw, db: at most rows / 64 + 32 additions in turn in fp32 (never more than the rows), the rest in 64 bits, 3 roundings a term."""

import numpy as np
import pytest

from oracle import dense as od

pytestmark = pytest.mark.gpu

E = 2.0**-24
HALF_STEP = {0: 2.0**-24, 1: 2.0**-8, 2: 2.0**-11}
TINY = {0: 2.0**-149, 1: 2.0**-134, 2: 2.0**-25}
EPS = 1e-5


def _torch_type(k):
    import torch
    return (torch.float32, torch.bfloat16, torch.float16)[k]


class Case:
    """Inputs on the GPU with guard elements around every output, and the same numbers in 64 bits."""

    def __init__(self, rows, dim, xt=0, yt=0, wt=0, weight=True, bias=True, pad=0, shift=0, seed=0, x=None, dy=None, broadcast=False):
        import torch
        self.rows, self.dim, self.xt, self.yt, self.wt, self.pad = rows, dim, xt, yt, wt, pad
        rng = np.random.default_rng(1000 * rows + dim + seed)
        if x is None:
            x = rng.standard_normal((rows, dim)) * np.exp(rng.standard_normal((rows, 1))) + rng.standard_normal((rows, 1))
        if dy is None:
            dy = rng.standard_normal((1 if broadcast else rows, dim))
        self.broadcast = broadcast
        self.x = self.put(x, xt, shift)
        self.dy = self.put(dy, yt, shift)
        self.w = torch.from_numpy(1 + 0.3 * rng.standard_normal(dim)).to(_torch_type(wt)).cuda() if weight else None
        self.b = torch.from_numpy(0.3 * rng.standard_normal(dim)).to(_torch_type(wt)).cuda() if bias else None

    def put(self, a, kind, shift):
        """[rows] rows at a stride of dim + pad, the first `shift` elements behind the start of an allocation."""
        import torch
        rows = a.shape[0]
        flat = torch.full((shift + rows * (self.dim + self.pad) + 8,), 7.0, dtype=_torch_type(kind), device="cuda")
        view = flat[shift:shift + rows * (self.dim + self.pad)].view(rows, self.dim + self.pad)
        view[:, :self.dim] = torch.from_numpy(np.ascontiguousarray(a)).to(_torch_type(kind)).cuda()
        return flat, view

    def blank(self, kind, shift=0):
        import torch
        flat = torch.full((shift + self.rows * (self.dim + self.pad) + 8,), -77.0, dtype=_torch_type(kind), device="cuda")
        return flat, flat[shift:shift + self.rows * (self.dim + self.pad)].view(self.rows, self.dim + self.pad)

    def numbers(self, a):
        return a.double().cpu().numpy()

    @property
    def x64(self):
        return self.numbers(self.x[1][:, :self.dim])

    @property
    def dy64(self):
        d = self.numbers(self.dy[1][:, :self.dim])
        return np.repeat(d, self.rows, 0) if self.broadcast else d

    @property
    def w64(self):
        return None if self.w is None else self.numbers(self.w)

    @property
    def b64(self):
        return None if self.b is None else self.numbers(self.b)

    def args(self, **more):
        from paper_2505_09258_amd import binding as L
        a = dict(rows=self.rows, dim=self.dim, x=self.x[1].data_ptr(), x_stride=self.dim + self.pad, x_type=self.xt, weight_type=self.wt, eps=EPS,
                 weight=None if self.w is None else self.w.data_ptr(), bias=None if self.b is None else self.b.data_ptr())
        a.update(more)
        return L.make_layer_norm(**a)


def guards_kept(case, out):
    flat, view = out
    rest = flat.clone()
    first = view.data_ptr() - flat.data_ptr()
    k = first // flat.element_size()
    rest[k:k + view.numel()].view_as(view)[:, :case.dim] = -77.0
    return bool((rest == -77.0).all())


@pytest.fixture(scope="module")
def ctx():
    from paper_2505_09258_amd import binding as L
    cfg = L.make_config(num_nodes=3, dim=4, batch_size=64, chunk_size=16, num_negs=16, init_std=0.1, seed=1)
    c = L.legend_init_partitions(cfg, None, None)
    yield c
    L.legend_destroy(c)


def chain(d):
    return -(-d // 64) + 26


def forward(ctx, case, in_place=False, statistics=True):
    import torch
    from paper_2505_09258_amd import binding as L
    y = case.x if in_place else case.blank(case.yt, 1 if case.pad else 0)
    mean, rstd = (torch.full((case.rows + 2,), -77.0, device="cuda") for _ in range(2))
    torch.cuda.synchronize()
    L.legend_layer_norm_forward(ctx, case.args(y=y[1].data_ptr(), y_stride=case.dim + case.pad, y_type=case.yt,
                                               **(dict(mean=mean[1:].data_ptr(), rstd=rstd[1:].data_ptr()) if statistics else {})))
    L.legend_sync(ctx)
    if statistics:
        assert all(float(t[0]) == float(t[-1]) == -77.0 for t in (mean, rstd))
    if not in_place:
        assert guards_kept(case, y)
    return y[1][:, :case.dim], mean[1:-1], rstd[1:-1]


def check_forward(case, y, mean, rstd, x64=None):
    x = case.x64 if x64 is None else x64
    want, wm, wr = od.layer_norm(x, case.w64, case.b64, EPS)
    n, c = chain(case.dim), np.abs(x - wm[:, None]).mean(1)
    k = n * E * n * E * np.abs(x).mean(1)
    xh = np.abs(x - wm[:, None]) * wr[:, None]
    w = 1.0 if case.w is None else np.abs(case.w64)
    tol = ((2 * n + 6) * E * (xh + 1) + (k * wr)[:, None]) * w + E * (xh * w + np.abs(want)) + HALF_STEP[case.yt] * np.abs(want) * (1 + 1e-3) + TINY[case.yt]
    err = np.abs(case.numbers(y) - want)
    assert np.all(err <= tol), float((err / tol).max())
    assert np.all(np.abs(case.numbers(mean) - wm) <= n * E * c + k + E * np.abs(wm) + 2.0**-149)
    assert np.all(np.abs(case.numbers(rstd) - wr) <= (n / 2 + 6) * E * wr + 0.5 * (k + n * E * c) ** 2 * wr**3)


def backward(ctx, case, mean, rstd, dx_in=None, sums=True, kind=0, accumulate=None, want_bias=True):
    import torch
    from paper_2505_09258_amd import binding as L
    rows, dim = case.rows, case.dim
    out = {}
    more = dict(mean=mean.data_ptr(), rstd=rstd.data_ptr(), dy=case.dy[1].data_ptr(), dy_stride=0 if case.broadcast else dim + case.pad, dy_type=case.yt)
    if dx_in != "none":
        dx = {"x": case.x, "dy": case.dy, None: case.blank(case.xt, 3 if case.pad else 0) if dx_in is None else None}[dx_in]
        out["dx"] = dx
        more.update(dx=dx[1].data_ptr(), dx_stride=dim + case.pad)
    if sums:
        out["dweight"], out["dbias"] = (torch.full((dim + 2,), -77.0, dtype=_torch_type(kind), device="cuda") for _ in range(2))
        if accumulate is not None:
            out["dweight"][1:-1], out["dbias"][1:-1] = accumulate, -accumulate
        size = L.legend_layer_norm_workspace(rows, dim)
        space = torch.full((size // 4 + 4,), float("nan"), device="cuda")
        space[size // 4:] = -77.0
        more.update(dweight=out["dweight"][1:].data_ptr(), dweight_type=kind, workspace=space.data_ptr(), workspace_bytes=size, accumulate=accumulate is not None)
        if want_bias:
            more.update(dbias=out["dbias"][1:].data_ptr())
    args = case.args(**more)
    torch.cuda.synchronize()
    L.legend_layer_norm_backward(ctx, args)
    L.legend_sync(ctx)
    if dx_in is None:
        assert guards_kept(case, out["dx"])
    if sums:
        assert bool((space[size // 4:] == -77.0).all())
        for k in ("dweight", "dbias"):
            assert float(out[k][0]) == float(out[k][-1]) == -77.0
            out[k] = out[k][1:-1]
    if "dx" in out:
        out["dx"] = out["dx"][1][:, :dim]
    return out


def check_backward(case, out, x, dy, mean, rstd, kind=0, added=0.0):
    m64, r64 = case.numbers(mean), case.numbers(rstd)
    dx, dw, db = od.layer_norm_backward(x, dy, m64, r64, case.w64)
    n, r = chain(case.dim), r64[:, None]
    xh = np.abs(x - m64[:, None]) * r
    u = np.abs(dy if case.w is None else dy * case.w64)
    if "dx" in out:
        tol = r * E * (4 * u + (n + 4) * u.mean(1, keepdims=True) + xh * (n + 8) * (u * xh).mean(1, keepdims=True))
        tol = tol + (3 * E + HALF_STEP[case.xt] * (1 + 1e-3)) * np.abs(dx) + TINY[case.xt]
        err = np.abs(case.numbers(out["dx"]) - dx)
        assert np.all(err <= tol), float((err / tol).max())
    turns = min(case.rows, case.rows / 64 + 32) + 3
    for k, want, terms, sign in (("dweight", dw, np.abs(dy) * xh, 1), ("dbias", db, np.abs(dy), -1)):
        if k in out:
            want = want + sign * added
            tol = turns * E * terms.sum(0) + (E + HALF_STEP[kind]) * np.abs(want) + TINY[kind]
            err = np.abs(case.numbers(out[k]) - want)
            assert np.all(err <= tol), (k, float((err / tol).max()))


SHAPES = [(1, 1), (5, 2), (1, 3), (3, 4), (17, 5), (9, 31), (64, 32), (33, 33), (7, 50), (1, 64), (130, 100), (5, 127), (260, 128), (3, 129), (11, 200),
          (2, 255), (67, 256), (3, 257), (64, 400), (9, 511), (20, 512), (13, 513), (41, 777), (3, 1_000), (37, 1_001), (6, 1_024), (5, 1_025),
          (3, 2_047), (70, 2_048), (3, 2_050), (9, 4_096), (2, 4_100), (5, 5_001), (3, 8_192), (2, 8_194), (3, 16_384), (2, 16_387), (2, 40_000), (1, 100_001),
          (3_001, 8), (2_053, 100), (1_030, 513), (600, 4_096)]


@pytest.mark.parametrize("rows,dim", SHAPES, ids=lambda v: str(v))
def test_forward_and_backward(ctx, rows, dim):
    case = Case(rows, dim)
    y, mean, rstd = forward(ctx, case)
    check_forward(case, y, mean, rstd)
    check_backward(case, backward(ctx, case, mean, rstd), case.x64, case.dy64, mean, rstd)


@pytest.mark.parametrize("rows,dim", [(700, 5_000), (600, 9_001), (300, 16_384), (600, 20_000), (2_500, 1_028)], ids=lambda v: str(v))
def test_many_wide_rows(ctx, rows, dim):
    """Every workgroup takes several rows: what its threads add up from row to row."""
    case = Case(rows, dim, 1, 1)
    y, mean, rstd = forward(ctx, case)
    check_forward(case, y, mean, rstd)
    check_backward(case, backward(ctx, case, mean, rstd), case.x64, case.dy64, mean, rstd)


@pytest.mark.parametrize("wt", [0, 1, 2], ids=["wf", "wb", "wh"])
@pytest.mark.parametrize("xt,yt", [(0, 0), (0, 1), (0, 2), (1, 1), (1, 0), (2, 2), (2, 0)], ids=["ff", "fb", "fh", "bb", "bf", "hh", "hf"])
@pytest.mark.parametrize("rows,dim", [(37, 100), (21, 1_001), (9, 2_304), (4, 20_000)], ids=lambda v: str(v))
def test_types(ctx, rows, dim, xt, yt, wt):
    case = Case(rows, dim, xt, yt, wt)
    y, mean, rstd = forward(ctx, case)
    check_forward(case, y, mean, rstd)
    check_backward(case, backward(ctx, case, mean, rstd, kind=wt), case.x64, case.dy64, mean, rstd, kind=wt)


@pytest.mark.parametrize("pad,shift", [(1, 1), (3, 2), (8, 5)], ids=lambda v: str(v))
@pytest.mark.parametrize("dim", [12, 100, 101, 640, 2_050, 17_000], ids=lambda v: str(v))
@pytest.mark.parametrize("xt", [0, 1, 2], ids=["f", "b", "h"])
def test_strides_and_odd_addresses(ctx, dim, xt, pad, shift):
    case = Case(19, dim, xt, xt, 0, pad=pad, shift=shift)
    y, mean, rstd = forward(ctx, case)
    check_forward(case, y, mean, rstd)
    check_backward(case, backward(ctx, case, mean, rstd), case.x64, case.dy64, mean, rstd)


@pytest.mark.parametrize("weight,bias", [(False, False), (True, False), (False, True)], ids=["none", "weight", "bias"])
@pytest.mark.parametrize("dim", [100, 1_536, 20_001], ids=lambda v: str(v))
def test_without_weight_or_bias(ctx, dim, weight, bias):
    case = Case(11, dim, weight=weight, bias=bias)
    y, mean, rstd = forward(ctx, case)
    check_forward(case, y, mean, rstd)
    check_backward(case, backward(ctx, case, mean, rstd), case.x64, case.dy64, mean, rstd)
    y2, _, _ = forward(ctx, case, statistics=False)
    assert bool((y2 == y).all())
    only = backward(ctx, case, mean, rstd, sums=False)
    assert set(only) == {"dx"}
    check_backward(case, only, case.x64, case.dy64, mean, rstd)
    frozen = backward(ctx, case, mean, rstd, dx_in="none", want_bias=False)
    assert bool((frozen["dbias"] == -77.0).all())
    check_backward(case, {"dweight": frozen["dweight"]}, case.x64, case.dy64, mean, rstd)


@pytest.mark.parametrize("dim", [96, 101, 3_000, 18_000], ids=lambda v: str(v))
def test_in_place(ctx, dim):
    for dx_in in ("x", "dy"):
        case = Case(23, dim)
        x, dy = case.x64, case.dy64
        _, mean, rstd = forward(ctx, case)
        check_backward(case, backward(ctx, case, mean, rstd, dx_in=dx_in), x, dy, mean, rstd)
    case = Case(23, dim, pad=2)
    x = case.x64
    y, mean, rstd = forward(ctx, case, in_place=True)
    check_forward(case, y, mean, rstd, x64=x)
    assert bool((case.x[1][:, dim:] == 7.0).all())


@pytest.mark.parametrize("dim", [100, 700, 20_000], ids=lambda v: str(v))
def test_gradient_of_a_broadcast_output(ctx, dim):
    case = Case(77, dim, broadcast=True)
    _, mean, rstd = forward(ctx, case)
    check_backward(case, backward(ctx, case, mean, rstd), case.x64, case.dy64, mean, rstd)


@pytest.mark.parametrize("dim", [100, 1_500, 20_000], ids=lambda v: str(v))
@pytest.mark.parametrize("kind", [0, 1, 2], ids=["f", "b", "h"])
def test_accumulated_gradients(ctx, dim, kind):
    case = Case(50, dim)
    _, mean, rstd = forward(ctx, case)
    check_backward(case, backward(ctx, case, mean, rstd, kind=kind, accumulate=2.5), case.x64, case.dy64, mean, rstd, kind=kind, added=2.5)


@pytest.mark.parametrize("dim", [100, 2_000, 20_000], ids=lambda v: str(v))
def test_rows_with_an_offset_or_without_spread(ctx, dim):
    rng = np.random.default_rng(dim)
    x = rng.standard_normal((6, dim))
    x[0] = 1e4 + x[0]              # an offset of ten thousand times the spread
    x[1] = 3.25                    # no spread: xh is zero, y is the bias
    x[2] = 0.0
    x[3] *= 1e-6                   # a spread below sqrt(eps)
    x[4] = 1e6
    case = Case(6, dim, x=x)
    y, mean, rstd = forward(ctx, case)
    check_forward(case, y, mean, rstd)
    for r in (1, 2):
        assert np.array_equal(case.numbers(y)[r], case.b64)
    check_backward(case, backward(ctx, case, mean, rstd), case.x64, case.dy64, mean, rstd)


@pytest.mark.parametrize("dim", [100, 2_000, 20_000], ids=lambda v: str(v))
def test_numbers_that_are_not_finite_stay_in_their_row(ctx, dim):
    case = Case(9, dim)
    clean_y, clean_mean, clean_rstd = (t.clone() for t in forward(ctx, case))
    case.x[1][2, 5], case.x[1][6, dim - 1] = float("nan"), float("inf")
    y, mean, rstd = forward(ctx, case)
    fine = [k for k in range(9) if k not in (2, 6)]
    assert bool((y[fine] == clean_y[fine]).all()) and bool((mean[fine] == clean_mean[fine]).all()) and bool((rstd[fine] == clean_rstd[fine]).all())
    assert bool(y[2].isnan().all()) and bool(y[6].isnan().all())
    out = backward(ctx, case, mean, rstd)
    assert bool(out["dx"][fine].isfinite().all()) and bool(out["dx"][2].isnan().all()) and bool(out["dweight"].isnan().all())
    assert bool(out["dbias"].isfinite().all())


def test_no_rows(ctx):
    import torch
    from paper_2505_09258_amd import binding as L
    dw, db = torch.full((40,), 3.0, device="cuda"), torch.full((40,), 4.0, device="cuda")
    torch.cuda.synchronize()
    L.legend_layer_norm_forward(ctx, L.make_layer_norm(rows=0, dim=40))
    L.legend_layer_norm_backward(ctx, L.make_layer_norm(rows=0, dim=40, dweight=dw.data_ptr(), dbias=db.data_ptr(), accumulate=True))
    L.legend_sync(ctx)
    assert bool((dw == 3.0).all()) and bool((db == 4.0).all())
    L.legend_layer_norm_backward(ctx, L.make_layer_norm(rows=0, dim=40, dweight=dw.data_ptr(), dbias=db.data_ptr()))
    L.legend_sync(ctx)
    assert not bool(dw.any()) and not bool(db.any())


@pytest.mark.parametrize("rows,dim", [(500, 100), (40, 3_000), (3, 30_000)], ids=lambda v: str(v))
def test_the_same_bits_again(ctx, rows, dim):
    case = Case(rows, dim, 1, 1)
    y, mean, rstd = (t.clone() for t in forward(ctx, case))
    a = {k: v.clone() for k, v in backward(ctx, case, mean, rstd).items()}
    y2, mean2, rstd2 = forward(ctx, case)
    b = backward(ctx, case, mean2, rstd2)
    assert bool((y == y2).all()) and all(bool((a[k] == b[k]).all()) for k in a)


def test_rows_more_than_two_to_the_32_elements_apart(ctx):
    """Three rows of half precision, 2^31 + 8 elements from one to the next; what lies between them is never touched."""
    import torch
    from paper_2505_09258_amd import binding as L
    dim, stride = 333, 2**31 + 8
    case = Case(3, dim, 2, 2)
    far = [torch.empty(2 * stride + dim + 8, dtype=torch.float16, device="cuda") for _ in range(4)]
    row = lambda t: torch.as_strided(t, (3, dim), (stride, 1))  # noqa: E731
    x, dy, y, dx = (row(t) for t in far)
    x.copy_(case.x[1][:, :dim])
    dy.copy_(case.dy[1][:, :dim])
    mean, rstd = torch.empty(3, device="cuda"), torch.empty(3, device="cuda")
    dw, db = torch.empty(dim, device="cuda"), torch.empty(dim, device="cuda")
    size = L.legend_layer_norm_workspace(3, dim)
    space = torch.empty(size // 4, device="cuda")
    args = case.args(x=x.data_ptr(), x_stride=stride, y=y.data_ptr(), y_stride=stride, dy=dy.data_ptr(), dy_stride=stride, dy_type=2, dx=dx.data_ptr(), dx_stride=stride,
                     mean=mean.data_ptr(), rstd=rstd.data_ptr(), dweight=dw.data_ptr(), dbias=db.data_ptr(), workspace=space.data_ptr(), workspace_bytes=size)
    torch.cuda.synchronize()
    L.legend_layer_norm_forward(ctx, args)
    L.legend_layer_norm_backward(ctx, args)
    L.legend_sync(ctx)
    check_forward(case, y, mean, rstd)
    check_backward(case, dict(dx=dx, dweight=dw, dbias=db), case.x64, case.dy64, mean, rstd)


# ---- rows of the tables -----------------------------------------------------------------------------------------------


@pytest.fixture()
def tables():
    """Five partitions of which three are resident (0, 2 and 4), seven relations."""
    from paper_2505_09258_amd import binding as L
    rng = np.random.default_rng(9)
    V, d = 4_003, 100
    node, rel = rng.standard_normal((V, d)).astype(np.float32), rng.standard_normal((7, d)).astype(np.float32)
    cfg = L.make_config(num_nodes=V, dim=d, num_partitions=5, buffer_capacity=3, num_relations=7, score=L.SCORE_DISTMULT, batch_size=64, chunk_size=16, num_negs=16, seed=1)
    c = L.legend_init_partitions(cfg, node, rel)
    for p in (0, 2, 4):
        L.legend_swap_partition(c, -1, p)
    yield c, node, rel
    L.legend_destroy(c)


class TableCase(Case):
    """The oracle's x is the table rows; bad rows count as rows without a say."""

    def __init__(self, rows_of, **kw):
        super().__init__(rows_of.shape[0], rows_of.shape[1], x=rows_of, **kw)


def table_call(c, case, table, ids, direction, mean, rstd, **more):
    import torch
    from paper_2505_09258_amd import binding as L
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    args = case.args(x=None, x_stride=None, x_type=0, table=table, ids=None if ids is None else ids.data_ptr(), status=status.data_ptr(),
                     mean=mean.data_ptr(), rstd=rstd.data_ptr(), **more)
    torch.cuda.synchronize()
    direction(c, args)
    L.legend_sync(c)
    return int(status[0])


@pytest.mark.parametrize("yt", [0, 1, 2], ids=["f", "b", "h"])
@pytest.mark.parametrize("bad", [False, True], ids=["good", "bad"])
def test_rows_of_the_node_table(tables, bad, yt):
    import torch
    from paper_2505_09258_amd import binding as L
    c, node, _ = tables
    V, d = node.shape
    part = -(-V // 5)
    rng = np.random.default_rng(3)
    ids = np.concatenate([rng.integers(0, part, 200), 2 * part + rng.integers(0, part, 200), rng.integers(4 * part, V, 101), [0, 0, V - 1, V - 1]])
    rng.shuffle(ids)
    wrong = np.zeros(len(ids), bool)
    want_status = 0
    if bad:
        ids[[3, 77, 400]] = [-1, V, 1 << 40]
        ids[[5, 250]] = [part, 3 * part + 1]                     # partitions 1 and 3 are not resident
        wrong[[3, 77, 400, 5, 250]] = True
        want_status = 3
    rows_of = node[np.where(wrong, 0, ids)]
    case = TableCase(rows_of, yt=yt)
    dids = torch.from_numpy(ids).cuda()
    y, (mean, rstd) = case.blank(yt), (torch.full((len(ids),), -77.0, device="cuda") for _ in range(2))
    assert table_call(c, case, L.TABLE_NODE_EMB, dids, L.legend_layer_norm_forward, mean, rstd, y=y[1].data_ptr(), y_type=yt) == want_status
    assert guards_kept(case, y)
    good = ~wrong
    sub = TableCase(rows_of[good], yt=yt)
    sub.w, sub.b = case.w, case.b
    tg = torch.from_numpy(good).cuda()
    check_forward(sub, y[1][tg], mean[tg], rstd[tg])
    assert not bool(y[1][~tg].any()) and not bool(mean[~tg].any()) and not bool(rstd[~tg].any())
    dx, dw, db = case.blank(0), torch.full((d,), -77.0, device="cuda"), torch.full((d,), -77.0, device="cuda")
    size = L.legend_layer_norm_workspace(len(ids), d)
    space = torch.full((size // 4,), float("nan"), device="cuda")
    assert table_call(c, case, L.TABLE_NODE_EMB, dids, L.legend_layer_norm_backward, mean, rstd, dy=case.dy[1].data_ptr(), dy_type=yt, dx=dx[1].data_ptr(),
                      dweight=dw.data_ptr(), dbias=db.data_ptr(), workspace=space.data_ptr(), workspace_bytes=size) == want_status
    assert guards_kept(case, dx) and not bool(dx[1][~tg].any())
    check_backward(sub, {"dx": dx[1][tg], "dweight": dw, "dbias": db}, sub.x64, case.dy64[good], mean[tg], rstd[tg])


def test_rows_of_the_relation_table_and_rows_in_order(tables):
    import torch
    from paper_2505_09258_amd import binding as L
    c, node, rel = tables
    for table, rows_of, ids, status in ((L.TABLE_REL_EMB, rel, None, 0), (L.TABLE_REL_EMB, rel[[6, 0, 6]], np.array([6, 0, 6]), 0), (L.TABLE_NODE_EMB, node[:300], None, 0)):
        case = TableCase(rows_of)
        y, (mean, rstd) = case.blank(0), (torch.empty(case.rows, device="cuda") for _ in range(2))
        dids = None if ids is None else torch.from_numpy(ids.astype(np.int64)).cuda()
        assert table_call(c, case, table, dids, L.legend_layer_norm_forward, mean, rstd, y=y[1].data_ptr()) == status
        check_forward(case, y[1], mean, rstd)
    case = TableCase(rel[[0, 0]])
    y = case.blank(0)
    assert table_call(c, case, L.TABLE_REL_EMB, torch.tensor([7, -1], device="cuda"), L.legend_layer_norm_forward, mean, rstd, y=y[1].data_ptr()) == 1
    assert not bool(y[1].any())


def test_rows_follow_a_swap(tables):
    import torch
    from paper_2505_09258_amd import binding as L
    c, node, _ = tables
    part = -(-node.shape[0] // 5)
    ids = np.arange(part, part + 150)
    case = TableCase(node[ids])
    y, (mean, rstd) = case.blank(0), (torch.empty(150, device="cuda") for _ in range(2))
    dids = torch.from_numpy(ids).cuda()
    assert table_call(c, case, L.TABLE_NODE_EMB, dids, L.legend_layer_norm_forward, mean, rstd, y=y[1].data_ptr()) == 2
    L.legend_swap_partition(c, 2, 1)                              # the call itself waits for the copy
    assert table_call(c, case, L.TABLE_NODE_EMB, dids, L.legend_layer_norm_forward, mean, rstd, y=y[1].data_ptr()) == 0
    check_forward(case, y[1], mean, rstd)


# ---- graphs -----------------------------------------------------------------------------------------------------------


@pytest.mark.parametrize("rows,dim", [(300, 100), (20, 3_000), (3, 20_000)], ids=lambda v: str(v))
def test_replayed_graphs(rows, dim):
    """Two graphs over the same weights, each with a workspace of its own, replayed with other inputs and eager calls between."""
    import torch
    from paper_2505_09258_amd import binding as L
    stream = torch.cuda.Stream()
    cfg = L.make_config(num_nodes=3, dim=4, batch_size=64, chunk_size=16, num_negs=16, init_std=0.1, seed=1, compute_stream=stream.cuda_stream)
    c = L.legend_init_partitions(cfg, None, None)
    try:
        with torch.cuda.stream(stream):
            cases = [Case(rows, dim, seed=k) for k in range(2)]
            made = []
            for case in cases:
                size = L.legend_layer_norm_workspace(rows, dim)
                out = dict(y=torch.zeros(rows, dim, device="cuda"), mean=torch.zeros(rows, device="cuda"), rstd=torch.zeros(rows, device="cuda"),
                           dx=torch.zeros(rows, dim, device="cuda"), dweight=torch.zeros(dim, device="cuda"), dbias=torch.zeros(dim, device="cuda"),
                           workspace=torch.zeros(size // 4, device="cuda"))
                args = case.args(dy=case.dy[1].data_ptr(), workspace_bytes=size, **{k: v.data_ptr() for k, v in out.items()})
                stream.synchronize()
                graph = torch.cuda.CUDAGraph()
                with torch.cuda.graph(graph, stream=stream):
                    L.legend_layer_norm_forward(c, args)
                    L.legend_layer_norm_backward(c, args)
                made.append((case, out, args, graph))
            for turn in range(4):
                for case, out, args, graph in made:
                    case.x[1].add_(0.25)
                    case.dy[1].mul_(0.5)
                    graph.replay()
                torch.cuda.synchronize()
                for case, out, args, graph in made:
                    got = {k: v.clone() for k, v in out.items() if k != "workspace"}
                    for v in out.values():
                        v.zero_()
                    L.legend_layer_norm_forward(c, args)
                    L.legend_layer_norm_backward(c, args)
                    stream.synchronize()
                    assert all(torch.equal(got[k], out[k]) for k in got), turn
                    check_forward(case, out["y"], out["mean"], out["rstd"])
    finally:
        L.legend_destroy(c)


def test_two_calls_on_the_librarys_own_stream_in_order(ctx):
    """A chain without a wait in between: the second call reads what the first one writes."""
    import torch
    from paper_2505_09258_amd import binding as L
    case = Case(2_000, 100)
    mid, out = torch.empty(2_000, 100, device="cuda"), torch.empty(2_000, 100, device="cuda")
    torch.cuda.synchronize()
    for _ in range(3):
        L.legend_layer_norm_forward(ctx, case.args(y=mid.data_ptr()))
        L.legend_layer_norm_forward(ctx, case.args(x=mid.data_ptr(), y=out.data_ptr()))
    L.legend_sync(ctx)
    x = mid.double().cpu().numpy()
    want, _, wr = od.layer_norm(x, case.w64, case.b64, EPS)
    assert np.all(np.abs(out.double().cpu().numpy() - want) <= (2 * chain(100) + 9) * E * (np.abs(want - case.b64) + np.abs(case.w64) + np.abs(want)))
