"""The host side of the dense operators (csrc/dense.hip) on the CPU, compiled against a stub of the runtime: every argument that
must be refused is, before anything is enqueued, and what the documentation allows is not."""

import ctypes as C
import os
import re
import shutil
import subprocess

import pytest

HERE = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(HERE)
CSRC = os.path.join(ROOT, "paper_2505_09258_amd", "csrc")
OK, INVAL, NOMEM, STATE = 0, -1, -2, -6
BASE = 1 << 40                      # addresses that nothing dereferences


def at(k):
    """The k-th of a row of addresses 16 MB apart."""
    return BASE + (k << 24)


@pytest.fixture(scope="module")
def lib(tmp_path_factory):
    if shutil.which("g++") is None:
        pytest.skip("needs g++")
    from paper_2505_09258_amd import binding as L
    so = tmp_path_factory.mktemp("dense") / "libdense_stub.so"
    native = os.path.join(HERE, "native")
    subprocess.run(["g++", "-std=c++17", "-O1", "-g", "-Wall", "-Wno-unknown-pragmas", "-shared", "-fPIC", "-I", os.path.join(native, "dense"),
                    "-I", CSRC, "-I", os.path.join(ROOT, "include"), os.path.join(native, "dense_stub.cpp"), "-o", str(so)], check=True, timeout=120)
    lib = C.CDLL(str(so))
    for name in ("legend_layer_norm_forward", "legend_layer_norm_backward", "legend_layer_norm_workspace", "legend_adamw_create",
                 "legend_adamw_destroy", "legend_adamw_step", "legend_adamw_set_gradients", "legend_adamw_get_steps", "legend_adamw_set_steps"):
        getattr(lib, name).argtypes = getattr(L._lib, name).argtypes
        getattr(lib, name).restype = getattr(L._lib, name).restype
    lib.legend_last_error.restype = C.c_char_p
    lib.stub_context.restype = C.c_void_p
    lib.stub_context.argtypes = [C.c_int, C.c_int64, C.c_int]
    lib.stub_context_gone.argtypes = [C.c_void_p]
    lib.stub_set.argtypes = [C.c_void_p, C.c_int, C.c_int, C.c_int]
    lib.stub_grad.restype = C.c_void_p
    return lib


@pytest.fixture()
def ctx(lib):
    c = lib.stub_context(100, 5_000, 7)
    lib.stub_set(c, 0, 0, 0)
    yield c
    lib.stub_set(c, 0, 0, 0)
    lib.stub_context_gone(c)


def forward(**change):
    from paper_2505_09258_amd import binding as L
    a = dict(rows=10, dim=64, x=at(0), y=at(1), mean=at(2), rstd=at(3), weight=at(4), bias=at(5))
    return L.make_layer_norm(**{**a, **change})


def backward(**change):
    from paper_2505_09258_amd import binding as L
    a = dict(rows=10, dim=64, x=at(0), dy=at(1), mean=at(2), rstd=at(3), weight=at(4), dx=at(6), dweight=at(7), dbias=at(8),
             workspace=at(9), workspace_bytes=1 << 20)
    return L.make_layer_norm(**{**a, **change})


TABLE = dict(x=None, dim=100, ids=at(10), status=at(11))

ALLOWED_FORWARD = {
    "plain": {}, "no_statistics": dict(mean=None, rstd=None), "no_weight": dict(weight=None), "no_bias": dict(bias=None),
    "in_place": dict(y=at(0)), "same_row_again": dict(x_stride=0), "no_rows": dict(rows=0, x=None, y=None),
    "half": dict(x_type=2, y_type=2), "half_to_float": dict(x_type=2, y_type=0), "float_to_bfloat": dict(y_type=1), "odd_address": dict(x_type=1, y_type=1, x=at(0) + 2),
    "one_row_short_stride_ok": dict(rows=1), "nodes": dict(TABLE, table=0), "relations": dict(TABLE, table=2), "no_ids": dict(TABLE, table=0, ids=None),
    "behind_one_another": dict(y=at(0) + 10 * 64 * 4), "widest": dict(dim=1 << 20, rows=2),
}
REFUSED_FORWARD = {
    "dim_zero": dict(dim=0), "dim_large": dict(dim=(1 << 20) + 1), "rows_negative": dict(rows=-1), "rows_many": dict(rows=(1 << 40) + 1),
    "x_null": dict(x=None), "y_null": dict(y=None), "x_type": dict(x_type=3), "x_type_negative": dict(x_type=-1), "y_type": dict(y_type=7),
    "types": dict(x_type=1, y_type=2), "weight_type": dict(weight_type=9), "eps_zero": dict(eps=0.0), "eps_negative": dict(eps=-1.0),
    "eps_nan": dict(eps=float("nan")), "eps_infinite": dict(eps=float("inf")), "x_stride": dict(x_stride=63), "x_stride_negative": dict(x_stride=-64),
    "y_stride": dict(y_stride=63), "y_stride_zero": dict(y_stride=0), "stride_overflow": dict(x_stride=1 << 60), "x_misaligned": dict(x=at(0) + 2),
    "half_misaligned": dict(x_type=2, y_type=2, x=at(0) + 1), "y_misaligned": dict(y=at(1) + 2), "mean_misaligned": dict(mean=at(2) + 1),
    "weight_misaligned": dict(weight=at(4) + 2), "y_over_x": dict(y=at(0) + 256), "y_on_x_other_stride": dict(y=at(0), y_stride=65),
    "y_on_x_other_size": dict(y=at(0), y_type=1), "mean_in_y": dict(mean=at(1) + 64), "rstd_is_mean": dict(rstd=at(2)), "mean_in_x": dict(mean=at(0) + 4),
    "y_over_weight": dict(y=at(4)), "mean_over_bias": dict(mean=at(5) + 4),
    "table_unknown": dict(TABLE, table=4), "table_state": dict(TABLE, table=1), "table_and_x": dict(TABLE, table=0, x=at(0)), "table_dim": dict(TABLE, table=0, dim=64),
    "table_type": dict(TABLE, table=0, x_type=1), "table_no_status": dict(TABLE, table=0, status=None), "table_status_misaligned": dict(TABLE, table=0, status=at(11) + 2),
    "table_ids_misaligned": dict(TABLE, table=0, ids=at(10) + 4), "table_y_over_ids": dict(TABLE, table=0, y=at(10)), "table_status_in_y": dict(TABLE, table=0, status=at(1) + 8),
}
ALLOWED_BACKWARD = {
    "plain": {}, "only_rows": dict(dweight=None, dbias=None, workspace=None, workspace_bytes=0), "only_weight": dict(dx=None, dbias=None),
    "only_bias": dict(dx=None, dweight=None), "dx_is_dy": dict(dx=at(1)), "dx_is_x": dict(dx=at(0)), "no_rows": dict(rows=0, x=None, dy=None, mean=None, rstd=None, workspace=None, workspace_bytes=0),
    "broadcast_gradient": dict(dy_stride=0), "accumulate": dict(accumulate=True), "half_sums": dict(dweight_type=2),
    "nodes": dict(TABLE, table=0), "frozen_nodes": dict(TABLE, table=0, dx=None), "enough": dict(workspace_bytes=10 * 2 * 64 * 4),
}
REFUSED_BACKWARD = {
    "nothing": dict(dx=None, dweight=None, dbias=None), "no_mean": dict(mean=None), "no_rstd": dict(rstd=None), "dy_null": dict(dy=None), "x_null": dict(x=None),
    "dy_type": dict(dy_type=5), "types": dict(x_type=1, dy_type=2), "dy_stride": dict(dy_stride=5), "dx_stride": dict(dx_stride=0), "dweight_type": dict(dweight_type=3),
    "accumulate": dict(accumulate=2), "no_workspace": dict(workspace=None), "small_workspace": dict(workspace_bytes=10 * 2 * 64 * 4 - 1), "workspace_misaligned": dict(workspace=at(9) + 8),
    "workspace_in_x": dict(workspace=at(0)), "dweight_in_workspace": dict(dweight=at(9) + 64), "dweight_is_dbias": dict(dbias=at(7)), "dweight_over_weight": dict(dweight=at(4)),
    "dx_over_dy": dict(dx=at(1) + 256), "dx_over_x": dict(dx=at(0) + 4), "dx_on_broadcast": dict(dx=at(1), dy_stride=0), "dx_over_mean": dict(dx=at(2)), "dx_over_weight": dict(dx=at(4)),
    "dx_over_workspace": dict(dx=at(9)), "dbias_in_dy": dict(dbias=at(1) + 8), "dx_misaligned": dict(dx=at(6) + 1), "dweight_misaligned": dict(dweight=at(7) + 2),
    "table_dx_over_ids": dict(TABLE, table=0, dx=at(10)), "table_status_in_dweight": dict(TABLE, table=0, status=at(7)), "table_status_in_dx": dict(TABLE, table=0, status=at(6) + 4),
}


@pytest.mark.parametrize("name", ALLOWED_FORWARD)
def test_forward_takes(lib, ctx, name):
    before = lib.stub_launches()
    n = forward(**ALLOWED_FORWARD[name])
    assert lib.legend_layer_norm_forward(ctx, n) == OK, lib.legend_last_error()
    assert lib.stub_launches() - before == (1 if n.rows else 0) and lib.stub_current_device() == 0


@pytest.mark.parametrize("name", REFUSED_FORWARD)
def test_forward_refuses(lib, ctx, name):
    before = lib.stub_launches()
    assert lib.legend_layer_norm_forward(ctx, forward(**REFUSED_FORWARD[name])) == INVAL
    assert lib.legend_last_error() and lib.stub_launches() == before and lib.stub_current_device() == 0


@pytest.mark.parametrize("name", ALLOWED_BACKWARD)
def test_backward_takes(lib, ctx, name):
    before = lib.stub_launches()
    assert lib.legend_layer_norm_backward(ctx, backward(**ALLOWED_BACKWARD[name])) == OK, lib.legend_last_error()
    assert lib.stub_launches() == before + 1 and lib.stub_current_device() == 0


@pytest.mark.parametrize("name", REFUSED_BACKWARD)
def test_backward_refuses(lib, ctx, name):
    before = lib.stub_launches()
    assert lib.legend_layer_norm_backward(ctx, backward(**REFUSED_BACKWARD[name])) == INVAL
    assert lib.legend_last_error() and lib.stub_launches() == before


def test_layer_norm_of_nothing(lib, ctx):
    assert lib.legend_layer_norm_forward(None, forward()) == INVAL
    assert lib.legend_layer_norm_forward(ctx, None) == INVAL and lib.legend_layer_norm_backward(ctx, None) == INVAL
    n = forward()
    n.struct_size -= 8
    assert lib.legend_layer_norm_forward(ctx, n) == INVAL


def test_recorded_calls_on_tables_wait_for_no_swap(lib, ctx):
    n = forward(**dict(TABLE, table=0))
    lib.stub_set(ctx, 1, 0, 1)
    assert lib.legend_layer_norm_forward(ctx, n) == STATE
    assert lib.legend_layer_norm_backward(ctx, backward(**dict(TABLE, table=0))) == STATE
    assert lib.legend_layer_norm_forward(ctx, forward()) == OK           # no table, no swap to wait for
    lib.stub_set(ctx, 0, 0, 1)
    assert lib.legend_layer_norm_forward(ctx, n) == OK
    lib.stub_set(ctx, 1, 0, 0)
    assert lib.legend_layer_norm_forward(ctx, n) == OK


def test_workspace_of_impossible_sizes():
    from paper_2505_09258_amd import binding as L
    assert L.legend_layer_norm_workspace(-1, 4) == L.legend_layer_norm_workspace(4, 0) == L.legend_layer_norm_workspace(4, (1 << 20) + 1) == -1
    assert L.legend_layer_norm_workspace(0, 8) >= 0
    for rows in (1, 7, 64, 1_000, 50_000, 1 << 40):
        for dim in (1, 100, 1_001, 4_096, 1 << 20):
            size = L.legend_layer_norm_workspace(rows, dim)
            assert size % (8 * dim) == 0 and 0 < size <= 1024 * 8 * dim


def tensor(k=0, **change):
    from paper_2505_09258_amd import binding as L
    a = dict(count=1_000, param=at(10 * k), grad=at(10 * k + 1), m=at(10 * k + 2), v=at(10 * k + 3))
    return L.make_adamw_tensor(**{**a, **change})


def block(k=0, **change):
    from paper_2505_09258_amd import binding as L
    return tensor(k, **{**dict(state_type=L.STATE_BLOCK, m_scale=at(10 * k + 4), v_scale=at(10 * k + 5)), **change})


def create(lib, ctx, tensors, n=None, size=None, reserved=0, **cfg):
    from paper_2505_09258_amd import binding as L
    c = dict(beta1=0.9, beta2=0.999, eps=1e-8, max_norm=0.0)
    c.update(cfg)
    conf = L.legend_adamw_config(C.sizeof(L.legend_adamw_config) if size is None else size, reserved, c["beta1"], c["beta2"], c["eps"], c["max_norm"], 5)
    out = C.c_void_p(123)
    rc = lib.legend_adamw_create(ctx, C.byref(conf), (L.legend_adamw_tensor * max(1, len(tensors)))(*tensors), len(tensors) if n is None else n, C.byref(out))
    assert (out.value is None) == (rc != OK)
    return rc, out


ALLOWED_TENSORS = {
    "one": lambda: [tensor()], "mixed": lambda: [tensor(0), block(1, param_type=1, grad_type=1, master=at(16)), tensor(2, param_type=2, grad_type=2)],
    "empty_among": lambda: [tensor(0), tensor(1, count=0, param=None, grad=None, m=None, v=None), block(2)],
    "only_empty": lambda: [tensor(0, count=0, param=None, grad=None, m=None, v=None)],
    "shared_gradient": lambda: [tensor(0), tensor(1, grad=at(1))], "tight": lambda: [tensor(0), tensor(1, param=at(0) + 4_000)],
    "codes_at_odd_addresses": lambda: [block(m=at(2) + 1, v=at(3) + 3)],
    "units_of_a_long_one": lambda: [tensor(0, count=100_001), tensor(20), block(40, count=5_000)],
}
REFUSED_TENSORS = {
    "count": lambda: [tensor(count=-1)], "count_large": lambda: [tensor(count=(1 << 48) + 1)], "param_type": lambda: [tensor(param_type=3)], "grad_type": lambda: [tensor(grad_type=-1)],
    "state_type": lambda: [tensor(state_type=2)], "decay": lambda: [tensor(weight_decay=-0.1)], "decay_nan": lambda: [tensor(weight_decay=float("nan"))],
    "lr_scale": lambda: [tensor(lr_scale=float("inf"))], "lr_scale_negative": lambda: [tensor(lr_scale=-1.0)], "master_of_float": lambda: [tensor(master=at(6))],
    "no_param": lambda: [tensor(param=None)], "no_grad": lambda: [tensor(grad=None)], "no_m": lambda: [tensor(m=None)], "no_v": lambda: [tensor(v=None)],
    "no_scale": lambda: [block(m_scale=None)], "scale_of_float": lambda: [tensor(v_scale=at(5))], "param_misaligned": lambda: [tensor(param=at(0) + 2)],
    "half_misaligned": lambda: [tensor(grad_type=2, grad=at(1) + 1)], "m_misaligned": lambda: [tensor(m=at(2) + 1)], "scale_misaligned": lambda: [block(m_scale=at(4) + 2)],
    "same_param_twice": lambda: [tensor(0), tensor(1, param=at(0))], "states_overlap": lambda: [tensor(0), tensor(1, m=at(3) + 3_996)], "m_is_v": lambda: [tensor(v=at(2))],
    "gradient_in_param": lambda: [tensor(0), tensor(1, grad=at(0) + 64)], "scales_shared": lambda: [block(0), block(1, m_scale=at(4))], "codes_in_scales": lambda: [block(m=at(4) + 15)],
    "master_is_param": lambda: [tensor(param_type=1, master=at(0))], "last_element": lambda: [tensor(0), tensor(1, param=at(0) + 3_996)],
}


@pytest.mark.parametrize("name", ALLOWED_TENSORS)
def test_adamw_takes(lib, ctx, name):
    rc, opt = create(lib, ctx, ALLOWED_TENSORS[name]())
    assert rc == OK, lib.legend_last_error()
    before = lib.stub_launches()
    assert lib.legend_adamw_step(opt, 1e-3, None, None, None) == OK, lib.legend_last_error()
    assert lib.stub_launches() == before + 1 and lib.stub_current_device() == 0
    steps, skipped = C.c_int64(-1), C.c_int64(-1)
    assert lib.legend_adamw_get_steps(opt, C.byref(steps), C.byref(skipped)) == OK and (steps.value, skipped.value) == (1, 0)
    assert lib.legend_adamw_destroy(opt) == OK and lib.stub_live() == 0


@pytest.mark.parametrize("name", REFUSED_TENSORS)
def test_adamw_refuses(lib, ctx, name):
    assert create(lib, ctx, REFUSED_TENSORS[name]())[0] == INVAL
    assert lib.legend_last_error() and lib.stub_live() == 0


@pytest.mark.parametrize("cfg", [dict(beta1=1.0), dict(beta1=-0.1), dict(beta2=1.0), dict(beta2=float("nan")), dict(eps=0.0), dict(eps=float("inf")),
                                 dict(max_norm=-1.0), dict(max_norm=float("nan")), dict(n=0), dict(n=-1), dict(n=(1 << 24) + 1), dict(size=8), dict(reserved=1)],
                         ids=lambda c: "%s_%s" % next(iter(c.items())))
def test_adamw_refuses_configurations(lib, ctx, cfg):
    assert create(lib, ctx, [tensor()], **cfg)[0] == INVAL and lib.stub_live() == 0


def test_adamw_refuses_steps_and_gradients(lib, ctx):
    rc, opt = create(lib, ctx, [tensor(0), tensor(1, grad_type=2)])
    assert rc == OK
    for lr in (-1e-3, float("nan"), float("inf")):
        assert lib.legend_adamw_step(opt, lr, None, None, None) == INVAL
    for k in range(3):
        assert lib.legend_adamw_step(opt, 1e-3, *[at(30) + 2 if j == k else None for j in range(3)]) == INVAL

    def set_gradients(*g):
        return lib.legend_adamw_set_gradients(opt, (C.c_void_p * max(1, len(g)))(*g), len(g))

    assert set_gradients(at(31), at(32)) == OK
    assert lib.legend_adamw_step(opt, 1e-3, None, None, None) == OK and lib.stub_grad(0) == at(31) and lib.stub_grad(1) == at(32)
    for bad in ((at(31),), (at(31), None), (at(31) + 2, at(32)), (at(31), at(32) + 1), (at(0), at(32)), (at(31), at(13) + 16), (at(31), at(32), at(33))):
        assert set_gradients(*bad) == INVAL
    assert lib.legend_adamw_step(opt, 1e-3, None, None, None) == OK and lib.stub_grad(0) == at(31)        # refused ones left no trace
    assert lib.legend_adamw_set_gradients(opt, None, 2) == INVAL
    assert lib.legend_adamw_set_steps(opt, -1) == INVAL and lib.legend_adamw_set_steps(opt, 41) == OK
    steps = C.c_int64()
    assert lib.legend_adamw_get_steps(opt, C.byref(steps), None) == OK and steps.value == 41
    for f in (lambda: lib.legend_adamw_step(None, 1e-3, None, None, None), lambda: lib.legend_adamw_set_steps(None, 1),
              lambda: lib.legend_adamw_get_steps(None, None, None), lambda: lib.legend_adamw_set_gradients(None, None, 0)):
        assert f() == INVAL
    assert lib.legend_adamw_destroy(opt) == OK and lib.legend_adamw_destroy(None) == OK


def test_adamw_refuses_scalars_in_its_memory(lib, ctx):
    rc, opt = create(lib, ctx, [tensor(0), block(1)])
    assert rc == OK
    last = at(0) + 4 * 999                                            # of the first tensor's parameter
    for k in (0, 1, 2):
        for p in (at(0), last, at(1) + 8, at(12) + 996, at(14), at(15) + 12):
            assert lib.legend_adamw_step(opt, 1e-3, *[p if j == k else None for j in range(3)]) == INVAL
        for p in (last + 4, at(12) + 1_000, at(14) + 16, at(0) - 4):
            assert lib.legend_adamw_step(opt, 1e-3, *[p if j == k else None for j in range(3)]) == OK
    assert lib.legend_adamw_step(opt, 1e-3, at(60), None, at(60)) == lib.legend_adamw_step(opt, 1e-3, None, at(60), at(60)) == INVAL
    assert lib.legend_adamw_step(opt, 1e-3, at(60), at(60), at(61)) == OK
    assert lib.legend_adamw_set_gradients(opt, (C.c_void_p * 2)(at(62), at(63)), 2) == OK
    assert lib.legend_adamw_step(opt, 1e-3, None, None, at(62)) == INVAL and lib.legend_adamw_step(opt, 1e-3, None, None, at(1)) == OK
    assert lib.legend_adamw_destroy(opt) == OK


def test_adamw_while_recording(lib, ctx):
    rc, opt = create(lib, ctx, [tensor()])
    lib.stub_set(ctx, 1, 0, 0)
    assert lib.legend_adamw_step(opt, 1e-3, None, None, None) == OK
    assert create(lib, ctx, [tensor(1)])[0] == STATE
    assert lib.legend_adamw_set_gradients(opt, (C.c_void_p * 1)(at(31)), 1) == STATE
    assert lib.legend_adamw_get_steps(opt, None, None) == STATE and lib.legend_adamw_set_steps(opt, 1) == STATE
    assert lib.legend_adamw_destroy(opt) == STATE                      # and it is still there
    lib.stub_set(ctx, 0, 0, 0)
    assert lib.legend_adamw_step(opt, 1e-3, None, None, None) == OK and lib.legend_adamw_destroy(opt) == OK


def test_adamw_outlives_its_context(lib):
    c = lib.stub_context(100, 5_000, 7)
    rc, opt = create(lib, c, [tensor()])
    lib.stub_context_gone(c)
    assert lib.legend_adamw_step(opt, 1e-3, None, None, None) == STATE and lib.legend_adamw_get_steps(opt, None, None) == STATE
    assert lib.legend_adamw_destroy(opt) == OK and lib.stub_live() == 0


def test_adamw_without_memory(lib, ctx):
    lib.stub_set(ctx, 0, 1, 0)
    assert create(lib, ctx, [tensor()])[0] == NOMEM
    lib.stub_set(ctx, 0, 0, 0)
    rc, opt = create(lib, ctx, [tensor()])                           # the context is still usable
    assert rc == OK and lib.legend_adamw_destroy(opt) == OK


@pytest.mark.parametrize("name", ["legend_layer_norm", "legend_adamw_config", "legend_adamw_tensor"])
def test_struct_layout_matches_header_field_order(name):
    from paper_2505_09258_amd import binding as L
    text = re.sub(r"/\*.*?\*/", "", open(os.path.join(ROOT, "include", "legend.h")).read(), flags=re.S)
    body = text[text.index("typedef struct %s {" % name):text.index("} %s;" % name)].split("{", 1)[1]
    fields = []
    for line in filter(None, (part.strip() for part in body.split(";"))):
        first, *more = line.split(",")
        fields.append(first.split()[-1].lstrip("*"))
        fields += [m.strip() for m in more]
    assert fields == [f[0] for f in getattr(L, name)._fields_]
