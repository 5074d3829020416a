"""AdamW over sets of 4 Mi elements and more, which take kernels and a hand-over of the step's state of their own, against the same step by
small optimisers: every tensor alone in one, at its own place among empty ones (the place goes into the random words), with what the
gradients are multiplied by handed to it.  Elementwise the arithmetic is the same, so every bit has to be; the small optimisers are
compared with the 64-bit oracle in test_gpu_adamw.  The norm and the factor are taken here in 64 bits."""

import numpy as np
import pytest

pytestmark = pytest.mark.gpu

HYPER = dict(beta1=0.9, beta2=0.999, eps=1e-8)
LR, SEED = 0.003, 13
LARGE, STREAM_BYTES = 4 << 20, 128 << 20
# (elements, 8-bit states, 16-bit parameter with a master copy): a tensor stays below 4 Mi elements, a set is above, once below and once above
# 128 MB of parameters, states and gradients
SETS = {
    "float": [(2_000_003, 0, 0), (1, 0, 0), (0, 0, 0), (2_047, 0, 1), (2_300_001, 0, 0), (2_049, 0, 0)],
    "float_streamed": [(3_999_999, 0, 0), (257, 0, 0), (4_000_000, 0, 1), (3_000_001, 0, 0)],
    "block": [(2_500_001, 1, 1), (255, 1, 0), (2_000_000, 1, 0), (2_305, 1, 1)],
    "block_streamed": [(4_000_255, 1, 1), (4_000_000, 1, 1), (1, 1, 0), (4_100_001, 1, 0), (3_000_000, 1, 1)],
    "both": [(2_500_001, 1, 1), (1_900_003, 0, 0), (300, 1, 0), (300, 0, 1)],
    "both_streamed": [(4_000_001, 1, 0), (4_100_003, 0, 0), (2_500_000, 0, 1), (2_600, 1, 1)],
}


class Tensors:
    """One set's tensors on the GPU; the same for the same name and seed."""

    def __init__(self, name):
        import torch
        self.shapes, self.all = SETS[name], []
        gen = torch.Generator(device="cuda")
        gen.manual_seed(5)
        r = lambda n: torch.randn(n, generator=gen, device="cuda")  # noqa: E731
        for n, block, half in self.shapes:
            t = dict(master=r(n) * 0.1) if half else {}
            t["param"] = t["master"].bfloat16() if half else r(n) * 0.1
            t["grad"] = torch.empty(n, dtype=torch.bfloat16 if half else torch.float32, device="cuda")
            if block:
                t.update({k: torch.zeros(n, dtype=torch.uint8, device="cuda") for k in ("m", "v")})
                t.update({k: torch.zeros(-(-n // 256), device="cuda") for k in ("m_scale", "v_scale")})
            else:
                t.update({k: torch.zeros(n, device="cuda") for k in ("m", "v")})
            self.all.append(t)
        self.elements = sum(s[0] for s in self.shapes)
        self.bytes = sum(v.numel() * v.element_size() for t in self.all for k, v in t.items() if not k.endswith("scale"))

    def new_gradients(self, turn):
        import torch
        gen = torch.Generator(device="cuda")
        gen.manual_seed(100 + turn)
        for t in self.all:
            t["grad"].copy_(torch.randn(t["grad"].numel(), generator=gen, device="cuda") * 0.01)

    def describe(self, only=None):
        from paper_2505_09258_amd import binding as L
        out = []
        for k, ((n, block, half), t) in enumerate(zip(self.shapes, self.all)):
            a = {key: v.data_ptr() if n else None for key, v in t.items()}
            if only is not None and k != only:
                n, a = 0, dict.fromkeys(("param", "grad", "m", "v"))
            out.append(L.make_adamw_tensor(count=n, param_type=half, grad_type=half, state_type=block, weight_decay=0.01 * (k % 2), lr_scale=1.0 - 0.25 * (k % 3), **a))
        return out

    def norm(self):
        return float(sum((t["grad"].double() ** 2).sum() for t in self.all).sqrt())

    def written(self):
        return [v for t in self.all for k, v in t.items() if k != "grad"]


def same(a, b):
    import torch
    return all(torch.equal(x, y) for x, y in zip(a.written(), b.written()))


@pytest.fixture()
def stream():
    """A stream of torch's that the context computes on too, and the context."""
    import torch
    from paper_2505_09258_amd import binding as L
    s = torch.cuda.Stream()
    cfg = L.make_config(num_nodes=3, dim=4, batch_size=64, chunk_size=16, num_negs=16, init_std=0.1, seed=1, compute_stream=s.cuda_stream)
    c = L.legend_init_partitions(cfg, None, None)
    with torch.cuda.stream(s):
        yield c, s
    torch.cuda.synchronize()
    L.legend_destroy(c)


class Small:
    """The set's step by one optimiser a tensor."""

    def __init__(self, ctx, tensors):
        from paper_2505_09258_amd import binding as L
        import torch
        self.L, self.scale = L, torch.ones(1, device="cuda")
        self.opts = [L.legend_adamw_create(ctx, tensors.describe(k), seed=SEED, **HYPER) for k in range(len(tensors.shapes))]

    def step(self, scale=1.0):
        self.scale.fill_(float(np.float32(scale)))
        for o in self.opts:
            self.L.legend_adamw_step(o, LR, grad_scale=self.scale.data_ptr())

    def close(self):
        for o in self.opts:
            self.L.legend_adamw_destroy(o)


def create(ctx, tensors, max_norm=0.0):
    from paper_2505_09258_amd import binding as L
    return L.legend_adamw_create(ctx, tensors.describe(), max_norm=max_norm, seed=SEED, **HYPER)


@pytest.mark.parametrize("name", SETS)
def test_sets_are_on_both_sides_of_the_rules(name):
    t = Tensors(name)
    assert t.elements >= LARGE and (t.bytes > STREAM_BYTES) == name.endswith("streamed") and max(s[0] for s in t.shapes) < LARGE


@pytest.mark.parametrize("name", SETS)
def test_steps_with_and_without_a_norm_in_turn(stream, name):
    import torch
    from paper_2505_09258_amd import binding as L
    ctx, _ = stream
    a, b = Tensors(name), Tensors(name)
    opt, small = create(ctx, a), Small(ctx, b)
    norm = torch.zeros(1, device="cuda")
    for turn in range(1, 6):
        a.new_gradients(turn)
        b.new_gradients(turn)
        L.legend_adamw_step(opt, LR, norm=norm.data_ptr() if turn in (2, 3, 5) else None)
        small.step()
        assert same(a, b), turn
        if turn in (2, 3, 5):
            assert float(norm) == pytest.approx(a.norm(), rel=2.0**-23)
    assert L.legend_adamw_get_steps(opt) == (5, 0)
    small.close()
    L.legend_adamw_destroy(opt)


@pytest.mark.parametrize("value", [float("nan"), float("inf")], ids=["nan", "inf"])
@pytest.mark.parametrize("name", SETS)
def test_clipped_and_skipped_steps(stream, name, value):
    """Clipped, skipped, skipped, clipped, not clipped: a skipped one leaves every bit and the number of steps."""
    import torch
    from paper_2505_09258_amd import binding as L
    ctx, _ = stream
    a, b = Tensors(name), Tensors(name)
    opt, small = create(ctx, a, max_norm=1.0), Small(ctx, b)
    norm = torch.zeros(1, device="cuda")
    made = skipped = 0
    for turn in range(1, 6):
        a.new_gradients(turn)
        if turn == 5:
            for t in a.all:
                t["grad"].mul_(2.0**-8)
        for t, u in zip(a.all, b.all):
            u["grad"].copy_(t["grad"])
        size = a.norm()
        assert (size > 1.0) == (turn < 5)
        if turn in (2, 3):
            a.all[-1 if turn == 2 else 0]["grad"][-1] = value
            skipped += 1
        else:
            made += 1
        L.legend_adamw_step(opt, LR, norm=norm.data_ptr() if turn != 3 else None)
        if turn not in (2, 3):
            small.step(1.0 / (size + 1e-6) if size > 1.0 else 1.0)
            assert float(norm) == pytest.approx(size, rel=2.0**-23)
        elif turn == 2:
            assert not bool(torch.isfinite(norm))
        assert same(a, b), turn
        assert L.legend_adamw_get_steps(opt) == (made, skipped)
    small.close()
    L.legend_adamw_destroy(opt)


@pytest.mark.parametrize("name", ["float", "float_streamed", "block_streamed", "both"])
def test_replayed_steps(stream, name):
    """A recorded step among eager ones, one of the replays with a gradient that is not finite, against eager steps alone."""
    import torch
    from paper_2505_09258_amd import binding as L
    ctx, s = stream
    a, b = Tensors(name), Tensors(name)
    opts = [create(ctx, a, max_norm=1.0), create(ctx, b, max_norm=1.0)]
    factor, norm, other_norm = torch.ones(1, device="cuda"), torch.zeros(1, device="cuda"), torch.zeros(1, device="cuda")
    s.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=s):
        L.legend_adamw_step(opts[0], LR, lr_factor=factor.data_ptr(), norm=norm.data_ptr())
    assert L.legend_adamw_get_steps(opts[0]) == (0, 0)
    made = skipped = 0
    for turn in range(1, 7):
        factor.fill_(1.0 / turn)
        for t in (a, b):
            t.new_gradients(turn)
            if turn == 4:
                t.all[0]["grad"][7] = float("inf")
        made, skipped = made + (turn != 4), skipped + (turn == 4)
        if turn == 3:
            L.legend_adamw_step(opts[0], LR, lr_factor=factor.data_ptr(), norm=norm.data_ptr())
        else:
            graph.replay()
        L.legend_adamw_step(opts[1], LR, lr_factor=factor.data_ptr(), norm=other_norm.data_ptr())
        torch.cuda.synchronize()
        assert same(a, b), turn
        assert torch.equal(norm, other_norm) and [L.legend_adamw_get_steps(o) for o in opts] == [(made, skipped)] * 2
    for o in opts:
        L.legend_adamw_destroy(o)


def test_as_many_tensors_as_an_optimiser_takes(stream):
    """2^24 tensors of one element: more units than one launch has workgroups."""
    import ctypes as C
    import torch
    from paper_2505_09258_amd import binding as L
    ctx, _ = stream
    n = 1 << 24
    kinds = {C.c_void_p: "u8", C.c_int64: "i8", C.c_int32: "i4", C.c_uint32: "u4", C.c_double: "f8"}
    fields = L.legend_adamw_tensor._fields_
    all_of_them = np.zeros(n, np.dtype(dict(names=[f for f, _ in fields], formats=[kinds[t] for _, t in fields],
                                            offsets=[getattr(L.legend_adamw_tensor, f).offset for f, _ in fields], itemsize=C.sizeof(L.legend_adamw_tensor))))
    dev = {k: torch.zeros(n, device="cuda") for k in ("param", "m", "v")}
    dev["grad"] = 1.0 + torch.arange(n, device="cuda") % 3
    for k, t in dev.items():
        all_of_them[k] = t.data_ptr() + 4 * np.arange(n, dtype=np.uint64)
    all_of_them["count"] = all_of_them["lr_scale"] = 1
    conf, opt = L.legend_adamw_config(C.sizeof(L.legend_adamw_config), 0, 0.9, 0.999, 1e-8, 0.0, 0), C.c_void_p()
    assert L._lib.legend_adamw_create(ctx, C.byref(conf), all_of_them.ctypes.data_as(C.c_void_p), n, C.byref(opt)) == 0
    del all_of_them
    L.legend_adamw_step(opt, 0.5)
    assert L.legend_adamw_get_steps(opt) == (1, 0)
    # three gradients, three results: the first step of each is 0.5 times its sign, but for eps and a few roundings
    for t in dev.values():
        assert all(bool((t[k::3] == t[k]).all()) for k in range(3))
    assert float((dev["param"] + 0.5).abs().max()) <= 0.5 * (1e-8 + 24 * 2.0**-24)
    assert torch.allclose(dev["m"], 0.1 * dev["grad"], rtol=2.0**-22, atol=0)
    L.legend_adamw_destroy(opt)
