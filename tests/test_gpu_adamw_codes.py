"""The 8-bit states bit for bit: what the header promises of every operation up to a code, fp32 and rounded to nearest in the order written."""

import numpy as np
import pytest

from oracle import dense as od
from tests.test_gpu_adamw import ctx  # noqa: F401

pytestmark = pytest.mark.gpu

F = np.float32


def codes_of(x, scale, share):
    """e4m3 codes (without the sign of zero) of |x| / scale with `share` of a step added and cut off: exact, x and the scale being fp32."""
    with np.errstate(divide="ignore", invalid="ignore"):
        q = np.where(scale > 0, x / scale, F(0.0)).astype(F)                  # fp32 by fp32, rounded once
    a = np.minimum(np.abs(q), F(448.0)).astype(np.float64)
    step = np.exp2(np.maximum(np.frexp(a)[1] - 1, -6) - 3.0)
    return np.sign(q) * np.minimum(np.floor(a / step + share) * step, 448.0), a


@pytest.mark.parametrize("size", [1.0, 1e-6, 1e-17, 1e6], ids=["ones", "small", "tiny", "large"])
@pytest.mark.parametrize("n", [300 * 256, 1_000_003], ids=str)
def test_codes_and_scales(ctx, n, size):  # noqa: F811
    """No element is left out, near a boundary or not.  Gradients over six decades, so that the small codes are met as well."""
    import torch
    from paper_2505_09258_amd import binding as L
    b1, b2, seed, gs = 0.9, 0.999, 31, 0.3
    rng = np.random.default_rng(n)
    dev = {k: torch.zeros(n, dtype=t, device="cuda") for k, t in (("param", torch.float32), ("grad", torch.float32), ("m", torch.uint8), ("v", torch.uint8))}
    dev.update({k: torch.zeros(-(-n // 256), device="cuda") for k in ("m_scale", "v_scale")})
    scale = torch.tensor([gs], device="cuda")
    torch.cuda.synchronize()
    opt = L.legend_adamw_create(ctx, [L.make_adamw_tensor(count=n, state_type=1, **{k: t.data_ptr() for k, t in dev.items()})], beta1=b1, beta2=b2, eps=1e-8, seed=seed)
    values, word = od.e4m3_values().astype(F), None
    spread = lambda s: np.repeat(s, 256)[:n]  # noqa: E731
    tops = lambda x: np.pad(np.abs(x), (0, -n % 256)).reshape(-1, 256).max(1)  # noqa: E731
    for step in range(1, 5):
        g = (rng.standard_normal(n) * np.exp(2.0 * rng.standard_normal(n)) * size).astype(F)
        dev["grad"].copy_(torch.from_numpy(g))
        cm, cr, sm, sr = (dev[k].cpu().numpy() for k in ("m", "v", "m_scale", "v_scale"))
        torch.cuda.synchronize()
        L.legend_adamw_step(opt, 0.0, grad_scale=scale.data_ptr())
        L.legend_sync(ctx)
        g = g * F(gs)
        m, root = values[cm] * spread(sm), values[cr] * spread(sr)
        v = root * root
        m = F(b1) * m + F(1 - b1) * g
        v = F(b2) * v + (F(1 - b2) * g) * g
        assert m.dtype == v.dtype == F
        root = np.sqrt(v)
        word = od.random_words(seed, step, 0, n)
        for key, x, share, least in (("m", m, (word >> np.uint64(12)) / 2.0**20, False), ("v", root, (word & np.uint64(0xFFFF)) / 2.0**16, True)):
            want_scale = tops(x) * F(1 / 448)
            assert np.array_equal(dev[key + "_scale"].cpu().numpy(), want_scale), (key, step)
            want, a = codes_of(x, spread(want_scale), share)
            if least:
                low = (a > 0) & (a < od.LEAST)
                want[low] = od.LEAST * np.floor(1.0 + share[low])
            got = od.e4m3_values()[dev[key].cpu().numpy()]
            assert np.array_equal(got, want), (key, step, int((got != want).sum()))
    L.legend_adamw_destroy(opt)


@pytest.mark.parametrize("octave", [0, 1])
@pytest.mark.parametrize("power", [-127, -104, -101, -40, 0, 60], ids=lambda p: "2^%d" % p)
def test_the_root_of_every_mantissa(ctx, octave, power):  # noqa: F811
    """v runs through every fp32 number of an octave (first the numbers below 2^-126), one a block, whose scale is then sqrt(v) rounded, times 1 / 448 rounded.  With beta2 = 1/2
    v = v_before / 2 + (g / 2) g; v_before / 2 lies at the begin of an eighth of the octave, g adds the rest, so small that its roundings fall away."""
    import torch
    from paper_2505_09258_amd import binding as L
    part = 1 << 20
    n = part * 256
    dev = {k: torch.zeros(n, dtype=t, device="cuda") for k, t in (("param", torch.bfloat16), ("grad", torch.float32), ("m", torch.uint8), ("v", torch.uint8))}
    dev.update({k: torch.zeros(part, device="cuda") for k in ("m_scale", "v_scale")})
    opt = L.legend_adamw_create(ctx, [L.make_adamw_tensor(count=n, param_type=1, state_type=1, **{k: t.data_ptr() for k, t in dev.items()})],
                                beta1=0.5, beta2=0.5, eps=1e-8, seed=1)
    first = (127 + octave + power) << 23
    for eighth in range(8):
        v = torch.arange(first + eighth * part, first + (eighth + 1) * part, dtype=torch.int32, device="cuda").view(torch.float32)
        before = torch.sqrt(2.0 * v[:1].double()).float() * (1 - 2.0**-22)                 # its square, halved, is just below the first v
        half = 0.5 * (before * before)
        rest = v.double() - half.double()
        assert float(rest.min()) >= 0
        g = torch.sqrt(2.0 * rest).float()
        assert torch.equal(half + (0.5 * g) * g, v)
        for k in ("m", "v", "grad", "m_scale"):
            dev[k].zero_()
        dev["grad"][::256] = g
        dev["v"][::256] = 0x38                                                             # the code of 1
        dev["v_scale"].copy_(before.expand(part))
        torch.cuda.synchronize()
        L.legend_adamw_step(opt, 0.0)
        L.legend_sync(ctx)
        want = torch.sqrt(v.double()).float() * torch.tensor(1 / 448, dtype=torch.float32, device="cuda")
        assert torch.equal(dev["v_scale"], want), (eighth, int((dev["v_scale"] != want).sum()))
    L.legend_adamw_destroy(opt)
