"""What the operators for a model's dense parts are measured on: layer norm, forward and backward, and the AdamW step.

A case is a dict of plain values.  `kind` says which operator it runs:

    norm        layer norm's forward pass over rows of a matrix, or of the resident node table by id
    norm_grad   its backward pass: gradients of the rows (where asked for), of the weight and of the bias
    adamw       one AdamW step over many tensors, states in 32 bits or in blocks of 8-bit codes, with clipping to a norm

The sizes are those of this repository's workloads where it has them (embedding dimensions 32 to 512, batches of up to
50 000 rows) and generic ones beyond: rows from one to tens of thousands, widths from eight to 16 384, parameters from a
few thousand to a hundred million in one to three hundred tensors.
"""

from __future__ import annotations

import math

import numpy as np
import torch

own = False

TYPES = {"float": torch.float32, "bfloat": torch.bfloat16, "half": torch.float16}
SIZE = {"float": 4, "bfloat": 2, "half": 2}
EPS = 1e-5                          # layer norm
BETA1, BETA2, ADAM_EPS, LR = 0.9, 0.999, 1e-8, 1e-3
STEPS_BEFORE = 100                  # the step that is measured is the 101st
BLOCK, TOP = 256, 448.0             # elements that share a scale; the largest e4m3 value
NODES = 200_000                     # rows of the node table that cases read from
TABLE_DIMS = (32, 50, 64, 100, 128, 200, 400)
SR_SEED = 11


def _norm(name, kind, rows, dim, *, x="float", y="float", source="matrix", pad=0, affine="both", weight="float", want_dx=True):
    """y: type of the output, of its gradient in the backward pass.  pad: unused columns between rows."""
    return dict(name=name, kind=kind, rows=rows, dim=dim, x=x, y=y, source=source, pad=pad, affine=affine, weight=weight, want_dx=want_dx)


def _adamw(name, tensors, elements, *, state="float", param="float", grad="float", master=False, max_norm=1.0, loss_scale=1.0):
    """elements: of all tensors together.  State "float": 32 bits; "block": 8-bit codes.  max_norm 0: no clipping."""
    return dict(name=name, kind="adamw", tensors=tensors, elements=elements, state=state, param=param, grad=grad, master=master,
                max_norm=max_norm, loss_scale=loss_scale)


def listed():
    return [
        # one query's row before it is answered: all latency
        _norm("norm_one_row", "norm", 1, 128),
        # a batch's rows of the learned table (d = 100, 50 000 rows), normalised for a matrix product in bfloat16
        _norm("norm_table_rows", "norm", 50_000, 100, y="bfloat", source="table"),
        # a wide hidden layer's activations
        _norm("norm_wide", "norm", 16_384, 4_096, x="bfloat", y="bfloat", weight="bfloat"),
        # odd widths in a padded buffer
        _norm("norm_ragged", "norm", 4_099, 1_001, x="half", y="half", pad=3, affine="weight"),
        # a short evaluation batch of the widest table rows
        _norm("norm_grad_small", "norm_grad", 64, 400),
        # the same batch as norm_table_rows: the head's gradients, table rows frozen
        _norm("norm_grad_table_rows", "norm_grad", 50_000, 100, y="bfloat", source="table", want_dx=False),
        # the wide hidden layer again
        _norm("norm_grad_wide", "norm_grad", 16_384, 4_096, x="bfloat", y="bfloat", weight="bfloat"),
        # a small head: weight and bias of a norm, a projection and its bias; all latency
        _adamw("adamw_head", 4, 41_000),
        # many small tensors that lie tight behind one another, gradients of a scaled loss in half precision
        _adamw("adamw_many_ragged", 300, 3_000_001, grad="half", loss_scale=1024.0),
        # a large model's parameters
        _adamw("adamw_large", 40, 60_000_000),
        # states in 8 bits: many odd tensors
        _adamw("adamw_block_ragged", 200, 2_500_003, state="block"),
        # states in 8 bits: a large model in bfloat16 with its parameters kept in 32 bits beside
        _adamw("adamw_block_large", 60, 120_000_000, state="block", param="bfloat", grad="bfloat", master=True),
    ]


def _spread(rng, low, high):
    """A whole number between low and high, spread over its logarithm."""
    return int(round(math.exp(rng.uniform(math.log(low), math.log(high)))))


def draw(rng):
    kind = rng.choice(("norm", "norm_grad", "adamw"))
    if kind == "adamw":
        state = rng.choice(("float", "block"))
        param = rng.choice(("float", "bfloat", "half"))
        case = _adamw("", _spread(rng, 1, 300), _spread(rng, 5_000, 60_000_000), state=state, param=param,
                      grad=rng.choice(("float", param)), master=param != "float" and rng.random() < 0.7,
                      max_norm=rng.choice((0.0, 1.0, 1.0)), loss_scale=rng.choice((1.0, 256.0)))
    elif rng.random() < 0.3:
        case = _norm("", kind, _spread(rng, 1, 100_000), rng.choice(TABLE_DIMS), y=rng.choice(("float", "bfloat")), source="table",
                     affine=rng.choice(("both", "weight", "none")), want_dx=rng.random() < 0.5)
    else:
        x = rng.choice(("float", "bfloat", "half"))
        dim = _spread(rng, 8, 16_384)     # with fewer columns the rows' gradient is what is left of terms that cancel
        case = _norm("", kind, max(1, min(_spread(rng, 1, 65_536), 48_000_000 // dim)), dim, x=x, y=rng.choice((x, "float")),
                     pad=rng.choice((0, 0, 0, 1, 8)), affine=rng.choice(("both", "both", "weight", "none")), weight=rng.choice(("float", x)))
    del case["name"]
    return case


# ---- inputs ---------------------------------------------------------------------------------------------------------


def _tensor_sizes(case):
    """Sizes of a case's tensors: a few large ones and many small ones, odd ones among them."""
    n, total = case["tensors"], case["elements"]
    share = np.random.RandomState(n).pareto(1.0, n) + 0.05
    sizes = np.maximum(1, np.floor(share / share.sum() * total).astype(np.int64))
    sizes[0] += max(0, total - int(sizes.sum()))
    return sizes


def _values(gen, *shape, dtype=torch.float32):
    return torch.randn(*shape, generator=gen, device="cuda", dtype=torch.float32).to(dtype)


def _prepare_norm(case, gen, seed):
    rows, dim, s = case["rows"], case["dim"], {"case": case}
    if case["source"] == "table":
        s["table"] = _values(gen, NODES, dim) * 0.3 + 0.1
        s["ids"] = torch.randint(0, NODES, (rows,), generator=gen, device="cuda")
    else:
        wide = torch.zeros(rows, dim + case["pad"], device="cuda", dtype=TYPES[case["x"]])
        wide[:, :dim] = _values(gen, rows, dim) * torch.exp(0.5 * _values(gen, rows, 1)) + 0.5 * _values(gen, rows, 1)
        s["x"] = wide[:, :dim]
    wt = TYPES[case["weight"]]
    s["weight"] = (1 + 0.1 * _values(gen, dim)).to(wt) if case["affine"] != "none" else None
    s["bias"] = (0.1 * _values(gen, dim)).to(wt) if case["affine"] == "both" else None
    if case["kind"] == "norm_grad":
        s["dy"] = _values(gen, rows, dim, dtype=TYPES[case["y"]])
        x = _rows(s).double()
        mean = x.mean(1)
        s["mean"], s["rstd"] = mean.float(), (x.var(1, unbiased=False) + EPS).rsqrt().float()    # what the forward pass left
        del x
    if own:
        s["call"] = _OwnNorm(s)
    return s


def _prepare_adamw(case, gen, seed):
    sizes = _tensor_sizes(case)
    block = case["state"] == "block"
    # in blocks a tensor begins on a whole block of one buffer; otherwise tensors lie tight
    room = -(-sizes // BLOCK) * BLOCK if block else sizes
    starts = np.concatenate([[0], np.cumsum(room)])
    total = int(starts[-1])
    s = {"case": case, "sizes": sizes, "starts": starts, "steps": STEPS_BEFORE,
         "decay": np.where(np.arange(len(sizes)) % 3 == 1, 0.0, 0.01), "lr_scale": np.where(np.arange(len(sizes)) % 5 == 2, 0.5, 1.0)}
    pt, gt = TYPES[case["param"]], TYPES[case["grad"]]
    # the plain form's plan: which tensor an element (a block) belongs to
    s["owner"] = torch.repeat_interleave(torch.from_numpy(room // BLOCK if block else room).cuda())
    used = 1.0
    if block:       # elements behind a tensor's last one stay zero
        place = torch.arange(total, device="cuda").view(-1, BLOCK) - torch.from_numpy(starts[:-1]).cuda()[s["owner"], None]
        used = (place < torch.from_numpy(sizes).cuda()[s["owner"], None]).float().view(-1)
        del place
    p = _values(gen, total) * 0.05 * used
    s["param"] = p.to(pt)
    if case["master"]:
        s["master"] = p
    size = torch.exp(_values(gen, total))                     # gradients' sizes differ from element to element
    s["grad"] = (_values(gen, total) * size * (1e-3 * case["loss_scale"]) * used).to(gt)
    s["grad_scale"] = torch.full((1,), 1.0 / case["loss_scale"], device="cuda")
    m = _values(gen, total) * size * 2e-4 * used
    root = size * 1e-3 * (1 + 0.1 * _values(gen, total).abs()) * used
    if block:
        for key, v in (("m", m), ("root", root)):
            v = v.view(-1, BLOCK)
            scale = v.abs().amax(1) / TOP
            s[key + "_scale"] = scale
            s[key] = (v / scale.clamp_min(1e-30)[:, None]).clamp(-TOP, TOP).to(torch.float8_e4m3fn).view(-1)
    else:
        s["m"], s["v"] = m, root * root
    s["norm"] = torch.zeros(1, device="cuda")
    if own:
        s["call"] = _OwnAdamW(s)
    return s


def prepare(case, seed):
    if own:
        _stream()
    gen = torch.Generator(device="cuda")
    gen.manual_seed(int(seed))
    return (_prepare_adamw if case["kind"] == "adamw" else _prepare_norm)(dict(case), gen, int(seed))


# ---- the framework's calls ------------------------------------------------------------------------------------------

_kept = {}


def _stream():
    """The one stream of a program that mixes torch and this library: torch's current one, handed to every context."""
    if "stream" not in _kept:
        _kept["stream"] = torch.cuda.Stream()
        torch.cuda.synchronize()
        torch.cuda.set_stream(_kept["stream"])
    return _kept["stream"]


def _context(table=None):
    from paper_2505_09258_amd import binding as L
    nodes, dim = (3, 4) if table is None else table.shape
    cfg = L.make_config(num_nodes=nodes, dim=dim, batch_size=64, chunk_size=16, num_negs=16, init_std=0.1, seed=1,
                        compute_stream=_stream().cuda_stream)
    ctx = L.legend_init_partitions(cfg, None if table is None else table.cpu().numpy(), None)
    L.legend_swap_partition(ctx, -1, 0)
    L.legend_sync(ctx)
    return ctx


def _shared_context():
    if "context" not in _kept:
        _kept["context"] = _context()
    return _kept["context"]


def _kind_of(t):
    from paper_2505_09258_amd import binding as L
    return {torch.float32: L.TYPE_FLOAT, torch.bfloat16: L.TYPE_BFLOAT, torch.float16: L.TYPE_HALF}[t.dtype]


class _OwnNorm:
    """A layer norm's arguments as a program keeps them: buffers in place, one call a pass."""

    def __init__(self, s):
        from paper_2505_09258_amd import binding as L
        case = s["case"]
        rows, dim = case["rows"], case["dim"]
        self.L, self.private = L, case["source"] == "table"
        self.ctx = _context(s["table"]) if self.private else _shared_context()
        at = dict(rows=rows, dim=dim, eps=EPS)
        if self.private:
            self.status = torch.zeros(1, dtype=torch.int32, device="cuda")
            at.update(table=L.TABLE_NODE_EMB, ids=s["ids"].data_ptr(), status=self.status.data_ptr())
        else:
            at.update(x=s["x"].data_ptr(), x_stride=s["x"].stride(0), x_type=_kind_of(s["x"]))
        if s["weight"] is not None:
            at.update(weight=s["weight"].data_ptr(), weight_type=_kind_of(s["weight"]))
        if s["bias"] is not None:
            at.update(bias=s["bias"].data_ptr())
        if case["kind"] == "norm":
            y = torch.empty(rows, dim, dtype=TYPES[case["y"]], device="cuda")
            self.out = {"y": y, "mean": torch.empty(rows, device="cuda"), "rstd": torch.empty(rows, device="cuda")}
            at.update(y=y.data_ptr(), y_type=_kind_of(y), mean=self.out["mean"].data_ptr(), rstd=self.out["rstd"].data_ptr())
            self.go = L.legend_layer_norm_forward
        else:
            self.out = {}
            at.update(dy=s["dy"].data_ptr(), dy_type=_kind_of(s["dy"]), mean=s["mean"].data_ptr(), rstd=s["rstd"].data_ptr())
            if case["want_dx"]:
                self.out["dx"] = torch.empty(rows, dim, dtype=TYPES[case["x"]], device="cuda")
                at.update(dx=self.out["dx"].data_ptr())
            if s["weight"] is not None:
                self.out["dweight"] = torch.empty(dim, device="cuda")
                at.update(dweight=self.out["dweight"].data_ptr())
            if s["bias"] is not None or s["weight"] is None:
                self.out["dbias"] = torch.empty(dim, device="cuda")
                at.update(dbias=self.out["dbias"].data_ptr())
            size = L.legend_layer_norm_workspace(rows, dim)
            self.workspace = torch.empty(max(size, 4) // 4, device="cuda")
            at.update(workspace=self.workspace.data_ptr(), workspace_bytes=size)
            self.go = L.legend_layer_norm_backward
        self.args = L.make_layer_norm(**at)

    def __call__(self):
        self.go(self.ctx, self.args)
        return self.out

    def __del__(self):
        if self.private:
            self.L.legend_destroy(self.ctx)


class _OwnAdamW:
    def __init__(self, s):
        from paper_2505_09258_amd import binding as L
        case, n = s["case"], len(s["sizes"])
        self.L, block = L, case["state"] == "block"

        def at(key, k, scales=False):
            t = s[key]
            return t.data_ptr() + int(s["starts"][k]) // (BLOCK if scales else 1) * t.element_size()

        tensors = [L.make_adamw_tensor(
            count=int(s["sizes"][k]), param=at("param", k), param_type=_kind_of(s["param"]), grad=at("grad", k), grad_type=_kind_of(s["grad"]),
            master=at("master", k) if case["master"] else None, m=at("m", k), v=at("root" if block else "v", k),
            state_type=L.STATE_BLOCK if block else L.STATE_FLOAT, m_scale=at("m_scale", k, True) if block else None,
            v_scale=at("root_scale", k, True) if block else None, weight_decay=float(s["decay"][k]), lr_scale=float(s["lr_scale"][k]))
            for k in range(n)]
        self.opt = L.legend_adamw_create(_shared_context(), tensors, beta1=BETA1, beta2=BETA2, eps=ADAM_EPS, max_norm=case["max_norm"], seed=SR_SEED)
        L.legend_adamw_set_steps(self.opt, s["steps"])
        self.scale, self.norm = s["grad_scale"].data_ptr(), s["norm"].data_ptr() if case["max_norm"] else None

    def __call__(self):
        self.L.legend_adamw_step(self.opt, LR, grad_scale=self.scale, norm=self.norm)

    def __del__(self):
        if hasattr(self, "opt"):
            self.L.legend_adamw_destroy(self.opt)


# ---- plain forms ----------------------------------------------------------------------------------------------------


def _rows(s):
    return s["table"][s["ids"]] if "table" in s else s["x"]


def _norm_plain(s):
    x = _rows(s).float()
    mean = x.sum(1, keepdim=True) / x.shape[1]
    c = x - mean
    rstd = 1.0 / torch.sqrt((c * c).sum(1, keepdim=True) / x.shape[1] + EPS)
    y = c * rstd
    if s["weight"] is not None:
        y = y * s["weight"].float()
    if s["bias"] is not None:
        y = y + s["bias"].float()
    return {"y": y.to(TYPES[s["case"]["y"]]), "mean": mean[:, 0], "rstd": rstd[:, 0]}


def _norm_grad_plain(s):
    case = s["case"]
    rstd = s["rstd"][:, None]
    xh = (_rows(s).float() - s["mean"][:, None]) * rstd
    dy = s["dy"].float()
    out = {}
    if s["weight"] is not None:
        out["dweight"] = (dy * xh).sum(0)
    if s["bias"] is not None or s["weight"] is None:
        out["dbias"] = dy.sum(0)
    if case["want_dx"]:
        u = dy if s["weight"] is None else dy * s["weight"].float()
        a, b = u.sum(1, keepdim=True) / case["dim"], (u * xh).sum(1, keepdim=True) / case["dim"]
        out["dx"] = (rstd * (u - a - xh * b)).to(TYPES[case["x"]])
    return out


def _fold(h, x):
    """One step of the library's counter hash: the splitmix64 output function of h + golden ratio + x."""
    z = h + np.uint64(0x9E3779B97F4A7C15) + x
    z = (z ^ (z >> np.uint64(30))) * np.uint64(0xBF58476D1CE4E5B9)
    z = (z ^ (z >> np.uint64(27))) * np.uint64(0x94D049BB133111EB)
    return z ^ (z >> np.uint64(31))


def _random_words(s, steps):
    """The 32-bit word of every element: a mix of its place in its tensor and of a key of (seed, step, tensor)."""
    n = len(s["sizes"])
    base = _fold(np.array([SR_SEED], np.uint64), np.uint64(steps))
    keys = _fold(np.repeat(base, n), np.arange(n, dtype=np.uint64)) & np.uint64(0xFFFFFFFF)
    start = torch.from_numpy(s["starts"][:-1]).cuda()[s["owner"], None]
    place = torch.arange(start.shape[0] * BLOCK, device="cuda").view(-1, BLOCK) - start
    w = place ^ torch.from_numpy(keys.astype(np.int64)).cuda()[s["owner"], None]
    w = w ^ (w >> 16)
    w = (w * 0x9E3779B1) & 0xFFFFFFFF
    w = w ^ (w >> 15)
    w = (w * 0x85157AF5) & 0xFFFFFFFF
    return w ^ (w >> 16)


def _to_codes(v, u, least):
    """[blocks, 256] values as e4m3 codes and a scale a block; u in [0, 1) decides between the two codes around a value."""
    scale = v.abs().amax(1) / TOP
    scale = torch.where(scale > 2.0**-100, scale, torch.zeros_like(scale))
    x = torch.where(scale[:, None] > 0, v / scale[:, None], torch.zeros_like(v)).clamp(-TOP, TOP)
    if least:        # a second moment above zero keeps a code above zero
        x = torch.where(x > 0, x.clamp_min(2.0**-9), x)
    a = x.abs()
    step = (((torch.frexp(a)[1] - 1).clamp_min(-6) - 3 + 127) << 23).view(torch.float32)      # of the value's octave: 2^(e - 3)
    q = torch.floor(a / step + u) * step
    return torch.where(x < 0, -q, q).to(torch.float8_e4m3fn).view(-1), scale


def _adamw_plain(s):
    case, block = s["case"], s["case"]["state"] == "block"
    s["steps"] += 1
    t = s["steps"]
    g = s["grad"].float()
    scale = s["grad_scale"]
    if case["max_norm"]:
        norm = g.double().square().sum().sqrt() * scale.double()
        scale = torch.where(norm > case["max_norm"], case["max_norm"] / (norm + 1e-6), torch.ones_like(norm)).float() * scale
        s["norm"].copy_(norm)
    g = g * scale
    # what belongs to a tensor, once for each of its elements (for each of its blocks)
    lr = LR * s["lr_scale"]
    step = torch.from_numpy((lr / (1 - BETA1**t)).astype(np.float32)).cuda()[s["owner"]]
    keep = torch.from_numpy((1 - lr * s["decay"]).astype(np.float32)).cuda()[s["owner"]]
    m, p = s["m"], (s["master"] if case["master"] else s["param"]).float()
    if block:
        g, p, step, keep = g.view(-1, BLOCK), p.view(-1, BLOCK), step[:, None], keep[:, None]
        m = m.float().view(-1, BLOCK) * s["m_scale"][:, None]
        root = s["root"].float().view(-1, BLOCK) * s["root_scale"][:, None]
        v = root * root
    else:
        v = s["v"]
    m = BETA1 * m + (1 - BETA1) * g
    v = BETA2 * v + (1 - BETA2) * g * g
    root = torch.sqrt(v)
    p = p * keep - step * (m / (root * (1 / math.sqrt(1 - BETA2**t)) + ADAM_EPS))
    s["param"].copy_(p.view(-1))
    if case["master"]:
        s["master"].copy_(p.view(-1))
    if block:
        words = _random_words(s, t)
        s["m"], s["m_scale"] = _to_codes(m, (words >> 12).float() * 2.0**-20, False)
        s["root"], s["root_scale"] = _to_codes(root, (words & 0xFFFF).float() * 2.0**-16, True)
    else:
        s["m"], s["v"] = m, v


def run(state):
    kind = state["case"]["kind"]
    if own:
        out = state["call"]()
        if kind != "adamw":
            return out
    elif kind == "adamw":
        _adamw_plain(state)
    else:
        return _norm_plain(state) if kind == "norm" else _norm_grad_plain(state)
    return {k: state[k] for k in ("param", "master", "m", "m_scale", "root", "root_scale", "v") if k in state} | (
        {"norm": state["norm"]} if state["case"]["max_norm"] else {})


# ---- the definition in 64 bits --------------------------------------------------------------------------------------


def _exact_norm(s):
    case = s["case"]
    x = (s["table"].index_select(0, s["ids"]) if "table" in s else s["x"]).to(torch.float64)
    w = torch.ones(case["dim"], dtype=torch.float64, device="cuda") if s["weight"] is None else s["weight"].to(torch.float64)
    if case["kind"] == "norm":
        var, mean = torch.var_mean(x, 1, correction=0)
        rstd = (var + EPS).pow(-0.5)
        y = torch.addcmul(torch.zeros_like(w) if s["bias"] is None else s["bias"].to(torch.float64), (x - mean[:, None]) * rstd[:, None], w)
        return {"y": y, "mean": mean, "rstd": rstd}
    rstd = s["rstd"].to(torch.float64).unsqueeze(1)
    xh = x.sub_(s["mean"].to(torch.float64).unsqueeze(1)).mul_(rstd)
    dy = s["dy"].to(torch.float64)
    out = {"dweight": torch.einsum("rc,rc->c", dy, xh)} if s["weight"] is not None else {}
    if s["bias"] is not None or s["weight"] is None:
        out["dbias"] = torch.einsum("rc->c", dy)
    if case["want_dx"]:
        u = dy.mul_(w)
        out["dx"] = rstd * (u - u.mean(1, keepdim=True) - xh * (u * xh).mean(1, keepdim=True))
    return out


def _exact_codes(v, word, bits, least):
    """Values in units of their block's scale, rounded up where the word's fraction reaches the next e4m3 value."""
    top = v.abs().max(1).values
    x = v * torch.where(top > 0, TOP / top, 0.0).unsqueeze(1)
    a = x.abs()
    if least:
        a = torch.where(a > 0, torch.clamp(a, min=2.0**-9), a)
    octave = torch.clamp(torch.floor(torch.log2(torch.clamp(a, min=1e-300))), min=-6.0)
    unit = torch.exp2(octave - 3.0)
    q = torch.floor(a / unit + word.to(torch.float64) / 2.0**bits) * unit
    return (torch.sign(x) * torch.clamp(q, max=TOP)).reshape(-1), top / TOP


def _exact_adamw(s):
    case, block = s["case"], s["case"]["state"] == "block"
    t = STEPS_BEFORE + 1
    f = torch.float64
    g = s["grad"].to(f) * float(s["grad_scale"].item())
    out = {}
    if case["max_norm"]:
        norm = torch.linalg.vector_norm(g)
        out["norm"] = norm.reshape(1)
        g = g * min(1.0, case["max_norm"] / (norm.item() + 1e-6)) if norm.item() > case["max_norm"] else g
    p = (s["master"] if case["master"] else s["param"]).to(f).clone()
    if block:
        m = (s["m"].to(f).view(-1, BLOCK) * s["m_scale"].to(f)[:, None]).view(-1)
        v = (s["root"].to(f).view(-1, BLOCK) * s["root_scale"].to(f)[:, None]).view(-1).square()
    else:
        m, v = s["m"].to(f), s["v"].to(f)
    m = torch.lerp(g, m, BETA1)
    v = torch.lerp(g.square(), v, BETA2)
    for k, size in enumerate(s["sizes"]):
        a, b = int(s["starts"][k]), int(s["starts"][k]) + int(size)
        lr = LR * float(s["lr_scale"][k])
        hat = (m[a:b] / (1 - BETA1**t)) / ((v[a:b] / (1 - BETA2**t)).sqrt() + ADAM_EPS)
        p[a:b] = p[a:b] * (1 - lr * float(s["decay"][k])) - lr * hat
    out["param"] = p
    if case["master"]:
        out["master"] = p
    if block:
        words = _random_words(s, t)
        out["m"], out["m_scale"] = _exact_codes(m.view(-1, BLOCK), words >> 12, 20, False)
        out["root"], out["root_scale"] = _exact_codes(v.sqrt().view(-1, BLOCK), words & 0xFFFF, 16, True)
    else:
        out["m"], out["v"] = m, v
    return out


def exact(case, seed):
    s = prepare(case, seed)
    return _exact_adamw(s) if case["kind"] == "adamw" else _exact_norm(s)


# ---- what a pass cannot do without ----------------------------------------------------------------------------------


def work(case):
    if case["kind"] == "adamw":
        n = case["elements"]
        p, g = SIZE[case["param"]], SIZE[case["grad"]]
        each = g + (p + 8 if case["master"] else 2 * p) + (4 + 16 / BLOCK if case["state"] == "block" else 16)
        return {"bytes": n * each, "flops": n * (18 + (2 if case["max_norm"] else 0))}
    n, sx, sy = case["rows"] * case["dim"], SIZE[case["x"]], SIZE[case["y"]]
    params = {"both": 2, "weight": 1, "none": 0}[case["affine"]] * case["dim"]
    rows = case["rows"] * (8 + (8 if case["source"] == "table" else 0))
    if case["kind"] == "norm":
        return {"bytes": n * (sx + sy) + rows + params * SIZE[case["weight"]], "flops": 8 * n}
    return {"bytes": n * (sx + sy + (sx if case["want_dx"] else 0)) + rows + case["dim"] * SIZE[case["weight"]] + 8 * case["dim"],
            "flops": (14 if case["want_dx"] else 5) * n}
