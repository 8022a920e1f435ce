"""The operators of a language-model job's residual blocks, timed: what stands between the lookup of its rows and its loss, and what of
it is remembered for the backward pass in 8 bits.

  keep        rows in 8 bits, 32 neighbours sharing a power of two, and the rows restored from them
  edge        the edge between two blocks: a norm of the block's result, its gate, the scaled residual, the norm before the next block
  edge_step   the same, and its gradients, from rows as they are or kept in 8 bits
  gated       a gated activation
  gated_step  the same, and its gradients, from inputs as they are or kept in 8 bits
  kept_grad   the gradient of a layer's weights from its input kept in 8 bits

A case is a dict of plain values.  `prepare` draws its inputs on the GPU from a seed alone, `run` is one pass (in elementary torch
operations, or through the package's entry points where `own` is true), `work` says what a pass cannot do without, `exact` gives
the outputs in 64 bits.
"""
import math

import torch

own = False

TYPES = {"fp32": torch.float32, "bf16": torch.bfloat16, "fp16": torch.float16}
SIZE = {"fp32": 4, "bf16": 2, "fp16": 2}
GROUP = 32                              # neighbours that share a scale
KEPT = (GROUP + 1) / GROUP              # bytes an element
EPS = 1e-6
LARGEST = 16384 * 4096 * 16384          # tokens x width x width of the largest listed gradient


def listed():
    """The listed cases; each stands for the use its comment names."""
    return [
        # the rows of a short prompt: the calls are latency
        dict(name="keep_few", kind="keep", N=5, D=1003, type="fp32", form="e4m3"),
        # a large micro-batch's widest rows, remembered and restored
        dict(name="keep_large", kind="keep", N=16384, D=8192, type="bf16", form="i8"),
        # four tokens that a trained model is asked to go on from: the edge of a block is latency
        dict(name="edge_few", kind="edge", N=4, D=2048, type="bf16", x_type="bf16", centred=False, after=True, gates=1),
        # scoring a batch, a gate for each token
        dict(name="edge_gates", kind="edge", N=4096, D=5120, type="fp16", x_type="fp16", centred=False, after=True, gates=4096),
        # a small job: three sequences of 1001 tokens with a gate each, norms with means and biases, the residual stream in single precision
        dict(name="edge_step_odd", kind="edge_step", N=3003, D=1000, type="bf16", x_type="fp32", centred=True, after=True, gates=3, form=""),
        # a large micro-batch, all that is remembered of it in 8 bits
        dict(name="edge_step_large", kind="edge_step", N=16384, D=4096, type="bf16", x_type="bf16", centred=False, after=True, gates=1, form="i8"),
        # a few tokens through an activation of odd width
        dict(name="gated_few", kind="gated", N=3, F=5461, type="fp32", act="gelu"),
        # a small job in half precision
        dict(name="gated_step_odd", kind="gated_step", N=1501, F=2731, type="fp16", act="gelu", form="e4m3"),
        # a large micro-batch, the widest rows of a block
        dict(name="gated_step_large", kind="gated_step", N=8192, F=16384, type="bf16", act="silu", form="i8"),
        # a small job in single precision
        dict(name="kept_grad_small", kind="kept_grad", N=512, D=512, M=2048, type="fp32", form="e4m3", weighted=False),
        # a ragged batch in half precision, of odd widths; the kept rows are a norm's, its weights and biases applied after the product
        dict(name="kept_grad_odd", kind="kept_grad", N=4999, D=1000, M=2731, type="fp16", form="e4m3", weighted=True),
        # a large model's micro-batch
        dict(name="kept_grad_large", kind="kept_grad", N=16384, D=4096, M=16384, type="bf16", form="i8", weighted=False),
    ]


def draw(rng):
    """One more case of the ranges the listed ones stand for."""
    def log_int(lo, hi):
        return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))

    def width(lo, hi):
        d = log_int(lo, hi)
        return d if rng.random() < 0.35 else max(lo, d // 64 * 64)

    def sizes(lo, hi, most):
        while True:
            n, d = log_int(1, 65536), width(lo, hi)
            if n * d <= most:
                return n, d

    kind = rng.choice(["keep", "edge", "edge_step", "edge_step", "gated", "gated_step", "kept_grad", "kept_grad"])
    type_ = rng.choice(["bf16", "bf16", "fp16", "fp32"])
    form = rng.choice(["i8", "e4m3"])
    if kind == "keep":
        N, D = sizes(64, 32768, 1 << 27)
        return dict(kind=kind, N=N, D=D, type=type_, form=form)
    if kind in ("edge", "edge_step"):
        N, D = sizes(64, 8192, 1 << 26)
        x_type = "fp32" if rng.random() < 0.25 else type_
        gates = rng.choice([0, 1, N] + [g for g in range(2, 33) if N % g == 0][-1:])
        case = dict(kind=kind, N=N, D=D, type=type_, x_type=x_type, centred=rng.random() < 0.4, after=rng.random() < 0.6, gates=gates)
        if kind == "edge_step":
            case["form"] = form if x_type != "fp32" and rng.random() < 0.7 else ""
        return case
    if kind in ("gated", "gated_step"):
        N, F = sizes(64, 32768, 1 << 27)
        case = dict(kind=kind, N=N, F=F, type=type_, act=rng.choice(["silu", "gelu", "gelu_tanh"]))
        if kind == "gated_step":
            case["form"] = rng.choice(["i8", "e4m3", ""])
        return case
    while True:
        N, D, M = log_int(1, 65536), width(64, 16384), width(64, 16384)
        if N * D * M <= LARGEST // (16 if type_ == "fp32" else 1) and D * M <= 1 << 27 and N * max(D, M) <= 1 << 28:
            return dict(kind=kind, N=N, D=D, M=M, type=type_, form=form, weighted=rng.random() < 0.5)


# ---- inputs --------------------------------------------------------------------------------------------------------

def prepare(case, seed):
    g = torch.Generator("cuda").manual_seed(seed)
    kind, dt = case["kind"], TYPES[case["type"]]

    def normal(*shape, std=1.0, dtype=dt):
        return (torch.randn(shape, generator=g, device="cuda", dtype=torch.float32) * std).to(dtype)

    def rows(n, d, dtype=dt):
        """Rows of a model in training: some columns several times as large as others."""
        size = torch.exp(0.7 * torch.randn(d, generator=g, device="cuda"))
        return (torch.randn((n, d), generator=g, device="cuda") * size).to(dtype)

    def around_one(d, dtype):
        return (1.0 + 0.1 * torch.randn(d, generator=g, device="cuda")).to(dtype)

    s = dict(case=case)
    N = case["N"]
    if kind == "keep":
        s["rows"] = rows(N, case["D"])
    elif kind in ("edge", "edge_step"):
        D, G = case["D"], case["gates"]
        xt = TYPES[case["x_type"]]
        # parameters in single precision where the residual stream is, but for rows that are remembered in 8 bits
        wt = torch.float32 if case["x_type"] == "fp32" and not case.get("form") else dt
        s["x"], s["branch"] = rows(N, D, xt), rows(N, D)
        s["gate"] = None if G == 0 else normal(D, std=0.5, dtype=wt) if G == 1 else normal(G, D, std=0.5, dtype=wt)
        biased = case["centred"]
        s["after"] = (around_one(D, wt), normal(D, std=0.1, dtype=wt) if biased else None) if case["after"] else None
        s["before"] = (around_one(D, wt), normal(D, std=0.1, dtype=wt) if biased else None)
        if kind == "edge_step":
            s["y_grad"], s["rows_grad"] = normal(N, D, std=0.02, dtype=xt), normal(N, D, std=0.02)
    elif kind in ("gated", "gated_step"):
        # one product's result, its halves the gate's input and what is gated
        s["both"] = rows(N, 2 * case["F"])
        if kind == "gated_step":
            s["rows_grad"] = normal(N, case["F"], std=0.02)
    else:
        # the kept rows a norm's, as an earlier call of the same iteration left them
        N, D, M = case["N"], case["D"], case["M"]
        s["values"], s["scales"] = _kept_bytes(normal(N, D, dtype=torch.float32), case["form"])
        s["rows_grad"] = normal(N, M, std=0.02)
        s["weight"], s["bias"] = (around_one(D, dt), normal(D, std=0.1)) if case["weighted"] else (None, None)
    return s


def _grouped(rows):
    """[N, groups, 32] in fp32, zeros beyond the row's end."""
    N, D = rows.shape
    groups = -(-D // GROUP)
    whole = torch.zeros((N, groups * GROUP), dtype=torch.float32, device=rows.device)
    whole[:, :D] = rows
    return whole.view(N, groups, GROUP)


def _exponent(groups, form):
    """Of each group's scale: the least power of two that brings its largest element to a code."""
    part, exponent = torch.frexp(groups.abs().amax(2, keepdim=True))           # part 1/2 .. 1
    if form == "i8":
        return exponent - 7 + (part >= 255 / 256).int()
    return exponent - 9 + (part > 0.875).int()


def _codes(groups, exponent, form):
    """What the codes stand for, in units of the scale."""
    scaled = torch.ldexp(groups, -exponent)
    if form == "i8":
        return torch.round(scaled)
    step = torch.frexp(scaled)[1].clamp_(min=-5) - 4                           # e4m3: three bits after the first, none below 2^-9
    return torch.ldexp(torch.round(torch.ldexp(scaled, -step)), step)


def _plain_kept(rows, form):
    """The rows as 8 bits hold them, in fp32."""
    if not form:
        return rows.float()
    groups = _grouped(rows)
    exponent = _exponent(groups, form)
    return torch.ldexp(_codes(groups, exponent, form), exponent).flatten(1)[:, :rows.shape[1]]


def _kept_bytes(rows, form):
    """(values [N, whole groups], scales [N, groups]), uint8: a code each, and the scale's exponent + 127."""
    groups = _grouped(rows)
    exponent = _exponent(groups, form)
    codes = _codes(groups, exponent, form).flatten(1)
    codes = codes.to(torch.int8) if form == "i8" else codes.to(torch.float8_e4m3fn)
    return codes.view(torch.uint8), (exponent + 127).clamp(0, 254).to(torch.uint8).flatten(1)


# ---- one pass ------------------------------------------------------------------------------------------------------

def run(state):
    c = state["case"]
    return (_own if own else _plain)[c["kind"]](c, state)


def _own_keep(c, s):
    import paper_2008_12260_amd as px
    return px.restore(px.keep(s["rows"], c["form"]), s["rows"].dtype)


def _edge_of(px, c, s):
    norm = lambda parts: None if parts is None else px.Norm(*parts)
    return dict(gate=s["gate"], after=norm(s["after"]), before=norm(s["before"]), residual=1.0, scale=0.5, centred=c["centred"])


def _own_edge(c, s):
    import paper_2008_12260_amd as px
    y, rows, _ = px.block_edge(s["x"], s["branch"], **_edge_of(px, c, s), eps=EPS)
    return dict(y=y, rows=rows)


def _own_edge_step(c, s):
    import paper_2008_12260_amd as px
    edge, form = _edge_of(px, c, s), c["form"] or None
    y, rows, state = px.block_edge(s["x"], s["branch"], **edge, eps=EPS, keep=form)
    grads = px.block_edge_grad(s["y_grad"], s["rows_grad"], state, y=None if form else y, branch=None if form else s["branch"], **edge)
    return dict(y=y, rows=rows, **grads._asdict())


def _own_gated(c, s):
    import paper_2008_12260_amd as px
    return px.gated(s["both"][:, :c["F"]], s["both"][:, c["F"]:], c["act"])[0]


def _own_gated_step(c, s):
    import paper_2008_12260_amd as px
    gate, up, form = s["both"][:, :c["F"]], s["both"][:, c["F"]:], c["form"] or None
    rows, gate_kept, up_kept = px.gated(gate, up, c["act"], keep=form)
    gate_grad, up_grad, again = px.gated_grad(s["rows_grad"], gate_kept if form else gate, up_kept if form else up, c["act"], want_rows=True)
    return dict(rows=rows, gate_grad=gate_grad, up_grad=up_grad, again=again)


def _own_kept_grad(c, s):
    import paper_2008_12260_amd as px
    return px.kept_grad(px.Kept(s["values"], s["scales"], c["D"], c["form"]), s["rows_grad"], s["weight"], s["bias"])


_own = dict(keep=_own_keep, edge=_own_edge, edge_step=_own_edge_step, gated=_own_gated, gated_step=_own_gated_step, kept_grad=_own_kept_grad)


def _plain_keep(c, s):
    return _plain_kept(s["rows"], c["form"]).to(s["rows"].dtype)


def _normed(v, centred):
    """(the normalised rows, 1 / their spread) in fp32."""
    if centred:
        v = v - v.mean(1, keepdim=True)
    r = torch.rsqrt(v.square().mean(1, keepdim=True) + EPS)
    return v * r, r


def _weighted(n, parts):
    out = n * parts[0].float()
    return out if parts[1] is None else out + parts[1].float()


def _gate_rows(c, s):
    """The gate of each row, or 1."""
    if s["gate"] is None:
        return 1.0
    gate = s["gate"].float()
    return gate if c["gates"] <= 1 or c["gates"] == c["N"] else gate.repeat_interleave(c["N"] // c["gates"], 0)


def _plain_edge_forward(c, s):
    z = s["branch"].float()
    n, r = _normed(z, c["centred"]) if c["after"] else (z, None)
    b = _weighted(n, s["after"]) if c["after"] else n
    y = s["x"].float() + 0.5 * _gate_rows(c, s) * b
    n_y, r_y = _normed(y, c["centred"])
    return n, r, y, n_y, r_y, _weighted(n_y, s["before"])


def _plain_edge(c, s):
    _, _, y, _, _, h = _plain_edge_forward(c, s)
    return dict(y=y.to(s["x"].dtype), rows=h.to(s["branch"].dtype))


def _norm_grad(d, n, r, centred):
    out = d - n * (d * n).mean(1, keepdim=True)
    return r * (out - d.mean(1, keepdim=True) if centred else out)


def _plain_edge_step(c, s):
    n, r, y, n_y, r_y, h = _plain_edge_forward(c, s)
    xt, dt, wt = s["x"].dtype, s["branch"].dtype, s["before"][0].dtype
    y_out = y.to(xt)
    if c["form"]:
        n, n_y = _plain_kept(n, c["form"]), _plain_kept(n_y, c["form"])
    else:
        n_y = (y_out.float() - (y.mean(1, keepdim=True) if c["centred"] else 0.0)) * r_y
    dh = s["rows_grad"].float()
    g = s["y_grad"].float() + _norm_grad(dh * s["before"][0].float(), n_y, r_y, c["centred"])
    t = 0.5 * g
    b = _weighted(n, s["after"]) if c["after"] else n
    gate_grad = None if s["gate"] is None else (t * b).view(c["gates"], -1, c["D"]).sum(1).view(s["gate"].shape)
    t = t * _gate_rows(c, s)
    total = lambda rows: rows.sum(0).to(wt)
    biased = c["centred"]
    z_grad = _norm_grad(t * s["after"][0].float(), n, r, c["centred"]) if c["after"] else t
    return dict(y=y_out, rows=h.to(dt), x=g.to(xt), branch=z_grad.to(dt), gate=None if gate_grad is None else gate_grad.to(wt),
                after_weight=total(t * n) if c["after"] else None, after_bias=total(t) if c["after"] and biased else None,
                before_weight=total(dh * n_y), before_bias=total(dh) if biased else None)


def _activated(g, act):
    """(the activation, its derivative) in fp32."""
    if act == "silu":
        p = 1.0 / (1.0 + torch.exp(-g))
        return g * p, p * (1.0 + g * (1.0 - p))
    if act == "gelu":
        p = 0.5 * (1.0 + torch.erf(g * math.sqrt(0.5)))
        return g * p, p + g * torch.exp(-0.5 * g * g) * (1.0 / math.sqrt(2.0 * math.pi))
    k = math.sqrt(2.0 / math.pi)
    p = 0.5 * (1.0 + torch.tanh(k * (g + 0.044715 * g * g * g)))
    return g * p, p + 2.0 * g * p * (1.0 - p) * k * (1.0 + 3 * 0.044715 * g * g)


def _plain_gated(c, s):
    g, u = s["both"][:, :c["F"]].float(), s["both"][:, c["F"]:].float()
    return (_activated(g, c["act"])[0] * u).to(s["both"].dtype)


def _plain_gated_step(c, s):
    F, form, dt = c["F"], c["form"], s["both"].dtype
    rows = _plain_gated(c, s)
    g, u, d = _plain_kept(s["both"][:, :F], form), _plain_kept(s["both"][:, F:], form), s["rows_grad"].float()
    a, slope = _activated(g, c["act"])
    return dict(rows=rows, gate_grad=(d * u * slope).to(dt), up_grad=(d * a).to(dt), again=(a * u).to(dt))


def _plain_kept_grad(c, s):
    codes = s["values"].view(torch.int8 if c["form"] == "i8" else torch.float8_e4m3fn).float()
    x = torch.ldexp(codes, s["scales"].int().repeat_interleave(GROUP, 1) - 127)[:, :c["D"]]
    d = s["rows_grad"].float()
    out = d.t() @ x
    if c["weighted"]:
        out = out * s["weight"].float() + d.sum(0)[:, None] * s["bias"].float()
    return out.to(s["rows_grad"].dtype)


_plain = dict(keep=_plain_keep, edge=_plain_edge, edge_step=_plain_edge_step, gated=_plain_gated, gated_step=_plain_gated_step, kept_grad=_plain_kept_grad)


# ---- what a pass cannot do without ---------------------------------------------------------------------------------

def work(case):
    kind, e, N = case["kind"], SIZE[case["type"]], case["N"]
    kept = KEPT if case.get("form") else None
    if kind == "keep":
        n = N * case["D"]
        return dict(bytes=int(n * (2 * e + 2 * kept)), flops=4 * n)
    if kind in ("edge", "edge_step"):
        n, G, ex = N * case["D"], case["gates"], SIZE[case["x_type"]]
        w = ex if case["x_type"] == "fp32" and not kept else e
        parameters = ((2 if case["centred"] else 1) * (2 if case["after"] else 1) + G) * case["D"] * w
        forward, flops = n * (2 * ex + 2 * e) + parameters, 12 * n
        if kind == "edge":
            return dict(bytes=forward, flops=flops)
        # what is remembered is written and read; without a form the rows themselves are read again
        remembered = 4 * n * kept if kept else n * (ex + e)
        return dict(bytes=int(forward + remembered + n * (2 * ex + 2 * e) + 2 * parameters), flops=flops + 24 * n)
    if kind in ("gated", "gated_step"):
        n = N * case["F"]
        if kind == "gated":
            return dict(bytes=3 * n * e, flops=8 * n)
        return dict(bytes=int(3 * n * e + (4 * n * kept if kept else 2 * n * e) + 4 * n * e), flops=24 * n)
    D, M = case["D"], case["M"]
    return dict(bytes=int(N * D * kept + N * M * e + D * M * e), flops=2 * N * D * M)


# ---- the outputs in 64 bits ----------------------------------------------------------------------------------------

def _exact_kept(rows, form):
    """Rows as 8 bits hold them.  The scale from the largest element's bits; rounding by a sum with a number whose last bit is the step."""
    v = rows.double()
    if not form:
        return v
    N, D = v.shape
    v = torch.nn.functional.pad(v, (0, -D % GROUP)).unflatten(1, (-1, GROUP))
    bits = v.abs().amax(2, keepdim=True).view(torch.int64)
    # one more where the fraction is from 127/128 (above 3/4) on
    bits = bits + ((1 << 45) if form == "i8" else (1 << 50) - 1)
    scale = torch.exp2(((bits >> 52) - 1023 - (6 if form == "i8" else 8)).clamp(min=-127).double())
    q = v / scale
    step = 1.0
    if form != "i8":
        exponent = ((q.abs().view(torch.int64) >> 52) - 1023).clamp(min=-6)
        step = torch.exp2((exponent - 3).double())
    magic = step * (1.5 * 2.0 ** 52)
    return (((q + magic) - magic) * scale).flatten(1)[:, :D]


def exact(case, seed):
    s, kind = prepare(case, seed), case["kind"]
    N = case["N"]
    if kind == "keep":
        return _exact_kept(s["rows"], case["form"])
    if kind in ("edge", "edge_step"):
        D, G, centred = case["D"], case["gates"], case["centred"]

        def normed(v):
            mean = v.sum(1, keepdim=True) / D if centred else torch.zeros((N, 1), dtype=v.dtype, device=v.device)
            spread = (torch.linalg.vector_norm(v - mean, dim=1, keepdim=True) ** 2 / D + EPS) ** 0.5
            return (v - mean) / spread, spread

        double = lambda t: None if t is None else t.double()
        part = lambda parts, k: double(parts[k]) if parts is not None and parts[k] is not None else None
        w_a, b_a, w_b, b_b = part(s["after"], 0), part(s["after"], 1), part(s["before"], 0), part(s["before"], 1)
        gate = torch.ones((1, D), dtype=torch.float64, device="cuda") if s["gate"] is None else double(s["gate"]).view(-1, D)
        of_row = torch.arange(N, device="cuda") // max(1, N // gate.shape[0])
        z = double(s["branch"])
        n_z, spread_z = normed(z) if case["after"] else (z, None)

        def after(n):
            if w_a is None:
                return n
            return n * w_a if b_a is None else torch.addcmul(b_a, n, w_a)

        y = torch.addcmul(double(s["x"]), gate[of_row], after(n_z), value=0.5)
        n_y, spread_y = normed(y)
        h = n_y * w_b if b_b is None else torch.addcmul(b_b, n_y, w_b)
        out = dict(y=y, rows=h)
        if kind == "edge":
            return out
        if case["form"]:
            n_z, n_y = _exact_kept(n_z, case["form"]), _exact_kept(n_y, case["form"])

        def through(d, n, spread):
            """What remains of d without its parts along n and, with means, along ones."""
            along = torch.einsum("ij,ij->i", d, n)[:, None] / D
            d = torch.addcmul(d, n, along, value=-1.0)
            return (d - d.sum(1, keepdim=True) / D - (n.sum(1, keepdim=True) / D) * along if centred else d) / spread

        dh = double(s["rows_grad"])
        g = double(s["y_grad"]) + through(dh * w_b, n_y, spread_y)
        b = after(n_z)
        shared = torch.zeros((gate.shape[0], D), dtype=torch.float64, device="cuda").index_add_(0, of_row, g * b) * 0.5
        t = g * gate[of_row] * 0.5
        ones = torch.ones((1, N), dtype=torch.float64, device="cuda")
        out.update(x=g, branch=through(t * w_a, n_z, spread_z) if case["after"] else t, gate=None if s["gate"] is None else shared.view(s["gate"].shape),
                   after_weight=torch.mm(ones, t * n_z)[0] if case["after"] else None, after_bias=torch.mm(ones, t)[0] if b_a is not None else None,
                   before_weight=torch.mm(ones, dh * n_y)[0], before_bias=torch.mm(ones, dh)[0] if b_b is not None else None)
        return out
    if kind in ("gated", "gated_step"):
        F = case["F"]
        act = dict(silu=torch.nn.functional.silu, gelu=torch.nn.functional.gelu,
                   gelu_tanh=lambda v: torch.nn.functional.gelu(v, approximate="tanh"))[case["act"]]
        rows = act(s["both"][:, :F].double()) * s["both"][:, F:].double()
        if kind == "gated":
            return rows
        g, u, d = _exact_kept(s["both"][:, :F], case["form"]).requires_grad_(), _exact_kept(s["both"][:, F:], case["form"]), s["rows_grad"].double()
        a = act(g)
        slope, = torch.autograd.grad(a, g, d * u)
        a = a.detach()
        return dict(rows=rows, gate_grad=slope, up_grad=d * a, again=a * u)
    # products of some tokens at a time, the scales multiplied in last
    D, M = case["D"], case["M"]
    codes = s["values"].view(torch.int8 if case["form"] == "i8" else torch.float8_e4m3fn)
    out, sums = torch.zeros((M, D), dtype=torch.float64, device="cuda"), torch.zeros(M, dtype=torch.float64, device="cuda")
    for at in range(0, N, 4096):
        scale = torch.exp2(s["scales"][at:at + 4096].double() - 127.0)
        x = (codes[at:at + 4096].double().unflatten(1, (-1, GROUP)) * scale[:, :, None]).flatten(1)[:, :D]
        d = s["rows_grad"][at:at + 4096].double()
        out += torch.mm(d.t(), x)
        sums += d.sum(0)
    if case["weighted"]:
        out = out * s["weight"].double() + torch.outer(sums, s["bias"].double())
    return out
