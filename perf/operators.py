"""The operators of a language-model job's training iteration, timed: what a job's agent runs to obtain the gradients whose
noise scale, and the iterations whose times, the scheduler is given.

  embed          rows of a table looked up by token and scaled
  embed_grad     the table's gradient from the rows' gradients
  loss           cross entropy of each token over a vocabulary, from hidden rows and the projection's weights
  loss_step      the same, and the gradients of the hidden rows and of the weights
  noise          the mean of several gradients and the gradient noise scale that they show
  orthogonalize  an update orthogonalised by Newton-Schulz products

A case is a dict of plain values.  `prepare` draws its inputs on the GPU from a seed alone, `run` is one pass (in elementary torch
operations, or through the package's entry points where `own` is true), `work` says what a pass cannot do without, `exact` gives
the outputs in 64 bits.
"""
import math

import torch

own = False

TYPES = {"fp32": torch.float32, "bf16": torch.bfloat16, "fp16": torch.float16}
SIZE = {"fp32": 4, "bf16": 2, "fp16": 2}
NEWTON_SCHULZ = (3.4445, -4.7750, 2.0315)
LARGEST = 8192 * 131072 * 4096          # tokens x vocabulary x width of the largest listed loss


def listed():
    """The listed cases; each stands for the use its comment names."""
    return [
        # eight sequences asked for their next token: the call is latency
        dict(name="lookup_few", kind="embed", N=8, V=32768, D=1024, type="bf16", scale=32.0),
        # the first operator of a large micro-batch, rows scaled by the root of the width
        dict(name="lookup_batch", kind="embed", N=16384, V=131072, D=4096, type="bf16", scale=64.0),
        # a small job in single precision whose sizes are nobody's round numbers, a tenth of its tokens padding
        dict(name="lookup_grad_odd", kind="embed_grad", N=5003, V=20011, D=1000, type="fp32", scale=1.0, ignored=0.1),
        # the last operator of a micro-batch: tokens as frequent as words are, a few of them in thousands of places
        dict(name="lookup_grad", kind="embed_grad", N=16384, V=65536, D=2048, type="bf16", scale=1.0),
        # the losses of a few tokens under a large model's projection: reading the weights is all there is
        dict(name="score_few", kind="loss", N=3, V=131072, D=4096, type="bf16"),
        # a small job in single precision: loss and gradients of a micro-batch
        dict(name="step_small_fp32", kind="loss_step", N=512, V=8192, D=512, type="fp32"),
        # odd sizes in half precision with a scaled loss, a fifth of the targets masked (prompts that are not trained on)
        dict(name="step_odd_fp16", kind="loss_step", N=1501, V=50021, D=1000, type="fp16", ignored=0.2, loss_scale=4096.0),
        # a large model's micro-batch of 8192 tokens
        dict(name="step_large", kind="loss_step", N=8192, V=131072, D=4096, type="bf16"),
        # the estimate of a small job: the gradients of two micro-batches
        dict(name="noise_small", kind="noise", B=2, n=1000003, type="bf16", examples=8.0),
        # a large job with eight micro-batches an iteration (seven accumulation steps), pre-conditioned
        dict(name="noise_large", kind="noise", B=8, n=1 << 27, type="bf16", examples=16.0, preconditioned=True),
        # the layers of a small model, updated in one call
        dict(name="update_small", kind="orthogonalize", batch=12, rows=384, cols=640, type="fp32", steps=5),
        # one large matrix of a large model, taller than wide
        dict(name="update_large", kind="orthogonalize", batch=1, rows=8192, cols=4096, type="bf16", steps=5),
    ]


def draw(rng):
    """One more case of the ranges the listed ones stand for."""
    def log_int(lo, hi):
        return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))

    def width(lo, hi):
        d = log_int(lo, hi)
        return d if rng.random() < 0.35 else max(lo, d // 64 * 64)

    kind = rng.choice(["embed", "embed_grad", "loss", "loss_step", "loss_step", "noise", "orthogonalize"])
    if kind in ("embed", "embed_grad"):
        D = width(64, 4096)
        return dict(kind=kind, N=log_int(1, 16384), V=min(log_int(1000, 131072), (1 << 28) // D), D=D,
                    type=rng.choice(["bf16", "bf16", "fp16", "fp32"]), scale=rng.choice([1.0, math.sqrt(D)]),
                    ignored=rng.choice([0.0, 0.0, 0.1]))
    if kind in ("loss", "loss_step"):
        type_ = rng.choice(["bf16", "bf16", "fp16", "fp32"])
        while True:
            N, V, D = log_int(1, 16384), log_int(1000, 131072), width(64, 4096)
            if N * V * D <= LARGEST // (16 if type_ == "fp32" else 1):
                break
        case = dict(kind=kind, N=N, V=V, D=D, type=type_, ignored=rng.choice([0.0, 0.0, 0.2]))
        if type_ == "fp16":
            case["loss_scale"] = 4096.0
        return case
    if kind == "noise":
        B = rng.randint(2, 16)
        return dict(kind=kind, B=B, n=min(log_int(1000, 1 << 27), (1 << 30) // B), type=rng.choice(["bf16", "bf16", "fp16", "fp32"]),
                    examples=float(log_int(1, 512)), preconditioned=rng.random() < 0.5)
    while True:
        rows, cols, batch = width(64, 8192), width(64, 8192), log_int(1, 24)
        if batch * min(rows, cols) ** 2 * max(rows, cols) <= 4096 * 4096 * 8192:
            return dict(kind=kind, batch=batch, rows=rows, cols=cols, type=rng.choice(["bf16", "bf16", "fp32"]), steps=5)


# ---- inputs --------------------------------------------------------------------------------------------------------

def _tokens(N, V, ignored, g):
    """Tokens as frequent as words are (the k-th most frequent about 1/k as often as the first), the frequent ones anywhere in the
    vocabulary; a share of them -1, which stands for none."""
    u = torch.rand(N, generator=g, device="cuda", dtype=torch.float64)
    rank = (torch.exp(u * math.log(V + 1.0)) - 1.0).long().clamp_(0, V - 1)
    tokens = torch.randperm(V, generator=g, device="cuda")[rank]
    if ignored:
        tokens = torch.where(torch.rand(N, generator=g, device="cuda") < ignored, -1, tokens)
    return tokens


def prepare(case, seed):
    g = torch.Generator("cuda").manual_seed(seed)
    kind, dt = case["kind"], TYPES[case["type"]]

    def normal(*shape, std=1.0):
        return (torch.randn(shape, generator=g, device="cuda", dtype=torch.float32) * std).to(dt)

    state = dict(case=case)
    if kind in ("embed", "embed_grad"):
        N, V, D = case["N"], case["V"], case["D"]
        state["tokens"] = _tokens(N, V, case.get("ignored", 0.0), g)
        if kind == "embed":
            state["table"] = normal(V, D, std=0.02)
        else:
            state["rows_grad"] = normal(N, D, std=0.01)
    elif kind in ("loss", "loss_step"):
        # weights of the usual scale; hidden rows that lean towards their target's weights, as those of a model in training do
        N, V, D = case["N"], case["V"], case["D"]
        state["targets"] = _tokens(N, V, case.get("ignored", 0.0), g)
        state["weight"] = normal(V, D, std=D ** -0.5)
        towards = state["weight"][state["targets"].clamp(min=0)].float()
        lean = 6.0 * torch.rand((N, 1), generator=g, device="cuda")
        state["hidden"] = (torch.randn((N, D), generator=g, device="cuda") * 1.5 + lean * towards).to(dt)
        # the mean over the tokens that count, times the scale that half precision needs
        counts = (state["targets"] >= 0).sum().clamp(min=1)
        state["row_weight"] = torch.where(state["targets"] >= 0, case.get("loss_scale", 1.0) / counts, 0.0).float()
    elif kind == "noise":
        # gradients with a common part, and elements of very different sizes
        B, n = case["B"], case["n"]
        size = torch.exp(torch.randn(n, generator=g, device="cuda")) * 1e-3
        common = torch.randn(n, generator=g, device="cuda")
        grads = torch.empty((B, n), dtype=dt, device="cuda")
        for i in range(B):
            grads[i] = (size * (common + torch.randn(n, generator=g, device="cuda"))).to(dt)
        state["grads"] = grads
        state["precondition"] = 1.0 / (size + 1e-4) if case.get("preconditioned") else None
    else:
        # a gradient of a few strong directions over noise
        batch, rows, cols = case["batch"], case["rows"], case["cols"]
        strong = torch.matmul(torch.randn((batch, rows, 8), generator=g, device="cuda"), torch.randn((batch, 8, cols), generator=g, device="cuda"))
        state["grads"] = ((torch.randn((batch, rows, cols), generator=g, device="cuda") + 0.3 * strong) * 1e-3).to(dt)
    return state


# ---- one pass ------------------------------------------------------------------------------------------------------

def run(state):
    c = state["case"]
    return (_own if own else _plain)[c["kind"]](c, state)


def _own_loss_step(c, s):
    import paper_2008_12260_amd as px
    loss, lse = px.token_loss(s["hidden"], s["weight"], s["targets"])
    hidden_grad, weight_grad = px.token_loss_grad(s["hidden"], s["weight"], s["targets"], lse, s["row_weight"])
    return dict(loss=loss, lse=lse, hidden_grad=hidden_grad, weight_grad=weight_grad)


def _own_embed(c, s):
    import paper_2008_12260_amd as px
    return px.embed(s["tokens"], s["table"], c["scale"])


def _own_embed_grad(c, s):
    import paper_2008_12260_amd as px
    return px.embed_grad(s["tokens"], s["rows_grad"], c["V"], c["scale"])


def _own_loss(c, s):
    import paper_2008_12260_amd as px
    loss, lse = px.token_loss(s["hidden"], s["weight"], s["targets"])
    return dict(loss=loss, lse=lse)


def _own_noise(c, s):
    import paper_2008_12260_amd as px
    mean, scale = px.noise_scale(s["grads"], c["examples"], s["precondition"])
    return dict(mean=mean, scale=scale)


def _own_orthogonalize(c, s):
    import paper_2008_12260_amd as px
    return px.orthogonalize(s["grads"], c["steps"], NEWTON_SCHULZ)


_own = dict(embed=_own_embed, embed_grad=_own_embed_grad, loss=_own_loss, loss_step=_own_loss_step, noise=_own_noise,
            orthogonalize=_own_orthogonalize)


def _plain_embed(c, s):
    tokens, table = s["tokens"], s["table"]
    rows = table[tokens.clamp(min=0)].float() * c["scale"]
    return torch.where(tokens[:, None] >= 0, rows, 0.0).to(table.dtype)


def _plain_embed_grad(c, s):
    tokens, rows_grad = s["tokens"], s["rows_grad"]
    rows = torch.where(tokens[:, None] >= 0, rows_grad.float(), 0.0)
    total = torch.zeros((c["V"], c["D"]), dtype=torch.float32, device=rows.device)
    total.index_add_(0, tokens.clamp(min=0), rows)
    return (total * c["scale"]).to(rows_grad.dtype)


def _plain_logits(s):
    """(logits less the row's largest, that largest, the sum of their exponentials, the logits' logsumexp, the loss)."""
    logits = s["hidden"].float() @ s["weight"].float().T
    top = logits.amax(1, keepdim=True)
    logits -= top
    picked = logits.gather(1, s["targets"].clamp(min=0)[:, None])[:, 0] + top[:, 0]
    logits.exp_()
    total = logits.sum(1, keepdim=True)
    lse = (top + torch.log(total))[:, 0]
    loss = torch.where(s["targets"] >= 0, lse - picked, 0.0)
    return logits, total, lse, loss


def _plain_loss(c, s):
    _, _, lse, loss = _plain_logits(s)
    return dict(loss=loss, lse=lse)


def _plain_loss_step(c, s):
    q, total, lse, loss = _plain_logits(s)
    q /= total
    q.scatter_add_(1, s["targets"].clamp(min=0)[:, None], torch.full_like(total, -1.0))
    q *= s["row_weight"][:, None]
    dt = s["hidden"].dtype
    return dict(loss=loss, lse=lse, hidden_grad=(q @ s["weight"].float()).to(dt), weight_grad=(q.T @ s["hidden"].float()).to(dt))


def _noise(grads, mean, squares, precondition, examples):
    """[tr(P Sigma P'), |P g|^2, their quotient] from the sum over the gradients of the squared deviations, element by element."""
    weight = 1.0 if precondition is None else precondition.double().square()
    B = grads.shape[0]
    trace = examples / (B - 1) * (squares * weight).sum()
    norm = (mean.square() * weight).sum() - trace / (examples * B)
    return torch.stack([trace, norm, trace / norm])


def _plain_noise(c, s):
    # sums of 10^8 squares, and a difference of two of them: 64 bits
    grads = s["grads"]
    mean = grads.sum(0, dtype=torch.float64) / c["B"]
    squares = (grads[0].double() - mean).square()
    for i in range(1, c["B"]):
        squares += (grads[i].double() - mean).square()
    return dict(mean=mean.float(), scale=_noise(grads, mean, squares, s["precondition"], c["examples"]))


def _plain_orthogonalize(c, s):
    a, b, d = NEWTON_SCHULZ
    x = s["grads"].float()
    tall = c["rows"] > c["cols"]
    if tall:
        x = x.transpose(1, 2).contiguous()
    x = x / torch.sqrt(x.square().sum((1, 2), keepdim=True))
    for _ in range(c["steps"]):
        xx = torch.matmul(x, x.transpose(1, 2).contiguous())
        x = a * x + torch.matmul(b * xx + d * torch.matmul(xx, xx), x)
    if tall:
        x = x.transpose(1, 2)
    return x.to(torch.bfloat16).contiguous()


_plain = dict(embed=_plain_embed, embed_grad=_plain_embed_grad, loss=_plain_loss, loss_step=_plain_loss_step, noise=_plain_noise,
              orthogonalize=_plain_orthogonalize)


# ---- what a pass cannot do without ---------------------------------------------------------------------------------

def work(case):
    kind, e = case["kind"], SIZE[case["type"]]
    if kind == "embed":
        N, V, D = case["N"], case["V"], case["D"]
        return dict(bytes=8 * N + min(N, V) * D * e + N * D * e, flops=N * D)
    if kind == "embed_grad":
        N, V, D = case["N"], case["V"], case["D"]
        return dict(bytes=8 * N + N * D * e + V * D * e, flops=N * D)
    if kind in ("loss", "loss_step"):
        # logits once, and for the gradients one product each for the hidden rows and the weights
        N, V, D = case["N"], case["V"], case["D"]
        read = (N + V) * D * e + 16 * N
        return dict(bytes=read, flops=2 * N * V * D) if kind == "loss" else dict(bytes=read + (N + V) * D * e, flops=6 * N * V * D)
    if kind == "noise":
        B, n = case["B"], case["n"]
        return dict(bytes=B * n * e + 4 * n + (4 * n if case.get("preconditioned") else 0), flops=5 * B * n)
    # two symmetric products (half of each) and a full one a step
    m, n = min(case["rows"], case["cols"]), max(case["rows"], case["cols"])
    return dict(bytes=case["batch"] * m * n * (e + 2), flops=case["batch"] * case["steps"] * (3 * m * m * n + m ** 3))


# ---- the outputs in 64 bits ----------------------------------------------------------------------------------------

def exact(case, seed):
    s, kind = prepare(case, seed), case["kind"]
    if kind == "embed":
        kept = (s["tokens"] >= 0).double()[:, None]
        return s["table"].double().index_select(0, s["tokens"].clamp(min=0)) * (kept * case["scale"])
    if kind == "embed_grad":
        # tokens in order, the running sum's differences at their borders: a slice of the width at a time
        order = torch.argsort(s["tokens"], stable=True)
        ordered = s["tokens"][order]
        last = torch.searchsorted(ordered, torch.arange(case["V"], device="cuda"), right=True)
        first = torch.searchsorted(ordered, torch.arange(case["V"], device="cuda"), right=False)
        out = torch.empty((case["V"], case["D"]), dtype=torch.float64, device="cuda")
        for at in range(0, case["D"], 256):
            run_sum = torch.cumsum(s["rows_grad"][order, at:at + 256].double(), 0)
            run_sum = torch.cat([torch.zeros_like(run_sum[:1]), run_sum])
            out[:, at:at + 256] = (run_sum[last] - run_sum[first]) * case["scale"]
        return out
    if kind in ("loss", "loss_step"):
        hidden, weight, targets = s["hidden"].double(), s["weight"].double(), s["targets"]
        N, V = case["N"], case["V"]
        counted = targets >= 0
        lse, loss = torch.empty(N, dtype=torch.float64, device="cuda"), torch.zeros(N, dtype=torch.float64, device="cuda")
        grads = kind == "loss_step"
        hidden_grad, weight_grad = torch.empty_like(hidden) if grads else None, torch.zeros_like(weight) if grads else None
        for at in range(0, N, 1024):                      # some tokens at a time, all of their logits
            to = min(N, at + 1024)
            logits = torch.mm(hidden[at:to], weight.t())
            lse[at:to] = torch.logsumexp(logits, 1)
            here = torch.nonzero(counted[at:to])[:, 0]
            loss[at + here] = lse[at + here] - logits[here, targets[at + here]]
            if grads:
                q = torch.exp(logits - lse[at:to, None])
                q[here, targets[at + here]] -= 1.0
                q *= s["row_weight"][at:to, None].double()
                hidden_grad[at:to] = torch.mm(q, weight)
                weight_grad += torch.mm(q.t(), hidden[at:to])
        return dict(loss=loss, lse=lse, hidden_grad=hidden_grad, weight_grad=weight_grad) if grads else dict(loss=loss, lse=lse)
    if kind == "noise":
        # the mean over all pairs of half their squared distance is the variance; here through sums and products of the gradients
        B, b, grads = case["B"], case["examples"], s["grads"]
        p = torch.ones(case["n"], dtype=torch.float64, device="cuda") if s["precondition"] is None else s["precondition"].double()
        total = torch.zeros(case["n"], dtype=torch.float64, device="cuda")
        spread = torch.zeros((), dtype=torch.float64, device="cuda")
        for i in range(B):
            total += grads[i]
            for k in range(i):
                spread += torch.linalg.vector_norm((grads[i].double() - grads[k].double()) * p) ** 2
        trace = b * spread / (B * (B - 1))
        mean = total / B
        norm = torch.linalg.vector_norm(mean * p) ** 2 - trace / (b * B)
        return dict(mean=mean, scale=torch.stack([trace, norm, trace / norm]))
    a, b, d = NEWTON_SCHULZ
    out = []
    for g in s["grads"].double():
        x = g / torch.linalg.matrix_norm(g)
        for _ in range(case["steps"]):
            if case["rows"] <= case["cols"]:              # a X + b (X X') X + c (X X')^2 X, from whichever side is smaller
                y = torch.mm(x, x.t())
                x = a * x + torch.mm(b * y + d * torch.mm(y, y), x)
            else:
                y = torch.mm(x.t(), x)
                x = a * x + torch.mm(x, b * y + d * torch.mm(y, y))
        out.append(x)
    return torch.stack(out)
