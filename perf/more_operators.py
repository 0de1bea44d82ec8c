"""The end of a language model's training step as users of this library call it, as timed cases.

A case is a dict of plain values. Three kinds:

  norm  root-mean-square norm of a sum (an input and the residual stream), forward
        or backward
  head  softmax cross entropy of the head layer without keeping its logits: the
        loss alone, or the loss and every gradient; the layer's inputs may carry a
        row pattern
  muon  momentum update of a weight matrix by the orthogonalised kept block of the
        layer's row patterns

With ``own`` true, run() makes the calls of paper_1805_08939_amd.api; otherwise
it computes the same from elementary torch operations in 32 bits. A pattern's
period is part of the case (it sets the work); a pattern's offset, like every
input, comes from the seed.
"""

import math

import torch

own = False

DEV = "cuda:0"
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16}
EPS = 1e-5
LR, MOMENTUM, DECAY, NORM_EPS = 0.02, 0.95, 0.01, 1e-7
A, B, C = 3.4445, -4.7750, 2.0315  # of the polynomial that an iteration applies to the singular values
ITERATIONS = 5


def listed():
    return [
        # serving a single token: latency
        dict(name="norm-fwd-1024-bf16-b1", kind="norm", way="fwd", dtype="bf16", batch=1, features=1024, residual=True),
        # training next to the wide layers, forward and backward
        dict(name="norm-fwd-8192-bf16-b2048", kind="norm", way="fwd", dtype="bf16", batch=2048, features=8192,
             residual=True),
        dict(name="norm-bwd-8192-bf16-b2048", kind="norm", way="bwd", dtype="bf16", batch=2048, features=8192,
             residual=True),
        # the ten classes behind a 2048-unit layer, one batch
        dict(name="head-10-f32-b128", kind="head", way="train", dtype="f32", batch=128, inputs=2048, classes=10,
             period=2, major="in"),
        # the 8800-word head behind 1500 recurrent units of which every other is dropped, 35 steps of batch 20
        dict(name="head-8800-f32-b700", kind="head", way="train", dtype="f32", batch=700, inputs=1500, classes=8800,
             period=2, major="in"),
        # sizes that fit no tile and rows that fit no 16 bytes
        dict(name="head-5001-bf16-b331", kind="head", way="train", dtype="bf16", batch=331, inputs=1023, classes=5001,
             period=1, major="out"),
        # scoring a text: the loss alone
        dict(name="head-loss-32000-bf16-b512", kind="head", way="loss", dtype="bf16", batch=512, inputs=1024,
             classes=32000, period=1, major="out"),
        # a large vocabulary and a long batch of tokens in training
        dict(name="head-32000-bf16-b4096", kind="head", way="train", dtype="bf16", batch=4096, inputs=4096,
             classes=32000, period=1, major="out"),
        # a small layer: latency of a chain of small products
        dict(name="muon-512x784-f32", kind="muon", dtype="f32", outputs=512, inputs=784, out_period=1, in_period=1,
             major="out", grad="full"),
        # odd sizes, a third of the outputs kept
        dict(name="muon-1537x1023-bf16", kind="muon", dtype="bf16", outputs=1537, inputs=1023, out_period=3,
             in_period=1, major="out", grad="full"),
        # the gates of 1500 recurrent units in fp32, every input kept
        dict(name="muon-6000x1500-f32", kind="muon", dtype="f32", outputs=6000, inputs=1500, out_period=1, in_period=1,
             major="out", grad="full"),
        # the wide layer, every other unit kept on both sides, with the gradient of the compact weights
        dict(name="muon-8192x8192-bf16", kind="muon", dtype="bf16", outputs=8192, inputs=8192, out_period=2,
             in_period=2, major="out", grad="compact"),
    ]


def _log(rng, lo, hi):
    return max(lo, min(hi, round(math.exp(rng.uniform(math.log(lo), math.log(hi))))))


def draw(rng):
    """One more case of the same ranges; never more work than the largest listed one of its kind."""
    kind = rng.choice(["norm", "head", "head", "muon", "muon"])
    most = max(_cost(c) for c in listed() if c["kind"] == kind)
    whole = lambda n, of: (n + of - 1) // of * of if rng.random() < 0.6 else n  # noqa: E731
    while True:
        dtype = rng.choice(["f32", "bf16", "bf16"])
        if kind == "norm":
            c = dict(kind="norm", way=rng.choice(["fwd", "bwd"]), dtype=dtype, batch=_log(rng, 1, 8192),
                     features=whole(_log(rng, 64, 8192), 64), residual=rng.random() < 0.7)
            if c["batch"] > 16:
                c["batch"] = whole(c["batch"], 8)
        elif kind == "head":
            c = dict(kind="head", way=rng.choice(["train", "train", "loss"]), dtype=dtype,
                     batch=whole(_log(rng, 8, 4096), 8), inputs=whole(_log(rng, 64, 4096), 32),
                     classes=whole(_log(rng, 10, 32000), 8), period=rng.choice([1, 1, 1, 2, 3]),
                     major=rng.choice(["out", "out", "in"]))
        else:
            c = dict(kind="muon", dtype=dtype, outputs=whole(_log(rng, 64, 8192), 64),
                     inputs=whole(_log(rng, 64, 8192), 64), out_period=rng.choice([1, 1, 2, 3]),
                     in_period=rng.choice([1, 1, 2, 3]), major="out", grad="full")
            if c["in_period"] > 1 and rng.random() < 0.7:
                c["grad"] = "compact"
            elif c["out_period"] == 1 and rng.random() < 0.4:
                c["major"] = "in"
        if _cost(c) <= most:
            return c


# --------------------------------------------------------------------- shared

def _kept(n, period, offset):
    return len(range(offset, n, period))


def _cost(case):
    w = work(case)
    rate = 1e14 if case["dtype"] == "f32" else 1e15
    if case["kind"] == "muon":
        rate = min(rate, 4e14)
    return max(w["bytes"] / 4e12, w["flops"] / rate)


def work(case):
    es = 4 if case["dtype"] == "f32" else 2
    if case["kind"] == "norm":
        n = case["batch"] * case["features"]
        arrays = 4 if case["residual"] else (2 if case["way"] == "fwd" else 3)
        return {"bytes": es * arrays * n + 4 * case["batch"] + 8 * case["features"],
                "flops": (5 if case["way"] == "fwd" else 10) * n}
    if case["kind"] == "head":
        v, b, p = case["classes"], case["batch"], case["period"]
        k = _kept(case["inputs"], p, p // 2)
        if case["way"] == "loss":
            return {"bytes": es * (v * k + k * b) + 4 * v + 8 * b, "flops": 2 * v * k * b}
        # the logits, dX and dW; the gradients are written whole
        return {"bytes": es * (v * k + k * b + case["inputs"] * (v + b)) + 8 * v + 12 * b, "flops": 6 * v * k * b}
    n, k = _kept(case["outputs"], case["out_period"], case["out_period"] // 2), \
        _kept(case["inputs"], case["in_period"], case["in_period"] // 2)
    m, l = min(n, k), max(n, k)
    # both products of a matrix with its own transpose are symmetric
    return {"bytes": n * k * (2 * es + 12), "flops": ITERATIONS * (m * m * l + m * m * m + 2 * m * m * l)}


class _Draws:
    def __init__(self, seed):
        self.g = torch.Generator(device=DEV)
        self.g.manual_seed(seed)

    def normal(self, *shape, std=1.0, dtype=torch.float32):
        return (torch.randn(*shape, generator=self.g, device=DEV) * std).to(dtype)

    def below(self, n, *shape):
        return torch.randint(0, n, shape, generator=self.g, device=DEV, dtype=torch.int64)

    def gradient(self, rows, cols, std):
        """A few strong directions above noise, as gradients of weights are."""
        r = max(1, min(rows, cols) // 16)
        return (self.normal(rows, r) @ self.normal(r, cols) / math.sqrt(r) + self.normal(rows, cols, std=0.3)) * std


def prepare(case, seed):
    d, t = _Draws(seed), TYPES[case["dtype"]]
    s = {"case": case}
    if case["kind"] == "norm":
        k, b = case["features"], case["batch"]
        # a residual stream with a few features far larger than the others
        wide = 1.0 + 20.0 * (torch.arange(k, device=DEV) % 97 == seed % 97)[:, None]
        s["gain"] = 1.0 + d.normal(k, std=0.2)
        if case["way"] == "fwd":
            s["X"] = d.normal(k, b, dtype=t)
            s["R"] = (d.normal(k, b) * wide).to(t) if case["residual"] else None
        else:
            s["S"] = (d.normal(k, b) * wide).to(t)
            s["inv"] = (s["S"].double().square().mean(0) + EPS).rsqrt().float()
            s["dY"] = d.normal(k, b, std=1e-3, dtype=t)
            s["dS"] = d.normal(k, b, std=1e-3, dtype=t) if case["residual"] else None
    elif case["kind"] == "head":
        v, k, b = case["classes"], case["inputs"], case["batch"]
        s["offset"] = seed % case["period"]
        s["X"] = d.normal(k, b, dtype=t)
        std = 2.5 / math.sqrt(k / case["period"])  # logits of a trained model spread by a few units
        s["W"] = d.normal(v, k, std=std, dtype=t) if case["major"] == "out" else d.normal(k, v, std=std, dtype=t)
        s["bias"] = d.normal(v, std=0.5)
        s["labels"] = d.below(v, b).to(torch.int32)
        s["labels"][3::16] = -1  # padding
        s["dloss"] = torch.full((b,), 1.0 / b, device=DEV)
    else:
        n, k = case["outputs"], case["inputs"]
        s["out_offset"], s["in_offset"] = seed % case["out_period"], seed % case["in_period"]
        shape = (n, k) if case["major"] == "out" else (k, n)
        s["W0"] = d.normal(*shape, std=1.0 / math.sqrt(k), dtype=t)
        s["V0"] = d.gradient(*shape, 1e-2)
        if case["grad"] == "compact":
            rows = _kept(n, case["out_period"], s["out_offset"])
            cols = _kept(k, case["in_period"], s["in_offset"])
            s["dW"] = d.gradient(rows, (cols + 7) // 8 * 8, 1e-3)
        else:
            s["dW"] = d.gradient(*shape, 1e-3)
        s["W"], s["V"] = torch.empty_like(s["W0"]), torch.empty_like(s["V0"])
    return s


def run(state):
    case = state["case"]
    if own:
        if "call" not in state:  # descriptors, outputs and workspaces that a program makes once
            state["call"] = {"norm": _own_norm, "head": _own_head, "muon": _own_muon}[case["kind"]](state)
        return state["call"]()
    return {"norm": _plain_norm, "head": _plain_head, "muon": _plain_muon}[case["kind"]](state)


# --------------------------------------------------------------------- the framework's calls
# Addresses are looked up once, the stream at each pass.

def _at(*tensors):
    return tuple(None if x is None else x.data_ptr() for x in tensors)


def _stream():
    return torch.cuda.current_stream().cuda_stream


def _space(nbytes):
    ws = torch.empty(max(nbytes, 16) // 4 + 4, dtype=torch.float32, device=DEV)
    return ws, (ws.data_ptr(), ws.numel() * 4)


def _own_norm(s):
    from paper_1805_08939_amd import api

    case = s["case"]
    k, b, t = case["features"], case["batch"], TYPES[case["dtype"]]
    desc = api.rmsnorm_desc(api.ARD_BF16 if case["dtype"] == "bf16" else api.ARD_F32, b, k, EPS)
    s["space"], ws = _space(api.ard_rmsnorm_workspace_bytes(desc))
    if case["way"] == "fwd":
        Y, inv = torch.empty(k, b, dtype=t, device=DEV), torch.empty(b, device=DEV)
        S = torch.empty_like(Y) if case["residual"] else None
        out = (Y, S, inv) if case["residual"] else (Y, inv)
        at = _at(s["X"], s["R"], s["gain"], S, Y, inv)

        def fwd():
            api.ard_rmsnorm_fwd(desc, *at, ws, _stream())
            return out
        return fwd
    out = (torch.empty(k, b, dtype=t, device=DEV), torch.empty(k, device=DEV))
    at = _at(s["S"], s["gain"], s["inv"], s["dY"], s["dS"], *out)

    def bwd():
        api.ard_rmsnorm_bwd(desc, *at, ws, _stream())
        return out
    return bwd


def _own_head(s):
    from paper_1805_08939_amd import api

    case = s["case"]
    v, k, b, t = case["classes"], case["inputs"], case["batch"], TYPES[case["dtype"]]
    dt = api.ARD_BF16 if case["dtype"] == "bf16" else api.ARD_F32
    plan = api.ard_plan_rows(k, case["period"], s["offset"], None)
    layout = api.ARD_WEIGHTS_FULL if case["major"] == "out" else api.ARD_WEIGHTS_INPUT_MAJOR
    desc = api.headloss_desc(dt, b, k, v, plan, layout, api.ARD_DROPPED_ZERO, grad_dtype=dt)
    s["space"], ws = _space(api.ard_headloss_workspace_bytes(desc))
    s["stats"] = torch.empty(2, b, device=DEV)
    loss = torch.empty(b, device=DEV)
    told = _at(s["X"], s["W"], s["bias"], s["labels"])
    fwd = _at(loss, s["stats"])
    if case["way"] == "loss":
        def score():
            api.ard_headloss_fwd(desc, *told, fwd[0], None, ws, _stream())
            return loss
        return score
    grads = (torch.empty(k, b, dtype=t, device=DEV), torch.empty_like(s["W"]), torch.empty(v, device=DEV))
    bwd = _at(s["stats"], s["dloss"], *grads)

    def step():
        stream = _stream()
        api.ard_headloss_fwd(desc, *told, *fwd, ws, stream)
        api.ard_headloss_bwd(desc, *told, *bwd, ws, stream)
        return (loss, *grads)
    return step


def _own_muon(s):
    from paper_1805_08939_amd import api

    case = s["case"]
    n, k = case["outputs"], case["inputs"]
    dt = api.ARD_BF16 if case["dtype"] == "bf16" else api.ARD_F32
    layout = api.ARD_WEIGHTS_FULL
    if case["major"] == "in":
        layout = api.ARD_WEIGHTS_INPUT_MAJOR
    elif case["grad"] == "compact":
        layout = api.ARD_WEIGHTS_COMPACT_GRAD
    desc = api.fc_desc(dt, 1, k, n, api.ard_plan_rows(k, case["in_period"], s["in_offset"], None),
                       api.ard_plan_rows(n, case["out_period"], s["out_offset"], None), weight_layout=layout)
    opts = api.ard_muon_opts_default()
    opts.lr, opts.momentum, opts.weight_decay, opts.nesterov, opts.eps = LR, MOMENTUM, DECAY, 1, NORM_EPS
    s["space"], ws = _space(api.ard_fc_muon_workspace_bytes(desc))
    at = _at(s["W"], s["V"], s["dW"])

    def update():
        s["W"].copy_(s["W0"])  # the call updates in place; a pass starts from the same weights each time
        s["V"].copy_(s["V0"])
        api.ard_fc_muon(desc, opts, *at, None, None, None, ws, _stream())
        return s["W"], s["V"]
    return update


# --------------------------------------------------------------------- the plain form, in 32 bits

def _plain_norm(s):
    t = TYPES[s["case"]["dtype"]]
    if s["case"]["way"] == "fwd":
        x = s["X"].float()
        if s["R"] is not None:
            x = x + s["R"].float()
        inv = torch.rsqrt((x * x).mean(0) + EPS)
        y = (s["gain"][:, None] * (x * inv)).to(t)
        return (y, inv) if s["R"] is None else (y, x.to(t), inv)
    xh = s["S"].float() * s["inv"]
    dy = s["dY"].float()
    u = s["gain"][:, None] * dy
    dx = s["inv"] * (u - xh * (u * xh).mean(0))
    if s["dS"] is not None:
        dx = dx + s["dS"].float()
    return dx.to(t), (dy * xh).sum(1)


def _plain_head(s):
    case, t = s["case"], TYPES[s["case"]["dtype"]]
    kept = slice(s["offset"], None, case["period"])
    x = s["X"][kept].float()
    w = s["W"][:, kept].float() if case["major"] == "out" else s["W"][kept].float().t()
    z = w @ x + s["bias"][:, None]
    top = z.max(0).values
    e = torch.exp(z - top)
    total = e.sum(0)
    on = s["labels"] >= 0
    label = s["labels"].long().clamp(min=0)[None]
    loss = torch.where(on, torch.log(total) - (z.gather(0, label)[0] - top), torch.zeros_like(total))
    if case["way"] == "loss":
        return loss
    g = torch.where(on, s["dloss"], torch.zeros_like(total))
    p = e * (g / total)
    p.scatter_add_(0, label, -g[None])
    dX, dW = torch.zeros_like(s["X"]), torch.zeros_like(s["W"])
    dX[kept] = (w.t() @ p).to(t)
    if case["major"] == "out":
        dW[:, kept] = (p @ x.t()).to(t)
    else:
        dW[kept] = (x @ p.t()).to(t)
    return loss, dX, dW, p.sum(1)


def _block(case, s):
    """The kept rows and columns of the matrices as they are stored."""
    out, inp = slice(s["out_offset"], None, case["out_period"]), slice(s["in_offset"], None, case["in_period"])
    return (out, inp) if case["major"] == "out" else (inp, out)


def _plain_muon(s):
    case, t = s["case"], TYPES[s["case"]["dtype"]]
    block = _block(case, s)
    w, v = s["W0"][block].float(), s["V0"][block]
    g = s["dW"][:, :v.shape[1]] if case["grad"] == "compact" else s["dW"][block]
    v = MOMENTUM * v + g
    u = g + MOMENTUM * v
    x = u / (u.double().square().sum().sqrt() + NORM_EPS).float()
    tall = x.shape[0] > x.shape[1]
    if tall:
        x = x.t()
    for _ in range(ITERATIONS):
        a = x @ x.t()
        x = A * x + (B * a + C * (a @ a)) @ x
    if tall:
        x = x.t()
    outs, ins = x.shape if case["major"] == "out" else x.shape[::-1]
    W, V = s["W0"].clone(), s["V0"].clone()
    W[block] = ((1.0 - LR * DECAY) * w - LR * math.sqrt(max(1.0, outs / ins)) * x).to(t)
    V[block] = v
    return W, V


# --------------------------------------------------------------------- the definition, in 64 bits

def exact(case, seed):
    s = prepare(case, seed)
    return {"norm": _exact_norm, "head": _exact_head, "muon": _exact_muon}[case["kind"]](s)


def _exact_norm(s):
    if s["case"]["way"] == "fwd":
        v = s["X"].double() + (s["R"].double() if s["R"] is not None else 0.0)
        root = torch.sqrt(torch.einsum("kb,kb->b", v, v) / v.shape[0] + EPS)
        y = v / root * s["gain"].double()[:, None]
        return (y, 1.0 / root) if s["R"] is None else (y, v, 1.0 / root)
    # with the reciprocal root that the call is given as a function of S
    v, i, k = s["S"].double(), s["inv"].double(), s["S"].shape[0]
    u = s["dY"].double() * s["gain"].double()[:, None]
    dx = u * i - v * (i ** 3 / k * torch.einsum("kb,kb->b", u, v))
    if s["dS"] is not None:
        dx = dx + s["dS"].double()
    return dx, torch.einsum("kb,kb->k", s["dY"].double(), v * i)


def _exact_head(s):
    case = s["case"]
    v, b = case["classes"], case["batch"]
    keep = torch.zeros(case["inputs"], dtype=torch.bool, device=DEV)
    keep[s["offset"]::case["period"]] = True
    W = (s["W"] if case["major"] == "out" else s["W"].t()).double() * keep
    X = torch.where(keep[:, None], s["X"].double(), torch.zeros((), dtype=torch.float64, device=DEV))
    losses, dX = [], torch.zeros_like(X)
    dW, db = torch.zeros_like(W), torch.zeros(v, dtype=torch.float64, device=DEV)
    for c in torch.arange(b, device=DEV).split(1024):
        x, label = X[:, c], s["labels"][c].long()
        logq = torch.log_softmax(torch.addmm(s["bias"].double()[:, None], W, x), 0)
        told = (torch.arange(v, device=DEV)[:, None] == label).double()
        losses.append(-torch.where(told > 0, logq, torch.zeros_like(logq)).sum(0))
        if case["way"] == "train":
            dz = (logq.exp() - told) * (s["dloss"][c].double() * (label >= 0))
            dX[:, c] = W.t() @ dz
            dW += dz @ x.t()
            db += dz.sum(1)
    loss = torch.cat(losses)
    if case["way"] == "loss":
        return loss
    dW = dW * keep
    return loss, dX, dW if case["major"] == "out" else dW.t().contiguous(), db


def _exact_muon(s):
    case = s["case"]
    block = _block(case, s)
    W, V = s["W0"].double(), s["V0"].double()
    g = s["dW"].double()
    g = g[:, :V[block].shape[1]] if case["grad"] == "compact" else g[block]
    V[block] = MOMENTUM * V[block] + g
    X = g + MOMENTUM * V[block]
    X = X / (torch.linalg.vector_norm(X) + NORM_EPS)
    rows, cols = X.shape
    for _ in range(ITERATIONS):
        if rows <= cols:
            S = X @ X.t()
            X = A * X + B * (S @ X) + C * (S @ (S @ X))
        else:
            S = X.t() @ X
            X = A * X + B * (X @ S) + C * ((X @ S) @ S)
    ratio = rows / cols if case["major"] == "out" else cols / rows
    W[block] = W[block] * (1.0 - LR * DECAY) - LR * max(1.0, ratio) ** 0.5 * X
    return W, V
