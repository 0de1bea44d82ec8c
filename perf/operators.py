"""The language-model operators as users of this library call them, as timed cases.

A case is a dict of plain values. Three kinds:

  glu      a gated feed-forward layer under a row pattern on its hidden units:
           forward (with or without the pre-activations that training keeps) or
           backward
  distill  the loss against a teacher's top logits and the labels, forward and
           backward
  linattn  linear attention with a decay for each head: forward over prompts,
           backward, or a step of one token for each sequence

With ``own`` true, run() makes the calls of paper_1805_08939_amd.api; otherwise
it computes the same from elementary torch operations in 32 bits. A pattern's
period and the sequence lengths are part of the case (they set the work); a
pattern's offset, like every input, comes from the seed.
"""

import math

import torch

own = False

DEV = "cuda:0"
CHUNK = 64  # tokens per block of the plain linear attention
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16}


def listed():
    return [
        # serving a single token: a small layer, every hidden unit kept
        dict(name="glu-step-1024x2048-bf16-b1", kind="glu", way="fwd", dtype="bf16", batch=1, inputs=1024, hidden=2048,
             period=1, act="silu", train=False),
        # serving sixteen sequences: the weights are read once for all of them
        dict(name="glu-step-4096x8192-bf16-b16", kind="glu", way="fwd", dtype="bf16", batch=16, inputs=4096,
             hidden=8192, period=1, act="silu", train=False),
        # training in fp32 next to the 1500-unit recurrent layers, 35 steps of batch 20, half of the hidden units
        dict(name="glu-fwd-1500x4000-f32-b700", kind="glu", way="fwd", dtype="f32", batch=700, inputs=1500, hidden=4000,
             period=2, act="gelu", train=True),
        # sizes that fit no tile and rows that fit no 16 bytes
        dict(name="glu-bwd-1023x1537-bf16-b100", kind="glu", way="bwd", dtype="bf16", batch=100, inputs=1023,
             hidden=1537, period=3, act="gelu", train=True),
        # the wide layer in training, half of the hidden units, forward and backward
        dict(name="glu-fwd-8192x8192-bf16-b2048", kind="glu", way="fwd", dtype="bf16", batch=2048, inputs=8192,
             hidden=8192, period=2, act="silu", train=True),
        dict(name="glu-bwd-8192x8192-bf16-b2048", kind="glu", way="bwd", dtype="bf16", batch=2048, inputs=8192,
             hidden=8192, period=2, act="silu", train=True),
        # a ten-class network distilled from a larger one, one batch
        dict(name="distill-10-f32-b128", kind="distill", dtype="f32", batch=128, classes=10, top=5, temperature=4.0,
             weight=0.9),
        # the 8800-word head of the recurrent language model, 35 steps of batch 20
        dict(name="distill-8800-f32-b700", kind="distill", dtype="f32", batch=700, classes=8800, top=20,
             temperature=2.0, weight=0.5),
        # a large vocabulary and a long batch of tokens
        dict(name="distill-32000-bf16-b4096", kind="distill", dtype="bf16", batch=4096, classes=32000, top=64,
             temperature=1.0, weight=0.7),
        # generation: one token for each of 64 sequences
        dict(name="linattn-step-16x128-bf16-s64", kind="linattn", way="step", dtype="bf16", seqs=64, tokens=64,
             ragged=False, heads=16, shared=1, key=128, value=128, initial=True),
        # prompts of different lengths behind a state each, keys and values shared by four heads
        dict(name="linattn-fwd-16x64-bf16-ragged", kind="linattn", way="fwd", dtype="bf16", seqs=9, tokens=16411,
             ragged=True, heads=16, shared=4, key=64, value=64, initial=True),
        # training on four long sequences
        dict(name="linattn-bwd-16x128-bf16-4x4096", kind="linattn", way="bwd", dtype="bf16", seqs=4, tokens=16384,
             ragged=False, heads=16, shared=1, key=128, value=128, initial=False),
    ]


def _log(rng, lo, hi):
    return max(lo, min(hi, round(math.exp(rng.uniform(math.log(lo), math.log(hi))))))


def draw(rng):
    """One more case of the same ranges; never more work than the largest listed one of its kind."""
    kind = rng.choice(["glu", "glu", "distill", "linattn", "linattn"])
    most = {k: max(_cost(c) for c in listed() if c["kind"] == k) for k in ("glu", "distill", "linattn")}[kind]
    while True:
        if kind == "glu":
            c = dict(kind="glu", way=rng.choice(["fwd", "bwd"]), dtype=rng.choice(["f32", "bf16", "bf16"]),
                     batch=_log(rng, 1, 2048), inputs=_log(rng, 256, 8192), hidden=_log(rng, 256, 8192),
                     period=rng.choice([1, 1, 2, 2, 3, 5]), act=rng.choice(["silu", "gelu", "relu", "sigmoid"]),
                     train=True)
            if rng.random() < 0.6:  # the sizes that networks are usually given; the others are odd ones too
                for k in ("inputs", "hidden"):
                    c[k] = (c[k] + 63) // 64 * 64
                if c["batch"] > 16:
                    c["batch"] = (c["batch"] + 15) // 16 * 16
            if c["way"] == "fwd":
                c["train"] = c["batch"] > 16 and rng.random() < 0.5
        elif kind == "distill":
            c = dict(kind="distill", dtype=rng.choice(["f32", "bf16"]), batch=_log(rng, 1, 4096),
                     classes=_log(rng, 10, 32000), top=_log(rng, 1, 64), temperature=rng.choice([1.0, 2.0, 4.0]),
                     weight=rng.choice([0.5, 0.9, 1.0]))
            c["top"] = min(c["top"], c["classes"])
            if rng.random() < 0.5:
                c["batch"] = (c["batch"] + 7) // 8 * 8
        else:
            way = rng.choice(["fwd", "fwd", "bwd", "step"])
            seqs = _log(rng, 1, 64 if way == "step" else 16)
            heads = rng.choice([2, 4, 8, 16])
            c = dict(kind="linattn", way=way, dtype=rng.choice(["f32", "bf16", "bf16"]), seqs=seqs,
                     tokens=seqs if way == "step" else seqs * _log(rng, 1, 4096), ragged=False, heads=heads,
                     shared=rng.choice([1, 1, 2]), key=rng.choice([32, 64, 64, 80, 96, 128]),
                     value=rng.choice([32, 64, 64, 80, 96, 128]), initial=way == "step" or rng.random() < 0.5)
            if way != "step" and seqs > 1 and rng.random() < 0.5:
                c["ragged"] = True
                c["tokens"] += rng.randrange(8)
        if _cost(c) <= most:
            return c


# --------------------------------------------------------------------- shared

def _cost(case):
    w = work(case)
    rate = 1e14 if case["dtype"] == "f32" else 1e15
    return max(w["bytes"] / 4e12, w["flops"] / rate)


def _kept(case, offset):
    return range(offset, case["hidden"], case["period"])


def _lengths(case):
    """Tokens of each sequence, first to last: growing ones where they are ragged."""
    n, total = case["seqs"], case["tokens"]
    if not case["ragged"]:
        return [total // n] * n
    ends = [round(total * (i / n) ** 2) for i in range(n + 1)]
    return [b - a for a, b in zip(ends, ends[1:])]


def work(case):
    es = 4 if case["dtype"] == "f32" else 2
    if case["kind"] == "glu":
        b, k = case["batch"], case["inputs"]
        h, n = case["hidden"], len(_kept(case, case["period"] // 2))
        if case["way"] == "fwd":
            moved = es * (b * k + 2 * n * k + b * h + (2 * b * n if case["train"] else 0)) + 8 * n
            return {"bytes": moved, "flops": 4 * n * k * b}
        moved = es * (b * k + 2 * n * k + 3 * b * n + b * k + 2 * h * k) + 8 * h
        return {"bytes": moved, "flops": 8 * n * k * b}
    if case["kind"] == "distill":
        b, v, top = case["batch"], case["classes"], case["top"]
        return {"bytes": 2 * es * b * v + 8 * b * top + 12 * b, "flops": 12 * b * v}
    h, hk, dk, dv = case["heads"], case["heads"] // case["shared"], case["key"], case["value"]
    row = h * dk + hk * dk + hk * dv  # q, k, v of a token
    state = 4 * case["seqs"] * h * dk * dv
    states = 2 if case["initial"] else 1
    if case["way"] == "bwd":
        return {"bytes": es * case["tokens"] * (2 * row + h * dv) + state * 2 * states,
                "flops": 10 * case["tokens"] * h * dk * dv}
    return {"bytes": es * case["tokens"] * (row + h * dv) + state * states,
            "flops": 4 * case["tokens"] * h * dk * dv}


class _Draws:
    def __init__(self, seed):
        self.g = torch.Generator(device=DEV)
        self.g.manual_seed(seed)

    def normal(self, *shape, std=1.0, dtype=torch.float32):
        return (torch.randn(*shape, generator=self.g, device=DEV) * std).to(dtype)

    def below(self, n, *shape):
        return torch.randint(0, n, shape, generator=self.g, device=DEV, dtype=torch.int64)


def prepare(case, seed):
    d, t = _Draws(seed), TYPES[case["dtype"]]
    s = {"case": case}
    if case["kind"] == "glu":
        k, h, b = case["inputs"], case["hidden"], case["batch"]
        s["offset"] = seed % case["period"]
        s["X"] = d.normal(k, b, dtype=t)
        s["W"] = d.normal(2, h, k, std=math.sqrt(1.0 / k), dtype=t)
        s["bias"] = d.normal(2, h, std=0.1)
        s["scale"] = float(case["period"])  # the inverse of the kept share
        if case["way"] == "bwd":
            s["Z"] = d.normal(2, h, b, dtype=t)
            s["dH"] = d.normal(h, b, dtype=t)
    elif case["kind"] == "distill":
        v, b, top = case["classes"], case["batch"], case["top"]
        s["Z"] = d.normal(v, b, std=3.0, dtype=t)
        first, step = d.below(v, 1, b), max(1, v // top)
        idx = (first + step * torch.arange(top, device=DEV)[:, None]) % v
        s["logits"] = d.normal(top, b, std=2.0).sort(dim=0, descending=True).values + 6.0
        s["labels"] = d.below(v, b).to(torch.int32)
        # tokens without a label (padding) and without a teacher's answer
        s["labels"][3::16] = -1
        idx[:, 5::16] = -1
        s["idx"] = idx.to(torch.int32)
        s["dloss"] = torch.full((b,), 1.0 / b, device=DEV)
    else:
        h, hk, dk, dv, n = case["heads"], case["heads"] // case["shared"], case["key"], case["value"], case["tokens"]
        lens = _lengths(case)
        s["lens"], s["max_len"] = lens, max(lens)
        s["lengths"] = torch.tensor(lens, device=DEV)
        s["starts"] = s["lengths"].cumsum(0) - s["lengths"]
        s["offsets"] = torch.tensor([sum(lens[:i]) for i in range(len(lens) + 1)], device=DEV, dtype=torch.int32)
        s["scale"] = dk ** -0.5
        s["Q"], s["K"] = d.normal(h * dk, n, dtype=t), d.normal(hk * dk, n, dtype=t)
        s["V"] = d.normal(hk * dv, n, dtype=t)
        # heads that remember from 32 to 1024 tokens
        s["decay"] = torch.log1p(-torch.pow(2.0, -torch.linspace(5.0, 10.0, h, device=DEV)))
        s["S0"] = d.normal(case["seqs"], h, dk, dv) if case["initial"] else None
        if case["way"] == "bwd":
            s["dO"] = d.normal(h * dv, n, dtype=t)
            s["dST"] = d.normal(case["seqs"], h, dk, dv) if case["initial"] else None
    return s


def run(state):
    case = state["case"]
    if own:
        if "call" not in state:  # descriptors, outputs and workspaces that a program makes once
            state["call"] = {"glu": _own_glu, "distill": _own_distill, "linattn": _own_linattn}[case["kind"]](state)
        return state["call"]()
    return {"glu": _plain_glu, "distill": _plain_distill, "linattn": _plain_linattn}[case["kind"]](state)


# --------------------------------------------------------------------- the framework's calls
# Addresses are looked up once, the stream at each pass.

def _at(*tensors):
    return tuple(None if x is None else x.data_ptr() for x in tensors)


def _stream():
    return torch.cuda.current_stream().cuda_stream


def _space(nbytes):
    ws = torch.empty(max(nbytes, 16) // 4 + 4, dtype=torch.float32, device=DEV)
    return ws, (ws.data_ptr(), ws.numel() * 4)


def _own_glu(s):
    from paper_1805_08939_amd import api

    case = s["case"]
    k, h, b, t = case["inputs"], case["hidden"], case["batch"], TYPES[case["dtype"]]
    dt = api.ARD_BF16 if case["dtype"] == "bf16" else api.ARD_F32
    act = {"silu": api.ARD_GLU_SILU, "gelu": api.ARD_GLU_GELU, "relu": api.ARD_GLU_RELU,
           "sigmoid": api.ARD_GLU_SIGMOID}[case["act"]]
    plan = api.ard_plan_rows(h, case["period"], s["offset"], None)
    desc = api.glu_desc(dt, b, k, h, plan, s["scale"], act, api.ARD_DROPPED_ZERO, grad_dtype=dt)
    s["space"], ws = _space(api.ard_glu_workspace_bytes(desc))
    if case["way"] == "fwd":
        H = torch.empty(h, b, dtype=t, device=DEV)
        Z = torch.zeros(2, h, b, dtype=t, device=DEV) if case["train"] else None
        out = (H, Z) if case["train"] else H
        at = _at(s["X"], s["W"], s["bias"], Z, H)

        def fwd():
            api.ard_glu_fwd(desc, *at, ws, _stream())
            return out
        return fwd
    out = (torch.empty(k, b, dtype=t, device=DEV), torch.empty(2, h, k, dtype=t, device=DEV),
           torch.empty(2, h, device=DEV))
    at = _at(s["X"], s["W"], s["Z"], s["dH"], *out)

    def bwd():
        api.ard_glu_bwd(desc, *at, ws, _stream())
        return out
    return bwd


def _own_distill(s):
    from paper_1805_08939_amd import api

    case = s["case"]
    v, b = case["classes"], case["batch"]
    dt = api.ARD_BF16 if case["dtype"] == "bf16" else api.ARD_F32
    desc = api.distill_desc(dt, b, v, case["top"], case["temperature"], case["weight"])
    s["space"], ws = _space(api.ard_distill_workspace_bytes(desc))
    s["stats"] = torch.empty(5, b, device=DEV)
    loss, dZ = torch.empty(b, device=DEV), torch.empty_like(s["Z"])
    told = _at(s["Z"], s["idx"], s["logits"], s["labels"])
    fwd, bwd = _at(loss, s["stats"]), _at(s["stats"], s["dloss"], dZ)

    def step():
        stream = _stream()
        api.ard_distill_fwd(desc, *told, *fwd, ws, stream)
        api.ard_distill_bwd(desc, *told, *bwd, stream)
        return loss, dZ
    return step


def _own_linattn(s):
    from paper_1805_08939_amd import api

    case = s["case"]
    h, hk, dk, dv = case["heads"], case["heads"] // case["shared"], case["key"], case["value"]
    dt = api.ARD_BF16 if case["dtype"] == "bf16" else api.ARD_F32
    desc = api.linattn_desc(dt, case["seqs"], s["max_len"], case["tokens"], h, hk, dk, dv, s["scale"],
                            s["offsets"] if case["ragged"] else None)
    told = _at(s["Q"], s["K"], s["V"], s["decay"], s["S0"])
    O = torch.empty(h * dv, case["tokens"], dtype=TYPES[case["dtype"]], device=DEV)
    ST = torch.empty(case["seqs"], h, dk, dv, device=DEV)
    if case["way"] == "step":
        out = _at(O, ST)

        def step():
            api.ard_linattn_step(desc, *told, *out, _stream())
            return O, ST
        return step
    s["space"], ws = _space(api.ard_linattn_workspace_bytes(desc))
    if case["way"] == "fwd":
        out = _at(O, ST)

        def fwd():
            api.ard_linattn_fwd(desc, *told, *out, ws, _stream())
            return O, ST
        return fwd
    grads = [torch.empty_like(s[x]) for x in ("Q", "K", "V")] + ([torch.empty_like(s["S0"])] if case["initial"] else [])
    given = _at(s["dO"], s["dST"])
    out = _at(*grads) if case["initial"] else (*_at(*grads), None)

    def bwd():
        api.ard_linattn_bwd(desc, *told, *given, *out, ws, _stream())
        return tuple(grads)
    return bwd


# --------------------------------------------------------------------- the plain form, in 32 bits

def _act(name, g):
    """The activation and its derivative."""
    if name == "relu":
        return g.clamp(min=0), (g > 0).to(g.dtype)
    if name == "gelu":
        cdf = 0.5 * (1 + torch.erf(g * math.sqrt(0.5)))
        return g * cdf, cdf + g * torch.exp(-0.5 * g * g) / math.sqrt(2 * math.pi)
    sig = 1 / (1 + torch.exp(-g))
    if name == "sigmoid":
        return sig, sig * (1 - sig)
    return g * sig, sig * (1 + g * (1 - sig))


def _plain_glu(s):
    case = s["case"]
    t, keep = TYPES[case["dtype"]], slice(s["offset"], None, case["period"])
    h, b = case["hidden"], case["batch"]
    w, x = s["W"][:, keep].float(), s["X"].float()
    if case["way"] == "fwd":
        g = w[0] @ x + s["bias"][0, keep, None]
        u = w[1] @ x + s["bias"][1, keep, None]
        H = torch.zeros(h, b, dtype=t, device=DEV)
        H[keep] = (s["scale"] * _act(case["act"], g)[0] * u).to(t)
        if not case["train"]:
            return H
        Z = torch.zeros(2, h, b, dtype=t, device=DEV)
        Z[0, keep], Z[1, keep] = g.to(t), u.to(t)
        return H, Z
    g, u = s["Z"][0, keep].float(), s["Z"][1, keep].float()
    a, da = _act(case["act"], g)
    dh = s["dH"][keep].float() * s["scale"]
    dg, du = dh * u * da, dh * a
    dX = (w[0].T @ dg + w[1].T @ du).to(t)
    dW, db = torch.zeros(2, h, case["inputs"], dtype=t, device=DEV), torch.zeros(2, h, device=DEV)
    dW[0, keep], dW[1, keep] = (dg @ x.T).to(t), (du @ x.T).to(t)
    db[0, keep], db[1, keep] = dg.sum(1), du.sum(1)
    return dX, dW, db


def _plain_distill(s):
    case = s["case"]
    T, a = case["temperature"], case["weight"]
    z, idx = s["Z"].float(), s["idx"].long()
    valid = (idx >= 0) & (idx < case["classes"])
    taught = valid.any(0)
    at = idx.clamp(min=0)
    t = torch.where(valid, s["logits"] / T, -math.inf)
    e = torch.where(valid, torch.exp(t - torch.where(taught, t.amax(0), 0)), 0)
    p = e / torch.where(taught, e.sum(0), 1)
    logp = torch.where(p > 0, torch.log(torch.where(p > 0, p, 1)), 0)
    m = z.amax(0)
    e1, eT = torch.exp(z - m), torch.exp((z - m) / T)
    s1, sT = e1.sum(0), eT.sum(0)
    logq = (z.gather(0, at) - m) / T - torch.log(sT)
    soft = torch.where(taught, (p * (logp - logq)).sum(0), 0)
    told = s["labels"] >= 0
    label = s["labels"].long().clamp(min=0)[None]
    hard = torch.where(told, torch.log(s1) + m - z.gather(0, label)[0], 0)
    loss = a * T * T * soft + (1 - a) * hard
    cs, ch = s["dloss"] * a * T * taught, s["dloss"] * (1 - a) * told
    dz = eT * (cs / sT) + e1 * (ch / s1)
    dz.scatter_add_(0, at, -cs * p)
    dz.scatter_add_(0, label, -ch[None])
    return loss, dz.to(TYPES[case["dtype"]])


def _padded(s, x, heads):
    """[heads * d][tokens] as [seq][head][whole chunks of tokens][d] in 32 bits, zeros past each end."""
    length = -(-s["max_len"] // CHUNK) * CHUNK
    pos = torch.arange(length, device=DEV)
    inside = pos < s["lengths"][:, None]
    at = torch.where(inside, s["starts"][:, None] + pos, 0)
    y = x.float().view(heads, -1, x.shape[1])[:, :, at] * inside
    y = y.permute(2, 0, 3, 1)
    return y.repeat_interleave(s["case"]["heads"] // heads, dim=1).contiguous()


def _unpadded(s, x, shared, dtype):
    """Back to [heads * d][tokens]; shared heads added up."""
    n, h, length, d = x.shape
    x = x.view(n, h // shared, shared, length, d).sum(2).permute(1, 3, 0, 2).reshape(h // shared * d, n * length)
    pos = torch.arange(length, device=DEV)
    return x[:, (pos < s["lengths"][:, None]).reshape(-1)].to(dtype)


def _mix(g, q, k, v):
    """o_i = sum over j <= i of exp(g (i - j)) (q_i . k_j) v_j, chunk by chunk."""
    n, h, length, dk = q.shape
    c = length // CHUNK
    q, k, v = (x.reshape(n * h, c, CHUNK, -1) for x in (q, k, v))
    i = torch.arange(CHUNK, device=DEV, dtype=torch.float32)
    g = g.repeat(n)[:, None, None]
    inner = torch.where(i[:, None] >= i, torch.exp(g * (i[:, None] - i).clamp(min=0)), 0)
    o = ((q @ k.transpose(2, 3).contiguous()) * inner[:, None]) @ v
    u = (k * torch.exp(g * (CHUNK - 1 - i[:, None]))[:, None]).transpose(2, 3).contiguous() @ v
    j = torch.arange(c, device=DEV, dtype=torch.float32)
    outer = torch.where(j[:, None] > j, torch.exp(g * CHUNK * (j[:, None] - j - 1).clamp(min=0)), 0)
    before = (outer @ u.reshape(n * h, c, -1)).reshape(u.shape)
    o = o + (q * torch.exp(g * (i[:, None] + 1))[:, None]) @ before
    return o.reshape(n, h, length, -1)


def _plain_linattn(s):
    case = s["case"]
    h, shared, t, scale, g = case["heads"], case["shared"], TYPES[case["dtype"]], s["scale"], s["decay"]
    if case["way"] == "step":
        n = case["seqs"]
        q, k, v = (x.float().view(-1, d, n).permute(2, 0, 1).repeat_interleave(r, dim=1)
                   for x, d, r in ((s["Q"], case["key"], 1), (s["K"], case["key"], shared),
                                   (s["V"], case["value"], shared)))
        S = s["S0"] * torch.exp(g)[:, None, None] + k[..., None] * v[..., None, :]
        o = scale * (q[..., None] * S).sum(2)
        return o.permute(1, 2, 0).reshape(h * case["value"], n).to(t), S
    q, k, v = _padded(s, s["Q"], h), _padded(s, s["K"], h // shared), _padded(s, s["V"], h // shared)
    pos = torch.arange(q.shape[2], device=DEV, dtype=torch.float32)
    left = s["lengths"][:, None] - 1 - pos  # tokens behind each one
    since = torch.exp(g[:, None] * (pos + 1))[None, :, :, None]
    until = torch.where(left[:, None] >= 0, torch.exp(g[:, None] * left[:, None].clamp(min=0)), 0)[..., None]
    whole = torch.exp(g * s["lengths"][:, None])[..., None, None]
    if case["way"] == "fwd":
        o = _mix(g, q, k, v)
        S = (k * until).transpose(2, 3).contiguous() @ v
        if case["initial"]:
            o = o + (q * since) @ s["S0"]
            S = S + whole * s["S0"]
        return _unpadded(s, scale * o, 1, t), S
    do = _padded(s, s["dO"], h) * scale
    dq = _mix(g, do, v, k)
    dk, dv = (_mix(g, *(x.flip(2) for x in y)).flip(2) for y in ((v, do, q), (k, q, do)))
    out = ()
    if case["initial"]:
        dq = dq + (do * since) @ s["S0"].transpose(2, 3).contiguous()
        dk = dk + (v * until) @ s["dST"].transpose(2, 3).contiguous()
        dv = dv + (k * until) @ s["dST"]
        out = ((q * since).transpose(2, 3).contiguous() @ do + whole * s["dST"],)
    return (_unpadded(s, dq, 1, t), _unpadded(s, dk, shared, t), _unpadded(s, dv, shared, t), *out)


# --------------------------------------------------------------------- the definition, in 64 bits

def exact(case, seed):
    s = prepare(case, seed)
    return {"glu": _exact_glu, "distill": _exact_distill, "linattn": _exact_linattn}[case["kind"]](s)


def _exact_glu(s):
    case = s["case"]
    h, b, scale = case["hidden"], case["batch"], s["scale"]
    keep = torch.arange(h, device=DEV) % case["period"] == s["offset"]
    x, w = s["X"].double(), s["W"].double()
    fn = {"silu": lambda g: g * torch.sigmoid(g), "sigmoid": torch.sigmoid, "relu": torch.relu,
          "gelu": lambda g: 0.5 * g * torch.special.erfc(-g / math.sqrt(2))}[case["act"]]
    if case["way"] == "fwd":
        z = torch.stack([w[i] @ x + s["bias"][i].double()[:, None] for i in (0, 1)]) * keep[:, None]
        H = scale * fn(z[0]) * z[1] * keep[:, None]
        return (H, z) if case["train"] else H
    with torch.enable_grad():
        z = s["Z"].double().requires_grad_(True)
        (scale * fn(z[0]) * z[1] * keep[:, None] * s["dH"].double()).sum().backward()
    d = z.grad
    dX = w[0].T.contiguous() @ d[0] + w[1].T.contiguous() @ d[1]
    xt = x.T.contiguous()
    return dX, torch.stack([d[0] @ xt, d[1] @ xt]), d.sum(2)


def _exact_distill(s):
    case = s["case"]
    T, a, v = case["temperature"], case["weight"], case["classes"]
    taught = s["idx"][0] >= 0
    told = s["labels"] >= 0
    # a column at a time would be slow: a group of them
    losses, grads = [], []
    for c in torch.arange(case["batch"], device=DEV).split(1024):
        with torch.enable_grad():
            z = s["Z"][:, c].double().requires_grad_(True)
            logp = torch.log_softmax(s["logits"][:, c].double() / T, 0)
            logq = torch.log_softmax(z / T, 0).gather(0, s["idx"][:, c].long().clamp(min=0))
            soft = (logp.exp() * (logp - logq)).sum(0) * taught[c]
            hard = -torch.log_softmax(z, 0).gather(0, s["labels"][c].long().clamp(min=0)[None])[0] * told[c]
            loss = a * T * T * soft + (1 - a) * hard
            (loss * s["dloss"][c].double()).sum().backward()
        losses.append(loss.detach())
        grads.append(z.grad)
    return torch.cat(losses), torch.cat(grads, 1)


def _exact_linattn(s):
    """Token after token."""
    case = s["case"]
    h, hk, dk, dv, n = case["heads"], case["heads"] // case["shared"], case["key"], case["value"], case["tokens"]
    seqs, scale = case["seqs"], s["scale"]
    a = torch.exp(s["decay"].double())[None, :, None, None]
    cols = lambda x, hh, d: x.double().view(hh, d, n).repeat_interleave(h // hh, dim=0).permute(2, 0, 1).contiguous()  # noqa: E731,E501
    q, k, v = cols(s["Q"], h, dk), cols(s["K"], hk, dk), cols(s["V"], hk, dv)
    zero = torch.zeros(seqs, h, dk, dv, dtype=torch.float64, device=DEV)
    S = s["S0"].double() if s["S0"] is not None else zero.clone()
    rows = lambda x, hh: x.view(n, hh, h // hh, -1).sum(2).permute(1, 2, 0).reshape(-1, n)  # noqa: E731
    lengths, starts, bwd = s["lengths"], s["starts"], case["way"] == "bwd"
    do = cols(s["dO"], h, dv) * scale if bwd else None
    out = torch.zeros(n, h, dk if bwd else dv, dtype=torch.float64, device=DEV)
    for t in range(s["max_len"]):
        on = [i for i, m in enumerate(s["lens"]) if m > t]
        on = slice(None) if len(on) == seqs else torch.tensor(on, device=DEV)
        at = starts[on] + t
        S = S if isinstance(on, slice) else S.clone()
        S[on] = a * S[on] + k[at][..., None] * v[at][..., None, :]
        if bwd:
            out[at] = (S[on] * do[at][..., None, :]).sum(3)
        else:
            out[at] = scale * (S[on] * q[at][..., None]).sum(2)
    if not bwd:
        return rows(out, h), S
    dk_, dv_ = torch.zeros_like(k), torch.zeros_like(v)
    G = s["dST"].double() if s["dST"] is not None else zero
    for t in reversed(range(s["max_len"])):
        on = [i for i, m in enumerate(s["lens"]) if m > t]
        on = slice(None) if len(on) == seqs else torch.tensor(on, device=DEV)
        at = starts[on] + t
        G = G.clone()
        now = G[on] + q[at][..., None] * do[at][..., None, :]
        dk_[at] = (now * v[at][..., None, :]).sum(3)
        dv_[at] = (now * k[at][..., None]).sum(2)
        G[on] = a * now
    res = (rows(out, h), rows(dk_, hk), rows(dv_, hk))
    return (*res, G) if case["initial"] else res
