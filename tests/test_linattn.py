"""Linear attention with decays: the oracle against finite differences and the quadratic form (CPU), refusals (CPU), and
the kernels against the oracle (GPU).

Tolerances, per value, in units of the same formula on absolute values ("size"): fp32 sums, decays and products over a
sequence of T tokens, 2 (T + 200) 2^-24; bf16 inputs, 2^-9 for the rounded inner products and 2^-9 for the rounded
state, and 2^-9 of the value for the output's rounding (half of the largest possible each: a value is at its largest only
where all of its terms have one sign, and then the roundings have not). States have only the fp32 part.
"""
import numpy as np
import pytest
import torch

from oracle import linattn as ol
from paper_1805_08939_amd import api, synth

U32, UBF = 2.0 ** -24, 2.0 ** -9


# ---------------------------------------------------------------- the oracle

def test_oracle_is_the_quadratic_form():
    r = np.random.default_rng(1)
    T, a = 7, 0.83
    q, k, v, S = r.normal(size=(T, 3)), r.normal(size=(T, 3)), r.normal(size=(T, 2)), r.normal(size=(3, 2))
    i = np.arange(T)
    D = np.where(i[:, None] >= i, a ** np.clip(i[:, None] - i, 0, None).astype(float), 0)
    o, ST = ol.forward(q, k, v, a, S, 0.5)
    assert np.abs(o - 0.5 * (((q @ k.T) * D) @ v + (a ** (i + 1.0))[:, None] * (q @ S))).max() < 1e-12
    assert np.abs(ST - (a ** T * S + (k * (a ** (T - 1.0 - i))[:, None]).T @ v)).max() < 1e-12


def test_oracle_backward_is_the_forward_differenced():
    r = np.random.default_rng(2)
    T, a, sc = 5, 0.7, 0.6
    p = [r.normal(size=(T, 3)), r.normal(size=(T, 3)), r.normal(size=(T, 2)), r.normal(size=(3, 2))]
    do, dS = r.normal(size=(T, 2)), r.normal(size=(3, 2))

    def value(q, k, v, S):
        o, ST = ol.forward(q, k, v, a, S, sc)
        return float((o * do).sum() + (ST * dS).sum())
    grads = ol.backward(*p[:3], a, p[3], sc, do, dS)
    for n, d in enumerate(grads):
        for at in np.ndindex(d.shape):
            up, dn = [x.copy() for x in p], [x.copy() for x in p]
            up[n][at] += 1e-6
            dn[n][at] -= 1e-6
            assert abs((value(*up) - value(*dn)) / 2e-6 - d[at]) < 1e-7


# ---------------------------------------------------------------- refusals

def test_refuses_bad_calls():
    a = 4096
    good = dict(dtype=api.ARD_F32, n_seqs=2, max_len=8, tokens=16, q_heads=4, kv_heads=2, key_dim=8, value_dim=8)

    def refused(status, call, *args):
        with pytest.raises(api.ArdError) as e:
            call(*args, stream=0)
        assert e.value.status == status and e.value.message

    big = (a, 1 << 40)
    for bad, status in ((dict(dtype=2), 2), (dict(n_seqs=0), 1), (dict(max_len=0), 1), (dict(tokens=0), 1),
                        (dict(tokens=15), 1), (dict(q_heads=3), 1), (dict(kv_heads=0), 1), (dict(key_dim=0), 2),
                        (dict(key_dim=129), 2), (dict(value_dim=200), 2), (dict(scale=float("nan")), 1),
                        (dict(d_offsets=a + 2), 1)):
        d = api.linattn_desc(**{**good, **bad})
        assert api.ard_linattn_workspace_bytes(d) == 0
        refused(status, api.ard_linattn_fwd, d, a, a, a, a, None, a, None, big)
        refused(status, api.ard_linattn_bwd, d, a, a, a, a, None, a, None, a, a, a, None, big)
        refused(status, api.ard_linattn_step, d, a, a, a, a, None, a, a)
    d = api.linattn_desc(**good)
    for i in (0, 1, 2, 3, 5):
        args = [a, a, a, a, None, a, None]
        args[i] = None
        refused(1, api.ard_linattn_fwd, d, *args, big)
        args[i] = a + 4
        refused(1, api.ard_linattn_fwd, d, *args, big)
    for i in (0, 1, 2, 3, 5):
        args = [a, a, a, a, None, a, None, a, a, a, None]
        args[i] = None
        refused(1, api.ard_linattn_bwd, d, *args, big)
    for i in range(4, 11):
        args = [a, a, a, a, None, a, None, a, a, a, None]
        args[i] = a + 4
        refused(1, api.ard_linattn_bwd, d, *args, big)
    refused(5, api.ard_linattn_bwd, d, a, a, a, a, None, a, None, a, a, a, None, (a, 16))
    refused(1, api.ard_linattn_step, d, a, a, a, a, None, a, a)  # not one token for each sequence
    one = api.linattn_desc(**{**good, "max_len": 1, "tokens": 2})
    refused(1, api.ard_linattn_step, one, a, a, a, a, None, a, None)
    refused(1, api.ard_linattn_step, one, a, a, a, a, None, None, a)


# ---------------------------------------------------------------- the kernels

class Case:
    """Seeded inputs of sequences with the given lengths, `gap` columns that belong to none in front of each."""

    def __init__(self, dtype, lens, heads, kv, dk, dv, initial, decays=None, gap=0, equal=False, seed=0):
        g = synth.generator(1805 + seed)
        self.dtype, self.lens, self.heads, self.kv, self.dk, self.dv = dtype, lens, heads, kv, dk, dv
        starts, at = [], 0
        for n in lens:
            at += gap
            starts.append(at)
            at += n
        self.spans = [(b, b + n) for b, n in zip(starts, lens)]
        self.n = max(1, at + gap)
        t = lambda *s: synth.to_storage(synth.normal(g, s), dtype)  # noqa: E731
        self.Q, self.K, self.V = t(heads * dk, self.n), t(kv * dk, self.n), t(kv * dv, self.n)
        self.dO = t(heads * dv, self.n)
        self.S0 = synth.normal(g, (len(lens), heads, dk, dv)) if initial else None
        self.dST = synth.normal(g, (len(lens), heads, dk, dv)) if initial else None
        a = decays if decays is not None else [1 - 2.0 ** -(1 + 7 * (h + 1) / heads) for h in range(heads)]
        self.g = torch.log(torch.tensor(a, dtype=torch.float32))
        self.scale = dk ** -0.5
        # the spans as the kernel is told them; with a gap an offset's end is not the next one's start
        self.equal = equal
        assert gap == 0 or equal is False

    def desc(self):
        from gpu_util import ard_dtype, device
        off = None
        if not self.equal:
            off = torch.tensor([b for b, _ in self.spans] + [self.spans[-1][1]], dtype=torch.int32, device=device())
        return api.linattn_desc(ard_dtype(self.dtype), len(self.lens), max(1, max(self.lens)), self.n, self.heads,
                                self.kv, self.dk, self.dv, self.scale, off)

    def each(self):
        """(sequence, head, kv head, columns, decay) of every state."""
        for s, (b, e) in enumerate(self.spans):
            for h in range(self.heads):
                yield s, h, h // (self.heads // self.kv), slice(b, e), float(np.exp(np.float64(self.g[h])))

    def rows(self, x, h, d, cols):
        return x[h * d:(h + 1) * d, cols].double().numpy().T

    def forward(self, size=False):
        f = np.abs if size else (lambda x: x)
        O = np.zeros((self.heads * self.dv, self.n))
        ST = np.zeros((len(self.lens), self.heads, self.dk, self.dv))
        for s, h, hk, c, a in self.each():
            S = self.S0[s, h].double().numpy() if self.S0 is not None else np.zeros((self.dk, self.dv))
            o, ST[s, h] = ol.forward(f(self.rows(self.Q, h, self.dk, c)), f(self.rows(self.K, hk, self.dk, c)),
                                     f(self.rows(self.V, hk, self.dv, c)), a, f(S), self.scale)
            O[h * self.dv:(h + 1) * self.dv, c] = o.T
        return O, ST

    def backward(self, size=False):
        f = np.abs if size else (lambda x: x)
        dQ, dK, dV = (np.zeros((m * d, self.n)) for m, d in ((self.heads, self.dk), (self.kv, self.dk), (self.kv, self.dv)))
        dS = np.zeros((len(self.lens), self.heads, self.dk, self.dv))
        for s, h, hk, c, a in self.each():
            S = self.S0[s, h].double().numpy() if self.S0 is not None else np.zeros((self.dk, self.dv))
            G = self.dST[s, h].double().numpy() if self.dST is not None else np.zeros((self.dk, self.dv))
            q, k, v, dS[s, h] = ol.backward(
                f(self.rows(self.Q, h, self.dk, c)), f(self.rows(self.K, hk, self.dk, c)),
                f(self.rows(self.V, hk, self.dv, c)), a, f(S), self.scale, f(self.rows(self.dO, h, self.dv, c)), f(G))
            dQ[h * self.dk:(h + 1) * self.dk, c] += q.T
            dK[hk * self.dk:(hk + 1) * self.dk, c] += k.T
            dV[hk * self.dv:(hk + 1) * self.dv, c] += v.T
        return dQ, dK, dV, dS

    def inside(self, got, want, size, what, state=False):
        got = got.double().cpu().numpy()
        if not state:  # the columns of no sequence are not touched
            on = np.zeros(self.n, dtype=bool)
            for b, e in self.spans:
                on[b:e] = True
            assert (got[:, ~on] == 7.0).all(), what
            got, want, size = got[:, on], want[:, on], size[:, on]
        assert np.isfinite(got).all(), what
        bound = 2 * (max(self.lens) + 200) * U32 * size + 1e-30
        if self.dtype == "bf16" and not state:
            bound += 2 * UBF * size + UBF * np.abs(want)
        else:
            bound += U32 * np.abs(want)
        assert (np.abs(got - want) <= bound).all(), f"{what}: {np.abs(got - want).max():.3e}"


def _put(t):
    from gpu_util import device
    return None if t is None else t.contiguous().to(device())


def _fwd(c, with_state=True):
    from gpu_util import device, workspace
    d = c.desc()
    O = torch.full((c.heads * c.dv, c.n), 7.0, dtype=c.Q.dtype, device=device())
    ST = torch.full((len(c.lens), c.heads, c.dk, c.dv), 7.0, device=device()) if with_state else None
    api.ard_linattn_fwd(d, _put(c.Q), _put(c.K), _put(c.V), _put(c.g), _put(c.S0), O, ST,
                        workspace(api.ard_linattn_workspace_bytes(d)))
    torch.cuda.synchronize()
    return O, ST


def _bwd(c, which=(0, 1, 2, 3)):
    from gpu_util import device, workspace
    d, dev = c.desc(), device()
    outs = [torch.full_like(x, 7.0, device=dev) for x in (c.Q, c.K, c.V)]
    outs.append(torch.full((len(c.lens), c.heads, c.dk, c.dv), 7.0, device=dev))
    api.ard_linattn_bwd(d, _put(c.Q), _put(c.K), _put(c.V), _put(c.g), _put(c.S0), _put(c.dO), _put(c.dST),
                        *(o if i in which else None for i, o in enumerate(outs)),
                        workspace(api.ard_linattn_workspace_bytes(d)))
    torch.cuda.synchronize()
    return outs


SHAPES = [  # lens, heads, kv heads, key dim, value dim, initial state, gap of equal runs
    ([1], 1, 1, 1, 1, False), ([1], 2, 1, 3, 5, True), ([63], 1, 1, 64, 64, True), ([64], 2, 2, 64, 64, False),
    ([65], 1, 1, 64, 64, True), ([200], 3, 3, 40, 24, True), ([130, 1, 0, 64, 77], 4, 2, 32, 48, True),
    ([0, 0], 2, 2, 16, 16, True), ([127, 128, 129], 2, 1, 80, 96, False), ([300], 4, 1, 128, 128, True),
    ([90, 31], 2, 2, 128, 64, True), ([90, 31], 2, 2, 64, 128, True), ([33], 1, 1, 65, 127, True),
    ([700], 2, 1, 64, 64, True), ([1500], 1, 1, 128, 128, True), ([513, 1025], 2, 2, 72, 40, False),
]


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("shape", SHAPES)
def test_forward(dtype, shape):
    c = Case(dtype, *shape, seed=sum(shape[0]))
    O, ST = _fwd(c)
    want, size = c.forward(), c.forward(size=True)
    c.inside(O, want[0], size[0], "O")
    c.inside(ST, want[1], size[1], "ST", state=True)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("shape", SHAPES)
def test_backward(dtype, shape):
    c = Case(dtype, *shape, seed=sum(shape[0]) + 1)
    got, want, size = _bwd(c), c.backward(), c.backward(size=True)
    for g, w, s, what in zip(got, want, size, ("dQ", "dK", "dV")):
        c.inside(g, w, s, what)
    c.inside(got[3], want[3], size[3], "dS0", state=True)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_equal_runs_without_offsets(dtype):
    c = Case(dtype, [70, 70, 70], 2, 2, 48, 40, True, equal=True)
    d = Case(dtype, [70, 70, 70], 2, 2, 48, 40, True)
    for a, b in zip(_fwd(c) + tuple(_bwd(c)), _fwd(d) + tuple(_bwd(d))):
        assert torch.equal(a, b)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_columns_in_front_and_behind(dtype):
    """One sequence inside a longer row; offsets past the row are held to it."""
    c = Case(dtype, [100], 2, 1, 40, 40, True, gap=13)
    want, size = c.forward(), c.forward(size=True)
    O, ST = _fwd(c)
    c.inside(O, want[0], size[0], "O")
    c.inside(ST, want[1], size[1], "ST", state=True)
    for g, w, s, what in zip(_bwd(c)[:3], c.backward(), c.backward(size=True), ("dQ", "dK", "dV")):
        c.inside(g, w, s, what)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("decays", [[1.0, 1.0], [0.0, 0.5], [1e-4, 0.999]])
def test_extreme_decays(dtype, decays):
    c = Case(dtype, [150, 40], 2, 2, 32, 32, True, decays=decays, seed=9)
    O, ST = _fwd(c)
    want, size = c.forward(), c.forward(size=True)
    c.inside(O, want[0], size[0], "O")
    c.inside(ST, want[1], size[1], "ST", state=True)
    got, want, size = _bwd(c), c.backward(), c.backward(size=True)
    for g, w, s, what in zip(got, want, size, ("dQ", "dK", "dV")):
        c.inside(g, w, s, what)
    c.inside(got[3], want[3], size[3], "dS0", state=True)


@pytest.mark.gpu
def test_nothing_of_other_sequences_is_read():
    """NaN in the columns of no sequence and in a neighbouring sequence stays there."""
    c = Case("bf16", [100, 70, 40], 2, 1, 40, 64, True, seed=4)
    clean = _fwd(c) + tuple(_bwd(c))
    b, e = c.spans[1]
    for x in (c.Q, c.K, c.V, c.dO):
        x[:, b:e] = float("nan")
    spoilt = _fwd(c) + tuple(_bwd(c))
    for x, y in zip(clean, spoilt):
        if x.dim() == 2:
            keep = [i for i in range(c.n) if not b <= i < e]
            assert torch.equal(x[:, keep], y[:, keep])
        else:
            assert torch.equal(x[[0, 2]], y[[0, 2]])


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_outputs_left_out_and_runs_alike(dtype):
    c = Case(dtype, [600, 90], 2, 1, 64, 64, True, seed=6)
    whole = _bwd(c)
    for which in ((0, 1, 2, 3), (0,), (1,), (2,), (3,), (0, 3)):
        for i, t in enumerate(_bwd(c, which)):
            assert torch.equal(t, whole[i]) if i in which else (t == 7.0).all()
    a, b = _fwd(c), _fwd(c, with_state=False)
    assert torch.equal(a[0], b[0])


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("n,heads,kv,dk,dv", [(1, 1, 1, 1, 1), (3, 2, 1, 7, 9), (5, 4, 2, 64, 64), (2, 3, 3, 128, 128),
                                              (33, 2, 2, 80, 96), (4, 1, 1, 40, 126), (6, 2, 1, 128, 4)])
def test_step(dtype, n, heads, kv, dk, dv):
    """One token: a sequence of length one through the recurrent form; in place and not; from nothing."""
    from gpu_util import device
    dev = device()
    c = Case(dtype, [1] * n, heads, kv, dk, dv, True, equal=True, seed=n)
    want, size = c.forward(), c.forward(size=True)
    d = c.desc()
    args = (_put(c.Q), _put(c.K), _put(c.V), _put(c.g))
    O, S, ST = torch.full((heads * dv, n), 7.0, dtype=c.Q.dtype, device=dev), _put(c.S0), torch.zeros_like(_put(c.S0))
    api.ard_linattn_step(d, *args, S, O, ST)
    torch.cuda.synchronize()
    c.inside(O, want[0], size[0], "O")
    c.inside(ST, want[1], size[1], "ST", state=True)
    O2 = torch.zeros_like(O)
    api.ard_linattn_step(d, *args, S, O2, S)
    torch.cuda.synchronize()
    assert torch.equal(O, O2) and torch.equal(S, ST)
    c.S0 = None
    want, size = c.forward(), c.forward(size=True)
    api.ard_linattn_step(d, *args, None, O, ST)
    torch.cuda.synchronize()
    c.inside(O, want[0], size[0], "O")
    c.inside(ST, want[1], size[1], "ST", state=True)


@pytest.mark.gpu
def test_prompt_then_steps_are_one_sequence():
    from gpu_util import device
    c = Case("f32", [90], 2, 1, 32, 48, False, seed=3)
    whole, ST = _fwd(c)
    head = Case("f32", [80], 2, 1, 32, 48, False, seed=3)
    for n in ("Q", "K", "V"):
        setattr(head, n, getattr(c, n)[:, :80].contiguous())
    O, S = _fwd(head)
    d = api.linattn_desc(api.ARD_F32, 1, 1, 1, 2, 1, 32, 48, c.scale)
    outs = [O]
    for t in range(80, 90):
        o = torch.empty(96, 1, device=device())
        api.ard_linattn_step(d, *(_put(x[:, t:t + 1]) for x in (c.Q, c.K, c.V)), _put(c.g), S, o, S)
        outs.append(o)
    torch.cuda.synchronize()
    got, want, size = torch.cat(outs, 1), c.forward(), c.forward(size=True)
    c.inside(got, want[0], size[0], "O")
    c.inside(S, want[1], size[1], "ST", state=True)
    c.inside(whole, want[0], size[0], "O")


@pytest.mark.gpu
def test_offsets_past_two_to_the_31():
    """A sequence at the end of rows whose last head lies past 2^31 elements, against the same columns on their own."""
    from gpu_util import device, workspace
    dev, heads, dk, n, length = device(), 8, 128, (1 << 21) + 12, 130
    assert heads * dk * n > 2 ** 31
    c = Case("bf16", [length], heads, heads, dk, dk, True, seed=11)
    small = _fwd(c) + tuple(_bwd(c))

    def wide(x):
        t = torch.empty(heads * dk, n, dtype=torch.bfloat16, device=dev)
        t[:, n - length:] = x.to(dev)
        return t
    Q, K, V, dO = (wide(x) for x in (c.Q, c.K, c.V, c.dO))
    off = torch.tensor([n - length, n], dtype=torch.int32, device=dev)
    d = api.linattn_desc(api.ARD_BF16, 1, length, n, heads, heads, dk, dk, c.scale, off)
    ws = workspace(api.ard_linattn_workspace_bytes(d))
    O, ST, dS0 = torch.empty_like(Q), torch.empty(1, heads, dk, dk, device=dev), torch.empty(1, heads, dk, dk, device=dev)
    api.ard_linattn_fwd(d, Q, K, V, _put(c.g), _put(c.S0), O, ST, ws)
    grads = [torch.empty_like(Q) for _ in range(3)]
    api.ard_linattn_bwd(d, Q, K, V, _put(c.g), _put(c.S0), dO, _put(c.dST), *grads, dS0, ws)
    torch.cuda.synchronize()
    got = [O[:, n - length:], ST] + [x[:, n - length:] for x in grads] + [dS0]
    for a, b in zip(small, got):
        assert torch.equal(a, b)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("name", ["Q", "K", "V", "dO"])
@pytest.mark.parametrize("lens,heads,kv,dk,dv", [([150], 2, 1, 64, 64), ([110, 128], 1, 1, 128, 128), ([120], 2, 2, 64, 128),
                                                 ([128], 1, 1, 128, 40), ([700], 2, 1, 40, 64)])
def test_a_token_that_is_not_finite_spoils_nothing_that_does_not_read_it(dtype, name, lens, heads, kv, dk, dv):
    """An infinity in one row of a token and NaN in all rows of a later one, in each sequence: what is finite by the
    formula, token after token, is right, and nothing else is finite."""
    c = Case(dtype, lens, heads, kv, dk, dv, True, seed=15)
    x = getattr(c, name)
    for b, _ in c.spans:
        x[3, b + 37] = float("inf")
        x[:, b + 100] = float("nan")

    def right(got, want, size, what, state):
        got = got.double().cpu().numpy()
        on = np.isfinite(want)
        assert (np.isfinite(got) == on).all(), f"{what}: {np.argwhere(np.isfinite(got) != on)[:5]}"
        if not on.any():
            return
        got, want, size = got[on], want[on], size[on]
        bound = 2 * (max(lens) + 200) * U32 * size + (U32 if state or dtype == "f32" else UBF) * np.abs(want) + 1e-30
        if dtype == "bf16" and not state:
            bound = bound + 2 * UBF * size
        assert (np.abs(got - want) <= bound).all(), what
    with np.errstate(invalid="ignore"):
        forward, backward = (c.forward(), c.forward(size=True)), (c.backward(), c.backward(size=True))
    if name != "dO":
        for i, (g, what) in enumerate(zip(_fwd(c), ("O", "ST"))):
            right(g, forward[0][i], forward[1][i], what, i == 1)
    for i, (g, what) in enumerate(zip(_bwd(c), ("dQ", "dK", "dV", "dS0"))):
        right(g, backward[0][i], backward[1][i], what, i == 3)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype,lens,heads,kv", [("bf16", [700, 90], 2, 1), ("f32", [300, 1], 2, 2)])
def test_in_a_graph(dtype, lens, heads, kv):
    from gpu_util import device, workspace
    dev = device()
    c = Case(dtype, lens, heads, kv, 64, 48, True, seed=12)
    d = c.desc()
    put = [_put(x) for x in (c.Q, c.K, c.V, c.g, c.S0, c.dO, c.dST)]
    ws = workspace(api.ard_linattn_workspace_bytes(d))
    outs = [torch.empty_like(put[5]), torch.empty_like(put[4])] + [torch.empty_like(x) for x in put[:3]] + [
        torch.empty_like(put[4])]

    def step():
        api.ard_linattn_fwd(d, *put[:5], outs[0], outs[1], ws)
        api.ard_linattn_bwd(d, *put[:5], put[5], put[6], *outs[2:], ws)
    step()
    torch.cuda.synchronize()
    eager = [o.clone() for o in outs]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step()
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for _ in range(3):
        for o in outs:
            o.fill_(3.0)
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, o) for a, o in zip(eager, outs))


def _right(c, got, want, size, what, state):
    """What is finite by the formula is right, and nothing else is finite."""
    got = got.double().cpu().numpy()
    on = np.isfinite(want)
    assert (np.isfinite(got) == on).all(), f"{what}: {np.argwhere(np.isfinite(got) != on)[:5]}"
    got, want, size = got[on], want[on], size[on]
    bound = 2 * (max(c.lens) + 200) * U32 * size + (U32 if state or c.dtype == "f32" else UBF) * np.abs(want) + 1e-30
    if c.dtype == "bf16" and not state:
        bound = bound + 2 * UBF * size
    assert (np.abs(got - want) <= bound).all(), what


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("name", ["Q", "K", "V", "dO"])
def test_tokens_that_are_not_finite_in_every_chunk(dtype, name):
    """One row after the other is spoilt, late in every chunk: right where the formula is finite, and at most ten times
    as long as with finite tokens (a second computation of a chunk's outputs is less than once more; values computed one
    by one were a hundred times)."""
    from gpu_util import device, workspace
    c = Case(dtype, [1000], 2, 1, 128, 128, True, seed=16)
    d = c.desc()
    ws = workspace(api.ard_linattn_workspace_bytes(d))

    def calls():
        put = [_put(x) for x in (c.Q, c.K, c.V, c.g, c.S0, c.dO, c.dST)]
        O, ST = torch.empty_like(put[5]), torch.empty_like(put[4])
        grads = [torch.empty_like(x) for x in put[:3]] + [torch.empty_like(put[4])]

        def fwd():
            api.ard_linattn_fwd(d, *put[:5], O, ST, ws)

        def bwd():
            api.ard_linattn_bwd(d, *put[:5], *put[5:], *grads, ws)
        return fwd, bwd

    def shortest(call):
        times = []
        for _ in range(6):
            a, b = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
            a.record()
            call()
            b.record()
            torch.cuda.synchronize()
            times.append(a.elapsed_time(b))
        return min(times)
    clean = [shortest(call) for call in calls()]
    x = getattr(c, name)
    for i in range(0, 15):
        x[7 * i, 64 * i + 62] = float("nan") if i % 2 else float("inf")
    spoilt = [shortest(call) for call in calls()]
    with np.errstate(invalid="ignore"):
        forward, backward = (c.forward(), c.forward(size=True)), (c.backward(), c.backward(size=True))
    for i, (g, what) in enumerate(zip(_fwd(c), ("O", "ST"))):
        _right(c, g, forward[0][i], forward[1][i], what, i == 1)
    for i, (g, what) in enumerate(zip(_bwd(c), ("dQ", "dK", "dV", "dS0"))):
        _right(c, g, backward[0][i], backward[1][i], what, i == 3)
    for a, b in zip(clean, spoilt):
        assert b < 10 * a, (clean, spoilt)


@pytest.mark.parametrize("dtype", [api.ARD_F32, api.ARD_BF16])
def test_a_bound_of_the_length_past_the_tokens_is_the_tokens(dtype):
    for n, heads in ((640, 4), (640, 300), (5000, 1)):
        desc = lambda most: api.linattn_desc(dtype, 3, most, n, heads, heads, 64, 64, 1.0, 4096)  # noqa: E731
        need = api.ard_linattn_workspace_bytes(desc(n))
        for most in (n + 1, 1 << 20, (1 << 31) - 1):
            assert api.ard_linattn_workspace_bytes(desc(most)) == need


@pytest.mark.parametrize("dtype,dim", [(api.ARD_F32, 64), (api.ARD_F32, 128), (api.ARD_BF16, 64), (api.ARD_BF16, 128)])
def test_no_plan_passes_the_threads_of_a_launch(dtype, dim):
    """Many short sequences told with a loose bound: a workgroup of up to 512 threads for each state of a segment (fp32: for
    each 64 of its columns)."""
    tile = dim * (64 if dtype == api.ARD_F32 else dim) * 4
    for tokens in (1 << 20, 1 << 24, 1 << 27, (1 << 31) - 1):
        desc = api.linattn_desc(dtype, (1 << 22) - 1, tokens, tokens, 1, 1, dim, dim, 1.0, 4096)
        assert api.ard_linattn_workspace_bytes(desc) // tile * 512 < 1 << 32


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("heads", [2, 300])
def test_the_largest_bound_of_the_length(dtype, heads):
    """max_len 2^31 - 1, as of a caller that knows no bound: what the longest sequence's own length gives."""
    from gpu_util import device, workspace
    c = Case(dtype, [300, 1, 90], heads, heads, 8, 8, True, seed=17)
    desc, dev = c.desc(), device()
    desc.max_len = (1 << 31) - 1
    ws = workspace(api.ard_linattn_workspace_bytes(desc))
    put = [_put(x) for x in (c.Q, c.K, c.V, c.g, c.S0)]
    O, ST = torch.full((c.heads * c.dv, c.n), 7.0, dtype=c.Q.dtype, device=dev), torch.full_like(put[4], 7.0)
    grads = [torch.full_like(x, 7.0) for x in put[:3] + put[4:]]
    api.ard_linattn_fwd(desc, *put, O, ST, ws)
    api.ard_linattn_bwd(desc, *put, _put(c.dO), _put(c.dST), *grads, ws)
    torch.cuda.synchronize()
    want, size = c.forward() + c.backward(), c.forward(size=True) + c.backward(size=True)
    for got, w, s, what in zip([O, ST] + grads, want, size, ("O", "ST", "dQ", "dK", "dV", "dS0")):
        c.inside(got, w, s, what, state="S" in what)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("told", [[-7, 30, 200], [50, 20, 140], [200, 300, -4], [0, 126, 2 ** 31 - 1]])
def test_offsets_are_held_to_the_row_and_lengths_to_the_bound(dtype, told):
    """Offsets in front of the row, past it and decreasing, and a sequence longer than max_len (60, of 126 columns): the
    columns that are meant, and nothing anywhere else."""
    from gpu_util import ard_dtype, device, workspace
    dev, n, heads, dk, dv = device(), 126, 2, 24, 40
    c = Case(dtype, [n, 0], heads, 1, dk, dv, True, seed=18)
    put = [_put(x) for x in (c.Q, c.K, c.V, c.g, c.S0, c.dO, c.dST)]
    O, ST = torch.full_like(put[5], 7.0), torch.full_like(put[4], 7.0)
    grads = [torch.full_like(x, 7.0) for x in put[:3] + put[4:5]]
    off = torch.tensor(told, dtype=torch.int32, device=dev)
    d = api.linattn_desc(ard_dtype(dtype), 2, 60, n, heads, 1, dk, dv, c.scale, off)
    ws = workspace(api.ard_linattn_workspace_bytes(d))
    api.ard_linattn_fwd(d, *put[:5], O, ST, ws)
    api.ard_linattn_bwd(d, *put, *grads, ws)
    torch.cuda.synchronize()
    held = [[min(max(x, 0), n) for x in told[s:s + 2]] for s in (0, 1)]
    c.spans = [(b, b + min(max(e - b, 0), 60)) for b, e in held]
    want, size = c.forward() + c.backward(), c.forward(size=True) + c.backward(size=True)
    for g, w, s, what in zip((O, ST, *grads), want, size, ("O", "ST", "dQ", "dK", "dV", "dS0")):
        c.inside(g, w, s, what, state="S" in what)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("name", ["Q", "K", "V", "dO"])
@pytest.mark.parametrize("dim", [64, 128])
def test_a_token_that_is_not_finite_is_not_forgotten(dtype, name, dim):
    """Decays whose powers are 0 in 32 bits after some tokens, and 0 itself: what the formula has a token in that is not
    finite is not finite, however far behind it, and the rest is right."""
    c = Case(dtype, [200], 2, 2, dim, dim, True, decays=[1e-4, 0.0], seed=19)
    x = getattr(c, name)
    x[3, 37], x[dim + 5, 70], x[:, 130] = float("inf"), float("nan"), float("nan")
    with np.errstate(invalid="ignore"):
        forward, backward = (c.forward(), c.forward(size=True)), (c.backward(), c.backward(size=True))
    for i, (g, what) in enumerate(zip(_fwd(c), ("O", "ST"))):
        _right(c, g, forward[0][i], forward[1][i], what, i == 1)
    for i, (g, what) in enumerate(zip(_bwd(c), ("dQ", "dK", "dV", "dS0"))):
        _right(c, g, backward[0][i], backward[1][i], what, i == 3)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("shape", SHAPES)
def test_nothing_behind_the_operands_is_read(dtype, shape):
    """NaN behind each operand's end, in the workspace and in the outputs changes no bit of what is computed."""
    from gpu_util import device
    dev, nan = device(), float("nan")
    c = Case(dtype, *shape, seed=sum(shape[0]) + 2)
    d = c.desc()

    def inside(t, fill):  # on 16 bytes, `fill` behind it
        if t is None:
            return None
        whole = torch.full((t.numel() + 4096,), fill, dtype=t.dtype, device=dev)
        whole[:t.numel()] = t.contiguous().flatten().to(dev)
        return whole[:t.numel()].view(t.shape)

    def run(fill):
        put = [inside(x, fill) for x in (c.Q, c.K, c.V, c.g, c.S0, c.dO, c.dST)]
        ws = torch.full((api.ard_linattn_workspace_bytes(d) // 4 + 4,), fill, device=dev)
        O, ST = torch.full_like(put[5], fill), torch.full((len(c.lens), c.heads, c.dk, c.dv), fill, device=dev)
        grads = [torch.full_like(x, fill) for x in put[:3]] + [torch.full_like(ST, fill)]
        api.ard_linattn_fwd(d, *put[:5], O, ST, ws)
        ws.fill_(fill)
        api.ard_linattn_bwd(d, *put, *grads, ws)
        torch.cuda.synchronize()
        on = torch.zeros(c.n, dtype=torch.bool)
        for b, e in c.spans:
            on[b:e] = True
        return [x[:, on] for x in (O, *grads[:3])] + [ST, grads[3]]
    for got, want in zip(run(nan), run(0.0)):
        assert torch.equal(got, want)
