"""The end of a training step as a run of calls on one stream and in one workspace: FC layer -> norm of its output and a
residual stream -> the head's loss without logits, under a row pattern -> all gradients back to the FC layer ->
orthogonalised updates of both weight matrices.

Tolerances: every stage against the definition in 64 bits on the inputs that the stage before left, per value, with
u = 2^-24 a rounding to fp32 and 2^-8 one to bf16 (2^-24 is taken for fp32 outputs): a sum of n terms is off by n u of the
sum of their absolute values; the norm's inverse root 3 u, its product with s and gain 3 more; the norm's gradient three
roundings in each of its two terms, its mean three, the difference and the last product two.
"""
import pytest
import torch

import test_headloss as head
import test_muon as muon
from paper_1805_08939_amd import api, synth

U, UBF = 2.0 ** -24, 2.0 ** -8
B, K, N, V, PERIOD, OFFSET = 45, 96, 200, 333, 3, 1
KEPT = slice(OFFSET, None, PERIOD)


class Step:
    def __init__(self, dtype, seed=1):
        from gpu_util import ard_dtype, device
        self.dev, self.st, self.dt = device(), synth.storage_dtype(dtype), ard_dtype(dtype)
        gen = torch.Generator(device=self.dev).manual_seed(seed)
        rand = lambda *s, std=1.0: torch.randn(*s, generator=gen, device=self.dev) * std  # noqa: E731
        self.X, self.R = rand(K, B).to(self.st), rand(N, B, std=3.0).to(self.st)
        self.W, self.b = rand(N, K, std=K ** -0.5).to(self.st), rand(N, std=0.1)
        self.gain = 1.0 + rand(N, std=0.2)
        self.Wh, self.bh = rand(V, N, std=2.0 * (PERIOD / N) ** 0.5).to(self.st), rand(V, std=0.3)
        self.labels = torch.randint(0, V, (B,), generator=gen, device=self.dev, dtype=torch.int32)
        self.labels[::9] = -1
        self.share = torch.full((B,), 1.0 / B, device=self.dev)
        self.VW, self.VWh = rand(N, K, std=1e-3), rand(V, N, std=1e-3)
        e = lambda *s, t=torch.float32: torch.empty(*s, dtype=t, device=self.dev)  # noqa: E731
        self.H, self.S, self.Y, self.inv = e(N, B, t=self.st), e(N, B, t=self.st), e(N, B, t=self.st), e(B)
        self.loss, self.stats = e(B), e(2, B)
        self.dY, self.dS, self.dX = e(N, B, t=self.st), e(N, B, t=self.st), e(K, B, t=self.st)
        self.dWh, self.dbh, self.dgain, self.dW, self.db = e(V, N), e(V), e(N), e(N, K), e(N)
        self.fc = api.fc_desc(self.dt, B, K, N, None, None)
        self.norm = api.rmsnorm_desc(self.dt, B, N, 1e-5)
        self.plan = api.ard_plan_rows(N, PERIOD, OFFSET, None)
        self.head = api.headloss_desc(self.dt, B, N, V, self.plan)
        self.over = api.fc_desc(self.dt, B, N, V, self.plan, None)
        need = max(api.ard_fc_workspace_bytes(self.fc), api.ard_rmsnorm_workspace_bytes(self.norm),
                   api.ard_headloss_workspace_bytes(self.head), api.ard_fc_muon_workspace_bytes(self.fc),
                   api.ard_fc_muon_workspace_bytes(self.over))
        self.ws = torch.full((need // 4 + 4,), float("nan"), device=self.dev)

    def forward(self):
        api.ard_fc_fwd(self.fc, self.X, self.W, self.b, self.H, self.ws)
        api.ard_rmsnorm_fwd(self.norm, self.H, self.R, self.gain, self.S, self.Y, self.inv, self.ws)
        api.ard_headloss_fwd(self.head, self.Y, self.Wh, self.bh, self.labels, self.loss, self.stats, self.ws)

    def backward(self):
        api.ard_headloss_bwd(self.head, self.Y, self.Wh, self.bh, self.labels, self.stats, self.share, self.dY, self.dWh,
                             self.dbh, self.ws)
        api.ard_rmsnorm_bwd(self.norm, self.S, self.gain, self.inv, self.dY, None, self.dS, self.dgain, self.ws)
        api.ard_fc_bwd(self.fc, self.X, self.dS, None, self.W, self.dX, self.dW, self.db, self.ws)

    def update(self):
        api.ard_fc_muon(self.over, None, self.Wh, self.VWh, self.dWh, ws=self.ws)
        api.ard_fc_muon(self.fc, None, self.W, self.VW, self.dW, ws=self.ws)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_every_stage_on_what_the_one_before_left(dtype):
    s = Step(dtype)
    s.forward()
    s.backward()
    W0, Wh0, V0, Vh0 = s.W.double(), s.Wh.double(), s.VW.double(), s.VWh.double()
    s.update()
    torch.cuda.synchronize()
    d = lambda t: t.double()  # noqa: E731
    out = UBF if dtype == "bf16" else U
    inside = head._inside
    X, R, H, S, Y, dY, dS, gain = d(s.X), d(s.R), d(s.H), d(s.S), d(s.Y), d(s.dY), d(s.dS), d(s.gain)[:, None]
    want = W0 @ X + d(s.b)[:, None]
    inside(s.H, want, (K + 2) * U * (W0.abs() @ X.abs() + d(s.b).abs()[:, None]) + out * want.abs() * (1 + UBF), "H")
    v = H + R
    inv = (v.square().mean(0) + 1e-5).rsqrt()
    inside(s.S, v, (out + U) * v.abs(), "S")
    inside(s.Y, gain * v * inv, (8 * U + out * (1 + UBF)) * (gain * v * inv).abs(), "Y")
    inside(s.inv, inv, 4 * U * inv, "inv")
    Wk, Yk = Wh0[:, KEPT], Y[KEPT]
    loss, eloss, dz, edz = head._reference(Yk, Wk, d(s.bh), s.labels.long(), d(s.share))
    inside(s.loss, loss, eloss, "loss")
    inside(s.dbh, dz.sum(1), edz.sum(1) + B * U * dz.abs().sum(1), "dbias of the head")
    edz = edz + (UBF if dtype == "bf16" else 0) * dz.abs()
    want, bound = Wk.T @ dz, Wk.abs().T @ (edz + (V + 2) * U * dz.abs())
    inside(s.dY[KEPT], want, bound + out * (want.abs() + bound), "dY")
    on = (s.labels >= 0).double()
    want, bound = dz @ (Yk * on).T, (edz + (B + 2) * U * dz.abs()) @ (Yk.abs() * on).T
    inside(s.dWh[:, KEPT], want, bound + U * want.abs(), "dW of the head")
    drop = torch.ones(N, dtype=torch.bool, device=s.dev)
    drop[KEPT] = False
    assert (s.dY[drop] == 0).all() and (s.dWh[:, drop] == 0).all()
    xh, u = S * d(s.inv), gain * dY
    want = d(s.inv) * (u - xh * (u * xh).mean(0))
    size = d(s.inv) * (u.abs() + xh.abs() * (u * xh).abs().mean(0))
    inside(s.dS, want, 8 * U * size + out * want.abs() * (1 + UBF), "dS")
    inside(s.dgain, (dY * xh).sum(1), (B + 4) * U * (dY * xh).abs().sum(1), "dgain")
    want, bound = dS @ X.T, (B + 2) * U * (dS.abs() @ X.abs().T)
    inside(s.dW, want, bound + U * want.abs(), "dW")
    inside(s.db, dS.sum(1), (B + 2) * U * dS.abs().sum(1), "db")
    o = api.ard_muon_opts_default()
    muon._check(d(s.W), W0, V0, d(s.dW), o, dtype, N / K)
    kept = Wk.shape[1]
    muon._check(d(s.Wh)[:, KEPT], Wk, Vh0[:, KEPT], d(s.dWh)[:, KEPT], o, dtype, V / kept)
    assert torch.equal(d(s.Wh)[:, drop], Wh0[:, drop]) and torch.equal(d(s.VWh)[:, drop], Vh0[:, drop])


@pytest.mark.gpu
def test_gradients_of_the_run_against_differences():
    """Along each gradient's own values at half of its places: differences in 64 bits of the definition. The gradients are
    products of at most four matrices with up to 333 terms a sum, each off by (n + 2) u of its absolute values, and those are
    up to sqrt(n) of a product's own size: 4 x 335 x 2^-24 x 18.3 = 1.5e-3 of the gradient's norm; the differences'
    step of 1e-4 of the weights adds 1e-8 of the third derivative's."""
    s = Step("f32")
    s.forward()
    s.backward()
    torch.cuda.synchronize()
    drop = torch.ones(N, dtype=torch.bool, device=s.dev)
    drop[KEPT] = False

    def value(W, gain, Wh, R):
        v = W @ s.X.double() + s.b.double()[:, None] + R
        y = gain[:, None] * v / (v.square().mean(0) + 1e-5).sqrt()
        y[drop] = 0
        z = Wh @ y + s.bh.double()[:, None]
        each = torch.logsumexp(z, 0) - z.gather(0, s.labels.long().clamp(min=0)[None])[0]
        return float((each * s.share.double() * (s.labels >= 0)).sum())

    at = [s.W.double(), s.gain.double(), s.Wh.double(), s.R.double()]
    gen = torch.Generator(device=s.dev).manual_seed(9)
    for i, grad in enumerate((s.dW, s.dgain, s.dWh, s.dS)):
        grad = grad.double()
        step = grad * (torch.rand(grad.shape, generator=gen, device=s.dev) < 0.5)
        h = 1e-4 * float(at[i].norm() / step.norm())
        up, down = list(at), list(at)
        up[i], down[i] = at[i] + h * step, at[i] - h * step
        want, got = (value(*up) - value(*down)) / (2 * h), float((grad * step).sum())
        assert got > 0 and abs(got - want) <= 2e-3 * float(grad.norm() * step.norm()), (i, got, want)


@pytest.mark.gpu
def test_captured_steps_are_eager_ones():
    """Three replays of a captured step, with eager steps between them, leave what three eager steps leave."""
    one, two = Step("bf16"), Step("bf16")

    def step(s):
        s.forward()
        s.backward()
        s.update()

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step(Step("bf16", seed=2))  # loads every kernel
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step(one)
    for _ in range(3):
        graph.replay()
        step(two)
        torch.cuda.synchronize()
        for name in ("loss", "dY", "dWh", "dW", "dgain", "W", "Wh", "VW", "VWh"):
            assert torch.equal(getattr(one, name), getattr(two, name)), name
