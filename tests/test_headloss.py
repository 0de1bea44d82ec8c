"""The head's cross entropy without logits: the oracle against differences (CPU), refusals (CPU), and the kernels against
the definition in 64 bits (GPU).

Tolerances, per value, with u = 2^-24 a rounding to fp32 and 2^-8 one to bf16: a sum of n terms is off by at most n u of
the sum of their absolute values, an exponential by the rounding of its argument and 4 u.
"""
import numpy as np
import pytest
import torch

from oracle import headloss as ohead
from paper_1805_08939_amd import _ffi, api, synth

U, UBF = 2.0 ** -24, 2.0 ** -8
FULL, INPUT = api.ARD_WEIGHTS_FULL, api.ARD_WEIGHTS_INPUT_MAJOR


# ---------------------------------------------------------------- the oracle

def test_oracle_backward_is_the_forward_differenced():
    r = np.random.default_rng(4)
    X, W, b, dl = r.normal(size=(4, 5)), r.normal(size=(6, 5)), r.normal(size=6), r.normal(size=4)
    labels, keep = np.array([0, 5, -1, 3]), np.array([1.0, 0, 1, 0, 1])
    b[2] = -np.inf
    value = lambda X, W, b: float((ohead.forward(X, W, b, labels, keep)[0] * dl).sum())  # noqa: E731
    grads = ohead.backward(X, W, b, labels, keep, dl)
    for n, p in enumerate((X, W, b)):
        for at in np.ndindex(p.shape):
            if not np.isfinite(p[at]):
                assert grads[n][at] == 0
                continue
            e = np.zeros_like(p)
            e[at] = 1e-6
            up, down = [X, W, b], [X, W, b]
            up[n], down[n] = p + e, p - e
            assert abs((value(*up) - value(*down)) / 2e-6 - grads[n][at]) < 1e-7 * (1 + abs(grads[n][at]))


# ---------------------------------------------------------------- refusals

def test_refuses_bad_calls():
    a = 4096  # an aligned address; never read

    def refused(status, call, *args):
        with pytest.raises(api.ArdError) as e:
            call(*args, stream=0)
        assert e.value.status == status and e.value.message

    space = (a, 1 << 40)
    good = dict(dtype=api.ARD_F32, batch=4, in_features=8, classes=6)
    for bad, status in ((dict(dtype=7), 2), (dict(batch=0), 1), (dict(in_features=-1), 1), (dict(classes=0), 1),
                        (dict(weight_layout=api.ARD_WEIGHTS_COMPACT), 1), (dict(weight_layout=9), 1), (dict(dropped=3), 1),
                        (dict(grad_dtype=api.ARD_BF16), 1), (dict(grad_dtype=5), 1), (dict(batch=1 << 22), 2),
                        (dict(in_features=1 << 22), 2), (dict(weight_layout=INPUT, classes=1 << 22), 2),
                        (dict(in_plan=api.ard_plan_rows(7, 2, 0, None)), 1)):
        d = api.headloss_desc(**{**good, **bad})
        assert api.ard_headloss_workspace_bytes(d) == 0
        refused(status, api.ard_headloss_fwd, d, a, a, a, a, a, a, space)
        refused(status, api.ard_headloss_bwd, d, a, a, a, a, a, a, a, a, a, space)
    d = api.headloss_desc(**good)
    need = api.ard_headloss_workspace_bytes(d)
    assert need > 0
    fwd, bwd = (a,) * 6, (a,) * 9
    for at, x in ((0, None), (1, None), (3, None), (4, None), (0, a + 8), (1, a + 4), (2, a + 4), (3, a + 4), (4, a + 8), (5, a + 4)):
        refused(1, api.ard_headloss_fwd, d, *(x if i == at else g for i, g in enumerate(fwd)), space)
    for at, x in ((0, None), (1, None), (3, None), (4, None), *((i, a + 4) for i in range(9))):
        refused(1, api.ard_headloss_bwd, d, *(x if i == at else g for i, g in enumerate(bwd)), space)
    refused(5, api.ard_headloss_fwd, d, *fwd, None)
    refused(5, api.ard_headloss_bwd, d, *bwd, None)
    refused(5, api.ard_headloss_bwd, d, *bwd, (a, 16))
    refused(1, api.ard_headloss_bwd, d, *bwd, (a + 8, 1 << 40))
    assert _ffi.lib().ard_headloss_workspace_bytes(None) == 0


@pytest.mark.parametrize("classes", [6, 600])
def test_refuses_gradients_in_the_inputs_buffers(classes):
    X, W, b, labels, stats, dl, dX, dW, db = (4096 * (i + 1) for i in range(9))
    d = api.headloss_desc(api.ARD_F32, 4, 8, classes)
    for outs in ((X, dW, db), (dX, W, db), (dX, dW, b), (dX, dW, dl)):
        with pytest.raises(api.ArdError) as e:
            api.ard_headloss_bwd(d, X, W, b, labels, stats, dl, *outs, (1 << 20, 1 << 40), stream=0)
        assert e.value.status == 1 and "buffer" in e.value.message


# ---------------------------------------------------------------- the kernels

def _fenced(t, dev):
    """The tensor on the device between values that are not numbers (labels: that are classes)."""
    n, pad = t.numel(), 64 // t.element_size()
    whole = torch.full((n + 2 * pad,), float("nan") if t.is_floating_point() else 0, dtype=t.dtype, device=dev)
    whole[pad:pad + n] = t.reshape(-1).to(dev)
    return whole[pad:pad + n].view(t.shape)


def _guarded(shape, dtype, dev, fill=3.0):
    n = int(np.prod(shape))
    pad = 64 // torch.empty(0, dtype=dtype).element_size()
    whole = torch.full((n + 2 * pad,), fill, dtype=dtype, device=dev)

    def untouched():
        assert (whole[:pad] == fill).all() and (whole[pad + n:] == fill).all()
    return whole[pad:pad + n].view(shape), untouched


def _reference(X, W, bias, labels, dloss):
    """The definition and error bounds in 64 bits on the device; X[K][B], W[V][K] of kept inputs only."""
    V, K = W.shape
    z = W @ X + bias[:, None]
    ez = (K + 2) * U * (W.abs() @ X.abs() + torch.where(bias.isinf(), torch.zeros_like(bias), bias).abs()[:, None])
    top = z.max(0).values
    lse = torch.logsumexp(z, 0)
    on = (labels >= 0) & (labels < V)
    at = labels.clamp(0, V - 1).long()[None]
    zl = z.gather(0, at)[0]
    loss = torch.where(on, lse - zl, torch.zeros_like(lse))
    # the sum: terms of a tile's lane, tiles and merges, an exponential each, arguments no wider than the spread that matters
    spread = 30.0
    rel = (spread + 100 + V / 64) * 4 * U
    es = ez.max(0).values + rel
    eloss = on * (es + ez.gather(0, at)[0] + 4 * U * (loss.abs() + lse.abs() + top.abs() + zl.abs() + spread))
    p = torch.exp(z - lse)
    told = (torch.arange(V, device=z.device)[:, None] == labels[None]).double()
    dl = dloss * on
    dz = (p - told) * dl
    wide = torch.where(p > 0, (z - top).abs(), torch.zeros_like(z))
    ep = p * torch.expm1(ez + es + (wide + 8) * U)
    edz = dl.abs() * (ep + 2 * U * (p + told))
    return loss, eloss, dz, edz


def _inside(got, want, bound, what):
    got = got.double()
    if got.numel() == 0:
        return
    assert torch.isfinite(got).all(), what
    off = (got - want).abs()
    worst = (off - bound).argmax()
    assert (off <= bound).all(), f"{what}: {float(off.max()):.3e} off; {float(off.flatten()[worst]):.3e} where " \
                                 f"{float(bound.flatten()[worst]):.3e} is allowed"


def _run(dtype, B, K, V, period, offset, layout, seed=0, bias=True, dropped=api.ARD_DROPPED_ZERO, grad=None, std=2.5,
         fence=True):
    from gpu_util import ard_dtype, device, workspace
    dev, st = device(), synth.storage_dtype(dtype)
    gen = torch.Generator(device=dev).manual_seed(seed + B + K + V)
    rand = lambda *s: torch.randn(*s, generator=gen, device=dev)  # noqa: E731
    wrap = (lambda t: _fenced(t, dev)) if fence else (lambda t: t)
    plan = api.ard_plan_rows(K, period, offset, None)
    kept = slice(offset, None, period)
    X, W = rand(K, B).to(st), (rand(V, K) * std / max(1, K // period) ** 0.5).to(st)
    if period > 1:  # what is dropped is never read
        drop = torch.ones(K, dtype=torch.bool, device=dev)
        drop[kept] = False
        X[drop], W[:, drop] = float("nan"), float("nan")
    b = rand(V) * 0.5 if bias else None
    labels = torch.randint(0, V, (B,), generator=gen, device=dev, dtype=torch.int32)
    labels[2::7] = -1
    labels[3::11] = V
    X[kept, 2::7] = float("nan")  # padding holds anything
    dl = rand(B)
    g = grad or dtype
    desc = api.headloss_desc(ard_dtype(dtype), B, K, V, plan, layout, dropped, ard_dtype(g))
    ws = workspace(api.ard_headloss_workspace_bytes(desc))
    ws.fill_(float("nan"))
    stored = lambda t: t if layout == FULL else t.T.contiguous()  # noqa: E731
    given = [wrap(X), wrap(stored(W)), None if b is None else wrap(b), wrap(labels)]
    (loss, l_ok), (stats, s_ok) = _guarded((B,), torch.float32, dev), _guarded((2, B), torch.float32, dev)
    api.ard_headloss_fwd(desc, *given, loss, stats, ws)
    dld = wrap(dl)
    (dX, x_ok), (dW, w_ok) = _guarded((K, B), st, dev), _guarded((V, K) if layout == FULL else (K, V), synth.storage_dtype(g), dev)
    db, b_ok = _guarded((V,), torch.float32, dev)
    ws.fill_(float("nan"))
    api.ard_headloss_bwd(desc, *given, stats, dld, dX, dW, db, ws)
    torch.cuda.synchronize()
    for ok in (l_ok, s_ok, x_ok, w_ok, b_ok):
        ok()
    X[kept, 2::7] = 0
    return X, W, b, labels, dl, loss, dX, (dW if layout == FULL else dW.T), db, kept


SIZES = [  # dtype, B, K, V, period, offset, layout
    ("f32", 1, 1, 1, 1, 0, FULL), ("bf16", 1, 3, 2, 1, 0, FULL), ("bf16", 5, 64, 10, 1, 0, FULL), ("f32", 128, 200, 10, 2, 1, INPUT),
    ("f32", 33, 65, 70, 1, 0, FULL), ("bf16", 33, 65, 70, 1, 0, INPUT), ("f32", 64, 130, 203, 3, 2, FULL), ("bf16", 48, 136, 200, 3, 0, INPUT),
    ("bf16", 40, 1000, 333, 2, 0, FULL), ("f32", 700, 150, 880, 2, 1, INPUT), ("f32", 701, 75, 4001, 1, 0, FULL),
    ("f32", 1024, 40, 5000, 1, 0, FULL), ("f32", 2000, 24, 9000, 1, 0, INPUT), ("f32", 1030, 20, 6002, 2, 0, INPUT),
    ("bf16", 331, 1023, 501, 1, 0, FULL), ("bf16", 2048, 40, 2048, 1, 0, FULL), ("bf16", 4096, 24, 4100, 1, 0, FULL),
    ("bf16", 4090, 32, 2050, 1, 0, FULL), ("bf16", 128, 24, 65536, 1, 0, FULL), ("bf16", 2000, 72, 2056, 2, 1, INPUT),
    ("bf16", 2100, 33, 2053, 1, 0, INPUT), ("bf16", 4096, 40, 8192, 1, 0, INPUT), ("bf16", 4101, 39, 8200, 3, 1, FULL),
    ("bf16", 9, 4, 12, 8, 7, FULL), ("f32", 9, 4, 12, 8, 7, INPUT), ("bf16", 24, 520, 30000, 1, 0, FULL), ("f32", 12, 77, 20001, 1, 0, FULL),
    # dz in several pieces
    ("bf16", 40000, 16, 3500, 1, 0, FULL), ("f32", 40001, 12, 1700, 1, 0, FULL), ("bf16", 40008, 16, 3400, 2, 1, INPUT),
]


@pytest.mark.gpu
@pytest.mark.parametrize("size", SIZES, ids=lambda s: "-".join(map(str, s)))
def test_loss_and_gradients(size):
    dtype, B, K, V, period, offset, layout = size
    X, W, b, labels, dl, loss, dX, dW, db, kept = _run(*size, bias=V % 3 != 0, grad="f32" if K % 2 else None)
    bias = b.double() if b is not None else torch.zeros(V, dtype=torch.float64, device=X.device)
    Xk, Wk = X[kept].double(), W[:, kept].double()
    want, eloss, dz, edz = _reference(Xk, Wk, bias, labels.long(), dl.double())
    _inside(loss, want, eloss, "loss")
    assert (loss[2::7] == 0).all() and (loss[3::11] == 0).all()
    outX, outW = (UBF if t.dtype == torch.bfloat16 else U for t in (dX, dW))
    _inside(db, dz.sum(1), edz.sum(1) + B * U * dz.abs().sum(1), "dbias")
    edz = edz + (UBF if dtype == "bf16" else 0) * dz.abs()  # dz as an operand
    wantX, bound = Wk.T @ dz, Wk.abs().T @ (edz + (V + 2) * U * dz.abs())
    _inside(dX[kept], wantX, bound + outX * (wantX.abs() + bound), "dX")
    on = ((labels >= 0) & (labels < V)).double()
    wantW, bound = dz @ (Xk * on).T, (edz + (B + 2) * U * dz.abs()) @ (Xk.abs() * on).T
    _inside(dW[:, kept], wantW, bound + outW * (wantW.abs() + bound), "dW")
    if period > 1:
        drop = torch.ones(K, dtype=torch.bool, device=X.device)
        drop[kept] = False
        assert (dX[drop] == 0).all() and (dW[:, drop] == 0).all()


@pytest.mark.gpu
@pytest.mark.parametrize("size", [("bf16", 2100000, 6, 33, 2, 1, FULL), ("bf16", 24, 8, 2100000, 2, 0, INPUT),
                                  ("f32", 24, 8, 2100000, 2, 1, INPUT)], ids=lambda s: "-".join(map(str, s)))
def test_kept_rows_more_than_2_22_elements_apart(size):
    test_loss_and_gradients(size)


@pytest.mark.gpu
@pytest.mark.parametrize("size", [
    # 64 x 128 tiles of bf16
    ("bf16", 331, 520, 5001, 1, 0, FULL), ("bf16", 1024, 300, 1000, 1, 0, INPUT), ("bf16", 331, 522, 5001, 1, 0, INPUT),
    # 256 x 128 and 128 x 128 tiles of parts, in the products too
    ("f32", 700, 1500, 8800, 2, 1, INPUT), ("f32", 703, 500, 6001, 1, 0, FULL), ("f32", 1500, 400, 2000, 1, 0, FULL),
    ("f32", 1024, 64, 3100, 1, 0, INPUT),
    # few classes: one and two blocks of 16, rows of weights on and off 16 bytes, shares of dX's rows, more inputs than
    # a pass of the waves
    ("f32", 37, 130, 32, 1, 0, FULL), ("f32", 16, 260, 17, 1, 0, FULL), ("f32", 100, 777, 20, 2, 1, INPUT),
    ("f32", 20, 3000, 10, 1, 0, FULL), ("f32", 257, 1100, 25, 3, 2, FULL), ("f32", 5000, 300, 12, 1, 0, INPUT),
    ("f32", 1, 1024, 16, 2, 0, FULL), ("f32", 48, 2500, 31, 4, 3, INPUT), ("f32", 17, 36, 3, 40, 39, FULL),
], ids=lambda s: "-".join(map(str, s)))
def test_further_tiles_and_few_classes(size):
    test_loss_and_gradients(size)


@pytest.mark.gpu
@pytest.mark.parametrize("layout", [FULL, INPUT])
def test_few_classes_leave_dropped_inputs_and_masked_columns(layout):
    _, _, _, labels, _, loss, dX, dW, _, kept = _run("f32", 40, 600, 10, 3, 1, layout, dropped=api.ARD_DROPPED_SKIP)
    drop = torch.ones(600, dtype=torch.bool, device=dX.device)
    drop[kept] = False
    off = (labels < 0) | (labels >= 10)
    assert (dX[drop] == 3).all() and (dW[:, drop] == 3).all()
    assert off.any() and (loss[off] == 0).all() and (dX[kept][:, off] == 0).all() and not (dX[kept][:, ~off] == 0).any()


@pytest.mark.gpu
@pytest.mark.parametrize("size", [("bf16", 90000, 16, 3500, 1, 0, FULL), ("bf16", 90009, 24, 3333, 2, 1, FULL),
                                  ("bf16", 90008, 16, 3400, 2, 1, INPUT)], ids=lambda s: "-".join(map(str, s)))
def test_gradients_of_several_pieces_in_bf16(size):
    test_loss_and_gradients(size)


@pytest.mark.gpu
@pytest.mark.parametrize("layout", [FULL, INPUT])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_dropped_inputs_left_as_they_are(dtype, layout):
    _, _, _, _, _, _, dX, dW, _, kept = _run(dtype, 64, 48, 100, 3, 1, layout, dropped=api.ARD_DROPPED_SKIP)
    drop = torch.ones(48, dtype=torch.bool, device=dX.device)
    drop[kept] = False
    assert (dX[drop] == 3).all() and (dW[:, drop] == 3).all()
    assert not (dX[kept] == 3).all() and not (dW[:, kept] == 3).all()


@pytest.mark.gpu
@pytest.mark.parametrize("dtype,B,K,V", [("bf16", 40, 64, 90), ("f32", 40, 64, 90), ("bf16", 2048, 32, 2304), ("f32", 1100, 20, 5000)])
def test_masked_classes_and_values_that_are_not_finite(dtype, B, K, V):
    from gpu_util import ard_dtype, device, workspace
    dev, st = device(), synth.storage_dtype(dtype)
    gen = torch.Generator(device=dev).manual_seed(11)
    X = torch.randn(K, B, generator=gen, device=dev).to(st)
    W = torch.randn(V, K, generator=gen, device=dev).to(st)
    b = torch.randn(V, generator=gen, device=dev)
    b[V // 2:] = -float("inf")
    labels = torch.randint(0, V // 2, (B,), generator=gen, device=dev, dtype=torch.int32)
    labels[5] = V - 1                # a masked class
    X[:, 7] = 0
    X[3, 7], W[:V // 2, 3] = float("nan"), 0  # a column that is not finite
    desc = api.headloss_desc(ard_dtype(dtype), B, K, V)
    ws = workspace(api.ard_headloss_workspace_bytes(desc))
    loss, stats = torch.empty(B, device=dev), torch.empty(2, B, device=dev)
    dX, dW, db = torch.empty_like(X), torch.empty(V, K, device=dev), torch.empty(V, device=dev)
    api.ard_headloss_fwd(desc, X, W, b, labels, loss, stats, ws)
    api.ard_headloss_bwd(desc, X, W, b, labels, stats, None, dX, None, None, ws)
    torch.cuda.synchronize()
    assert torch.isinf(loss[5]) and loss[5] > 0 and torch.isnan(loss[7])
    ok = torch.ones(B, dtype=torch.bool, device=dev)
    ok[5] = ok[7] = False
    assert torch.isfinite(loss[ok]).all() and torch.isfinite(dX[:, ok]).all() and torch.isnan(dX[:, 7]).all()
    # the masked label pulls with its whole weight: dX = W^T (q - onehot)
    half = W[:V // 2].double()
    q = torch.softmax(half @ X[:, 5].double() + b[:V // 2].double(), 0)
    want = half.T @ q - W[V - 1].double()
    size = half.abs().T @ q + W[V - 1].double().abs()
    assert ((dX[:, 5].double() - want).abs() <= (2 * UBF + 2e-4) * size).all()
    # without the column that is not finite: masked classes have no gradient but the label's
    labels[7] = -1
    api.ard_headloss_fwd(desc, X, W, b, labels, loss, stats, ws)
    api.ard_headloss_bwd(desc, X, W, b, labels, stats, None, dX, dW, db, ws)
    assert loss[7] == 0 and (dX[:, 7] == 0).all()
    assert torch.isfinite(dW).all() and (dW[V // 2:V - 1] == 0).all() and (db[V // 2:V - 1] == 0).all() and db[V - 1] == -1
    # every class masked
    b.fill_(-float("inf"))
    X[3, 7] = 1
    api.ard_headloss_fwd(desc, X, W, b, labels, loss, stats, ws)
    api.ard_headloss_bwd(desc, X, W, b, labels, stats, None, dX, dW, db, ws)
    for t in (loss, dX, dW, db):
        assert (t == 0).all()


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_outputs_left_out_and_logits_far_from_zero(dtype):
    """Calls without some outputs give the same bits; logits of a few hundred do not overflow."""
    from gpu_util import ard_dtype, device, workspace
    dev, st = device(), synth.storage_dtype(dtype)
    B, K, V = 72, 96, 1000
    gen = torch.Generator(device=dev).manual_seed(5)
    X, W = torch.randn(K, B, generator=gen, device=dev).to(st), (20 * torch.randn(V, K, generator=gen, device=dev)).to(st)
    labels = torch.randint(0, V, (B,), generator=gen, device=dev, dtype=torch.int32)
    desc = api.headloss_desc(ard_dtype(dtype), B, K, V)
    ws = workspace(api.ard_headloss_workspace_bytes(desc))
    loss, stats = torch.empty(B, device=dev), torch.empty(2, B, device=dev)
    api.ard_headloss_fwd(desc, X, W, None, labels, loss, stats, ws)
    z = W.double() @ X.double()
    want = torch.logsumexp(z, 0) - z.gather(0, labels.long()[None])[0]
    assert z.max() > 500
    assert ((loss.double() - want).abs() <= (2 * K + 40) * U * (W.double().abs() @ X.double().abs()).max()).all()
    alone = torch.empty_like(loss)
    api.ard_headloss_fwd(desc, X, W, None, labels, alone, None, ws)
    assert torch.equal(alone, loss)
    outs = [torch.empty_like(X), torch.empty(V, K, device=dev), torch.empty(V, device=dev)]
    api.ard_headloss_bwd(desc, X, W, None, labels, stats, None, *outs, ws)
    for i in range(3):
        one = torch.empty_like(outs[i])
        api.ard_headloss_bwd(desc, X, W, None, labels, stats, None, *(one if j == i else None for j in range(3)), ws)
        assert torch.equal(one, outs[i])


@pytest.mark.gpu
def test_captured_and_on_another_stream():
    from gpu_util import device, workspace
    dev = device()
    B, K, V, period = 200, 96, 3000, 2
    desc = api.headloss_desc(api.ARD_BF16, B, K, V, api.ard_plan_rows(K, period, 1, None), FULL, grad_dtype=api.ARD_BF16)
    nbytes = api.ard_headloss_workspace_bytes(desc)
    ws, ws2 = workspace(nbytes), workspace(nbytes)
    X = torch.empty(K, B, dtype=torch.bfloat16, device=dev)
    W = torch.empty(V, K, dtype=torch.bfloat16, device=dev)
    labels = torch.empty(B, dtype=torch.int32, device=dev)
    make = lambda: [torch.empty(B, device=dev), torch.empty(2, B, device=dev), torch.empty_like(X), torch.empty_like(W),  # noqa: E731
                    torch.empty(V, device=dev)]
    outs, again = make(), make()

    def step(o, w):
        api.ard_headloss_fwd(desc, X, W, None, labels, o[0], o[1], w)
        api.ard_headloss_bwd(desc, X, W, None, labels, o[1], None, o[2], o[3], o[4], w)

    X.zero_(), W.zero_(), labels.zero_()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step(outs, ws)
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step(outs, ws)
    for seed in range(4):
        gen = torch.Generator(device=dev).manual_seed(seed)
        X.copy_(torch.randn(K, B, generator=gen, device=dev))
        W.copy_(torch.randn(V, K, generator=gen, device=dev))
        labels.copy_(torch.randint(-1, V, (B,), generator=gen, device=dev))
        graph.replay()
        with torch.cuda.stream(side):
            side.wait_stream(torch.cuda.current_stream())
            step(again, ws2)
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(outs, again))


@pytest.mark.gpu
@pytest.mark.parametrize("layout", [FULL, INPUT])
def test_weights_past_2_31_elements(layout):
    from gpu_util import device, workspace
    dev = device()
    B, K, V = 16, 4096, 600_064
    gen = torch.Generator(device=dev).manual_seed(2)
    W = torch.empty((V, K) if layout == FULL else (K, V), dtype=torch.bfloat16, device=dev).uniform_(-0.05, 0.05, generator=gen)
    X = torch.randn(K, B, generator=gen, device=dev).to(torch.bfloat16)
    labels = torch.tensor([0, V - 1, V // 2, 2 ** 31 // K + 5] * 4, dtype=torch.int32, device=dev)
    desc = api.headloss_desc(api.ARD_BF16, B, K, V, None, layout, grad_dtype=api.ARD_BF16)
    ws = workspace(api.ard_headloss_workspace_bytes(desc))
    loss, stats = torch.empty(B, device=dev), torch.empty(2, B, device=dev)
    dX, dW, db = torch.empty_like(X), torch.empty_like(W), torch.empty(V, device=dev)
    api.ard_headloss_fwd(desc, X, W, None, labels, loss, stats, ws)
    api.ard_headloss_bwd(desc, X, W, None, labels, stats, None, dX, dW, db, ws)
    rows = lambda v: (W[v] if layout == FULL else W[:, v].T).double()  # noqa: E731
    total = torch.zeros(B, dtype=torch.float64, device=dev)
    for v in torch.arange(V, device=dev).split(100_000):
        total += torch.exp(rows(slice(int(v[0]), int(v[-1]) + 1)) @ X.double()).sum(0)
    at = labels.long()
    zl = (rows(at) * X.double().T).sum(1)
    # sums of 4096 terms of at most 0.05 |x|, a rounding each at worst
    ez = K * U * 0.05 * X.double().abs().sum(0)
    assert ((loss.double() - (torch.log(total) - zl)).abs() <= 2 * ez + 1e-3).all()
    q = torch.exp(zl) / total
    told = q - 1
    others = [torch.exp((rows(at) @ X.double()))[i] / total for i in range(4)]
    for i in range(4):
        dz = others[i] - (at == at[i]).double()
        want = dz @ X.double().T
        got = (dW[at[i]] if layout == FULL else dW[:, at[i]]).double()
        assert ((got - want).abs() <= (3 * UBF + 1e-3) * (dz.abs() @ X.double().abs().T)).all()
        assert abs(float(db[at[i]]) - float(dz.sum())) <= 1e-3 * float(dz.abs().sum())
    assert told.max() < 0 and torch.isfinite(dX).all()


# ---------------------------------------------------------------- index limits, on the CPU

@pytest.mark.parametrize("dtype", [api.ARD_F32, api.ARD_BF16])
@pytest.mark.parametrize("classes", [10, 40])
def test_kept_inputs_of_input_major_weights_stay_in_32_bits(dtype, classes):
    """The kernels round the kept inputs up to their loops' steps in 32 bits: at most 2^31 - 2^16 of them."""
    a = 4096  # never read
    most = 2 ** 31 - 2 ** 16

    def desc(k, plan=None):
        return api.headloss_desc(dtype, 1, k, classes, plan, INPUT)
    assert api.ard_headloss_workspace_bytes(desc(most)) > 0
    assert api.ard_headloss_workspace_bytes(desc(2 ** 31 - 1, api.ard_plan_rows(2 ** 31 - 1, 2, 0, None))) > 0
    for k in (most + 1, 2 ** 31 - 3100, 2 ** 31 - 1):
        assert api.ard_headloss_workspace_bytes(desc(k)) == 0
        for call, n in ((api.ard_headloss_fwd, 6), (api.ard_headloss_bwd, 9)):
            with pytest.raises(api.ArdError) as e:
                call(desc(k), *(a * (i + 1) for i in range(n)), (a * 16, 1 << 60), stream=0)
            assert e.value.status == 2 and "kept inputs" in e.value.message


# ---------------------------------------------------------------- each argument, on the CPU

FWD = ("Xt", "W", "bias", "labels", "loss", "stats")
BWD = ("Xt", "W", "bias", "labels", "stats", "dloss", "dXt", "dW", "dbias")
NEEDED = {"fwd": {"Xt", "W", "labels", "loss"}, "bwd": {"Xt", "W", "labels", "stats"}}


@pytest.mark.parametrize("classes", [6, 600])
@pytest.mark.parametrize("way", ["fwd", "bwd"])
def test_refuses_each_argument_by_its_name(way, classes):
    """Arguments at addresses of their own, one of them wrong: no other check stands in for its own."""
    call, names = (api.ard_headloss_fwd, FWD) if way == "fwd" else (api.ard_headloss_bwd, BWD)
    d = api.headloss_desc(api.ARD_F32, 4, 8, classes)
    good, space = [4096 * (i + 1) for i in range(len(names))], (1 << 20, 1 << 40)

    def refused(status, what, args, ws):
        with pytest.raises(api.ArdError) as e:
            call(d, *args, ws, stream=0)
        assert e.value.status == status and what in e.value.message
    for at, name in enumerate(names):
        wrong = lambda x: [x if i == at else g for i, g in enumerate(good)]  # noqa: E731
        for off in (2, 4, 8):
            refused(1, name + " is not 16-byte aligned", wrong(good[at] + off), space)
        if name in NEEDED[way]:
            refused(1, name + " is NULL", wrong(None), space)
    need = api.ard_headloss_workspace_bytes(d)
    assert need > 0
    refused(5, "workspace", good, None)
    refused(5, "workspace", good, (1 << 20, need - 1))
    refused(1, "workspace", good, ((1 << 20) + 8, need))


# ---------------------------------------------------------------- buffers, on the CPU

@pytest.mark.parametrize("classes", [6, 600])
def test_refuses_outputs_in_the_buffers_of_other_arguments(classes):
    """As many columns as classes give loss and bias one shape: a workgroup would write what others still read."""
    d = api.headloss_desc(api.ARD_F32, classes, 8, classes)
    for call, n, outs in ((api.ard_headloss_fwd, 6, (4, 5)), (api.ard_headloss_bwd, 9, (6, 7, 8))):
        args = [4096 * (i + 1) for i in range(n)]
        for out in outs:
            for i in range(n):
                if i != out:
                    with pytest.raises(api.ArdError) as e:
                        call(d, *(args[i] if j == out else x for j, x in enumerate(args)), (1 << 20, 1 << 60), stream=0)
                    assert e.value.status == 1 and "buffer" in e.value.message


# ---------------------------------------------------------------- values next to the largest

@pytest.mark.gpu
@pytest.mark.parametrize("B,K,V", [(8, 40, 10), (33, 65, 70), (700, 100, 3000), (703, 500, 6001), (1500, 400, 2000)])
def test_fp32_operands_past_the_largest_bf16_number(B, K, V):
    """3.4e38 is finite in fp32 and rounds to infinity in bf16; so do weights and inputs of it, and dz."""
    from gpu_util import device, workspace
    dev = device()
    gen = torch.Generator(device=dev).manual_seed(B + V)
    rand = lambda *s: torch.randn(*s, generator=gen, device=dev)  # noqa: E731
    big = float(np.float32(3.4e38))
    assert torch.isinf(torch.tensor(big).bfloat16()) and torch.isfinite(torch.tensor(big))
    desc = api.headloss_desc(api.ARD_F32, B, K, V)
    ws = workspace(api.ard_headloss_workspace_bytes(desc))
    labels = torch.randint(0, V, (B,), generator=gen, device=dev, dtype=torch.int32)
    sign = torch.tensor([1.0, -1.0, 1.0, -1.0], device=dev)
    tiny = lambda *s: (1 + rand(*s).abs()).bfloat16().float()  # noqa: E731  one part of a product, above 2^-126
    for which in ("W", "X", "dloss"):
        W, X, b, dl = rand(V, K) / K ** 0.5, rand(K, B), rand(V), rand(B).clamp(-0.9, 0.9)
        rows = torch.arange(4, device=dev)
        if which == "W":     # four weights, each alone on its input, whose values are small
            W[:, :4] = 0
            W[2 * rows, rows], X[:4] = big * sign, 2.0 ** -120 * tiny(4, B)
        elif which == "X":
            X[rows, rows], W[:, :4] = big * sign, 2.0 ** -122 * tiny(V, 4)
        else:                # dz of the label is all of dloss
            dl[3], b[labels[3].long()] = big, -40.0
            X *= 2.0 ** -4
        loss, stats = torch.empty(B, device=dev), torch.empty(2, B, device=dev)
        dX, dW, db = torch.empty_like(X), torch.empty_like(W), torch.empty(V, device=dev)
        api.ard_headloss_fwd(desc, X, W, b, labels, loss, stats, ws)
        api.ard_headloss_bwd(desc, X, W, b, labels, stats, dl, dX, dW, db, ws)
        X, W = X.double(), W.double()
        want, eloss, dz, edz = _reference(X, W, b.double(), labels.long(), dl.double())
        edz = edz + 2.0 ** -126  # what parts hold
        _inside(loss, want, eloss, which + ": loss")
        _inside(db, dz.sum(1), edz.sum(1) + B * U * dz.abs().sum(1), which + ": dbias")
        # of each term six products, each lost below 2^-126
        want, bound = W.T @ dz, W.abs().T @ (edz + (V + 2) * U * dz.abs()) + (6 * V + 1) * 2.0 ** -126
        _inside(dX, want, bound + U * (want.abs() + bound), which + ": dX")
        want, bound = dz @ X.T, (edz + (B + 2) * U * dz.abs()) @ X.abs().T + (6 * B + 1) * 2.0 ** -126
        _inside(dW, want, bound + U * (want.abs() + bound), which + ": dW")


# ---------------------------------------------------------------- many columns

@pytest.mark.gpu
@pytest.mark.parametrize("dtype,V", [("f32", 10), ("f32", 32), ("f32", 40), ("f32", 200), ("bf16", 40), ("bf16", 200)])
def test_gradient_of_the_bias_over_many_columns(dtype, V):
    """The error does not grow with the columns, also where each of them adds the same: up to 64 columns are added in fp32 one
    after the other, their sums in 64 bits."""
    from gpu_util import ard_dtype, device, workspace
    dev, st, B, K = device(), synth.storage_dtype(dtype), 2 ** 21, 8
    gen = torch.Generator(device=dev).manual_seed(V)
    X = torch.full((K, B), 0.5, dtype=st, device=dev)
    W = torch.randn(V, K, generator=gen, device=dev).to(st)
    labels = torch.zeros(B, dtype=torch.int32, device=dev)
    desc = api.headloss_desc(ard_dtype(dtype), B, K, V)
    ws = workspace(api.ard_headloss_workspace_bytes(desc))
    loss, stats, db = torch.empty(B, device=dev), torch.empty(2, B, device=dev), torch.empty(V, device=dev)
    api.ard_headloss_fwd(desc, X, W, None, labels, loss, stats, ws)
    api.ard_headloss_bwd(desc, X, W, None, labels, stats, None, None, None, db, ws)
    one = torch.ones(1, dtype=torch.float64, device=dev)
    _, _, dz, edz = _reference(X[:, :1].double(), W.double(), 0 * one.repeat(V), labels[:1].long(), one)
    _inside(db, B * dz[:, 0], B * (edz[:, 0] + 66 * U * dz[:, 0].abs()), "dbias")


# ---------------------------------------------------------------- past 2^31 elements

@pytest.mark.gpu
@pytest.mark.parametrize("layout", [FULL, INPUT])
def test_input_gradients_of_weights_past_2_31_elements(layout):
    """dX against W^T dz in 64 bits; the labels' classes, all over the weights, carry most of it."""
    from gpu_util import device, workspace
    dev = device()
    B, K, V = 16, 4096, 600_064
    gen = torch.Generator(device=dev).manual_seed(3)
    W = torch.empty((V, K) if layout == FULL else (K, V), dtype=torch.bfloat16, device=dev).uniform_(-0.05, 0.05, generator=gen)
    X = torch.randn(K, B, generator=gen, device=dev).to(torch.bfloat16)
    labels = torch.tensor([0, V - 1, V // 2, 2 ** 31 // K + 5, 2 ** 31 // K - 1, V - 65, 1, 2 ** 30 // K] * 2, dtype=torch.int32, device=dev)
    desc = api.headloss_desc(api.ARD_BF16, B, K, V, None, layout)
    ws = workspace(api.ard_headloss_workspace_bytes(desc))
    loss, stats, dX = torch.empty(B, device=dev), torch.empty(2, B, device=dev), torch.empty_like(X)
    api.ard_headloss_fwd(desc, X, W, None, labels, loss, stats, ws)
    api.ard_headloss_bwd(desc, X, W, None, labels, stats, None, dX, None, None, ws)
    chunks = torch.arange(V, device=dev).split(100_000)
    rows = lambda v: (W[v[0]:v[-1] + 1] if layout == FULL else W[:, v[0]:v[-1] + 1].T.contiguous()).double()  # noqa: E731
    total = sum(torch.exp(rows(v) @ X.double()).sum(0) for v in chunks)
    # a logit: K terms of at most 0.05 |x|, a rounding each at worst; p: that twice, and the exponentials' 2^-17
    ez = 2 * K * U * 0.05 * X.double().abs().sum(0) + 2.0 ** -17
    want, bound = torch.zeros(K, B, dtype=torch.float64, device=dev), torch.zeros(K, B, dtype=torch.float64, device=dev)
    for v in chunks:
        w = rows(v)
        p = torch.exp(w @ X.double()) / total
        dz = p - (v[:, None] == labels[None].long()).double()
        want += w.T.contiguous() @ dz
        bound += w.abs().T.contiguous() @ (p * torch.expm1(ez) + (UBF + (V + 2) * U) * dz.abs())
    assert ((dX.double() - want).abs() <= bound + UBF * (want.abs() + bound)).all()
    assert (want.abs() > 4 * bound).float().mean() > 0.5  # the bound tells a wrong row from the right one
