"""The root-mean-square norm of a sum: the oracle against differences (CPU), refusals (CPU), and the kernels against the
oracle (GPU).

Tolerances, per value, with u = 2^-24 a rounding to fp32 and 2^-8 one to bf16. The sums over a column are 64 bits
wide and add nothing. s is one rounding off, its square two, the mean's root half of that and its own rounding: inv 3 u.
"""
import numpy as np
import pytest
import torch

from oracle import rmsnorm as onorm
from paper_1805_08939_amd import api, synth

U, UBF = 2.0 ** -24, 2.0 ** -8


# ---------------------------------------------------------------- the oracle

def test_oracle_backward_is_the_forward_differenced():
    r = np.random.default_rng(3)
    s, gain, dY, dS = r.normal(size=(3, 5)), r.normal(size=5), r.normal(size=(3, 5)), r.normal(size=(3, 5))
    value = lambda s, g: float((onorm.forward(s, None, g, 0.1)[1] * dY + s * dS).sum())  # noqa: E731
    grads = onorm.backward(s, gain, 0.1, dY, dS)
    for n, p in enumerate((s, gain)):
        for at in np.ndindex(p.shape):
            e = np.zeros_like(p)
            e[at] = 1e-6
            up, down = (value(s + e, gain), value(s - e, gain)) if n == 0 else (value(s, gain + e), value(s, gain - e))
            assert abs((up - down) / 2e-6 - grads[n][at]) < 1e-7 * (1 + abs(grads[n][at]))


# ---------------------------------------------------------------- refusals

def test_refuses_bad_calls():
    a, b = 4096, 8192  # aligned addresses; never read

    def refused(status, call, *args):
        with pytest.raises(api.ArdError) as e:
            call(*args, stream=0)
        assert e.value.status == status and e.value.message

    for bad, status in ((dict(dtype=7), 2), (dict(batch=0), 1), (dict(features=0), 1), (dict(batch=-3), 1),
                        (dict(eps=-1.0), 1), (dict(eps=float("nan")), 1), (dict(eps=float("inf")), 1)):
        d = api.rmsnorm_desc(**{**dict(dtype=api.ARD_F32, batch=4, features=8), **bad})
        assert api.ard_rmsnorm_workspace_bytes(d) == 0
        refused(status, api.ard_rmsnorm_fwd, d, a, a, a, a, b, a, (a, 1 << 30))
    d = api.rmsnorm_desc(api.ARD_BF16, 2048, 4096)
    assert api.ard_rmsnorm_workspace_bytes(d) > 0
    good, space = (a, a, a, a, b, a), (a, 1 << 30)
    for at, x in ((0, None), (4, None), (0, a + 8), (1, a + 2), (2, a + 4), (3, a + 8), (4, b + 8), (5, a + 4), (4, a)):
        refused(1, api.ard_rmsnorm_fwd, d, *(x if i == at else g for i, g in enumerate(good)), space)
    refused(5, api.ard_rmsnorm_fwd, d, *good, None)
    refused(5, api.ard_rmsnorm_fwd, d, *good, (a, 16))
    refused(1, api.ard_rmsnorm_fwd, d, *good, (a + 4, 1 << 30))
    good = (a,) * 7
    for at, x in ((0, None), (2, None), (3, None), (0, a + 8), (1, a + 4), (2, a + 4), (3, a + 2), (4, a + 8),
                  (5, a + 8), (6, a + 4)):
        refused(1, api.ard_rmsnorm_bwd, d, *(x if i == at else g for i, g in enumerate(good)), space)
    refused(5, api.ard_rmsnorm_bwd, d, *good, None)
    refused(5, api.ard_rmsnorm_bwd, d, *good, (a, api.ard_rmsnorm_workspace_bytes(d) - 1))


def test_refuses_the_gain_as_its_gradient():
    """The gain is read again after the first gradients of it are written."""
    a, b = 4096, 8192
    d = api.rmsnorm_desc(api.ARD_F32, 4, 8)
    with pytest.raises(api.ArdError) as e:
        api.ard_rmsnorm_bwd(d, a, b, a, a, None, a, b, (a, 1 << 30), stream=0)
    assert e.value.status == 1 and "dgain" in e.value.message


# ---------------------------------------------------------------- the kernels

def _inside(got, want, bound, what):
    got = got.double().cpu().numpy()
    assert np.isfinite(got).all(), what
    over = np.abs(got - want) - bound
    assert over.max() <= 0, f"{what}: {np.abs(got - want).max():.3e} off, bound there {bound.flat[over.argmax()]:.3e}"


def _guarded(shape, dtype, dev, fill=3.0):
    """A tensor of this shape within a larger one, and a check that nothing around it was written."""
    n = int(np.prod(shape))
    pad = 64 // torch.empty(0, dtype=dtype).element_size()
    whole = torch.full((n + 2 * pad,), fill, dtype=dtype, device=dev)

    def untouched():
        assert (whole[:pad] == fill).all() and (whole[pad + n:] == fill).all()
    return whole[pad:pad + n].view(shape), untouched


def _fenced(t, dev):
    """The tensor on the device between values that are not numbers."""
    n, pad = t.numel(), 64 // t.element_size()
    whole = torch.full((n + 2 * pad,), float("nan"), dtype=t.dtype, device=dev)
    whole[pad:pad + n] = t.reshape(-1).to(dev)
    return whole[pad:pad + n].view(t.shape)


SIZES = [  # dtype, B, K: one workgroup's rows, ranges of rows, many blocks; columns short of a chunk and of a block
    ("bf16", 1, 1), ("f32", 1, 5), ("bf16", 1, 1024), ("bf16", 1, 8191), ("f32", 1, 100003), ("bf16", 2, 77), ("bf16", 7, 4096),
    ("f32", 3, 300), ("bf16", 8, 33), ("bf16", 9, 1000), ("f32", 4, 64), ("f32", 17, 129), ("bf16", 64, 512), ("bf16", 65, 512),
    ("f32", 63, 700), ("bf16", 100, 2048), ("f32", 700, 1500), ("bf16", 331, 1023), ("bf16", 2048, 768), ("f32", 130, 4000),
    ("bf16", 33001, 16), ("f32", 33001, 3), ("bf16", 40, 20000),
]


def _case(dtype, B, K, seed):
    g = synth.generator(1805 + seed)
    x, r, dY, dS = (synth.to_storage(synth.normal(g, (B, K)), dtype) for _ in range(4))
    return x, r, 1.0 + synth.normal(g, (K,), 0.3), dY, dS


def _np(t):
    return None if t is None else t.double().numpy()


@pytest.mark.gpu
@pytest.mark.parametrize("residual,gained", [(True, True), (False, False)])
@pytest.mark.parametrize("size", SIZES)
def test_forward_and_backward(size, residual, gained):
    from gpu_util import ard_dtype, device, workspace
    dtype, B, K = size
    x, r, gain, dY, dS = _case(dtype, B, K, B + K)
    if not residual:
        r = dS = None
    g64 = gain.double().numpy() if gained else np.ones(K)
    dev, st, out = device(), synth.storage_dtype(dtype), UBF if dtype == "bf16" else U
    eps = 1e-3
    desc = api.rmsnorm_desc(ard_dtype(dtype), B, K, eps)
    ws = workspace(api.ard_rmsnorm_workspace_bytes(desc))
    put = lambda t: None if t is None else _fenced(t.T.contiguous(), dev)  # noqa: E731
    gd = _fenced(gain, dev) if gained else None
    (S, s_ok), (Y, y_ok), (inv, i_ok) = _guarded((K, B), st, dev), _guarded((K, B), st, dev), _guarded((B,), torch.float32, dev)
    api.ard_rmsnorm_fwd(desc, put(x), put(r), gd, S if residual else None, Y, inv, ws)
    torch.cuda.synchronize()
    s64, y64, i64 = onorm.forward(_np(x), _np(r), g64, eps)
    # y: s, inv, their product and that with the gain
    _inside(Y.T, y64, (out + 7 * U) * np.abs(y64), "Y")
    _inside(inv, i64, 3 * U * i64, "inv")
    if residual:
        _inside(S.T, s64, (out + 2 * U) * np.abs(s64), "S")
    for ok in (s_ok, y_ok, i_ok):
        ok()
    # the backward takes S as it is stored and inv with 3 u
    s = S.T.double().cpu().numpy() if residual else _np(x)
    i = 1.0 / np.sqrt((s * s).mean(1) + eps)
    invd = _fenced(torch.tensor(i, dtype=torch.float32), dev)
    (dX, x_ok), (dg, g_ok) = _guarded((K, B), st, dev), _guarded((K,), torch.float32, dev)
    Sd = put(torch.tensor(s).to(st))
    api.ard_rmsnorm_bwd(desc, Sd, gd, invd, put(dY), put(dS), dX, dg, ws)
    torch.cuda.synchronize()
    dX64, dg64 = onorm.backward(s, g64, eps, _np(dY), _np(dS))
    xh, u, iv = np.abs(s) * i[:, None], np.abs(_np(dY) * g64), i[:, None]
    mean = (u * xh).mean(1)[:, None]
    # w = dY xh: inv and two products, 3 u; its sum over 64 bits; the mean's rounding. dX: inv (twice for xh) 2 u, xh,
    # its product with the mean, u, the difference, the product with inv and dS: at most 7 u of u and 11 of xh mean
    bound = iv * (7 * U * u + 11 * U * xh * mean) + 2 * U * (0 if dS is None else np.abs(_np(dS)))
    _inside(dX.T, dX64, bound + out * (np.abs(dX64) + bound), "dX")
    blocks = (B + 63) // 64
    terms = (np.abs(_np(dY)) * xh).sum(0)
    _inside(dg, dg64, (3 + 8 + 6 + blocks) * U * terms, "dgain")
    x_ok(), g_ok()


@pytest.mark.gpu
@pytest.mark.parametrize("dtype,B,K", [("bf16", 100, 2048), ("f32", 5, 64), ("bf16", 520, 600)])
def test_outputs_in_place_and_left_out(dtype, B, K):
    """Outputs that are the inputs' buffers and calls without some outputs give the same bits."""
    from gpu_util import ard_dtype, device, workspace
    x, r, gain, dY, dS = _case(dtype, B, K, 7)
    dev = device()
    desc = api.rmsnorm_desc(ard_dtype(dtype), B, K)
    ws = workspace(api.ard_rmsnorm_workspace_bytes(desc))
    X, R, D, E = (t.T.contiguous().to(dev) for t in (x, r, dY, dS))
    gd = gain.to(dev)
    S, Y, inv = torch.empty_like(X), torch.empty_like(X), torch.empty(B, device=dev)
    api.ard_rmsnorm_fwd(desc, X, R, gd, S, Y, inv, ws)
    for s, y in ((0, 1), (1, 0)):
        bufs = [X.clone(), R.clone()]
        api.ard_rmsnorm_fwd(desc, bufs[0], bufs[1], gd, bufs[s], bufs[y], None, ws)
        assert torch.equal(bufs[s], S) and torch.equal(bufs[y], Y)
    only = torch.empty_like(Y)
    api.ard_rmsnorm_fwd(desc, X, R, gd, None, only, None, ws)
    assert torch.equal(only, Y)
    dX, dg = torch.empty_like(X), torch.empty(K, device=dev)
    api.ard_rmsnorm_bwd(desc, S, gd, inv, D, E, dX, dg, ws)
    for at in range(3):
        bufs = [S.clone(), D.clone(), E.clone()]
        g2 = torch.empty_like(dg)
        api.ard_rmsnorm_bwd(desc, bufs[0], gd, inv, bufs[1], bufs[2], bufs[at], g2, ws)
        assert torch.equal(bufs[at], dX) and torch.equal(g2, dg)
    a, b = torch.empty_like(dX), torch.empty_like(dg)
    api.ard_rmsnorm_bwd(desc, S, gd, inv, D, E, a, None, ws)
    api.ard_rmsnorm_bwd(desc, S, gd, inv, D, E, None, b, ws)
    assert torch.equal(a, dX) and torch.equal(b, dg)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype,B,K", [("bf16", 100, 2048), ("f32", 5, 64), ("bf16", 520, 600)])
def test_values_at_the_ends_of_the_range(dtype, B, K):
    """Squares past 2^128 and below 2^-149, columns of zeros, and one that is not finite beside finite ones."""
    from gpu_util import ard_dtype, device, workspace
    x, _, gain, dY, _ = _case(dtype, B, K, 9)
    x[0] = (x[0].double() * 2.0 ** 100).to(x.dtype)
    x[1] = (x[1].double() * 2.0 ** -90).to(x.dtype)
    x[2], x[3, 5], x[4, K - 1] = 0, float("nan"), float("inf")
    dev, out = device(), UBF if dtype == "bf16" else U
    for eps in (0.0, 1e-6):
        desc = api.rmsnorm_desc(ard_dtype(dtype), B, K, eps)
        ws = workspace(api.ard_rmsnorm_workspace_bytes(desc))
        X, D, gd = x.T.contiguous().to(dev), dY.T.contiguous().to(dev), gain.to(dev)
        Y, inv, dX = torch.empty_like(X), torch.empty(B, device=dev), torch.empty_like(X)
        api.ard_rmsnorm_fwd(desc, X, None, gd, None, Y, inv, ws)
        api.ard_rmsnorm_bwd(desc, X, gd, inv, D, None, dX, None, ws)
        torch.cuda.synchronize()
        Y, dX = Y.T.double().cpu().numpy(), dX.T.double().cpu().numpy()
        fine = [b for b in range(B) if b not in (2, 3, 4)]
        _, y64, _ = onorm.forward(_np(x)[fine], None, gain.double().numpy(), eps)
        tiny = 2.0 ** -126  # of results below the smallest normal number nothing is asked
        assert (np.abs(Y[fine] - y64) <= (out + 7 * U) * np.abs(y64) + tiny).all()
        assert np.isnan(Y[3]).all() and np.isnan(dX[3]).all()
        assert np.isnan(Y[4, K - 1]) and (Y[4, :K - 1] == 0).all()
        assert np.isnan(Y[2]).all() if eps == 0 else (Y[2] == 0).all()
        # columns of ordinary size: the neighbours left no trace
        plain = [b for b in fine if b > 1]
        i = 1.0 / np.sqrt((_np(x)[plain] ** 2).mean(1) + eps)[:, None]
        want, _ = onorm.backward(_np(x)[plain], gain.double().numpy(), eps, _np(dY)[plain])
        xh, u = np.abs(_np(x)[plain]) * i, np.abs(_np(dY)[plain] * gain.double().numpy())
        bound = i * (7 * U * u + 17 * U * xh * (u * xh).mean(1)[:, None]) + 3 * U * i * u
        assert (np.abs(dX[plain] - want) <= bound + out * (np.abs(want) + bound)).all()


@pytest.mark.gpu
def test_captured_and_on_another_stream():
    """A captured forward and backward, replayed on new inputs between eager calls, give the eager bits."""
    from gpu_util import device, workspace
    dev = device()
    B, K = 600, 2000
    desc = api.rmsnorm_desc(api.ARD_BF16, B, K)
    nbytes = api.ard_rmsnorm_workspace_bytes(desc)
    ws, ws2 = workspace(nbytes), workspace(nbytes)
    X, R, D = (torch.empty(K, B, dtype=torch.bfloat16, device=dev) for _ in range(3))
    gain = torch.ones(K, device=dev)
    outs = [torch.empty_like(X), torch.empty_like(X), torch.empty(B, device=dev), torch.empty_like(X), torch.empty(K, device=dev)]
    again = [torch.empty_like(t) for t in outs]

    def step(o, w):
        api.ard_rmsnorm_fwd(desc, X, R, gain, o[0], o[1], o[2], w)
        api.ard_rmsnorm_bwd(desc, o[0], gain, o[2], D, D, o[3], o[4], w)

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
        for t in (X, R, D):
            t.copy_(torch.randn(K, B, generator=gen, device=dev))
        graph.replay()
        with torch.cuda.stream(side):
            side.wait_stream(torch.cuda.current_stream())
            step(again, ws2)
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(outs, again))


@pytest.mark.gpu
def test_more_than_2_31_elements():
    from gpu_util import device, workspace
    dev, K, B = device(), 5, 460_000_009
    desc = api.rmsnorm_desc(api.ARD_BF16, B, K)
    ws = workspace(api.ard_rmsnorm_workspace_bytes(desc))
    X = torch.empty(K, B, dtype=torch.bfloat16, device=dev).uniform_(-2, 2)
    Y, inv, dg = torch.empty_like(X), torch.empty(B, device=dev), torch.empty(K, device=dev)
    api.ard_rmsnorm_fwd(desc, X, None, None, None, Y, inv, ws)
    for at in (0, 12345, B - 70, 2 ** 31 // K, 2 ** 32 // K // 2 * 1):
        x = X[:, at:at + 64].double()
        want = x / torch.sqrt((x * x).mean(0) + float(np.float32(1e-5)))
        assert ((Y[:, at:at + 64].double() - want).abs() <= (UBF + 7 * U) * want.abs()).all()
    api.ard_rmsnorm_bwd(desc, X, None, inv, Y, None, Y, dg, ws)
    assert torch.isfinite(dg).all() and torch.isfinite(Y[:, -64:]).all()


# ---------------------------------------------------------------- index limits, on the CPU

@pytest.mark.parametrize("dtype", [api.ARD_F32, api.ARD_BF16])
@pytest.mark.parametrize("batch", [1, 7, 64])
def test_plans_of_the_most_features(dtype, batch):
    """Up to 64 columns make one block of at most 1024 ranges of rows: 8 bytes of sums a range and column."""
    for features in (2 ** 31 - 1, 2 ** 31 - 2 ** 20, 2 ** 30 + 1):
        nbytes = api.ard_rmsnorm_workspace_bytes(api.rmsnorm_desc(dtype, batch, features))
        assert 512 * batch * 8 < nbytes <= 1024 * batch * 8 + 255


@pytest.mark.gpu
def test_most_features():
    from gpu_util import device, workspace
    dev, K, eps = device(), 2 ** 31 - 1, float(np.float32(1e-5))
    desc = api.rmsnorm_desc(api.ARD_BF16, 1, K)
    ws = workspace(api.ard_rmsnorm_workspace_bytes(desc))
    X, D = (torch.empty(K, 1, dtype=torch.bfloat16, device=dev).uniform_(-2, 2) for _ in range(2))
    Y, inv, dX, dg = torch.empty_like(X), torch.empty(1, device=dev), torch.empty_like(X), torch.empty(K, device=dev)
    api.ard_rmsnorm_fwd(desc, X, None, None, None, Y, inv, ws)
    squares = sum(float(x.double().square().sum()) for x in X.split(2 ** 27))
    i = 1.0 / np.sqrt(squares / K + eps)
    assert abs(float(inv[0]) - i) <= 3 * U * i
    api.ard_rmsnorm_bwd(desc, X, None, inv, D, None, dX, dg, ws)
    # u xh has 3 u; the mean is rounded once more
    mean = sum(float((x.double() * d.double()).sum()) for x, d in zip(X.split(2 ** 27), D.split(2 ** 27))) * i / K
    size = sum(float((x.double() * d.double()).abs().sum()) for x, d in zip(X.split(2 ** 27), D.split(2 ** 27))) * i / K
    for at in (0, 2 ** 30 - 32, 2 ** 31 - 2 ** 21 - 32, K - 64):
        x, d = X[at:at + 64].double(), D[at:at + 64].double()
        assert ((Y[at:at + 64].double() - x * i).abs() <= (UBF + 7 * U) * (x * i).abs()).all()
        want, bound = i * (d - x * i * mean), i * (7 * U * d.abs() + (x * i).abs() * 11 * U * size)
        assert ((dX[at:at + 64].double() - want).abs() <= bound + UBF * (want.abs() + bound)).all()
        want = (d * x * i)[:, 0]
        assert ((dg[at:at + 64].double() - want).abs() <= 6 * U * want.abs()).all()


def test_refuses_more_sums_of_the_gain_than_a_launch_takes():
    """dgain of several blocks of columns is joined by a workgroup of 256 threads for 64 features: below 2^32 threads."""
    args = [4096 * (i + 1) for i in range(7)]  # never read
    d = api.rmsnorm_desc(api.ARD_BF16, 65, 2 ** 30)
    with pytest.raises(api.ArdError) as e:
        api.ard_rmsnorm_bwd(d, *args, (1 << 20, 1 << 60), stream=0)
    assert e.value.status == 2 and "features" in e.value.message


# ---------------------------------------------------------------- each argument, on the CPU

FWD = ("Xt", "Rt", "gain", "St", "Yt", "inv_rms")
BWD = ("St", "gain", "inv_rms", "dYt", "dSt", "dXt", "dgain")
NEEDED = {"fwd": {"Xt", "Yt"}, "bwd": {"St", "inv_rms", "dYt"}}


@pytest.mark.parametrize("way", ["fwd", "bwd"])
def test_refuses_each_argument_by_its_name(way):
    """Arguments at addresses of their own, one of them wrong: no other check stands in for its own."""
    call, names = (api.ard_rmsnorm_fwd, FWD) if way == "fwd" else (api.ard_rmsnorm_bwd, BWD)
    d = api.rmsnorm_desc(api.ARD_BF16, 2048, 4096)
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
    refused(5, "workspace", good, None)
    refused(5, "workspace", good, (1 << 20, 16))
    refused(1, "workspace", good, ((1 << 20) + 8, 1 << 40))
    if way == "bwd":  # the forward needs none of dgain's part
        refused(5, "workspace", good, (1 << 20, api.ard_rmsnorm_workspace_bytes(d) - 1))


# ---------------------------------------------------------------- buffers, on the CPU

@pytest.mark.parametrize("dtype,batch,features", [(api.ARD_F32, 64, 64), (api.ARD_BF16, 64, 64), (api.ARD_F32, 1, 600),
                                                  (api.ARD_F32, 600, 1), (api.ARD_BF16, 2048, 8192)])
def test_refuses_sums_in_the_buffers_of_other_arguments(dtype, batch, features):
    """inv_rms and dgain are written while other workgroups still read every other array."""
    d = api.rmsnorm_desc(dtype, batch, features)
    space = (1 << 20, 1 << 60)

    def refused(call, args, at, name):
        for i in range(len(args)):
            if i == at:
                continue
            with pytest.raises(api.ArdError) as e:
                call(d, *(args[i] if j == at else x for j, x in enumerate(args)), space, stream=0)
            assert e.value.status == 1 and name in e.value.message and "buffer" in e.value.message
    refused(api.ard_rmsnorm_fwd, [4096 * (i + 1) for i in range(6)], 5, "inv_rms")
    refused(api.ard_rmsnorm_bwd, [4096 * (i + 1) for i in range(7)], 6, "dgain")


# ---------------------------------------------------------------- many columns

@pytest.mark.gpu
@pytest.mark.parametrize("dtype,B,K", [("bf16", 2 ** 23, 4), ("f32", 2 ** 23 + 5, 2), ("bf16", 2 ** 25, 1), ("bf16", 32000, 4000)])
@pytest.mark.parametrize("equal", [True, False])
def test_gradient_of_the_gain_over_many_columns(dtype, B, K, equal):
    """The error does not grow with the columns, also where each of them adds the same. w = dY xh 3 u, 64 columns in fp32 at
    most 7 and 4 u (eight of a thread and 16 threads), the join 64 bits wide, a rounding of the result."""
    from gpu_util import ard_dtype, device, workspace
    dev, st = device(), synth.storage_dtype(dtype)
    desc = api.rmsnorm_desc(ard_dtype(dtype), B, K)
    ws = workspace(api.ard_rmsnorm_workspace_bytes(desc))
    S, D = torch.full((K, B), 1.5, dtype=st, device=dev), torch.full((K, B), 0.7, dtype=st, device=dev)
    inv, dg = torch.full((B,), 0.6666, device=dev), torch.empty(K, device=dev)
    if not equal:
        S.uniform_(0.5, 2), D.uniform_(-0.1, 1), inv.uniform_(0.5, 1)
    api.ard_rmsnorm_bwd(desc, S, None, inv, D, None, None, dg, ws)
    for k in range(0, K, max(1, K // 8)):
        w = S[k].double() * D[k].double() * inv.double()
        assert abs(float(dg[k]) - float(w.sum())) <= 15 * U * float(w.abs().sum())


# ---------------------------------------------------------------- past 2^31 elements

@pytest.mark.gpu
@pytest.mark.parametrize("sparse", [False, True])
def test_gradients_past_2_31_elements(sparse):
    """dX in columns all over the arrays; dgain of every column and, with a dY of zeros elsewhere, of these columns alone."""
    from gpu_util import device, workspace
    dev, K, B = device(), 5, 460_000_009
    desc = api.rmsnorm_desc(api.ARD_BF16, B, K)
    ws = workspace(api.ard_rmsnorm_workspace_bytes(desc))
    S, D = (torch.empty(K, B, dtype=torch.bfloat16, device=dev).uniform_(-2, 2) for _ in range(2))
    inv, gain = torch.empty(B, device=dev).uniform_(0.5, 2), torch.empty(K, device=dev).uniform_(0.5, 2)
    spans = [slice(at, at + 64) for at in (0, 12345, 2 ** 31 // K - 32, 2 ** 31 % B - 32, B - 64)]
    if sparse:
        kept = [D[:, c].clone() for c in spans]
        D.zero_()
        for c, d in zip(spans, kept):
            D[:, c] = d
    dX, dg = torch.full_like(S, float("nan")), torch.empty(K, device=dev)
    api.ard_rmsnorm_bwd(desc, S, gain, inv, D, None, dX, dg, ws)
    for c in spans:
        s, d, i, g = S[:, c].double(), D[:, c].double(), inv[c].double(), gain.double()[:, None]
        xh, u = s * i, g * d
        want, bound = i * (u - xh * (u * xh).mean(0)), i * (7 * U * u.abs() + 11 * U * xh.abs() * (u * xh).abs().mean(0))
        assert ((dX[:, c].double() - want).abs() <= bound + UBF * (want.abs() + bound)).all()
    assert not any(torch.isnan(x).any() for row in dX for x in row.split(2 ** 28))
    for k in range(K):
        sums = [(w.sum(), w.abs().sum()) for w in (D[k, c].double() * S[k, c].double() * inv[c].double()
                                                   for c in (spans if sparse else
                                                             [slice(a, a + 2 ** 26) for a in range(0, B, 2 ** 26)]))]
        # as over many columns above
        assert abs(float(dg[k]) - sum(float(a) for a, _ in sums)) <= 15 * U * sum(float(b) for _, b in sums)
