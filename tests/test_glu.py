"""The gated feed-forward layer: the oracle against finite differences (CPU), refusals (CPU), and the kernels against
the oracle (GPU).

Tolerances, per value: fp32 sums of n terms are off by at most n 2^-24 of the sum of the terms' absolute values, each
rounding to bf16 (8 significant bits) by 2^-8 of what is rounded; an activation or its derivative by 16 units in the last place.
"""
import numpy as np
import pytest
import torch

from oracle import glu as oglu
from oracle import patterns as opat
from paper_1805_08939_amd import api, synth

U32, UBF = 2.0 ** -24, 2.0 ** -8
ACTS = {"silu": api.ARD_GLU_SILU, "gelu": api.ARD_GLU_GELU, "relu": api.ARD_GLU_RELU, "sigmoid": api.ARD_GLU_SIGMOID}


# ---------------------------------------------------------------- the oracle

@pytest.mark.parametrize("name", sorted(ACTS))
def test_oracle_backward_is_the_forward_differenced(name):
    r = np.random.default_rng(5)
    X, W, b = r.normal(size=(3, 4)), r.normal(size=(2, 6, 4)), r.normal(size=(2, 6))
    dH, keep = r.normal(size=(3, 6)), opat.row_mask(6, 2, 1).astype(np.float64)
    value = lambda X, W, b: float((oglu.forward(X, W, b, keep, 1.5, name)[0] * dH).sum())  # noqa: E731
    _, Z = oglu.forward(X, W, b, keep, 1.5, name)
    grads = oglu.backward(X, W, Z, dH, keep, 1.5, name)
    for n, (p, d) in enumerate(zip((X, W, b), grads)):
        for at in np.ndindex(p.shape):
            e = np.zeros_like(p)
            e[at] = 1e-6
            args = [X, W, b], [X, W, b]
            args[0][n], args[1][n] = p + e, p - e
            assert abs((value(*args[0]) - value(*args[1])) / 2e-6 - d[at]) < 1e-6 * (1 + abs(d[at]))


def test_oracle_forward_is_torch():
    r = np.random.default_rng(6)
    X, W = r.normal(size=(5, 7)), r.normal(size=(2, 3, 7))
    x, w = torch.tensor(X), torch.tensor(W)
    g, u = x @ w[0].T, x @ w[1].T
    for name, fn in (("silu", torch.nn.functional.silu), ("gelu", torch.nn.functional.gelu), ("relu", torch.relu),
                     ("sigmoid", torch.sigmoid)):
        H, _ = oglu.forward(X, W, None, 1.0, 1.0, name)
        assert np.abs(H - (fn(g) * u).numpy()).max() < 1e-12


# ---------------------------------------------------------------- refusals

def test_refuses_bad_calls():
    a = 4096  # an aligned address; never read
    good = dict(dtype=api.ARD_F32, batch=4, in_features=8, hidden_features=6)

    def refused(status, call, *args):
        with pytest.raises(api.ArdError) as e:
            call(*args, stream=0)
        assert e.value.status == status and e.value.message

    for bad, status in ((dict(dtype=7), 2), (dict(batch=0), 1), (dict(in_features=-1), 1), (dict(hidden_features=0), 1),
                        (dict(act=9), 1), (dict(dropped=3), 1), (dict(scale=float("nan")), 1),
                        (dict(scale=float("inf")), 1), (dict(grad_dtype=api.ARD_BF16), 1), (dict(grad_dtype=5), 1),
                        (dict(hidden_plan=api.ard_plan_rows(7, 2, 0, None)), 1)):
        d = api.glu_desc(**{**good, **bad})
        assert api.ard_glu_workspace_bytes(d) == 0
        refused(status, api.ard_glu_fwd, d, a, a, a, a, a, (a, 1 << 30))
    d = api.glu_desc(**good)
    need = api.ard_glu_workspace_bytes(d)
    for args in ((None, a, a, a, a), (a, None, a, a, a), (a, a, a, a, None), (a + 4, a, a, a, a), (a, a, a + 8, a, a),
                 (a, a, a, a + 2, a)):
        refused(1, api.ard_glu_fwd, d, *args, (a, 1 << 30))
    for args in ((None, a, a, a, a, a, a), (a, a, None, a, a, a, a), (a, a, a, None, a, a, a), (a, a, a, a, a + 4, a, a),
                 (a, a, a, a, a, a + 4, a), (a, a, a, a, a, a, a + 4)):
        refused(1, api.ard_glu_bwd, d, *args, (a, 1 << 30))
    if need:
        refused(5, api.ard_glu_bwd, d, a, a, a, a, a, a, a, None)
        refused(5, api.ard_glu_bwd, d, a, a, a, a, a, a, a, (a, 0))


# ---------------------------------------------------------------- the kernels

def _case(dtype, B, K, N, period, offset, name, bias=True, seed=1):
    g = synth.generator(1805 + seed)
    X = synth.to_storage(synth.normal(g, (B, K)), dtype)
    W = synth.to_storage(synth.normal(g, (2, N, K), 1.0 / np.sqrt(K)), dtype)
    b = synth.normal(g, (2, N), 0.3) if bias else None
    dH = synth.to_storage(synth.normal(g, (B, N)), dtype)
    Z = synth.to_storage(synth.normal(g, (2, B, N), 1.3), dtype)
    return X, W, b, dH, Z, opat.row_mask(N, period, offset).astype(np.float64)


def _f64(t):
    return None if t is None else t.double().numpy()


def _inside(got, want, bound, what):
    got = got.double().cpu().numpy()
    if got.size == 0:
        return
    assert np.isfinite(got).all(), what
    over = np.abs(got - want) - bound
    assert over.max() <= 0, f"{what}: {np.abs(got - want).max():.3e} off, bound there {bound.flat[over.argmax()]:.3e}"


SIZES = [  # dtype, B, K, N, period, offset, act
    ("bf16", 1, 1, 1, 1, 0, "silu"), ("f32", 1, 3, 2, 1, 0, "gelu"), ("bf16", 1, 64, 96, 1, 0, "silu"),
    ("bf16", 1, 1000, 130, 2, 1, "silu"), ("f32", 1, 257, 66, 3, 2, "gelu"), ("bf16", 2, 520, 72, 1, 0, "gelu"),
    ("bf16", 5, 136, 200, 1, 0, "relu"), ("f32", 7, 200, 33, 1, 0, "sigmoid"), ("bf16", 16, 1024, 512, 1, 0, "silu"),
    ("bf16", 16, 333, 100, 2, 0, "silu"), ("f32", 16, 1024, 100, 2, 0, "silu"), ("bf16", 17, 72, 40, 1, 0, "sigmoid"),
    ("bf16", 100, 1023, 153, 3, 1, "gelu"), ("f32", 100, 103, 153, 3, 1, "gelu"), ("bf16", 128, 256, 512, 2, 1, "silu"),
    ("f32", 96, 256, 512, 2, 1, "silu"), ("bf16", 200, 512, 1100, 5, 4, "silu"), ("bf16", 640, 320, 2100, 1, 0, "relu"),
    ("f32", 640, 320, 1300, 1, 0, "relu"), ("bf16", 33, 40, 5, 7, 6, "silu"), ("f32", 33, 40, 9, 2, 1, "silu"),
    # grids large enough for each tile of the one-product forward, rows on 16 bytes and off them
    ("bf16", 1280, 72, 4096, 1, 0, "silu"), ("bf16", 256, 40, 11000, 1, 0, "gelu"), ("bf16", 128, 72, 20600, 1, 0, "silu"),
    ("bf16", 643, 63, 4200, 2, 1, "sigmoid"), ("bf16", 1100, 33, 4999, 3, 2, "silu"), ("bf16", 65, 24, 300, 1, 0, "silu"),
    # the few-column kernel: blocks of 16 columns, 8 or 16 units of a workgroup, inputs that end inside a step
    ("bf16", 31, 95, 4200, 1, 0, "silu"), ("bf16", 64, 33, 9000, 2, 1, "gelu"), ("bf16", 3, 31, 4500, 1, 0, "relu"),
    ("f32", 2, 17, 4500, 1, 0, "silu"), ("bf16", 1, 31, 17, 1, 0, "silu"), ("bf16", 64, 1, 3, 1, 0, "silu"),
    ("bf16", 33, 2, 40, 1, 0, "silu"), ("bf16", 49, 700, 33, 2, 0, "gelu"), ("f32", 16, 15, 5, 2, 0, "gelu"),
    # products large enough for copies of rows off 16 bytes: of both operands, of one, more inputs than units
    ("bf16", 100, 1023, 640, 2, 1, "silu"), ("f32", 171, 1025, 1300, 1, 0, "gelu"), ("bf16", 104, 1023, 400, 1, 0, "silu"),
    ("bf16", 101, 1024, 400, 1, 0, "relu"), ("bf16", 77, 5003, 90, 1, 0, "silu"), ("f32", 203, 1024, 1000, 1, 0, "silu"),
    ("f32", 204, 1030, 2003, 2, 0, "sigmoid"), ("bf16", 643, 64, 4200, 2, 1, "silu"), ("bf16", 640, 65, 4200, 2, 1, "silu"),
    ("bf16", 333, 700, 450, 1, 0, "gelu"), ("f32", 333, 701, 451, 1, 0, "silu"), ("bf16", 331, 3001, 101, 1, 0, "silu"),
]


@pytest.mark.gpu
@pytest.mark.parametrize("train", [False, True])
@pytest.mark.parametrize("size", SIZES)
def test_forward(size, train):
    from gpu_util import ard_dtype, device, workspace
    dtype, B, K, N, period, offset, name = size
    X, W, b, _, _, keep = _case(dtype, B, K, N, period, offset, name, bias=N % 3 != 0)
    dev, st = device(), synth.storage_dtype(dtype)
    scale = 1.25
    desc = api.glu_desc(ard_dtype(dtype), B, K, N, api.ard_plan_rows(N, period, offset, None), scale, ACTS[name],
                        api.ARD_DROPPED_ZERO if train else api.ARD_DROPPED_SKIP)
    Ht = torch.full((N, B), 7.0, dtype=st, device=dev)
    Zt = torch.full((2, N, B), 7.0, dtype=st, device=dev) if train else None
    ws = workspace(api.ard_glu_workspace_bytes(desc))
    api.ard_glu_fwd(desc, X.T.contiguous().to(dev), W.to(dev), None if b is None else b.to(dev), Zt, Ht, ws)
    torch.cuda.synchronize()
    H, Z = oglu.forward(_f64(X), _f64(W), _f64(b), keep, scale, name)
    ab = np.zeros((2, N)) if b is None else np.abs(_f64(b))
    size_z = np.stack([np.abs(_f64(X)) @ np.abs(_f64(W))[i].T + ab[i] for i in (0, 1)])
    sums = (K + 16) * U32 * size_z
    a, da, _ = oglu.act(name, Z[0])
    out = UBF if dtype == "bf16" else U32
    bound = scale * ((1.2 * sums[0] + 16 * U32 * np.abs(a)) * (np.abs(Z[1]) + sums[1]) + np.abs(a) * sums[1])
    bound = (bound * (1 + out) + out * np.abs(H)) + 1e-30
    if train:
        _inside(Ht.T, H, bound * keep, "H")
        for i in (0, 1):
            on = keep > 0
            _inside(Zt[i].T[:, on], Z[i][:, on], (sums[i] * (1 + out) + out * np.abs(Z[i]))[:, on] + 1e-30, "Z")
            assert (Zt[i].T[:, ~on] == 7.0).all()
    else:
        on = keep > 0
        _inside(Ht.T[:, on], H[:, on], bound[:, on], "H")
        assert (Ht.T[:, ~on] == 7.0).all()


@pytest.mark.gpu
@pytest.mark.parametrize("size", SIZES)
@pytest.mark.parametrize("grad", ["f32", "same"])
def test_backward(size, grad):
    from gpu_util import ard_dtype, device, workspace
    dtype, B, K, N, period, offset, name = size
    X, W, _, dH, Z, keep = _case(dtype, B, K, N, period, offset, name, seed=2)
    dev, st = device(), synth.storage_dtype(dtype)
    scale, zero = 0.75, grad == "f32"
    gt = torch.float32 if grad == "f32" else st
    desc = api.glu_desc(ard_dtype(dtype), B, K, N, api.ard_plan_rows(N, period, offset, None), scale, ACTS[name],
                        api.ARD_DROPPED_ZERO if zero else api.ARD_DROPPED_SKIP,
                        grad_dtype=api.ARD_F32 if grad == "f32" else ard_dtype(dtype))
    dXt = torch.full((K, B), 7.0, dtype=st, device=dev)
    dW = torch.full((2, N, K), 7.0, dtype=gt, device=dev)
    db = torch.full((2, N), 7.0, device=dev)
    ws = workspace(api.ard_glu_workspace_bytes(desc))
    api.ard_glu_bwd(desc, X.T.contiguous().to(dev), W.to(dev), Z.transpose(1, 2).contiguous().to(dev),
                    dH.T.contiguous().to(dev), dXt, dW, db, ws)
    torch.cuda.synchronize()
    x, w, z, dh = _f64(X), _f64(W), _f64(Z), _f64(dH)
    dX, dWo, dbo = oglu.backward(x, w, z, dh, keep, scale, name)
    a, d, dabs = oglu.act(name, z[0])
    m = scale * np.abs(dh) * keep
    # the terms' sizes: 16 units for the activation, 1 - sigmoid cancels to a unit of its own
    size_d = np.stack([m * np.abs(z[1]) * (dabs + np.abs(d)) + 1e-6 * m * np.abs(z[1]), m * np.abs(a) + 1e-6 * m])
    err_d = 16 * U32 * size_d
    both = np.stack(oglu.derivatives(z, dh, keep, scale, name))
    rounded = err_d + ((UBF * np.abs(both) + UBF * err_d) if dtype == "bf16" else 0)
    out = UBF if dtype == "bf16" else U32
    n = int(keep.sum())
    ax, aw = np.abs(x), np.abs(w)
    ad = np.abs(both) + rounded
    bound = sum(rounded[i] @ aw[i] + (2 * n + 16) * U32 * (ad[i] @ aw[i]) for i in (0, 1))
    _inside(dXt.T, dX, bound * (1 + out) + out * np.abs(dX) + 1e-30, "dX")
    on = keep > 0
    gout = U32 if gt == torch.float32 else UBF
    for i in (0, 1):
        bw = rounded[i].T @ ax + (B + 16) * U32 * (ad[i].T @ ax)
        bw = bw * (1 + gout) + gout * np.abs(dWo[i]) + 1e-30
        _inside(dW[i][torch.tensor(on)], dWo[i][on], bw[on], "dW")
        bb = err_d[i].sum(0) + (B + 16) * U32 * np.abs(both[i]).sum(0) + 1e-30
        _inside(db[i][torch.tensor(on)], dbo[i][on], bb[on], "dbias")
        rest = 0.0 if zero else 7.0
        assert (dW[i][torch.tensor(~on)] == rest).all() and (db[i][torch.tensor(~on)] == rest).all()


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_no_unit_kept(dtype):
    from gpu_util import ard_dtype, device, workspace
    dev, st, B, K, N = device(), synth.storage_dtype(dtype), 9, 12, 4
    X, W, b, dH, Z, _ = _case(dtype, B, K, N, 1, 0, "silu")
    desc = api.glu_desc(ard_dtype(dtype), B, K, N, api.ard_plan_rows(N, 9, 7, None))
    Ht, dXt = (torch.full(s, 7.0, dtype=st, device=dev) for s in ((N, B), (K, B)))
    dW, db = torch.full((2, N, K), 7.0, device=dev), torch.full((2, N), 7.0, device=dev)
    ws = workspace(api.ard_glu_workspace_bytes(desc))
    x, w = X.T.contiguous().to(dev), W.to(dev)
    api.ard_glu_fwd(desc, x, w, b.to(dev), None, Ht, ws)
    api.ard_glu_bwd(desc, x, w, Z.transpose(1, 2).contiguous().to(dev), dH.T.contiguous().to(dev), dXt, dW, db, ws)
    torch.cuda.synchronize()
    assert not Ht.any() and not dXt.any() and not dW.any() and not db.any()


@pytest.mark.gpu
@pytest.mark.parametrize("size", [("bf16", 24, 200, 96, 2, 1, "silu"), ("f32", 100, 96, 64, 1, 0, "gelu")])
def test_outputs_left_out_and_runs_alike(size):
    """Each gradient may be left out; the others do not change, nor does anything from run to run."""
    from gpu_util import ard_dtype, device, workspace
    dtype, B, K, N, period, offset, name = size
    X, W, _, dH, Z, _ = _case(dtype, B, K, N, period, offset, name, seed=3)
    dev, st = device(), synth.storage_dtype(dtype)
    desc = api.glu_desc(ard_dtype(dtype), B, K, N, api.ard_plan_rows(N, period, offset, None), 1.0, ACTS[name])
    ws = workspace(api.ard_glu_workspace_bytes(desc))
    args = (X.T.contiguous().to(dev), W.to(dev), Z.transpose(1, 2).contiguous().to(dev), dH.T.contiguous().to(dev))

    def outs(which):
        o = [torch.zeros(K, B, dtype=st, device=dev), torch.zeros(2, N, K, device=dev), torch.zeros(2, N, device=dev)]
        api.ard_glu_bwd(desc, *args, *(t if i in which else None for i, t in enumerate(o)), ws)
        torch.cuda.synchronize()
        return o
    whole = outs((0, 1, 2))
    for which in ((0, 1, 2), (0,), (1,), (2,), (0, 2)):
        for i, t in enumerate(outs(which)):
            assert torch.equal(t, whole[i]) if i in which else not t.any()


@pytest.mark.gpu
def test_on_another_stream():
    from gpu_util import device, workspace
    dev = device()
    X, W, b, _, _, keep = _case("bf16", 40, 64, 96, 1, 0, "silu", seed=4)
    desc = api.glu_desc(api.ARD_BF16, 40, 64, 96)
    x, w, bb, Ht = X.T.contiguous().to(dev), W.to(dev), b.to(dev), torch.zeros(96, 40, dtype=torch.bfloat16, device=dev)
    ws = workspace(api.ard_glu_workspace_bytes(desc))
    api.ard_glu_fwd(desc, x, w, bb, None, Ht, ws)
    torch.cuda.synchronize()
    side, other = torch.cuda.Stream(), torch.zeros_like(Ht)
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        api.ard_glu_fwd(desc, x, w, bb, None, other, ws)
    side.synchronize()
    assert torch.equal(Ht, other)


@pytest.mark.gpu
@pytest.mark.parametrize("size", [("bf16", 4, 200, 96, 2, 1, "silu"), ("bf16", 200, 512, 1100, 2, 1, "silu"),
                                  ("f32", 100, 96, 64, 2, 0, "gelu")])
def test_in_a_graph(size):
    from gpu_util import ard_dtype, device, workspace
    dtype, B, K, N, period, offset, name = size
    X, W, b, dH, Z, _ = _case(dtype, B, K, N, period, offset, name, seed=5)
    dev, st = device(), synth.storage_dtype(dtype)
    desc = api.glu_desc(ard_dtype(dtype), B, K, N, api.ard_plan_rows(N, period, offset, None), 1.5, ACTS[name])
    ws = workspace(api.ard_glu_workspace_bytes(desc))
    x, w, bb, dh = X.T.contiguous().to(dev), W.to(dev), b.to(dev), dH.T.contiguous().to(dev)
    H, z = torch.empty(N, B, dtype=st, device=dev), torch.zeros(2, N, B, dtype=st, device=dev)
    dX, dW, db = torch.empty(K, B, dtype=st, device=dev), torch.empty(2, N, K, device=dev), torch.empty(2, N, device=dev)

    def step():
        api.ard_glu_fwd(desc, x, w, bb, z, H, ws)
        api.ard_glu_bwd(desc, x, w, z, dh, dX, dW, db, ws)
    outs = (H, z, dX, dW, db)
    step()
    torch.cuda.synchronize()
    eager = [o.clone() for o in outs]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.stream(side):
        step()
    torch.cuda.current_stream().wait_stream(side)
    with torch.cuda.graph(graph):
        step()
    for _ in range(3):
        for o in outs:
            o.fill_(3.0)
        z.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, o) for a, o in zip(eager, outs))


# ---------------------------------------------------------------- past the sizes of 32-bit offsets and launches

def test_the_plan_counts_weights_in_64_bits():
    """From 2^29 units on 4 N passes 32 bits: the tiles, whose offsets have 32 bits, must not be planned. What is asked
    for then are the sums of the batched products."""
    B = 100
    for N in (1 << 29, (1 << 30) - 1):
        desc = api.glu_desc(api.ARD_BF16, B, 8, N)
        assert api.ard_glu_workspace_bytes(desc) >= 2 * N * B * 4


def _torch_sums(x, w, rows, b=None):
    """Exact pre-activations of some units, and the sums of the terms' absolute values, in 64 bits on the device."""
    z = torch.stack([w[i, rows].double() @ x.double() for i in (0, 1)])
    size = torch.stack([w[i, rows].double().abs() @ x.double().abs() for i in (0, 1)])
    if b is not None:
        z, size = z + b[:, rows].double()[..., None], size + b[:, rows].double().abs()[..., None]
    return z.cpu().numpy(), size.cpu().numpy()


def _check_units(dtype, K, H, Z, z, size, scale, name, rows):
    out, sums = (UBF if dtype == "bf16" else U32), (K + 16) * U32 * size
    a = oglu.act(name, z[0])[0]
    bound = scale * ((1.2 * sums[0] + 16 * U32 * np.abs(a)) * (np.abs(z[1]) + sums[1]) + np.abs(a) * sums[1])
    want = scale * a * z[1]
    _inside(H[rows], want, bound * (1 + out) + out * np.abs(want) + 1e-30, "H")
    for i in (0, 1):
        _inside(Z[i, rows], z[i], sums[i] * (1 + out) + out * np.abs(z[i]) + 1e-30, "Z")


def _check_derivatives(dtype, K, grads, x, w, z, dh, kept, rows, columns, scale, name):
    """dW and dbias of some units and dX of some columns, in 64 bits on the device."""
    dX, dW, db = grads
    out = UBF if dtype == "bf16" else U32

    def derivatives(zz, dhh):
        zz, dhh = zz.double().cpu().numpy(), dhh.double().cpu().numpy()
        a, d, dabs = oglu.act(name, zz[0])
        m = scale * np.abs(dhh)
        size = np.stack([m * np.abs(zz[1]) * (dabs + np.abs(d) + 1e-6), m * (np.abs(a) + 1e-6)])
        both = np.stack([scale * dhh * zz[1] * d, scale * dhh * a])
        err = 16 * U32 * size
        return both, err, err + (UBF * (np.abs(both) + err) if dtype == "bf16" else 0)
    n, B = len(kept), x.shape[1]
    both, err, rounded = derivatives(z[:, rows], dh[rows])
    xs = x.double().cpu().numpy()
    for i in (0, 1):
        want, size = both[i] @ xs.T, (np.abs(both[i]) + rounded[i]) @ np.abs(xs).T
        bound = rounded[i] @ np.abs(xs).T + (B + 16) * U32 * size
        _inside(dW[i, rows], want, bound + U32 * np.abs(want) + 1e-30, "dW")
        _inside(db[i, rows], both[i].sum(1), err[i].sum(1) + (B + 16) * U32 * np.abs(both[i]).sum(1) + 1e-30, "dbias")
    both, _, rounded = derivatives(z[:, kept][:, :, columns], dh[kept][:, columns])
    ws = w[:, kept].double().cpu().numpy()
    want = sum(ws[i].T @ both[i] for i in (0, 1))
    size = sum(np.abs(ws[i]).T @ (np.abs(both[i]) + rounded[i]) for i in (0, 1))
    bound = sum(np.abs(ws[i]).T @ rounded[i] for i in (0, 1)) + (2 * n + 16) * U32 * size
    _inside(dX[:, columns], want, bound * (1 + out) + out * np.abs(want) + 1e-30, "dX")


def _large(dtype, B, K, N, period, offset, name, scale, backward=True):
    """Forward and backward of a layer whose tensors are made on the device; a few units and columns checked."""
    from gpu_util import ard_dtype, device, workspace
    dev, st = device(), synth.storage_dtype(dtype)
    gen = torch.Generator(device=dev).manual_seed(1805)
    r = lambda *s, std=1.0: torch.randn(*s, generator=gen, device=dev, dtype=st) * std  # noqa: E731
    x, w, b = r(K, B), r(2, N, K, std=K ** -0.5), torch.randn(2, N, generator=gen, device=dev)
    desc = api.glu_desc(ard_dtype(dtype), B, K, N, api.ard_plan_rows(N, period, offset, None), scale, ACTS[name])
    ws = workspace(api.ard_glu_workspace_bytes(desc))
    H, Z = torch.full((N, B), 7.0, dtype=st, device=dev), torch.full((2, N, B), 7.0, dtype=st, device=dev)
    api.ard_glu_fwd(desc, x, w, b, Z, H, ws)
    torch.cuda.synchronize()
    kept = torch.arange(offset, N, period, device=dev)
    rows = kept[[0, 1, len(kept) // 2, len(kept) - 2, len(kept) - 1]]
    _check_units(dtype, K, H, Z, *_torch_sums(x, w, rows, b), scale, name, rows)
    dropped = torch.arange(N, device=dev) % period != offset
    count = lambda t, value: int(sum((c == value).all(-1).sum() for c in t.split(1 << 20)))  # noqa: E731
    assert count(H[dropped] if N < 1 << 22 else H, 0.0) == int(dropped.sum())
    if not backward:
        return
    del H
    dh = r(N, B)
    dX, dW, db = torch.full_like(x, 7.0), torch.full((2, N, K), 7.0, device=dev), torch.full((2, N), 7.0, device=dev)
    api.ard_glu_bwd(desc, x, w, Z, dh, dX, dW, db, ws)
    torch.cuda.synchronize()
    columns = torch.tensor([0, 1, B // 2, B - 1], device=dev).unique()
    _check_derivatives(dtype, K, (dX, dW, db), x, w, Z, dh, kept, rows, columns, scale, name)
    for t in (dW[0], dW[1], db[0][:, None], db[1][:, None]):
        assert count(t, 0.0) == int(dropped.sum())


@pytest.mark.gpu
@pytest.mark.parametrize("dtype,B", [("f32", 17), ("bf16", 66), ("bf16", 3)])
def test_more_units_than_a_row_of_workgroups(dtype, B):
    """2^24 units and a few, one of 1024 kept: a launch with 256 threads for each would pass 2^32."""
    _large(dtype, B, 4, (1 << 24) + 3, 1024, 2, "silu", 1.5)


@pytest.mark.gpu
def test_weights_past_the_load_offsets():
    """A projection of more than 2^31 bytes: no tiles, and a forward product of the general kernel."""
    N, K = 70000, 16384
    assert 2 * N * K > 2 ** 31
    _large("bf16", 72, K, N, 1, 0, "gelu", 0.5, backward=False)


@pytest.mark.gpu
def test_columns_past_the_load_offsets():
    """Derivatives of more than 2^31 bytes, along which dW is summed, by the general kernel."""
    N, B = 8300, 1 << 18
    assert N // 2 * B * 2 > 2 ** 31
    _large("bf16", B, 8, N, 2, 1, "silu", 2.0)


@pytest.mark.gpu
def test_every_one_of_many_units():
    """More tiles of units than 2^16 in the products, and more groups of units than a row in the few-column kernel."""
    _large("f32", 17, 4, (1 << 23) + 5, 1, 0, "silu", 1.0)
    _large("bf16", 3, 4, (1 << 24) + 3, 1, 0, "gelu", 1.0, backward=False)


@pytest.mark.gpu
@pytest.mark.parametrize("size", SIZES)
def test_nothing_else_is_read(size):
    """NaN in the dropped rows of every operand, behind each operand's end, in the workspace and in the outputs changes no
    bit of what is computed."""
    from gpu_util import ard_dtype, device
    dtype, B, K, N, period, offset, name = size
    X, W, b, dH, Z, keep = _case(dtype, B, K, N, period, offset, name, seed=6)
    dev, st, nan = device(), synth.storage_dtype(dtype), float("nan")
    drop = torch.tensor(keep == 0)
    desc = api.glu_desc(ard_dtype(dtype), B, K, N, api.ard_plan_rows(N, period, offset, None), 1.5, ACTS[name])
    need = api.ard_glu_workspace_bytes(desc)

    def inside(t, fill):  # on 16 bytes, `fill` behind it
        t = t.contiguous()
        whole = torch.full((t.numel() + 4096,), fill, dtype=t.dtype, device=dev)
        whole[:t.numel()] = t.flatten().to(dev)
        return whole[:t.numel()].view(t.shape)

    def run(fill, spoil):
        w, z, dh, bias = W.clone(), Z.transpose(1, 2).contiguous(), dH.T.contiguous(), b.clone()
        if spoil:
            w[:, drop], z[:, drop], dh[drop], bias[:, drop] = nan, nan, nan, nan
        ws = torch.full((need // 4 + 4,), fill, device=dev)
        x, w, z, dh, bias = (inside(t, fill) for t in (X.T, w, z, dh, bias))
        H, Zt = torch.full((N, B), fill, dtype=st, device=dev), torch.zeros(2, N, B, dtype=st, device=dev)
        api.ard_glu_fwd(desc, x, w, bias, Zt, H, ws)
        dX, dW = torch.full((K, B), fill, dtype=st, device=dev), torch.full((2, N, K), fill, device=dev)
        db = torch.full((2, N), fill, device=dev)
        ws.fill_(fill)
        api.ard_glu_bwd(desc, x, w, z, dh, dX, dW, db, ws)
        torch.cuda.synchronize()
        return H, Zt, dX, dW, db
    for got, want in zip(run(nan, True), run(0.0, False)):
        assert torch.equal(got, want)
