"""The distillation loss: the oracle against finite differences and torch (CPU), refusals (CPU), and the kernels against
the oracle (GPU).

Tolerances, per column or value. Loss: the logarithms and sums of exponentials are off by a few units of 2^-24 (a sum's
terms are added in chains of at most V / 8 and joined pairwise; the largest term is 1): 64 units of the loss's terms and
of their factor weight T^2. Gradient: 64 units of the largest factor (weight T, 1) times the softmax value, and the
rounding to the logits' type.
"""
import numpy as np
import pytest
import torch

from oracle import distill as od
from paper_1805_08939_amd import api, synth

U32, UBF = 2.0 ** -24, 2.0 ** -8
INF = float("inf")


# ---------------------------------------------------------------- the oracle

def test_oracle_gradient_is_the_loss_differenced():
    r = np.random.default_rng(3)
    z, idx, t = r.normal(size=9), [4, 0, 4, -1, 11], r.normal(size=5)  # a class named twice, two entries that are none
    for T, a in ((1.0, 1.0), (2.5, 0.3), (0.7, 0.0)):
        _, dz, _ = od.column(z, idx, t, 2, T, a)
        for v in range(9):
            e = np.eye(9)[v] * 1e-6
            d = (od.column(z + e, idx, t, 2, T, a)[0] - od.column(z - e, idx, t, 2, T, a)[0]) / 2e-6
            assert abs(d - dz[v]) < 1e-7


def test_oracle_is_torch():
    r = np.random.default_rng(4)
    z, t = torch.tensor(r.normal(size=(6, 20))), torch.tensor(r.normal(size=(6, 20)))
    T = 2.0
    want = T * T * torch.nn.functional.kl_div(torch.log_softmax(z / T, 1), torch.softmax(t / T, 1), reduction="none").sum(1)
    hard = torch.nn.functional.cross_entropy(z, torch.arange(6), reduction="none")
    idx = np.tile(np.arange(20)[:, None], (1, 6))  # every class named: the whole teacher
    loss, _, _ = od.batch(z.numpy().T, idx, t.numpy().T, np.arange(6), T, 0.6)
    assert np.abs(loss - (0.6 * want + 0.4 * hard).numpy()).max() < 1e-12


# ---------------------------------------------------------------- refusals

def test_refuses_bad_calls():
    a = 4096
    good = dict(dtype=api.ARD_F32, batch=4, classes=9, top=3, temperature=2.0, soft_weight=0.5)

    def refused(status, call, *args):
        with pytest.raises(api.ArdError) as e:
            call(*args, stream=0)
        assert e.value.status == status and e.value.message

    for bad, status in ((dict(dtype=3), 2), (dict(batch=0), 1), (dict(classes=0), 1), (dict(top=-1), 1),
                        (dict(top=70000), 1), (dict(temperature=0.0), 1), (dict(temperature=float("nan")), 1),
                        (dict(temperature=INF), 1), (dict(temperature=-1.0), 1), (dict(soft_weight=1.5), 1),
                        (dict(soft_weight=float("nan")), 1)):
        d = api.distill_desc(**{**good, **bad})
        assert api.ard_distill_workspace_bytes(d) == 0
        refused(status, api.ard_distill_fwd, d, a, a, a, a, a, a, (a, 1 << 30))
        refused(status, api.ard_distill_bwd, d, a, a, a, a, a, a, 2 * a)
    d = api.distill_desc(**good)
    for i in (0, 1, 2, 4, 5):
        args = [a] * 6
        args[i] = None
        refused(1, api.ard_distill_fwd, d, *args, (a, 1 << 30))
        args[i] = a + 4
        refused(1, api.ard_distill_fwd, d, *args, (a, 1 << 30))
    refused(1, api.ard_distill_fwd, d, a, a, a, a, a, a, (a + 4, 1 << 30))
    assert api.ard_distill_workspace_bytes(d) == 0  # few classes: one launch, no sums to keep
    many = api.distill_desc(**{**good, "classes": 3000})
    assert api.ard_distill_workspace_bytes(many) > 0
    refused(5, api.ard_distill_fwd, many, a, a, a, a, a, a, None)
    refused(5, api.ard_distill_fwd, many, a, a, a, a, a, a, (a, 4))
    refused(1, api.ard_distill_bwd, d, a, a, a, a, a, None, a)  # in place
    refused(1, api.ard_distill_bwd, d, a, a, a, a, None, None, 2 * a)
    refused(1, api.ard_distill_bwd, d, a, a, a, a, a, None, None)


# ---------------------------------------------------------------- the kernels

def _run(dtype, Z, idx, t, labels, T, a, dloss):
    from gpu_util import ard_dtype, device, workspace
    dev = device()
    V, B = Z.shape
    desc = api.distill_desc(ard_dtype(dtype), B, V, idx.shape[0], T, a)
    put = lambda x: None if x is None or x.numel() == 0 else x.contiguous().to(dev)  # noqa: E731
    z, i, tl, lab, dl = put(Z), put(idx), put(t), put(labels), put(dloss)
    loss, stats = torch.full((B,), 7.0, device=dev), torch.empty(5, B, device=dev)
    dZ = torch.full_like(z, 7.0)
    ws = workspace(api.ard_distill_workspace_bytes(desc))
    api.ard_distill_fwd(desc, z, i, tl, lab, loss, stats, ws)
    api.ard_distill_bwd(desc, z, i, tl, lab, stats, dl, dZ)
    torch.cuda.synchronize()
    return loss.double().cpu().numpy(), dZ.double().cpu().numpy()


def _check(dtype, Z, idx, t, labels, T, a, dloss):
    got, dgot = _run(dtype, Z, idx, t, labels, T, a, dloss)
    z = Z.double().numpy()
    with np.errstate(invalid="ignore", over="ignore"):
        loss, dz, size = od.batch(z, idx.numpy(), t.double().numpy(), None if labels is None else labels.numpy(), T, a)
        loss[np.isinf(loss.astype(np.float32))] = INF  # past the range of the loss's type
    dl = np.ones(Z.shape[1]) if dloss is None else dloss.double().numpy()
    dz = dz * dl
    fine = np.isfinite(loss)
    assert np.array_equal(np.isposinf(loss), np.isposinf(got)) and np.isfinite(got[fine]).all()
    span = 1 + np.abs(np.where(np.isfinite(z), z, 0)).max() / min(T, 1.0)
    bound = 64 * U32 * (size + span * (a * T * T + 1 - a))
    assert (np.abs(got - loss)[fine] <= bound[fine]).all(), np.abs(got - loss)[fine].max()
    out = UBF if dtype == "bf16" else U32
    assert np.isfinite(dgot).all()
    bound = out * np.abs(dz) + (64 + 4 * span) * U32 * (a * T + 1 - a) * np.abs(dl) + 1e-38
    assert (np.abs(dgot - dz) <= bound).all(), np.abs(dgot - dz).max()


def _inputs(dtype, V, B, top, seed):
    g = synth.generator(1805 + seed)
    Z = synth.to_storage(synth.normal(g, (V, B), 3.0), dtype)
    r = np.random.default_rng(seed)
    idx = np.stack([r.permutation(V)[:top] if top <= V else r.integers(0, V, top) for _ in range(B)], 1)
    return (Z, torch.tensor(idx.reshape(top, B).astype(np.int32)), synth.normal(g, (top, B), 2.0) + 5,
            torch.tensor(r.integers(0, V, B).astype(np.int32)), synth.normal(g, (B,)))


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("V,B,top,T,a", [
    (1, 1, 1, 1.0, 0.5), (2, 1, 2, 3.0, 1.0), (10, 128, 5, 4.0, 0.9), (10, 3, 10, 1.0, 0.5), (50, 7, 3, 2.0, 0.0),
    (1000, 1, 64, 2.0, 0.5), (333, 9, 1, 1.0, 1.0), (257, 100, 17, 0.5, 0.5), (8800, 20, 20, 2.0, 0.5),
    (1031, 65, 8, 1.0, 0.7), (64, 700, 4, 2.0, 0.3), (40, 1030, 6, 1.0, 0.6), (5003, 16, 300, 1.5, 0.4),
    (7, 4, 12, 2.0, 0.5), (700, 12, 0, 2.0, 0.5)])
def test_loss_and_gradient(dtype, V, B, top, T, a):
    Z, idx, t, labels, dloss = _inputs(dtype, V, B, top, V + B)
    _check(dtype, Z, idx, t, labels, T, a, dloss)
    _check(dtype, Z, idx, t, None, T, a, None)


@pytest.mark.gpu
@pytest.mark.parametrize("top", [15, 16, 17, 31, 32, 127, 128, 129])
@pytest.mark.parametrize("V", [40, 400])
def test_entries_in_blocks_of_threads(V, top):
    """Entry counts on both sides of what a workgroup holds, classes named more than once."""
    Z, idx, t, labels, dloss = _inputs("bf16", V, 19, top, top)
    idx[: top // 3] = idx[top - top // 3:]
    _check("bf16", Z, idx, t, labels, 2.0, 0.5, dloss)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("T", [1.0, 2.0])
def test_masked_and_empty_columns(dtype, T):
    V, B, top = 300, 24, 6
    Z, idx, t, labels, dloss = _inputs(dtype, V, B, top, 77)
    Z[5:250, 1] = -INF                       # masked classes, some of them the teacher's
    Z[:, 2] = -INF                           # nothing left
    Z[:, 3] = torch.finfo(Z.dtype).min       # the type's lowest value everywhere
    Z[7:, 4] = torch.finfo(Z.dtype).min      # and as a mask
    Z[:, 5] = 100.0
    Z[17, 6] = 300.0                         # one class far above the others
    idx[:, 7] = -1                           # no entry
    idx[2:, 8] = V                           # entries outside
    idx[:, 9] = 11                           # one class in every entry
    idx[0, 10], idx[3, 10] = 5, 5            # a class named twice
    t[:, 11] = -INF                          # a teacher without a finite logit
    t[1:, 12] = -INF
    t[:, 13] = 80.0
    labels[14], labels[15], labels[16] = -1, V, -100
    labels[9] = 11                           # label and teacher in one place
    idx[:, 17], labels[17] = -1, -1          # no term at all
    Z[:, 18] = Z[:, 18] * 20
    _check(dtype, Z, idx, t, labels, T, 0.6, dloss)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_nan_stays_in_its_column(dtype):
    V, B, top = 120, 11, 4
    Z, idx, t, labels, dloss = _inputs(dtype, V, B, top, 5)
    clean, dclean = _run(dtype, Z, idx, t, labels, 2.0, 0.5, dloss)
    Z[33, 4] = float("nan")
    Z[70, 6] = INF
    got, dgot = _run(dtype, Z, idx, t, labels, 2.0, 0.5, dloss)
    rest = [b for b in range(B) if b not in (4, 6)]
    assert np.isnan(got[[4, 6]]).all() and np.isnan(dgot[:, 4]).all()
    assert np.array_equal(got[rest], clean[rest]) and np.array_equal(dgot[:, rest], dclean[:, rest])


@pytest.mark.gpu
def test_runs_alike():
    Z, idx, t, labels, dloss = _inputs("bf16", 3001, 333, 9, 8)
    idx[4] = idx[2]
    a, b = (_run("bf16", Z, idx, t, labels, 2.0, 0.5, dloss) for _ in range(2))
    assert np.array_equal(a[0], b[0]) and np.array_equal(a[1], b[1])


@pytest.mark.gpu
def test_logits_past_two_to_the_31():
    """More than 2^31 logits: zero everywhere but in the last class, whose softmax is known."""
    from gpu_util import device, workspace
    dev, V, B = device(), 65600, 32776
    assert V * B > 2 ** 31
    Z = torch.zeros(V, B, dtype=torch.bfloat16, device=dev)
    Z[V - 1] = 8.0
    idx = torch.full((1, B), V - 1, dtype=torch.int32, device=dev)
    tl, labels = torch.ones(1, B, device=dev), torch.full((B,), V - 1, dtype=torch.int32, device=dev)
    desc = api.distill_desc(api.ARD_BF16, B, V, 1, 1.0, 0.5)
    loss, stats, dZ = torch.empty(B, device=dev), torch.empty(5, B, device=dev), torch.empty_like(Z)
    ws = workspace(api.ard_distill_workspace_bytes(desc))
    api.ard_distill_fwd(desc, Z, idx, tl, labels, loss, stats, ws)
    api.ard_distill_bwd(desc, Z, idx, tl, labels, stats, None, dZ)
    torch.cuda.synchronize()
    total = np.exp(8.0) + V - 1
    want = np.log(total) - 8.0  # both terms are -log q of the last class
    assert (loss.double() - want).abs().max() < 64 * U32 * (8 + want)
    q = np.exp(8.0) / total
    assert (dZ[V - 1].double() - (q - 1)).abs().max() < UBF
    assert (dZ[V - 2].double() - 1 / total).abs().max() < UBF / total + 64 * U32 / total


@pytest.mark.gpu
@pytest.mark.parametrize("V,B", [(40, 20), (3000, 70)])
def test_in_a_graph(V, B):
    from gpu_util import device, workspace
    dev = device()
    Z, idx, t, labels, dloss = (x.contiguous().to(dev) for x in _inputs("bf16", V, B, 5, 21))
    desc = api.distill_desc(api.ARD_BF16, B, V, 5, 2.0, 0.5)
    ws = workspace(api.ard_distill_workspace_bytes(desc))
    loss, stats, dZ = torch.empty(B, device=dev), torch.empty(5, B, device=dev), torch.empty_like(Z)

    def step():
        api.ard_distill_fwd(desc, Z, idx, t, labels, loss, stats, ws)
        api.ard_distill_bwd(desc, Z, idx, t, labels, stats, dloss, dZ)
    step()
    torch.cuda.synchronize()
    eager = loss.clone(), dZ.clone()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step()
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for _ in range(3):
        loss.fill_(3.0)
        dZ.fill_(3.0)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(loss, eager[0]) and torch.equal(dZ, eager[1])


@pytest.mark.gpu
@pytest.mark.parametrize("top", [1, 17])
def test_more_columns_than_a_row_of_workgroups(top):
    """2^28 columns and a few of three classes: 16 threads for each would pass 2^32. Columns repeat after 1009."""
    from gpu_util import device, workspace
    dev, V, B, few = device(), 3, (1 << 28) + 5, 1009
    Z, idx, t, labels, _ = _inputs("bf16", V, few, top, 33)
    want, dwant = _run("bf16", Z, idx, t, labels, 2.0, 0.5, None)

    def wide(x):
        x = x.to(dev)
        out = torch.empty(*x.shape[:-1], B, dtype=x.dtype, device=dev)
        whole = B // few * few
        out[..., :whole].unflatten(-1, (-1, few)).copy_(x[..., None, :].expand(*x.shape[:-1], B // few, few))
        out[..., whole:] = x[..., :B - whole]
        return out
    desc = api.distill_desc(api.ARD_BF16, B, V, top, 2.0, 0.5)
    Z, idx, t, labels = (wide(x) for x in (Z, idx, t, labels))
    loss, stats, dZ = torch.full((B,), 7.0, device=dev), torch.empty(5, B, device=dev), torch.full_like(Z, 7.0)
    ws = workspace(api.ard_distill_workspace_bytes(desc))
    api.ard_distill_fwd(desc, Z, idx, t, labels, loss, stats, ws)
    api.ard_distill_bwd(desc, Z, idx, t, labels, stats, None, dZ)
    torch.cuda.synchronize()
    assert torch.equal(loss, wide(torch.tensor(want).float())) and torch.equal(dZ, wide(torch.tensor(dwant).bfloat16()))


def _terms(z, idx, t, labels, T, a):
    """The sums of the absolute values of each gradient value's terms, in 64 bits."""
    V, B = z.shape
    out = np.zeros((V, B))
    for b in range(B):
        if z[:, b].max() == -INF:
            continue
        ok = [j for j in range(idx.shape[0]) if 0 <= idx[j, b] < V]
        if a > 0 and ok and max(t[j, b] for j in ok) > -INF:
            out[:, b] += a * T * od._softmax(z[:, b] / T)
            for j, p in zip(ok, od._softmax(np.array([t[j, b] for j in ok]) / T)):
                out[idx[j, b], b] += a * T * p
        if a < 1 and labels is not None and 0 <= labels[b] < V:
            out[:, b] += (1 - a) * od._softmax(z[:, b])
            out[labels[b], b] += 1 - a
    return out


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("V,B,top,T,a", [
    (10, 128, 5, 4.0, 0.9), (333, 9, 1, 1.0, 1.0), (257, 100, 17, 0.5, 0.5), (8800, 20, 20, 2.0, 0.5),
    (1031, 65, 8, 1.0, 0.7), (64, 700, 4, 2.0, 0.3), (5003, 16, 300, 1.5, 0.4), (700, 12, 0, 2.0, 0.5)])
def test_each_value_of_the_gradient_for_its_size(dtype, V, B, top, T, a):
    """Small probabilities too: each value against its own terms. A term is an exponential (the rounding of its argument x,
    three times, is 3 |x| 2^-24 of it, |x| at most `span`) over a sum, times a factor: 64 + 4 span units of its size, and the
    rounding of the result; values below the smallest normal numbers may be 0."""
    Z, idx, t, labels, dloss = _inputs(dtype, V, B, top, V + B)
    for lab, dl in ((labels, dloss), (None, None)):
        _, dgot = _run(dtype, Z, idx, t, lab, T, a, dl)
        z, i, tt = Z.double().numpy(), idx.numpy(), t.double().numpy()
        ll, d = None if lab is None else lab.numpy(), 1.0 if dl is None else dl.double().numpy()
        want, terms = od.batch(z, i, tt, ll, T, a)[1] * d, _terms(z, i, tt, ll, T, a) * np.abs(d)
        span = 1 + (z.max(0) - z.min(0)).max() / min(T, 1.0)
        out = UBF if dtype == "bf16" else U32
        bound = (64 + 4 * span) * U32 * terms
        bound += out * (np.abs(want) + bound) + 2.0 ** -126 * (1 + a * T) * np.abs(d)
        assert (np.abs(dgot - want) <= bound).all(), (np.abs(dgot - want) / bound).max()


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("V", [6, 700])
def test_masked_classes_that_an_entry_or_the_label_names(dtype, V):
    """Logits of -inf: gradient 0, but for the classes of the teacher's entries (-a T p) and the label (-(1 - a)), whose
    columns have a loss of +inf. Powers of two, so that every value is exact."""
    Z = torch.full((V, 4), -INF, dtype=synth.storage_dtype(dtype))
    Z[0], Z[1] = 0.0, 0.0                                # q = q1 = 1/2 each
    idx = torch.tensor([[3, 0, 0, 3], [4, 1, 1, 0]], dtype=torch.int32)
    t = torch.tensor([[1.0, 1, 1, -INF], [1.0, 1, 1, 1]])  # p = 1/2 each, in the last column 0 and 1
    labels = torch.tensor([0, 5, 1, 1], dtype=torch.int32)
    loss, dZ = _run(dtype, Z, idx, t, labels, 2.0, 0.5, None)
    want = np.zeros((V, 4))
    want[0], want[1] = 0.75, 0.75                        # a T q + (1 - a) q1
    want[[3, 4], 0] = -0.5                               # - a T p
    want[0, 0] -= 0.5                                    # - (1 - a)
    want[[0, 1], 1] -= 0.5
    want[5, 1] = -0.5
    want[[0, 1], 2] -= 0.5
    want[1, 2] -= 0.5
    want[0, 3] -= 1.0
    want[1, 3] -= 0.5
    assert np.array_equal(np.isposinf(loss), [True, True, False, False]) and np.isfinite(loss[2:]).all()
    assert np.array_equal(dZ, want)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("V,B,top", [(1, 1, 1), (10, 3, 4), (256, 17, 16), (256, 17, 40), (257, 9, 5), (700, 1, 3), (5003, 13, 33),
                                     (8800, 20, 0)])
def test_nothing_else_is_read(dtype, V, B, top):
    """NaN behind each operand's end, in the logits of entries that are none, in the workspace and in the outputs changes no
    bit of what is computed."""
    from gpu_util import ard_dtype, device
    dev, nan = device(), float("nan")
    Z, idx, t, labels, dloss = _inputs(dtype, V, B, top, 91)
    if top > 1:
        idx[1, ::2] = -1
    desc = api.distill_desc(ard_dtype(dtype), B, V, top, 2.0, 0.5)

    def inside(x, fill):  # on 16 bytes, `fill` behind it
        whole = torch.full((x.numel() + 4096,), fill, dtype=x.dtype, device=dev)
        whole[:x.numel()] = x.contiguous().flatten().to(dev)
        return whole[:x.numel()].view(x.shape)

    def run(fill, spoil):
        tl = t.clone()
        if spoil:
            tl[idx < 0] = nan
        z, i, tl, lab, dl = inside(Z, fill), inside(idx, 0), inside(tl, fill), inside(labels, 0), inside(dloss, fill)
        ws = torch.full((api.ard_distill_workspace_bytes(desc) // 4 + 4,), fill, device=dev)
        loss, stats, dZ = (torch.full(s, fill, device=dev) for s in ((B,), (5, B), (V, B)))
        dZ = dZ.to(z.dtype)
        told = (z, i, tl, lab) if top else (z, None, None, lab)
        api.ard_distill_fwd(desc, *told, loss, stats, ws)
        api.ard_distill_bwd(desc, *told, stats, dl, dZ)
        torch.cuda.synchronize()
        return loss, dZ
    for got, want in zip(run(nan, True), run(0.0, False)):
        assert torch.equal(got, want)
