"""The example that runs the gated layer, linear attention and the distillation loss together."""
import os
import sys

import pytest
import torch

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
sys.path.insert(0, os.path.join(ROOT, "examples"))


def _model(**kw):
    import distilled_lm as lm
    return lm, lm.Model(**{**dict(vocab=61, width=64, heads=2, hidden=96), **kw})


@pytest.mark.gpu
def test_the_loss_falls():
    lm, model = _model()
    losses = lm.train(model, lm.Teacher(61, 6, model.dev), steps=300, seqs=6, length=35, log=None)
    assert all(x == x for x in losses)
    assert sum(losses[-5:]) < 0.8 * sum(losses[:5])


@pytest.mark.gpu
def test_a_prompt_at_once_is_its_tokens_one_by_one():
    _, model = _model()
    tokens = torch.randint(0, 61, (3, 9), device=model.dev, generator=torch.Generator(device=model.dev).manual_seed(2))
    whole, last, _ = model.forward(tokens)
    state, cols = None, []
    for t in range(9):
        logits, state, _ = model.forward(tokens[:, t:t + 1], state=state)
        cols.append(logits)
    steps = torch.stack(cols, 2)  # [vocab][seqs][length]
    size = whole.abs().max()
    assert (steps.reshape(whole.shape) - whole).abs().max() < 1e-4 * size
    assert (state - last).abs().max() < 1e-4 * last.abs().max()


@pytest.mark.gpu
def test_gradients_against_differences():
    """The whole chain, weight by weight: central differences of the mean loss in fp32 along a random direction."""
    from paper_1805_08939_amd import api
    lm, model = _model()
    dev, seqs, length = model.dev, 2, 20
    n = seqs * length
    teacher = lm.Teacher(61, 6, dev)
    tokens, idx, t, labels = teacher.batch(seqs, length, torch.Generator(device=dev).manual_seed(3))
    plan = api.ard_plan_rows(96, 2, 1, None)
    dist = api.distill_desc(lm.ARD_DTYPE, n, 61, 6, 1.0, 0.5)
    loss, stats, share = torch.empty(n, device=dev), torch.empty(5, n, device=dev), torch.full((n,), 1.0 / n, device=dev)

    def value():
        logits, _, saved = model.forward(tokens, plan, 2.0, train=True)
        ws = model._space(api.ard_distill_workspace_bytes(dist))
        api.ard_distill_fwd(dist, logits, idx, t, labels, loss, stats, ws)
        return logits, saved, float(loss.double().mean())

    logits, saved, _ = value()
    dlogits = torch.empty_like(logits)
    api.ard_distill_bwd(dist, logits, idx, t, labels, stats, share, dlogits)
    model.backward(dlogits, plan, saved)
    gen = torch.Generator(device=dev).manual_seed(4)
    for name in ("qkv", "mix", "glu", "down", "head"):
        p = getattr(model, name)
        W, grad = p.W.clone(), p.dW.double()
        step = torch.randn(W.shape, device=dev, generator=gen)
        step = step * (grad != 0)  # the kept weights
        h = 2e-3 * float(W.norm() / step.norm())
        p.W.copy_(W + h * step)
        up = value()[2]
        p.W.copy_(W - h * step)
        down = value()[2]
        p.W.copy_(W)
        want, got = (up - down) / (2 * h), float((grad * step).sum())
        # rounding of the two losses (2^-22 each of about 5) over 2 h, and the third derivative's part
        assert abs(got - want) < 2e-2 * float(grad.norm() * step.norm()) / W.numel() ** 0.5 + 2e-6 / h, (name, got, want)


@pytest.mark.gpu
def test_gradients_of_every_kept_weight():
    """As above along directions that follow from the pattern, not from the gradients: one that a call leaves at 0 by
    mistake counts. The three parts of the first projection (queries, keys, values) and the two of the gated layer each for
    themselves; dropped weights have no gradient."""
    from paper_1805_08939_amd import api
    lm, model = _model()
    dev, seqs, length, w = model.dev, 2, 20, model.width
    n = seqs * length
    teacher = lm.Teacher(61, 6, dev)
    tokens, idx, t, labels = teacher.batch(seqs, length, torch.Generator(device=dev).manual_seed(5))
    plan = api.ard_plan_rows(96, 2, 1, None)
    dist = api.distill_desc(lm.ARD_DTYPE, n, 61, 6, 1.0, 0.5)
    loss, stats, share = torch.empty(n, device=dev), torch.empty(5, n, device=dev), torch.full((n,), 1.0 / n, device=dev)

    def value():
        logits, _, saved = model.forward(tokens, plan, 2.0, train=True)
        ws = model._space(api.ard_distill_workspace_bytes(dist))
        api.ard_distill_fwd(dist, logits, idx, t, labels, loss, stats, ws)
        return logits, saved, float(loss.double().mean())

    logits, saved, _ = value()
    dlogits = torch.empty_like(logits)
    api.ard_distill_bwd(dist, logits, idx, t, labels, stats, share, dlogits)
    model.backward(dlogits, plan, saved)
    units = (torch.arange(96, device=dev) % 2 == 1).float()
    on = {name: torch.ones_like(getattr(model, name).W) for name in ("mix", "head")}
    on["down"] = units.expand(w, 96).clone()
    for i in (0, 1):
        on["glu", i] = torch.zeros_like(model.glu.W)
        on["glu", i][i] = units[:, None]
    for i in (0, 1, 2):
        on["qkv", i] = torch.zeros_like(model.qkv.W)
        on["qkv", i][i * w:(i + 1) * w] = 1.0
    gen = torch.Generator(device=dev).manual_seed(6)
    for name, mask in on.items():
        p = getattr(model, name if isinstance(name, str) else name[0])
        W, grad = p.W.clone(), p.dW.double()
        step = torch.randn(W.shape, device=dev, generator=gen) * mask
        h = 2e-3 * float((W * mask).norm() / step.norm())
        p.W.copy_(W + h * step)
        up = value()[2]
        p.W.copy_(W - h * step)
        down = value()[2]
        p.W.copy_(W)
        want, part = (up - down) / (2 * h), grad * mask
        got, size = float((part * step).sum()), float(part.norm() * step.norm()) / float(mask.sum()) ** 0.5
        # rounding of the two losses (2^-22 each of about 5) over 2 h, and the third derivative's part
        assert size > 0 and abs(got - want) < 2e-2 * size + 2e-6 / h, (name, got, want, size)
    assert not (model.glu.dW * (1 - units)[:, None]).any() and not (model.down.dW * (1 - units)).any()
