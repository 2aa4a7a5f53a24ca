"""The example training step (paper_2609_10549_amd/train_step.py): its loss and
gradients against the same model in fp64 through torch's automatic
differentiation, and the loss over a few steps."""
import math

import pytest

pytestmark = pytest.mark.gpu


def _reference(model, ids, target):
    """The loss and gradients in fp64 from the bf16 weights."""
    import torch
    w = {k: model.bf16.get(k, v).double().requires_grad_() for k, v in model.master.items()}

    def norm(x, g, b):
        m = x.mean(1, keepdim=True)
        return (x - m) / torch.sqrt((x - m).square().mean(1, keepdim=True) + 1e-5) * g + b

    x0 = model.scale * w["E"][ids]
    x1 = x0 + norm(x0, w["g1"], w["b1"]) @ w["W1"].T @ w["W2"].T
    z = norm(x1, w["g2"], w["b2"]) @ w["E"].T
    kept = target >= 0
    loss = (torch.logsumexp(z, 1) - z.gather(1, target.clamp(min=0)[:, None])[:, 0])[kept].mean()
    loss.backward()
    return float(loss.detach()), {k: v.grad for k, v in w.items()}


def test_first_step_against_automatic_differentiation():
    from paper_2609_10549_amd import train_step as T
    model = T.Model(tokens=512, hidden=128, vocab=600, shards=3, seed=1)
    ids, target = T.batch(model, 0)
    loss = model.forward(ids, target)
    got = float(loss.sum() / (target >= 0).sum())
    grads = model.backward(ids, target)
    want, ref = _reference(model, ids, target)
    # every activation and gradient between the operators is rounded to bf16
    # (2^-8 each); a dozen of them lie on the longest path
    tol = 12 * 2.0 ** -8
    assert abs(got - want) < tol
    for k, r in ref.items():
        err = float((grads[k].double() - r).norm() / r.norm())
        print(k, err, flush=True)
        assert err < tol, k


def test_loss_falls_towards_the_learned_rule():
    from paper_2609_10549_amd import train_step as T
    model = T.Model(tokens=1024, hidden=128, vocab=200, shards=2, seed=2)
    first = float(model.step(*T.batch(model, 0), 0.2))
    assert first > 0.5 * math.log(200)
    for i in range(1, 40):
        last = float(model.step(*T.batch(model, i), 0.2))
    assert last < 0.5 * first
