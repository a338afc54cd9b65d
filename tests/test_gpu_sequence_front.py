"""The recurrent stack in front of a Moonwalk net, trained with the orthogonalised update: gradients of the
whole model against automatic differentiation of the same formulas in 64 bits, and a short training run.

Tolerance of a gradient, relative in the Frobenius norm: the projections' products keep 16 bits of their
operands (2^-16 each, two products per block and direction) and the net's gradients are good to 1e-4 of
theirs; 1e-3 covers two blocks and three layers."""
import numpy as np
import pytest

from paper_2402_14212_b200 import sequence_front as SF

pytestmark = pytest.mark.gpu


def reference(trainer, x, target):
    import torch
    f = trainer.front
    D = f.width
    leaf = lambda t: t.double().clone().requires_grad_(True)
    proj, w_post, scale, w_pre = ([leaf(t) for t in ts] for ts in (f.proj, f.w_post, f.scale, f.w_pre))
    w_in, net, xin = leaf(f.w_in), [leaf(t) for t in trainer.params], leaf(x)
    B, T, _ = x.shape
    norm = lambda v, w: w * v / torch.sqrt(v.square().mean(-1, keepdim=True) + 1e-6)
    s = xin
    n = norm(s, w_in)
    for i, w in enumerate(proj):
        p = n @ w.T
        v, fl, z = p[..., :D], p[..., D:2 * D] + f.bias.double(), p[..., 2 * D:]
        a, u = torch.sigmoid(fl), torch.sigmoid(-fl)
        h, state = [], torch.zeros(B, D, dtype=torch.float64, device=x.device)
        for t in range(T):
            state = a[:, t] * state + u[:, t] * v[:, t]
            h.append(state)
        s = s + scale[i] * torch.nn.functional.silu(z) * norm(torch.stack(h, 1), w_post[i])
        if i < len(w_pre):
            n = norm(s, w_pre[i])
    y = s.reshape(B * T, D)
    for w in net:
        y = torch.nn.functional.leaky_relu(y @ w.T, 0.1)
    loss = (y - target.double()).square().mean()
    loss.backward()
    return float(loss.detach()), dict(net=net, proj=proj, w_post=w_post, scale=scale, w_pre=w_pre, w_in=[w_in], x=[xin])


def test_gradients_of_the_whole_model_match_autograd():
    t = SF.Trainer(width=128, blocks=2, depth=3, batch=4, time=64, seed=1)
    x, target = SF.make_task(128, 4, 64, 1)
    want_loss, want = reference(t, x, target)
    dW, front, dx = t.gradients(x, target)
    assert t.status() == 0
    assert abs(float(t.loss.item()) - want_loss) <= 1e-4 * want_loss
    got = dict(net=dW, proj=front["proj"], w_post=front["w_post"], scale=front["scale"], w_pre=front["w_pre"],
               w_in=[front["w_in"]], x=[dx])
    for name, leaves in want.items():
        assert len(leaves) == len(got[name]) > 0
        for a, b in zip(got[name], leaves):
            g = b.grad.cpu().numpy()
            err = np.linalg.norm(a.double().cpu().numpy().reshape(g.shape) - g) / np.linalg.norm(g)
            assert err <= 1e-3, (name, err)


def test_training_lowers_the_loss():
    t = SF.Trainer(width=128, blocks=2, depth=3, batch=4, time=64, seed=2)
    x, target = SF.make_task(128, 4, 64, 2)
    losses = []
    for _ in range(25):
        losses.append(float(t.step(x, target).item()))
        assert t.status() == 0
    assert losses[-1] < 0.9 * losses[0] and np.isfinite(losses).all()
