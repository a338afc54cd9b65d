"""The lookup, the vocabulary's loss and the clipping as the recurrent stack uses them: gradients of the whole token
model, and of the stack that takes tokens in front of a net, against automatic differentiation of the same formulas in
64 bits; and the operators in one captured step.

Tolerance of a gradient, relative in the Frobenius norm: the projections' products keep 16 bits of their operands (2^-16
each, two products per block and direction) and a net's gradients are good to 1e-4 of theirs; 1e-3 covers two blocks
and three layers.  The lookup, the loss (2^-18 of its terms) and the clipping add nothing to that."""
import math
import sys

import pytest
import torch

from paper_2402_14212_b200 import binding as mwb
from paper_2402_14212_b200 import sequence_front as SF

pytestmark = pytest.mark.gpu


def stack(f, x, leaves):
    """The blocks in 64 bits on x [batch, time, width]."""
    proj, w_post, scale, w_pre, w_in = leaves
    B, T, D = x.shape
    norm = lambda v, w: w * v / torch.sqrt(v.square().mean(-1, keepdim=True) + 1e-6)
    s, n = x, norm(x, w_in)
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
    return s


def leaf(t):
    return t.double().clone().requires_grad_(True)


def rows(tokens, table, width):
    on = tokens >= 0
    return torch.where(on[..., None], table[torch.where(on, tokens, 0)] * math.sqrt(width), 0.0)


def check(got, leaves):
    for name, want in leaves.items():
        assert len(want) == len(got[name]) > 0
        for a, b in zip(got[name], want):
            err = float((a.double().reshape(b.shape) - b.grad).norm() / b.grad.norm())
            assert err <= 1e-3, (name, err)


def front_leaves(f):
    lists = dict(proj=f.proj, w_post=f.w_post, scale=f.scale, w_pre=f.w_pre, w_in=[f.w_in])
    return {k: [leaf(t) for t in v] for k, v in lists.items()}


def test_gradients_of_the_token_model_match_autograd():
    vocab, width, B, T = 333, 128, 4, 64
    t = SF.TokenTrainer(vocab, width, 2, seed=1)
    t.w_out.add_(0.1 * torch.randn_like(t.w_out))
    tokens = SF.make_tokens(vocab, B, T, 1)
    r, got = t.gradients(tokens)
    L = front_leaves(t.front)
    table, w_out = leaf(t.table), leaf(t.w_out)
    s = stack(t.front, rows(tokens[:, :-1], table, width), (L["proj"], L["w_post"], L["scale"], L["w_pre"], L["w_in"][0]))
    n = (w_out * s / torch.sqrt(s.square().mean(-1, keepdim=True) + 1e-6)).reshape(B * T, width)
    loss = torch.nn.functional.cross_entropy(n @ table.T, tokens[:, 1:].reshape(-1), ignore_index=-1)
    loss.backward()
    assert abs(float(r.total) - float(loss)) <= 1e-4 * float(loss)
    L.update(table=[table], w_out=[w_out])
    check({k: v if isinstance(v, list) else [v] for k, v in got.items()}, L)
    same = t.losses(tokens)
    assert abs(float(same.total) - float(r.total)) <= 1e-5 * float(loss)
    assert bool((same.loss[(tokens[:, 1:].reshape(-1) < 0)] == 0).all())


def test_gradients_of_tokens_in_front_of_a_net_match_autograd():
    vocab, width, B, T = 50, 128, 4, 64
    t = SF.Trainer(width=width, blocks=1, depth=2, batch=B, time=T, seed=1, vocab=vocab)
    tokens = SF.make_tokens(vocab, B, T, 2)[:, :-1]
    _, target = SF.make_task(width, B, T, 1)
    dW, front, dx = t.gradients(tokens, target)
    assert t.status() == 0
    L = front_leaves(t.front)
    L.pop("w_pre")
    table, net = leaf(t.table), [leaf(w) for w in t.params]
    y = stack(t.front, rows(tokens, table, width), (L["proj"], L["w_post"], L["scale"], [], L["w_in"][0])).reshape(B * T, width)
    for w in net:
        y = torch.nn.functional.leaky_relu(y @ w.T, 0.1)
    (y - target.double()).square().mean().backward()
    L.update(table=[table], net=net)
    got = {k: v if isinstance(v, list) else [v] for k, v in front.items()}
    got["net"] = dW
    check(got, L)


@pytest.mark.parametrize("clip", [None, 1e-3, 1e9])
def test_clipping_bounds_a_step(clip):
    t = SF.Trainer(width=128, blocks=1, depth=2, batch=4, time=64, seed=3, vocab=40, clip=clip)
    tokens = SF.make_tokens(40, 4, 64, 3)[:, :-1]
    _, target = SF.make_task(128, 4, 64, 3)
    before = t.table.clone()
    dW, front, _ = t.gradients(tokens, target)
    grads = [g.clone() for g in list(dW) + SF._flat(front)]
    norm = math.sqrt(sum(float(g.double().square().sum()) for g in grads))
    t.step(tokens, target)
    assert t.status() == 0
    if clip is None:
        assert t.norm is None
    else:
        assert abs(float(t.norm) - norm) <= 1e-6 * norm
    k = 1.0 if clip is None else min(1.0, clip / norm)
    want = before.double() - t.lr * k * front["table"].double()
    assert float((t.table.double() - want).abs().max()) <= 2.0 ** -22 * float(before.abs().max())


def test_the_commands_run(capsys, monkeypatch):
    for extra in (["--tokens", "100", "--clip", "1"], ["--inputs", "60", "--clip", "1", "--depth", "2"]):
        monkeypatch.setattr(sys, "argv", ["sequence_front", "--steps", "2", "--batch", "2", "--blocks", "1"] + extra)
        SF.main()
    out = capsys.readouterr().out
    assert out.count("step") == 4 and "nan" not in out


def test_one_captured_step_of_lookup_loss_and_clipping():
    """The table is both ends' weight; a graph of the step gives what the calls give, on new tokens too."""
    V, D, N = 500, 128, 384
    g = torch.Generator(device="cuda").manual_seed(0)
    table = (torch.randn(V, D, generator=g, device="cuda") / D ** 0.5).bfloat16()
    tokens = torch.randint(0, V, (N + 1,), generator=g, device="cuda")

    def step():
        x = mwb.embedding(tokens[:-1], table, scale=D ** 0.5)
        r = mwb.token_loss_gradient(x, table, tokens[1:].contiguous(), grad_dtype=torch.float32)
        d = mwb.embedding_backward(tokens[:-1], r.dh, V, scale=D ** 0.5, dtable=r.dweight, accumulate=True)
        norm = mwb.clip_gradients([d], 1e-2)
        return r.loss, r.total, d, norm

    step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        held = step()
    for seed in (1, 2):
        g.manual_seed(seed)
        tokens.copy_(torch.randint(-1, V, (N + 1,), generator=g, device="cuda"))
        graph.replay()
        got = [t.clone() for t in held]
        assert all(torch.equal(a, b) for a, b in zip(got, step()))
        assert abs(float(got[2].double().norm()) - 1e-2) <= 1e-6
