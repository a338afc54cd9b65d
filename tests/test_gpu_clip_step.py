"""A training step whose gradients have no finite norm changes nothing, and the next one goes on."""
import pytest
import torch

from paper_2402_14212_b200 import sequence_front as SF

pytestmark = pytest.mark.gpu


def weights(t):
    f = t.front
    out = list(f.proj) + list(f.w_post) + list(f.scale) + list(f.w_pre) + [f.w_in, t.table]
    out += list(t.proj_momentum)
    return out + ([t.w_out] if isinstance(t, SF.TokenTrainer) else list(t.params) + list(t.momentum))


@pytest.mark.parametrize("bad", [float("inf"), float("nan")])
@pytest.mark.parametrize("kind", [SF.TokenTrainer, SF.Trainer])
def test_a_step_without_a_finite_norm_is_skipped(kind, bad):
    if kind is SF.TokenTrainer:
        t, args = kind(100, 128, 1, clip=1.0, seed=2), (SF.make_tokens(100, 4, 64, 2),)
    else:
        t = kind(width=128, blocks=1, depth=2, batch=4, time=64, seed=2, vocab=100, clip=1.0)
        args = (SF.make_tokens(100, 4, 64, 2)[:, :-1], SF.make_task(128, 4, 64, 2)[1])
    t.step(*args)
    assert t.skipped == 0
    word = int(args[0][0, 0])
    row = t.table[word].clone()
    t.table[word] = bad
    before = [w.clone() for w in weights(t)]
    t.step(*args)
    assert t.skipped == 1 and not bool(torch.isfinite(t.norm))
    assert all(torch.equal(a.nan_to_num(1.0, 2.0, 3.0), b.nan_to_num(1.0, 2.0, 3.0)) for a, b in zip(weights(t), before))
    t.table[word] = row
    t.step(*args)
    assert t.skipped == 1 and all(bool(torch.isfinite(w).all()) for w in weights(t))
    assert not all(torch.equal(a, b) for a, b in zip(weights(t), before))
