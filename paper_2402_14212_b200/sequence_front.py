"""A stack of recurrent blocks in front of a Moonwalk net, trained with the orthogonalised update.

`python -m paper_2402_14212_b200.sequence_front` trains it on a synthetic sequence task and prints the loss; with
`--inputs V` its inputs are tokens of a vocabulary of V, with `--tokens V` the stack alone learns to say the next token.

Block (x: residual stream [batch * time, width], n: its normed copy):

    (v, f, z) = n Wp^T           one product, three windows of its rows
    h         = gated_scan(v, f)
    x', n'    = residual_norm(x, h, gate z): x' = x + s silu(z) rmsnorm(h; w_post), n' = rmsnorm(x'; w_pre)

The net behind it sees every position as a sample.  Its `mw_input_cotangent` gives g0 = dL/dx_0, which is the
cotangent of the stack's output: the blocks' backward calls carry it on from there, while the net's forward
sweep forms its own gradients.  Products, recurrence, norms, the net and the updates of its weights and of the projections
run in the library; torch holds the memory, adds the fixed bias of f, puts dz beside dv and df, and takes the plain
gradient steps of the per-channel weights.

Tokens enter through rows of a table (embedding); a token model ends in the vocabulary's loss over the same table
(token_loss_gradient), whose gradient takes that of the lookup on top.  clip bounds the norm of all gradients of a step
together (clip_gradients); where that is not finite there is no step.
"""
from __future__ import annotations

import argparse
import math

from . import binding as mwb
from . import synth as S

TERMS = 2          # operand terms of the projections' products


class SequenceFront:
    """Weights of `blocks` recurrent blocks of one width (a multiple of 64), float32."""

    def __init__(self, width: int, blocks: int, seed: int = 0, device="cuda"):
        import torch
        g = torch.Generator(device="cpu").manual_seed(seed)
        self.width = width

        def normal(*shape, std):
            return (torch.randn(*shape, generator=g) * std).to(device)

        self.proj = [normal(3 * width, width, std=1.0 / math.sqrt(width)) for _ in range(blocks)]
        for w in self.proj:                     # memories of a few to a few dozen steps
            w[width:2 * width] *= 0.5
        self.bias = torch.linspace(0.0, 3.0, width, device=device)      # of f: fixed decay rates per channel
        self.w_in = torch.ones(width, device=device)
        self.w_post = [torch.ones(width, device=device) for _ in range(blocks)]
        self.scale = [torch.full((width,), 0.5, device=device) for _ in range(blocks)]
        self.w_pre = [torch.ones(width, device=device) for _ in range(blocks - 1)]

    def forward(self, x):
        """x [batch, time, width] -> (the stream after the last block, what backward() needs)."""
        B, T, D = x.shape
        x = x.reshape(B * T, D)
        _, n, rms = mwb.residual_norm(x, w_pre=self.w_in, keep_rms=True)
        tape = {"x": x, "rms_in": rms, "shape": (B, T), "blocks": []}
        for i, w in enumerate(self.proj):
            p = mwb.gemm_split_bf16(n, w, False, False, TERMS)
            p[:, D:2 * D] += self.bias
            seq = p.view(B, T, 3 * D)
            h, _, states = mwb.gated_scan(seq[:, :, :D], seq[:, :, D:2 * D], keep_states=True)
            h = h.view(B * T, D)
            w_pre = self.w_pre[i] if i < len(self.w_pre) else None
            out, n_next, rms = mwb.residual_norm(x, h, z=p[:, 2 * D:], w_post=self.w_post[i], scale=self.scale[i],
                                                 w_pre=w_pre, keep_rms=True)
            tape["blocks"].append((x, n, p, h, states, rms))
            x, n = out, n_next
        return x, tape

    def backward(self, g, tape):
        """g = dL/d(stream after the last block) -> (dL/dx, gradients by name of the weight lists)."""
        import torch
        B, T = tape["shape"]
        D = self.width
        grads = {k: [None] * len(self.proj) for k in ("proj", "w_post", "scale")}
        grads["w_pre"] = [None] * len(self.w_pre)
        dn = None
        for i in reversed(range(len(self.proj))):
            x, n, p, h, states, rms = tape["blocks"][i]
            w_pre = self.w_pre[i] if i < len(self.w_pre) else None
            r = mwb.residual_norm_backward(x, h, rms, z=p[:, 2 * D:], w_post=self.w_post[i], scale=self.scale[i],
                                           w_pre=w_pre, dx_out=g, dn=dn)
            grads["w_post"][i], grads["scale"][i] = r.dw_post, r.dscale
            if w_pre is not None:
                grads["w_pre"][i] = r.dw_pre
            dp = torch.empty_like(p)
            seq, dseq = p.view(B, T, 3 * D), dp.view(B, T, 3 * D)
            mwb.gated_scan_backward(seq[:, :, :D], seq[:, :, D:2 * D], r.db.view(B, T, D), states,
                                    dv=dseq[:, :, :D], df=dseq[:, :, D:2 * D])
            dp[:, 2 * D:] = r.dz
            grads["proj"][i] = mwb.gemm_split_bf16(dp, n, True, True, TERMS)
            dn = mwb.gemm_split_bf16(dp, self.proj[i], False, True, TERMS)
            g = r.dx
        r = mwb.residual_norm_backward(tape["x"], None, tape["rms_in"], w_pre=self.w_in, dx_out=g, dn=dn)
        grads["w_in"] = r.dw_pre
        return r.dx.view(B, T, D), grads


def _table(vocab, width, seed):
    import torch
    g = torch.Generator(device="cpu").manual_seed(seed + 1000)
    return (torch.randn(vocab, width, generator=g) / math.sqrt(width)).cuda()


def _flat(grads):
    """All tensors of a dict of gradients, lists among them."""
    return [t for g in grads.values() for t in (g if isinstance(g, list) else [g])]


class Clipping:
    """The bound of a step's gradients: `clip` (None: none), the last step's `norm`, how many steps were `skipped`."""

    def __init__(self, clip):
        self.clip, self.norm, self.skipped = clip, None, 0

    def _clipped(self, grads):
        """Clips them; whether they are to be applied.  A norm that is not finite bounds nothing: such a step, which the
        host waits for, changes no weight and no momentum."""
        if self.clip is None:
            return True
        self.norm = mwb.clip_gradients(grads, self.clip)
        if math.isfinite(float(self.norm)):
            return True
        self.skipped += 1
        return False


class Trainer(Clipping):
    """The stack, a dense Moonwalk net behind it, and their updates.  With `vocab` the inputs are tokens (of negative
    ones a row is zero); with `clip` the gradients of a step are scaled together to that norm at most, and steps whose
    norm is not finite are skipped."""

    def __init__(self, width=128, blocks=2, depth=3, batch=8, time=64, lr=2e-3, seed=0, vocab=None, clip=None):
        import torch
        super().__init__(clip)
        self.table = None if vocab is None else _table(vocab, width, seed)
        self.front = SequenceFront(width, blocks, seed)
        problem = S.deep_mlp(seed=seed, depth=depth, n=width, batch=batch * time, reseed_every=2)
        self.net = mwb.net_for(problem, backend="tensor")
        self.params, _, _ = mwb.to_device(problem)
        self.ws = self.net.alloc_workspace("moonwalk")
        self.loss = torch.zeros(1, dtype=torch.float64, device="cuda")
        self.lr = lr
        # every square weight of the net in one plan, the projections in another
        self.orth = mwb.Orth(width, width, depth, "f32")
        self.orth_proj = mwb.Orth(3 * width, width, blocks, "f32")
        self.orth_ws, self.orth_proj_ws = self.orth.alloc_workspace(), self.orth_proj.alloc_workspace()
        self.momentum = [torch.zeros_like(w) for w in self.params]
        self.proj_momentum = [torch.zeros_like(w) for w in self.front.proj]
        self.stepped = False

    def gradients(self, x, target):
        """(gradients of the net's weights, of the stack's, dL/dx); the loss lands in self.loss.  Of tokens x the
        table's gradient is among the stack's, and dL/dx is that of their rows."""
        tokens, scale = x, math.sqrt(self.front.width)
        if self.table is not None:
            x = mwb.embedding(tokens, self.table, scale=scale)
        x0, tape = self.front.forward(x)
        x0 = x0.contiguous()
        g0 = self.net.input_cotangent(self.params, x0, target, self.ws, loss_out=self.loss)
        dx, front = self.front.backward(g0, tape)
        if self.table is not None:
            front["table"] = mwb.embedding_backward(tokens, dx, self.table.shape[0], scale=scale)
        dW = self.net.forward_sweep(self.params, x0, g0, self.ws)
        return dW, front, dx

    def step(self, x, target):
        dW, front, _ = self.gradients(x, target)
        if not self._clipped(list(dW) + _flat(front)):
            return self.loss
        # orthogonalised updates move every direction of a weight alike, so the net's weights stay near a
        # multiple of an orthogonal matrix, where its inverse converges
        self.orth.step(self.params, dW, self.momentum, self.orth_ws, lr=self.lr)
        self.orth_proj.step(self.front.proj, front["proj"], self.proj_momentum, self.orth_proj_ws, lr=4 * self.lr)
        self.stepped = True
        for name in ("w_post", "scale", "w_pre"):
            for w, g in zip(getattr(self.front, name), front[name]):
                w.sub_(g, alpha=self.lr)
        self.front.w_in.sub_(front["w_in"], alpha=self.lr)
        if self.table is not None:
            self.table.sub_(front["table"], alpha=self.lr)
        return self.loss

    def status(self) -> int:
        """First device-side error of the last step (0: none)."""
        code = self.net.last_device_status(self.ws)[0]
        if code == 0 and self.stepped:
            code = self.orth.status(self.orth_ws) or self.orth_proj.status(self.orth_proj_ws)
        return code


class TokenTrainer(Clipping):
    """A token model of the stack alone: rows of a table, the blocks, a last norm, the vocabulary's loss by the same
    table; each position says the token after it.  Negative tokens are padding: they are no input and no target."""

    def __init__(self, vocab=1000, width=128, blocks=2, lr=2e-3, clip=1.0, seed=0):
        import torch
        self.front = SequenceFront(width, blocks, seed)
        self.table = _table(vocab, width, seed)
        self.w_out = torch.ones(width, device="cuda")
        super().__init__(clip)
        self.lr = lr
        self.orth_proj = mwb.Orth(3 * width, width, blocks, "f32")
        self.orth_proj_ws = self.orth_proj.alloc_workspace()
        self.proj_momentum = [torch.zeros_like(w) for w in self.front.proj]

    def _states(self, tokens):
        x = mwb.embedding(tokens, self.table, scale=math.sqrt(self.front.width))
        s, tape = self.front.forward(x)
        _, n, rms = mwb.residual_norm(s, w_pre=self.w_out, keep_rms=True)
        return s, n, rms, tape

    def losses(self, tokens):
        """TokenLoss of tokens [batch, time + 1], a loss for each of the [batch * time] positions."""
        _, n, _, _ = self._states(tokens[:, :-1])
        return mwb.token_loss(n, self.table, tokens[:, 1:].reshape(-1))

    def gradients(self, tokens):
        """(TokenLoss, gradients by name) of tokens [batch, time + 1]."""
        inputs, targets = tokens[:, :-1], tokens[:, 1:].reshape(-1)
        s, n, rms, tape = self._states(inputs)
        r = mwb.token_loss_gradient(n, self.table, targets)
        g = mwb.residual_norm_backward(s, None, rms, w_pre=self.w_out, dn=r.dh)
        dx, grads = self.front.backward(g.dx, tape)
        grads["w_out"] = g.dw_pre
        grads["table"] = mwb.embedding_backward(inputs, dx, self.table.shape[0], scale=math.sqrt(self.front.width),
                                                dtable=r.dweight, accumulate=True)
        return r, grads

    def step(self, tokens):
        """One update, unless the gradients' norm is not finite; returns the mean loss of the positions that have a target."""
        r, grads = self.gradients(tokens)
        if not self._clipped(_flat(grads)):
            return r.total
        f = self.front
        self.orth_proj.step(f.proj, grads["proj"], self.proj_momentum, self.orth_proj_ws, lr=4 * self.lr)
        for name in ("w_post", "scale", "w_pre"):
            for w, g in zip(getattr(f, name), grads[name]):
                w.sub_(g, alpha=self.lr)
        f.w_in.sub_(grads["w_in"], alpha=self.lr)
        self.w_out.sub_(grads["w_out"], alpha=self.lr)
        self.table.sub_(grads["table"], alpha=50 * self.lr)
        return r.total


def make_tokens(vocab, batch, time, seed):
    """Token sequences [batch, time + 1] that a fixed table of successors drives, one step in eight at random; the last
    sequence is padded from its middle on."""
    import torch
    g = torch.Generator(device="cpu").manual_seed(seed + 200)
    after = torch.randperm(vocab, generator=g)
    t = torch.empty(batch, time + 1, dtype=torch.int64)
    t[:, 0] = torch.randint(0, vocab, (batch,), generator=g)
    for i in range(1, time + 1):
        any_, pick = torch.randint(0, vocab, (batch,), generator=g), torch.rand(batch, generator=g) < 0.125
        t[:, i] = torch.where(pick, any_, after[t[:, i - 1]])
    t[-1, time // 2:] = -1
    return t.cuda()


def make_task(width, batch, time, seed):
    """Inputs, and targets that need memory: a leaky average of past inputs, turned by a fixed rotation."""
    import torch
    g = torch.Generator(device="cpu").manual_seed(seed + 100)
    x = torch.randn(batch, time, width, generator=g)
    q, _ = torch.linalg.qr(torch.randn(width, width, generator=g))
    y, state = torch.empty_like(x), torch.zeros(batch, width)
    for t in range(time):
        state = 0.8 * state + 0.6 * x[:, t]
        y[:, t] = state @ q
    return x.cuda(), y.reshape(batch * time, width).cuda()


def main():
    ap = argparse.ArgumentParser(description=__doc__.splitlines()[0])
    ap.add_argument("--width", type=int, default=128)
    ap.add_argument("--blocks", type=int, default=2)
    ap.add_argument("--depth", type=int, default=3)
    ap.add_argument("--batch", type=int, default=8)
    ap.add_argument("--time", type=int, default=64)
    ap.add_argument("--steps", type=int, default=60)
    ap.add_argument("--lr", type=float, default=2e-3)
    ap.add_argument("--inputs", type=int, default=0, metavar="V", help="inputs are tokens of a vocabulary of V")
    ap.add_argument("--tokens", type=int, default=0, metavar="V", help="the stack alone says the next of V tokens")
    ap.add_argument("--clip", type=float, default=None, help="bound of the gradients' norm")
    a = ap.parse_args()
    if a.tokens:
        t = TokenTrainer(a.tokens, a.width, a.blocks, a.lr, a.clip)
        tokens = make_tokens(a.tokens, a.batch, a.time, 0)
        for i in range(a.steps):
            loss = float(t.step(tokens))
            if i % 10 == 0 or i == a.steps - 1:
                print(f"step {i:4d}  loss {loss:.5f}" + (f"  norm {float(t.norm):.3f}" if a.clip is not None else ""))
        return
    t = Trainer(a.width, a.blocks, a.depth, a.batch, a.time, a.lr, vocab=a.inputs or None, clip=a.clip)
    x, target = make_task(a.width, a.batch, a.time, 0)
    if a.inputs:
        x = make_tokens(a.inputs, a.batch, a.time, 0)[:, :-1]
    for i in range(a.steps):
        loss = float(t.step(x, target).item())
        if i % 10 == 0 or i == a.steps - 1:
            print(f"step {i:4d}  loss {loss:.5f}  status {t.status()}")


if __name__ == "__main__":
    main()
