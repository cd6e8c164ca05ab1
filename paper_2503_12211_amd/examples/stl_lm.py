"""A small language model whose linear maps are STL layers, trained through the library end to end: residual steps between its blocks
(`stl_residual_norm_forward` / `_backward`) and the loss over its vocabulary (`stl_vocab_loss_backward`), from labels and from the stored
top logits of a dense teacher, the logits formed for a chunk of the tokens at a time.

The three `torch.autograd.Function`s here marshal arguments, as `stl_linear.py` does; PyTorch supplies device memory, the embedding's rows, the mixing
of neighbouring tokens, the autograd graph and the optimiser.

    model = STLLanguageModel(vocab=1000, width=256, hidden=512, blocks=2).cuda()
    loss = model.loss(tokens, labels, top_id, top_logit)      # labels -100: none; top_id -1: no entry
    loss.backward()

    python -m paper_2503_12211_amd.examples.stl_lm --steps 200
"""
from __future__ import annotations

import argparse

import torch
from torch.autograd.function import once_differentiable

import paper_2503_12211_amd as stl

from .stl_linear import _DT, STLLinear, _scratch


def _like(name, t, shape, dtype, X):
    """The library reads plain pointers: a tensor of another type or size, or on another device, would be read as what it is not."""
    if t.dtype != dtype:
        raise TypeError(f"{name} is {t.dtype}, not {dtype}")
    if tuple(t.shape) != tuple(shape) or t.device != X.device:
        raise ValueError(f"{name} of {tuple(t.shape)} on {t.device}, not {tuple(shape)} on {X.device}")


def _states(X):
    if X.dtype not in _DT:
        raise TypeError(f"X is {X.dtype}: float32 or bfloat16")
    if X.dim() != 2:
        raise ValueError(f"X of {tuple(X.shape)}: rows and columns")
    return X.shape


class _ResidualNorm(torch.autograd.Function):
    @staticmethod
    def forward(ctx, X, H, gate, w_post, w_pre, scale, flags):
        X, H, gate, w_post, w_pre = (t.contiguous() for t in (X, H, gate, w_post, w_pre))
        rows, n = X.shape
        prob = stl.ResidualProblem(rows, n, max(1, -(-rows // gate.shape[0])), 1.0, scale, 1e-6, _DT[X.dtype])
        Xout, Z = torch.empty_like(X), torch.empty_like(X)
        stl.stl_residual_norm_forward(prob, X, H, gate, w_post, None, w_pre, None, Xout, Z, flags)
        ctx.prob, ctx.flags = prob, flags
        ctx.save_for_backward(Xout, H, gate, w_post, w_pre)
        return Xout, Z

    @staticmethod
    @once_differentiable
    def backward(ctx, dXout, dZ):
        Xout, H, gate, w_post, w_pre = ctx.saved_tensors
        dXout, dZ = dXout.contiguous(), dZ.contiguous()
        dX, dH = torch.empty_like(Xout), torch.empty_like(Xout)
        # (without rows there is no row of the gate that the library would write)
        sums = [(torch.empty if ctx.prob.rows else torch.zeros)(t.shape, dtype=torch.float32, device=t.device) for t in (gate, w_post, w_pre)]
        nbytes = stl.stl_residual_norm_workspace_bytes(ctx.prob, ctx.flags)
        stl.stl_residual_norm_backward(ctx.prob, Xout, H, gate, w_post, None, w_pre, dXout, dZ, dX, dH, sums[0], sums[1], None, sums[2], None, 0,
                                       _scratch(nbytes, Xout.device), nbytes, ctx.flags)
        return dX, dH, sums[0].to(gate.dtype), sums[1].to(w_post.dtype), sums[2].to(w_pre.dtype), None, None


def residual_norm(X, H, gate, w_post, w_pre, scale=1.0, center=False):
    """(X + scale gate * norm(H) w_post, norm of that times w_pre) for X, H (rows, n), gate (groups of rows, n); differentiable in the five tensors.  The
    groups have ceil(rows / groups) rows each, the last one what is left, which has to be some."""
    rows, n = _states(X)
    groups = gate.shape[0]
    for name, t, shape in (("H", H, (rows, n)), ("gate", gate, (groups, n)), ("w_post", w_post, (n,)), ("w_pre", w_pre, (n,))):
        _like(name, t, shape, X.dtype, X)
    if groups < 1 or rows and -(-rows // -(-rows // groups)) != groups:
        raise ValueError(f"{rows} rows in groups of {-(-rows // max(groups, 1))} do not take {groups} rows of the gate")
    flags = stl.STL_FLAG_POST_NORM | stl.STL_FLAG_PRE_NORM | (stl.STL_FLAG_CENTER if center else 0)
    return _ResidualNorm.apply(X, H, gate, w_post, w_pre, scale, flags)


class _VocabLoss(torch.autograd.Function):
    @staticmethod
    def forward(ctx, X, W, label, top_id, top_logit, label_weight, top_weight, temperature, want_x, want_w):
        X, W, label, top_id, top_logit = (None if t is None else t.contiguous() for t in (X, W, label, top_id, top_logit))
        rows, d = X.shape
        ntop = 0 if top_id is None else top_id.shape[1]
        prob = stl.VocabProblem(rows, d, W.shape[0], ntop, temperature, _DT[X.dtype])
        losses = [torch.empty(rows, dtype=torch.float32, device=X.device) if t is not None else None for t in (label, top_id)]
        inputs = (prob, X, W, label, top_id, top_logit)
        train = want_x or want_w
        nbytes = stl.stl_vocab_loss_workspace_bytes(prob, stl.STL_OP_BACKWARD if train else stl.STL_OP_FORWARD)
        ws = _scratch(nbytes, X.device)
        if train:
            # the row weights are known here: losses and gradients come from one call, which forms the logits once (a factor that comes later, such as that of
            # a scaled loss, is multiplied into the rounded gradients)
            dX, dW = torch.empty_like(X) if want_x else None, torch.empty_like(W) if want_w else None
            stl.stl_vocab_loss_backward(*inputs, label_weight, top_weight, *losses, dX, dW, ws, nbytes)
            ctx.save_for_backward(dX, dW)
        else:
            stl.stl_vocab_loss_forward(*inputs, *losses, ws, nbytes)
        total = X.new_zeros((), dtype=torch.float32)
        for loss, weight in zip(losses, (label_weight, top_weight)):
            if loss is not None:
                total = total + (loss * weight).sum()
        return total

    @staticmethod
    @once_differentiable
    def backward(ctx, upstream):
        dX, dW = ctx.saved_tensors
        # (in fp32: the factor rounded to bf16 would be an error that all gradients have in common)
        scaled = lambda t: None if t is None else (t.float() * upstream).to(t.dtype)  # noqa: E731
        return scaled(dX), scaled(dW), *[None] * 8


def vocab_loss(X, W, label=None, top_id=None, top_logit=None, temperature=1.0, distill=1.0):
    """Mean cross entropy of the rows with a label, plus `distill` times the mean divergence from the teacher's top logits over the rows; X (rows, d), W
    (vocab, d), label (rows,) int64, top_id and top_logit (rows, ntop) int64 and float32.  Differentiable in X and W."""
    rows, d = _states(X)
    _like("W", W, (W.shape[0], d), X.dtype, X)
    label_weight = top_weight = None
    if (top_id is None) != (top_logit is None):
        raise ValueError("top_id and top_logit go together")
    if top_id is not None:
        _like("top_id", top_id, (rows, top_id.shape[-1]), torch.int64, X)
        _like("top_logit", top_logit, top_id.shape, torch.float32, X)
    if label is not None:
        _like("label", label, (rows,), torch.int64, X)
        has = (label >= 0) & (label < W.shape[0])
        label_weight = (has / has.sum().clamp_min(1)).float()
    if top_id is not None:
        top_weight = torch.full((rows,), distill / max(rows, 1), dtype=torch.float32, device=X.device)
    # (asked here: the function's own needs_input_grad is set for a parameter under no_grad too)
    want = [torch.is_grad_enabled() and t.requires_grad for t in (X, W)]
    return _VocabLoss.apply(X, W, label, top_id, top_logit, label_weight, top_weight, temperature, *want)


class STLLanguageModel(torch.nn.Module):
    """tokens (batch, length) -> hidden states, through `blocks` blocks of two STL layers with a GELU between; a block sees each token beside the one
    before it (a token's own past of one step: enough for a language of pairs, and all that this example needs of attention).  The four rows of an STL tile
    see each other, so they must not be neighbours in time, or a token is told what follows it: rows go by position first, and a tile holds four
    sequences at one position (batch a multiple of 4)."""

    def __init__(self, vocab: int, width: int, hidden: int, blocks: int, rank: int = 32, dtype=torch.bfloat16, seed: int = 0):
        super().__init__()
        g = torch.Generator().manual_seed(seed)
        self.embed = torch.nn.Parameter((torch.randn((vocab, width), generator=g)).to(dtype))
        self.head = torch.nn.Parameter((torch.randn((vocab, width), generator=g) * width ** -0.5).to(dtype))
        self.up = torch.nn.ModuleList(STLLinear(2 * width, hidden, rank, dtype, seed + 2 * i + 1) for i in range(blocks))
        self.down = torch.nn.ModuleList(STLLinear(hidden, width, rank, dtype, seed + 2 * i + 2) for i in range(blocks))
        ones = lambda value: torch.nn.ParameterList(torch.nn.Parameter(torch.full((width,), value, dtype=dtype)) for _ in range(blocks))  # noqa: E731
        self.post, self.pre, self.gate = ones(1.0), ones(1.0), torch.nn.ParameterList(torch.nn.Parameter(torch.full((1, width), 0.5, dtype=dtype))
                                                                                     for _ in range(blocks))

    def hidden_states(self, tokens):
        batch, length = tokens.shape
        if batch % 4:
            raise ValueError("the batch must be a multiple of the tile size 4")
        stream = self.embed[tokens.t().reshape(-1)]
        z = stream
        for up, down, post, pre, gate in zip(self.up, self.down, self.post, self.pre, self.gate):
            before = torch.nn.functional.pad(z, (0, 0, batch, 0))[:-batch]
            h = torch.nn.functional.gelu(up(torch.cat([z, before], -1)))
            stream, z = residual_norm(stream, down(h), gate, post, pre)
        return z                                             # (length * batch, width)

    def loss(self, tokens, labels, top_id=None, top_logit=None, temperature=2.0, distill=0.5):
        z = self.hidden_states(tokens)
        rows = lambda t: None if t is None else t.transpose(0, 1).reshape(z.shape[0], *t.shape[2:]).contiguous()  # noqa: E731
        return vocab_loss(z, self.head, rows(labels), rows(top_id), rows(top_logit), temperature, distill)


def language(vocab: int, ntop: int, seed: int):
    """A table of pairs: after token v one of `ntop` tokens follows, with the given logits (what a teacher that knows the language would store)."""
    g = torch.Generator().manual_seed(seed)
    ids = torch.stack([torch.randperm(vocab, generator=g)[:ntop] for _ in range(vocab)])
    logits = torch.randn((vocab, ntop), generator=g).mul(2.0).sort(1, descending=True).values.contiguous()
    return ids.cuda(), logits.cuda()


def train(steps: int = 200, batch: int = 16, length: int = 64, vocab: int = 1000, width: int = 256, hidden: int = 512, blocks: int = 2, distill: float = 0.5,
          lr: float = 3e-3, seed: int = 0, log_every: int = 0):
    """Returns the label losses of every step on tokens that the model has not seen (before the step's update), and the entropy of what followed those
    tokens, below which no model's expected loss can be."""
    ids, logits = language(vocab, 8, seed)
    p = torch.softmax(logits, 1)
    entropy_of = -(p * p.log()).sum(1)
    g = torch.Generator(device="cuda").manual_seed(seed + 1)
    model = STLLanguageModel(vocab, width, hidden, blocks, seed=seed).cuda()
    opt = torch.optim.Adam(model.parameters(), lr=lr)
    history, entropy = [], []
    for step in range(steps):
        tokens = torch.empty((batch, length + 1), dtype=torch.int64, device="cuda")
        tokens[:, 0] = torch.randint(0, vocab, (batch,), generator=g, device="cuda")
        for t in range(length):
            pick = torch.multinomial(p[tokens[:, t]], 1, generator=g)
            tokens[:, t + 1] = ids[tokens[:, t]].gather(1, pick)[:, 0]
        x, y = tokens[:, :-1], tokens[:, 1:].clone()
        y[:, : length // 8] = -100                           # a prompt: nothing is learned from it but what the teacher says
        opt.zero_grad()
        loss = model.loss(x, y, ids[x], logits[x], 1.0, distill)
        loss.backward()
        with torch.no_grad():
            history.append(float(vocab_loss(model.hidden_states(x), model.head, y.t().reshape(-1))))
            entropy.append(float(entropy_of[x][y >= 0].mean()))
        opt.step()
        if log_every and step % log_every == 0:
            print(f"  step {step:4d}  cross entropy {history[-1]:.3f}  (entropy of what follows {entropy[-1]:.3f})", flush=True)
    return history, entropy


def main():
    ap = argparse.ArgumentParser()
    ap.add_argument("--steps", type=int, default=200)
    ap.add_argument("--width", type=int, default=256)
    ap.add_argument("--vocab", type=int, default=1000)
    ap.add_argument("--distill", type=float, default=0.5)
    args = ap.parse_args()
    history, entropy = train(args.steps, width=args.width, vocab=args.vocab, distill=args.distill, log_every=max(1, args.steps // 10))
    print(f"cross entropy {history[0]:.3f} -> {history[-1]:.3f}; the entropy of what follows is {entropy[-1]:.3f}")


if __name__ == "__main__":
    main()
