"""Trains all of a small LLaMA-style decoder's weights with the library's operators: RMSNorm with the residual's sum and its gain's
gradient, windowed attention, the loss over the vocabulary straight from hidden states, and updates of the layers'
matrices orthogonalised by Newton-Schulz products (the embedding and the gains by Adam).

    python examples/train.py [--steps N]

Linear layers, SiLU and Adam are plain torch.  Weights are random and the text to train on is a repeated pattern: what is
shown is how the calls fit together."""
import argparse
import math
import os
import sys

import torch
import torch.nn.functional as F

sys.path.insert(0, os.path.dirname(os.path.abspath(__file__)))
from answer import BF16, R, WindowAttention, _workspace, rotate, text  # noqa: E402

EPS = 1e-6


class Norm(torch.autograd.Function):
    """RMSNorm of x + residual over the last dimension, and that sum: (y, sum)."""

    @staticmethod
    def forward(ctx, x, residual, gamma):
        x, residual = x.contiguous(), residual.contiguous()
        H = x.shape[-1]
        rows = x.numel() // H
        y, total = torch.empty_like(x), torch.empty_like(x)
        rstd = torch.empty(rows, device="cuda")
        args = R.ra_norm_args(x_dev=x.data_ptr(), x_stride=H, residual_dev=residual.data_ptr(), residual_stride=H,
                              sum_dev=total.data_ptr(), sum_stride=H, gamma_dev=gamma.data_ptr(), y_dev=y.data_ptr(), y_stride=H,
                              rstd_dev=rstd.data_ptr(), rows=rows, hidden=H, kind=R.RA_NORM_RMS, dtype=R.RA_BF16,
                              w_dtype=R.RA_F32, eps=EPS)
        R.ra_norm_forward(args, torch.cuda.current_stream())
        ctx.save_for_backward(total, gamma, rstd)
        ctx.args = args
        return y, total

    @staticmethod
    def backward(ctx, dy, dtotal):
        total, gamma, _ = ctx.saved_tensors  # (the backward reads the sum, not what it is of)
        args, dy, dtotal = ctx.args, dy.contiguous(), dtotal.contiguous()
        dx, dgamma = torch.empty_like(total), torch.empty_like(gamma)
        args.dy_dev, args.dy_stride, args.dsum_dev, args.dsum_stride = dy.data_ptr(), args.hidden, dtotal.data_ptr(), args.hidden
        args.dx_dev, args.dx_stride, args.dgamma_dev = dx.data_ptr(), args.hidden, dgamma.data_ptr()
        ws = _workspace(R.ra_norm_workspace_bytes(args))
        args.workspace_dev, args.workspace_bytes = ws.data_ptr(), ws.numel()
        R.ra_norm_backward(args, torch.cuda.current_stream())
        return dx, dx, dgamma


class VocabLoss(torch.autograd.Function):
    """The loss of each token of x [tokens, hidden] under softmax(x w^T); 0 for those of a negative label."""

    @staticmethod
    def forward(ctx, x, w, labels, err):
        x, w = x.contiguous(), w.contiguous()
        loss, lse = (torch.empty(x.shape[0], device="cuda") for _ in "ab")
        args = R.ra_vocab_loss_args(x_dev=x.data_ptr(), x_stride=x.shape[1], w_dev=w.data_ptr(), w_stride=w.shape[1],
                                    labels_dev=labels.data_ptr(), loss_dev=loss.data_ptr(), lse_dev=lse.data_ptr(),
                                    err_dev=err.data_ptr(), tokens=x.shape[0], vocab=w.shape[0], hidden=x.shape[1],
                                    dtype=R.RA_BF16)
        ws = _workspace(R.ra_vocab_loss_workspace_bytes(args))
        args.workspace_dev, args.workspace_bytes = ws.data_ptr(), ws.numel()
        R.ra_vocab_loss_forward(args, torch.cuda.current_stream())
        ctx.save_for_backward(x, w, labels, lse, err)
        ctx.args = args
        return loss

    @staticmethod
    def backward(ctx, dloss):
        x, w, _, _, _ = ctx.saved_tensors
        args, dloss = ctx.args, dloss.contiguous()
        dx, dw = torch.empty_like(x), torch.empty_like(w)
        args.dloss_dev = dloss.data_ptr()
        args.dx_dev, args.dx_stride, args.dw_dev, args.dw_stride = dx.data_ptr(), x.shape[1], dw.data_ptr(), w.shape[1]
        ws = _workspace(R.ra_vocab_loss_workspace_bytes(args))  # (larger, now that there are gradients to write)
        args.workspace_dev, args.workspace_bytes = ws.data_ptr(), ws.numel()
        R.ra_vocab_loss_backward(args, torch.cuda.current_stream())
        return dx, dw, None, None


def orthogonalize(x, err, steps=5, coefficients=(3.4445, -4.775, 2.0315)):
    """Matrices [n, rows, cols] (fp32 or bf16) with their singular values brought to about 1."""
    n, rows, cols = x.shape
    out = torch.empty_like(x)
    a, b, c = coefficients
    args = R.ra_orthogonalize_args(x_dev=x.data_ptr(), x_stride=cols, x_matrix_stride=rows * cols, out_dev=out.data_ptr(),
                                   out_stride=cols, out_matrix_stride=rows * cols, err_dev=err.data_ptr(), n_matrices=n,
                                   rows=rows, cols=cols, steps=steps, dtype=R.RA_BF16 if x.dtype == BF16 else R.RA_F32,
                                   a=a, b=b, c=c, eps=1e-7)
    ws = _workspace(R.ra_orthogonalize_workspace_bytes(args))
    args.workspace_dev, args.workspace_bytes = ws.data_ptr(), ws.numel()
    R.ra_orthogonalize(args, torch.cuda.current_stream())
    return out


class Muon:
    """Momentum, orthogonalised, for the layers' matrices; those of one shape in one call."""

    def __init__(self, matrices, lr, err, momentum=0.9):
        self.lr, self.err, self.momentum, self.groups = lr, err, momentum, {}
        for w in matrices:
            self.groups.setdefault(tuple(w.shape), []).append(w)
        self.state = {k: torch.zeros(len(ws), *k, device="cuda") for k, ws in self.groups.items()}

    @torch.no_grad()
    def step(self):
        for shape, ws in self.groups.items():
            g = torch.stack([w.grad for w in ws]).float()
            m = self.state[shape].mul_(self.momentum).add_(g)
            update = orthogonalize((g + self.momentum * m).to(BF16), self.err)
            # (so that an update's elements are of the same size whatever the shape)
            scale = self.lr * math.sqrt(max(shape))
            for w, u in zip(ws, update):
                w.sub_(scale * u.to(w.dtype))


class Decoder:
    """Pre-norm layers of grouped-head windowed attention and a SiLU FFN, and a vocabulary head on the embedding."""

    def __init__(self, layers, hidden=256, heads=4, kv_heads=2, vocab=512, window=96, sinks=4, longest=2048, seed=0):
        g = torch.Generator("cuda").manual_seed(seed)
        self.H, self.KV, self.D, self.V, self.window, self.sinks = heads, kv_heads, hidden // heads, vocab, window, sinks

        def weight(n, m):
            return (torch.randn(n, m, device="cuda", generator=g) / math.sqrt(m)).to(BF16).requires_grad_()

        def gain():
            return torch.ones(hidden, device="cuda").requires_grad_()
        self.emb, self.last = weight(vocab, hidden), gain()
        self.layers = [dict(qkv=weight((heads + 2 * kv_heads) * self.D, hidden), o=weight(hidden, heads * self.D),
                            up=weight(4 * hidden, hidden), down=weight(hidden, 4 * hidden), before=gain(), between=gain())
                       for _ in range(layers)]
        freq = 10000.0 ** (-torch.arange(0, self.D, 2, device="cuda") / self.D)
        angle = torch.arange(longest, device="cuda")[:, None] * freq
        self.rope = torch.cat([angle.cos(), angle.sin()], 1).contiguous()
        self.err = torch.zeros(1, dtype=torch.int32, device="cuda")

    def matrices(self):
        return [layer[n] for layer in self.layers for n in ("qkv", "o", "up", "down")]

    def others(self):
        return [self.emb, self.last] + [layer[n] for layer in self.layers for n in ("before", "between")]

    def loss(self, tokens, labels):
        """The mean loss of the counted labels (int32, those below 0 are not) of whole sequences, with gradients."""
        x = F.embedding(tokens, self.emb)
        stream = torch.zeros_like(x)  # the residual stream; x is what the last block adds to it
        for layer in self.layers:
            y, stream = Norm.apply(x, stream, layer["before"])
            q, k, v = F.linear(y, layer["qkv"]).unflatten(-1, (-1, self.D)).split([self.H, self.KV, self.KV], 2)
            o = WindowAttention.apply(rotate(q, self.rope), rotate(k, self.rope), v, self.window, self.sinks, self.err)
            y, stream = Norm.apply(F.linear(o.flatten(2), layer["o"]), stream, layer["between"])
            x = F.linear(F.silu(F.linear(y, layer["up"])), layer["down"])
        y, _ = Norm.apply(x, stream, self.last)
        loss = VocabLoss.apply(y.flatten(0, 1), self.emb, labels.flatten().contiguous(), self.err)
        return loss.sum() / (labels >= 0).sum()


def next_tokens(tokens):
    """Labels: the token that follows; none for a sequence's last."""
    return torch.cat([tokens[:, 1:], torch.full_like(tokens[:, :1], -1)], 1).to(torch.int32)


def train(model, tokens, steps, lr=0.02):
    labels = next_tokens(tokens)
    muon = Muon(model.matrices(), lr / 16, model.err)
    adam = torch.optim.Adam(model.others(), lr=1e-3)
    losses = []
    for _ in range(steps):
        for w in model.matrices() + model.others():
            w.grad = None
        loss = model.loss(tokens, labels)
        loss.backward()
        muon.step()
        adam.step()
        losses.append(loss.detach())
    return [float(v) for v in losses]


def main():
    ap = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    ap.add_argument("--steps", type=int, default=40)
    a = ap.parse_args()
    model = Decoder(2)
    losses = train(model, text(4, 200, model.V), a.steps)
    print("loss %.3f -> %.3f in %d steps" % (losses[0], losses[-1], a.steps))
    if int(model.err):
        raise SystemExit("the device reported %d" % int(model.err))


if __name__ == "__main__":
    main()
