"""Tunes a small LLaMA-style decoder with windowed attention and answers with it: prompts by windowed attention
into paged caches, drafted tokens checked several at a time, and an eviction when a cache has grown past its limit.

    python examples/answer.py [--tokens N]

The attention, the caches and the verification are the library's operators; linear layers without gradients are its
bf16 GEMM.  Norms, activations and the tuning's linear layers are plain torch.  Weights are random and the text to tune
on is a repeated pattern: what is shown is how the calls fit together."""
import argparse
import math
import os
import sys
import time

import torch
import torch.nn.functional as F

sys.path.insert(0, os.path.join(os.path.dirname(os.path.abspath(__file__)), ".."))
from paper_2502_19864_gb300 import ringada as R  # noqa: E402

BF16 = torch.bfloat16


def _workspace(n):
    """`n` bytes, as a size function gave them for the whole argument block; it gives 0 for one that the call would refuse."""
    if n == 0:
        raise ValueError("the argument block is refused")
    return torch.zeros(max(n, 256), dtype=torch.uint8, device="cuda")


class WindowAttention(torch.autograd.Function):
    """Causal attention with a sliding window and sinks over [batch, seq, heads, head_dim], with its gradients."""

    @staticmethod
    def forward(ctx, q, k, v, window, sinks, err):
        q, k, v = q.contiguous(), k.contiguous(), v.contiguous()
        B, S, H, D = q.shape
        out = torch.empty_like(q)
        lse = torch.empty(B, H, S, dtype=torch.float32, device="cuda")
        args = R.ra_attention_window_args(
            q_dev=q.data_ptr(), k_dev=k.data_ptr(), v_dev=v.data_ptr(), q_stride=H * D, k_stride=k.shape[2] * D,
            v_stride=v.shape[2] * D, out_dev=out.data_ptr(), out_stride=H * D, lse_dev=lse.data_ptr(),
            err_dev=err.data_ptr(), batch=B, seq=S, n_heads=H, n_kv_heads=k.shape[2], head_dim=D, window=window,
            sinks=sinks, dtype=R.RA_BF16, scale=1 / math.sqrt(D))
        R.ra_attention_window_forward(args, torch.cuda.current_stream())
        ctx.save_for_backward(q, k, v, out, lse, err)
        ctx.args = args
        return out

    @staticmethod
    def backward(ctx, dout):
        q, k, v, _, _, _ = ctx.saved_tensors  # (the argument block points at all of them)
        args, dout = ctx.args, dout.contiguous()
        dq, dk, dv = torch.empty_like(q), torch.empty_like(k), torch.empty_like(v)
        args.dout_dev, args.dout_stride = dout.data_ptr(), args.q_stride
        args.dq_dev, args.dk_dev, args.dv_dev = dq.data_ptr(), dk.data_ptr(), dv.data_ptr()
        args.dq_stride, args.dk_stride, args.dv_stride = args.q_stride, args.k_stride, args.v_stride
        ws = _workspace(R.ra_attention_window_workspace_bytes(args))
        args.workspace_dev, args.workspace_bytes = ws.data_ptr(), ws.numel()
        R.ra_attention_window_backward(args, torch.cuda.current_stream())
        return dq, dk, dv, None, None, None


def rotate(x, rope):
    """Rotate-half RoPE of [batch, seq, heads, head_dim] at positions 0, 1, ..., as the append has it."""
    c, s = rope[:x.shape[1], None].chunk(2, -1)
    lo, hi = x.float().chunk(2, -1)
    return torch.cat([lo * c - hi * s, hi * c + lo * s], -1).to(x.dtype)


def linear(x, w):
    if torch.is_grad_enabled():
        return F.linear(x, w)
    x = x.contiguous()
    y = torch.empty(*x.shape[:-1], w.shape[0], dtype=BF16, device="cuda")
    R.ra_gemm_bf16(x.data_ptr(), w.data_ptr(), y.data_ptr(), x.numel() // x.shape[-1], w.shape[0], w.shape[1],
                   stream=torch.cuda.current_stream())
    return y


def norm(x):
    return (x.float() * torch.rsqrt(x.float().square().mean(-1, keepdim=True) + 1e-6)).to(x.dtype)


class Decoder:
    """Pre-norm layers of grouped-head attention and a SiLU FFN, and a vocabulary head on the embedding."""

    def __init__(self, layers, hidden=256, heads=4, kv_heads=2, vocab=512, window=96, sinks=4, longest=2048, seed=0):
        g = torch.Generator("cuda").manual_seed(seed)
        self.H, self.KV, self.D, self.V = heads, kv_heads, hidden // heads, vocab
        self.window, self.sinks = window, sinks

        def weight(n, m):
            return (torch.randn(n, m, device="cuda", generator=g) / math.sqrt(m)).to(BF16).requires_grad_()
        self.emb = weight(vocab, hidden)
        self.layers = [dict(qkv=weight((heads + 2 * kv_heads) * self.D, hidden), o=weight(hidden, heads * self.D),
                            up=weight(4 * hidden, hidden), down=weight(hidden, 4 * hidden)) for _ in range(layers)]
        freq = 10000.0 ** (-torch.arange(0, self.D, 2, device="cuda") / self.D)
        angle = torch.arange(longest, device="cuda")[:, None] * freq
        self.rope = torch.cat([angle.cos(), angle.sin()], 1).contiguous()
        self.err = torch.zeros(1, dtype=torch.int32, device="cuda")

    def parameters(self):
        return [self.emb] + [w for layer in self.layers for w in layer.values()]

    def _rest(self, x, o, layer):
        x = x + linear(o, layer["o"])
        return x + linear(F.silu(linear(norm(x), layer["up"])), layer["down"])

    def loss(self, tokens):
        """Next-token loss of whole sequences, with gradients."""
        x = F.embedding(tokens, self.emb)
        for layer in self.layers:
            q, k, v = linear(norm(x), layer["qkv"]).unflatten(-1, (-1, self.D)).split([self.H, self.KV, self.KV], 2)
            o = WindowAttention.apply(rotate(q, self.rope), rotate(k, self.rope), v, self.window, self.sinks, self.err)
            x = self._rest(x, o.flatten(2), layer)
        logits = linear(norm(x), self.emb)[:, :-1].float()
        return F.cross_entropy(logits.flatten(0, 1), tokens[:, 1:].flatten())


class Session:
    """A decoder answering a batch of sequences: a paged cache a layer, two pools of it where it is evicted."""

    def __init__(self, model, batch, capacity, page=32, evicts=False):
        self.m, self.batch, self.page, self.evicts = model, batch, page, evicts
        self.pages = -(-capacity // page)
        n = batch * self.pages
        # (any pages will do, and in any order)
        self.table = torch.randperm(n, device="cuda").to(torch.int32).view(batch, self.pages)
        shape = (n, model.KV, page, model.D)
        self.pools = [[torch.empty(2, *shape, dtype=BF16, device="cuda") for _ in range(2 if evicts else 1)] for _ in model.layers]
        self.lens = torch.zeros(batch, dtype=torch.int32, device="cuda")  # cached tokens
        self.pos = torch.zeros(batch, dtype=torch.int32, device="cuda")   # tokens seen
        self.weights = [torch.zeros(batch, model.KV, self.pages * page, device="cuda") for _ in model.layers] if evicts else None
        self.ws = None

    def cache(self, pool):
        return R.ra_kv_cache(k_dev=pool[0].data_ptr(), v_dev=pool[1].data_ptr(), block_table_dev=self.table.data_ptr(),
                             err_dev=self.m.err.data_ptr(), n_pages=pool.shape[1], max_pages=self.pages,
                             page_size=self.page, n_kv_heads=self.m.KV, head_dim=self.m.D, dtype=R.RA_BF16)

    @torch.no_grad()
    def step(self, tokens, prompt=False):
        """Logits after each of the newest tokens [batch, n]: put into the caches, attended over them; a prompt, the
        first tokens of all, by windowed attention."""
        m, B, n, stream = self.m, self.batch, tokens.shape[1], torch.cuda.current_stream()
        self.lens += n
        self.pos += n
        width = (m.H + 2 * m.KV) * m.D
        x = F.embedding(tokens, m.emb)
        for i, layer in enumerate(m.layers):
            qkv = linear(norm(x), layer["qkv"])
            at = [qkv.data_ptr() + 2 * m.D * h for h in (0, m.H, m.H + m.KV)]
            # a prompt's keys are turned twice: into the pages, and next to the queries for its own attention
            heads = m.H + m.KV if prompt else m.H
            rot = torch.empty(B, n, heads * m.D, dtype=BF16, device="cuda")
            R.ra_kv_append(R.ra_kv_append_args(
                cache=self.cache(self.pools[i][0]), lens_dev=self.lens.data_ptr(), pos_dev=self.pos.data_ptr(), q_dev=at[0],
                k_dev=at[1], v_dev=at[2], q_out_dev=rot.data_ptr(), q_stride=width, k_stride=width, v_stride=width,
                q_out_stride=heads * m.D, rope_dev=m.rope.data_ptr(), rope_len=m.rope.shape[0], batch=B, n_new=n,
                n_heads=heads), stream)
            out = torch.empty(B, n, m.H * m.D, dtype=BF16, device="cuda")
            if prompt:
                R.ra_attention_window_forward(R.ra_attention_window_args(
                    q_dev=rot.data_ptr(), k_dev=rot.data_ptr() + 2 * m.H * m.D, v_dev=at[2], q_stride=heads * m.D,
                    k_stride=heads * m.D, v_stride=width, out_dev=out.data_ptr(), out_stride=m.H * m.D,
                    err_dev=m.err.data_ptr(), batch=B, seq=n, n_heads=m.H, n_kv_heads=m.KV, head_dim=m.D,
                    window=m.window, sinks=m.sinks, dtype=R.RA_BF16, scale=1 / math.sqrt(m.D)), stream)
            else:
                # a cache that is evicted holds what is worth seeing: all of it is seen; else the window is
                args = R.ra_attention_decode_args(
                    cache=self.cache(self.pools[i][0]), lens_dev=self.lens.data_ptr(), q_dev=rot.data_ptr(),
                    q_stride=m.H * m.D, out_dev=out.data_ptr(), out_stride=m.H * m.D, batch=B, n_new=n, n_heads=m.H,
                    window=0 if self.evicts else m.window, sinks=0 if self.evicts else m.sinks, scale=1 / math.sqrt(m.D))
                if self.evicts:
                    args.weights_in_dev = args.weights_out_dev = self.weights[i].data_ptr()
                    args.weights_stride = self.weights[i].shape[-1]
                need = R.ra_attention_decode_workspace_bytes(args)
                if self.ws is None or self.ws.numel() < need:
                    self.ws = _workspace(need)
                args.workspace_dev, args.workspace_bytes = self.ws.data_ptr(), self.ws.numel()
                R.ra_attention_decode(args, stream)
            x = m._rest(x, out, layer)
        return linear(norm(x), m.emb).float()

    def back(self, n):
        """Takes the newest n[b] tokens of each sequence back."""
        self.lens -= n
        self.pos -= n
        if self.evicts:  # (the slots are used again; what those tokens' queries added to older slots stays there)
            gone = torch.arange(self.weights[0].shape[-1], device="cuda") >= self.lens[:, None, None]
            for w in self.weights:
                w.masked_fill_(gone, 0)

    def evict(self, budget, recent):
        """Down to `budget` tokens a sequence.  (A prompt's windowed attention leaves no weights: its tokens have those that
        the tokens after it gave them, and a prompt that is evicted at once keeps its first and newest tokens and, all
        being equal, the lowest slots.)"""
        stream, lens = torch.cuda.current_stream(), torch.empty_like(self.lens)
        for i, pools in enumerate(self.pools):
            w = torch.zeros_like(self.weights[i])
            kept = torch.empty(self.batch, self.m.KV, budget, dtype=torch.int32, device="cuda")
            R.ra_kv_evict(R.ra_kv_evict_args(
                src=self.cache(pools[0]), dst=self.cache(pools[1]), lens_dev=self.lens.data_ptr(),
                weights_dev=self.weights[i].data_ptr(), weights_stride=w.shape[-1], lens_out_dev=lens.data_ptr(),
                kept_dev=kept.data_ptr(), weights_out_dev=w.data_ptr(), weights_out_stride=w.shape[-1],
                batch=self.batch, max_len=self.pages * self.page, budget=budget, first=self.m.sinks, recent=recent), stream)
            pools.reverse()
            self.weights[i] = w
        self.lens = lens


@torch.no_grad()
def answer(model, draft, prompt, tokens, n_draft=4, budget=128, limit=192, seed=0):
    """`tokens` more tokens of each sequence, sampled as `model` would, with `draft`'s proposals; how many of those stood,
    and the number of evictions.  A sequence that has all of its tokens waits for the others: what a round puts into its
    caches is taken back, so that they hold no more than its own answer."""
    B, V, stream = prompt.shape[0], model.V, torch.cuda.current_stream()
    g = torch.Generator("cuda").manual_seed(seed)
    length = prompt.shape[1] + tokens + n_draft + 1
    big = Session(model, B, max(limit, prompt.shape[1]) + 2 * n_draft + 2, evicts=True)
    small = Session(draft, B, length + n_draft)
    last = big.step(prompt, prompt=True)[:, -1].softmax(-1).multinomial(1, generator=g)
    small.step(prompt, prompt=True)
    answers = [[int(t)] for t in last[:, 0]]
    ws = None
    accepted = torch.empty(B, dtype=torch.int32, device="cuda")
    out = torch.empty(B, n_draft + 1, dtype=torch.int32, device="cuda")
    stood = drafts = evictions = 0
    while min(map(len, answers)) < tokens:
        if int(big.lens.max()) > limit:
            big.evict(budget, recent=budget // 4)
            evictions += 1
        live = [len(a) < tokens for a in answers]
        # the draft's tokens; its last step puts the last of them into its cache
        t, proposed, q = last, [], []
        for i in range(n_draft + 1):
            p = small.step(t)[:, -1].softmax(-1)
            if i < n_draft:
                t = p.multinomial(1, generator=g)
                q.append(p)
                proposed.append(t)
        proposed, q = torch.cat(proposed, 1), torch.stack(q, 1).contiguous()
        p = big.step(torch.cat([last, proposed], 1)).softmax(-1).contiguous()
        drafted = proposed.to(torch.int32).contiguous()
        uniform = torch.rand(B, n_draft, device="cuda", generator=g)
        noise = torch.empty(B, V, device="cuda").exponential_(generator=g).clamp_min_(1e-30)
        args = R.ra_verify_draft_args(
            target_dev=p.data_ptr(), target_stride=V, draft_dev=q.data_ptr(), draft_stride=V, tokens_dev=drafted.data_ptr(),
            uniform_dev=uniform.data_ptr(), noise_dev=noise.data_ptr(), accepted_dev=accepted.data_ptr(),
            out_tokens_dev=out.data_ptr(), batch=B, n_draft=n_draft, vocab=V, dtype=R.RA_F32)
        if ws is None:  # (the batch is the same every round)
            ws = _workspace(R.ra_verify_draft_workspace_bytes(args))
        args.workspace_dev, args.workspace_bytes = ws.data_ptr(), ws.numel()
        R.ra_verify_draft(args, stream)
        on = torch.tensor(live, device="cuda")
        gone = torch.where(on, n_draft - accepted, n_draft + 1)
        big.back(gone)
        small.back(gone)
        last = torch.where(on[:, None], out.gather(1, accepted[:, None].long()).long(), last)
        for b, (row, n) in enumerate(zip(out.tolist(), accepted.tolist())):
            if live[b]:
                answers[b] += row[:n + 1]
                stood += n
                drafts += n_draft
    for m in (model, draft):
        if int(m.err):
            raise RuntimeError("device error word %d" % int(m.err))
    return [a[:tokens] for a in answers], stood / max(drafts, 1), evictions


def tune(model, tokens, steps, lr=2e-3):
    """Adam on all weights; the losses."""
    master = [p.detach().float().requires_grad_() for p in model.parameters()]
    adam, losses = torch.optim.Adam(master, lr=lr), []
    for _ in range(steps):
        loss = model.loss(tokens)
        for p, w, g in zip(model.parameters(), master, torch.autograd.grad(loss, model.parameters())):
            w.grad = g.float()
        adam.step()
        with torch.no_grad():
            for p, w in zip(model.parameters(), master):
                p.copy_(w)
        losses.append(float(loss.detach()))
    return losses


def text(batch, length, vocab, seed=0):
    """A pattern of 24 tokens a sequence, over and over."""
    g = torch.Generator("cuda").manual_seed(seed)
    p = torch.randint(0, vocab, (batch, 24), device="cuda", generator=g)
    return p.repeat(1, -(-length // 24))[:, :length].contiguous()


def main():
    ap = argparse.ArgumentParser(description=__doc__.splitlines()[0])
    ap.add_argument("--tokens", type=int, default=256)
    n = ap.parse_args().tokens
    model, draft = Decoder(2, seed=1), Decoder(1, seed=2)
    data = text(8, 200, model.V)
    for name, m in (("decoder", model), ("draft", draft)):
        losses = tune(m, data, 60)
        print("%s: loss %.3f -> %.3f in %d steps" % (name, losses[0], losses[-1], len(losses)))
    answer(model, draft, data[:4, :100], 16)
    torch.cuda.synchronize()
    t0 = time.perf_counter()
    answers, stood, evictions = answer(model, draft, data[:4, :100], n)
    took = time.perf_counter() - t0
    right = sum(a == b for row, want in zip(answers, text(8, 100 + n, model.V)[:4, 100:].tolist()) for a, b in zip(row, want))
    print("%d tokens of 4 sequences in %.2f s: %.0f%% of the drafted stood, %d evictions, %.0f%% continue the pattern"
          % (n, took, 100 * stood, evictions, 100 * right / (4 * n)))


if __name__ == "__main__":
    main()
