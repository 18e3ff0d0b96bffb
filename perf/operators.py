"""What the speed of the operators that answer with a tuned decoder is measured on, through the C ABI
binding: the paged key-value cache and the attention that reads it, the cache's eviction, windowed
attention over whole sequences (a prompt, or a training step with its gradients) and the verification
of drafted tokens.

A case is one call (``"op"``; ``window`` with ``"train"`` two):

``append``  ra_kv_append: rotates the queries and keys of the new tokens and puts their keys and
            values into the pages.  Rotated queries and both caches come back.
``decode``  ra_attention_decode: attention of the newest tokens of each sequence over its pages.
            Outputs, and with ``"weights"`` the accumulated weight of every cached token.
``evict``   ra_kv_evict: the tokens with the largest accumulated weight, beside the first and the
            newest, into other pages.  What was kept, lengths, weights and both caches.
``window``  ra_attention_window_forward (outputs and log-sum-exp), and with ``"train"``
            ra_attention_window_backward (outputs and the gradients of q, k and v).
``verify``  ra_verify_draft: how many drafted tokens stand, and the tokens that come out.

Values: unit-variance keys and values, queries scaled so that attention scores have a standard
deviation of 2 (a token attends to some tokens and not to all alike), accumulated weights with the
heavy tail that they have in use and some exact zeros, softmax probabilities of logits with a standard
deviation of 4 over the vocabulary, a draft that is near its target.
"""
import math

import torch

own = False  # True: the framework's operators; False: the same in elementary torch operations

DT = {"f32": torch.float32, "bf16": torch.bfloat16}
PAGE = 16


# ---- cases --------------------------------------------------------------------------------

def _append(name, dtype, B, T, heads, kv, dh, length):
    return {"name": name, "op": "append", "dtype": dtype, "batch": B, "new": T, "heads": heads, "kv_heads": kv,
            "head_dim": dh, "len": length, "page": PAGE}


def _decode(name, dtype, B, T, heads, kv, dh, length, ragged=True, weights=False, window=0, sinks=0, page=PAGE):
    return {"name": name, "op": "decode", "dtype": dtype, "batch": B, "new": T, "heads": heads, "kv_heads": kv,
            "head_dim": dh, "len": length, "ragged": ragged, "weights": weights, "window": window, "sinks": sinks,
            "page": page}


def _evict(name, dtype, B, kv, dh, length, budget, first, recent):
    return {"name": name, "op": "evict", "dtype": dtype, "batch": B, "kv_heads": kv, "head_dim": dh, "len": length,
            "budget": budget, "first": first, "recent": recent, "page": PAGE}


def _window(name, dtype, B, S, heads, kv, dh, window, sinks, train, ragged=False):
    return {"name": name, "op": "window", "dtype": dtype, "batch": B, "seq": S, "heads": heads, "kv_heads": kv,
            "head_dim": dh, "window": window, "sinks": sinks, "train": train, "ragged": ragged}


def _verify(name, dtype, B, drafted, vocab):
    return {"name": name, "op": "verify", "dtype": dtype, "batch": B, "drafted": drafted, "vocab": vocab}


def listed():
    return [
        # one new token of one sequence of a small fp32 model: the latency of the smallest call
        _append("append_f32_b1", "f32", 1, 1, 2, 2, 64, 100),
        # the prompts of a batch, 8 x 1024 tokens of 16 heads that share 4 key-value heads
        _append("append_bf16_prompt", "bf16", 8, 1024, 16, 4, 128, 1024),
        # one new token of one sequence of a thousand, 16 heads with keys of their own: latency
        _decode("decode_bf16_b1", "bf16", 1, 1, 16, 16, 128, 1000, ragged=False),
        # a serving batch with ragged lengths to 32768 and shared heads, whose accumulated weights an
        # eviction will go by
        _decode("decode_bf16_ragged", "bf16", 16, 1, 16, 4, 128, 32768, weights=True),
        # a fp32 model checks four drafted tokens and the one before them, with a window and first
        # tokens that stay visible; head dim 96, a page size that is no power of two
        _decode("decode_f32_draft_window", "f32", 6, 5, 12, 6, 96, 3000, window=1024, sinks=4, page=24),
        # one sequence outgrows a small budget
        _evict("evict_bf16_b1", "bf16", 1, 16, 128, 700, 512, 4, 128),
        # a batch of long sequences down to a quarter
        _evict("evict_bf16_long", "bf16", 16, 4, 128, 16384, 4096, 4, 1024),
        # a training step's attention of a small fp32 model: ragged, 333 tokens, shared heads
        _window("window_f32_train", "f32", 3, 333, 4, 2, 64, 100, 2, True, ragged=True),
        # the attention of the LLaMA-style decoder at 8 x 1024 tokens, trained with a window
        _window("window_bf16_train", "bf16", 8, 1024, 16, 16, 128, 256, 4, True),
        # a long prompt of a tuned decoder with shared heads, the largest
        _window("window_bf16_prompt", "bf16", 1, 16384, 16, 4, 128, 4096, 4, False),
        # one sequence's four drafted tokens over a 32000-word vocabulary
        _verify("verify_f32_b1", "f32", 1, 4, 32000),
        # a batch with eight drafts and a vocabulary of odd size
        _verify("verify_bf16_b64", "bf16", 64, 8, 50001),
    ]


def _log(rng, lo, hi, to=1):
    """A multiple of ``to`` in [lo, hi], spread over the logarithm."""
    v = math.exp(rng.uniform(math.log(lo), math.log(hi)))
    return int(min(hi, max(lo, round(v / to) * to)))


def draw(rng):
    op = rng.choice(["append", "decode", "decode", "evict", "window", "window", "verify"])
    dtype = rng.choice(["bf16", "bf16", "f32"])
    kv, group = rng.choice([(1, 1), (2, 1), (3, 1), (16, 1), (12, 1), (4, 4), (2, 2), (6, 2), (8, 4), (1, 8), (2, 16)])
    dh = rng.choice([64, 64, 128, 128, 96, 32])
    most = max(max(w["flops"] / 250, w["bytes"]) for w in (work(c) for c in listed()))
    while True:
        if op == "append":
            c = _append("", dtype, _log(rng, 1, 64), _log(rng, 1, 2048), kv * group, kv, dh, 0)
            c["len"] = c["new"] + _log(rng, 1, 20000) - 1
        elif op == "decode":
            c = _decode("", dtype, _log(rng, 1, 128), rng.choice([1, 1, 1, 2, 5, 8]), kv * group, kv, dh,
                        _log(rng, 8, 100000), rng.random() < 0.7, rng.random() < 0.4,
                        page=rng.choice([16, 16, 32, 64, 24]))
            if rng.random() < 0.3:
                c["window"], c["sinks"] = _log(rng, 16, 8192), rng.choice([0, 1, 4, 20])
        elif op == "evict":
            c = _evict("", dtype, _log(rng, 1, 64), kv, dh, _log(rng, 64, 60000), 0, rng.choice([0, 1, 4]), 0)
            c["budget"] = _log(rng, 32, c["len"])
            c["recent"] = rng.randint(0, c["budget"] - c["first"])
        elif op == "window":
            f32 = dtype == "f32"
            c = _window("", dtype, _log(rng, 1, 16), _log(rng, 5, 1000 if f32 else 8192), kv * group, kv,
                        dh if f32 else rng.choice([64, 128]), _log(rng, 1, 4096), rng.choice([0, 1, 4, 130]),
                        rng.random() < 0.6, rng.random() < 0.4)
        else:
            c = _verify("", dtype, _log(rng, 1, 256), rng.choice([1, 2, 4, 5, 8]), _log(rng, 500, 130000))
        w = work(c)
        if op == "window":  # (the plain form holds every pair of tokens)
            if c["batch"] * c["heads"] * c["seq"] ** 2 > (1.5e9 if dtype == "bf16" else 1.2e8):
                continue
        elif w["bytes"] > (0.3e9 if op != "decode" else 1.2e9) or c["batch"] * c.get("len", 0) * kv > 4e6:
            continue
        if max(w["flops"] / 250, w["bytes"]) <= most:
            del c["name"]
            return c


# ---- inputs -------------------------------------------------------------------------------

def _lens(c, least=1):
    """The lengths of a case's sequences, spread evenly from a quarter of the longest to it."""
    B, n = c["batch"], c.get("len") or c["seq"]
    if not c.get("ragged") or B == 1:
        return [n] * B
    return [max(least, n - (3 * n // 4) * i // (B - 1)) for i in range(B)]


def _pages(c):
    return -(-c["len"] // c["page"])


def _rand(gen, shape, dtype=torch.float32, scale=1.0):
    return torch.randn(shape, generator=gen, device="cuda").mul_(scale).to(dtype)


def _table(gen, B, per):
    """A table of `per` pages for each sequence, scattered over the pool."""
    return torch.randperm(B * per, generator=gen, device="cuda").to(torch.int32).view(B, per)


def _inputs(c, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    dt, B = DT[c["dtype"]], c["batch"]
    ints = lambda v: torch.tensor(v, dtype=torch.int32, device="cuda")  # noqa: E731
    s = {}
    if c["op"] == "verify":
        K, V = c["drafted"], c["vocab"]
        z = _rand(gen, (B, K + 1, V), scale=4.0)
        s["target"] = z.softmax(-1).to(dt)
        s["draft"] = (z[:, :K] + _rand(gen, (B, K, V), scale=0.7)).softmax(-1).to(dt)
        race = torch.empty((B, K, V), device="cuda").exponential_(generator=gen)
        s["tokens"] = (s["draft"].float() / race).argmax(-1).to(torch.int32)
        s["uniform"] = torch.rand((B, K), generator=gen, device="cuda")
        s["noise"] = torch.empty((B, V), device="cuda").exponential_(generator=gen).clamp_(min=1e-30)
        return s
    if c["op"] == "window":
        S, h, kv, dh = c["seq"], c["heads"], c["kv_heads"], c["head_dim"]
        s["q"] = _rand(gen, (B, S, h, dh), dt, 2.0)
        s["k"], s["v"] = (_rand(gen, (B, S, kv, dh), dt) for _ in "kv")
        if c["train"]:
            s["dout"] = _rand(gen, (B, S, h, dh), dt, 1e-2)
        order = torch.randperm(B, generator=gen, device="cuda")
        s["lens"] = ints(_lens(c))[order]
        return s
    kv, dh, page, per = c["kv_heads"], c["head_dim"], c["page"], _pages(c)
    pool = (B * per, kv, page, dh)
    s["table"] = _table(gen, B, per)
    if c["op"] == "append":
        T, h = c["new"], c["heads"]
        # queries, keys and values side by side, as the fused projection leaves them
        s["qkv"] = _rand(gen, (B, T, (h + 2 * kv) * dh), dt)
        s["k_pages"], s["v_pages"] = (torch.zeros(pool, dtype=dt, device="cuda") for _ in "kv")
        s["lens"] = torch.randint(T, c["len"] + 1, (B,), generator=gen, device="cuda", dtype=torch.int32)
        at = torch.arange(c["len"], device="cuda", dtype=torch.float64)[:, None] * (
            10000.0 ** (-torch.arange(dh // 2, device="cuda", dtype=torch.float64) * 2 / dh))
        s["rope"] = torch.cat([at.cos(), at.sin()], -1).float()
        return s
    s["k_pages"], s["v_pages"] = (_rand(gen, pool, dt) for _ in "kv")
    s["lens"] = ints(_lens(c, c.get("new", 1)))[torch.randperm(B, generator=gen, device="cuda")]
    n = per * page
    if c["op"] == "decode":
        s["q"] = _rand(gen, (B, c["new"], c["heads"], dh), dt, 2.0)
    if c["op"] == "evict" or c["weights"]:
        w = torch.randn((B, kv, n), generator=gen, device="cuda").mul_(2).exp_()
        s["weights"] = w * (torch.rand((B, kv, n), generator=gen, device="cuda") > 0.05)
    if c["op"] == "evict":
        s["out_table"] = _table(gen, B, -(-c["budget"] // page))
    return s


def _outputs(c, s):
    """The buffers that a user's program keeps for the outputs."""
    dt, B = DT[c["dtype"]], c["batch"]
    new = lambda shape, t=dt: torch.zeros(shape, dtype=t, device="cuda")  # noqa: E731
    if c["op"] == "append":
        return {"q": new((B, c["new"], c["heads"], c["head_dim"])), "k_pages": s["k_pages"], "v_pages": s["v_pages"]}
    if c["op"] == "decode":
        o = {"out": new((B, c["new"], c["heads"], c["head_dim"]))}
        if c["weights"]:
            o["weights"] = s["weights"].clone()
        return o
    if c["op"] == "evict":
        kv, page, n = c["kv_heads"], c["page"], -(-c["budget"] // c["page"])
        pool = (B * n, kv, page, c["head_dim"])
        return {"kept": new((B, kv, c["budget"]), torch.int32), "lens": new((B,), torch.int32),
                "weights": new((B, kv, n * page), torch.float32), "k_pages": new(pool), "v_pages": new(pool)}
    if c["op"] == "window":
        S, h, kv, dh = c["seq"], c["heads"], c["kv_heads"], c["head_dim"]
        o = {"out": new((B, S, h, dh)), "lse": new((B, h, S), torch.float32)}
        if c["train"]:
            o.update(dq=new((B, S, h, dh)), dk=new((B, S, kv, dh)), dv=new((B, S, kv, dh)))
        return o
    return {"accepted": new((B,), torch.int32), "tokens": new((B, c["drafted"] + 1), torch.int32)}


def prepare(case, seed):
    s = _inputs(case, seed)
    s["case"], s["outputs"] = case, _outputs(case, s)
    if own:  # the argument block, with its workspace, that a program fills in once for its buffers
        s["call"] = _call(case, s)
    return s


def _returned(c, o):
    """lse is a step's own value between its two calls, and an answer where there is one call."""
    return {k: v for k, v in o.items() if not (k == "lse" and c["train"])}


# ---- the framework's operators ------------------------------------------------------------

def _call(c, s):
    from paper_2502_19864_gb300 import ringada as R
    o, B = s["outputs"], c["batch"]
    at = lambda t: t.data_ptr()  # noqa: E731
    dt = {"f32": R.RA_F32, "bf16": R.RA_BF16}[c["dtype"]]

    def cache(table, k, v):
        return R.ra_kv_cache(k_dev=at(k), v_dev=at(v), block_table_dev=at(table), n_pages=k.shape[0],
                             max_pages=table.shape[1], page_size=c["page"], n_kv_heads=c["kv_heads"],
                             head_dim=c["head_dim"], dtype=dt)

    if c["op"] == "append":
        h, kv, dh, T = c["heads"], c["kv_heads"], c["head_dim"], c["new"]
        row, es = (h + 2 * kv) * dh, s["qkv"].element_size()
        a = R.ra_kv_append_args(
            cache=cache(s["table"], s["k_pages"], s["v_pages"]), lens_dev=at(s["lens"]), q_dev=at(s["qkv"]),
            k_dev=at(s["qkv"]) + h * dh * es, v_dev=at(s["qkv"]) + (h + kv) * dh * es, q_stride=row, k_stride=row,
            v_stride=row, q_out_dev=at(o["q"]), q_out_stride=h * dh, rope_dev=at(s["rope"]),
            rope_len=s["rope"].shape[0], batch=B, n_new=T, n_heads=h)
        return R.ra_kv_append, (a,)
    if c["op"] == "decode":
        a = R.ra_attention_decode_args(
            cache=cache(s["table"], s["k_pages"], s["v_pages"]), lens_dev=at(s["lens"]), q_dev=at(s["q"]),
            q_stride=c["heads"] * c["head_dim"], out_dev=at(o["out"]), out_stride=c["heads"] * c["head_dim"], batch=B,
            n_new=c["new"], n_heads=c["heads"], max_len=c["len"], window=c["window"], sinks=c["sinks"],
            scale=c["head_dim"] ** -0.5)
        if c["weights"]:
            a.weights_in_dev, a.weights_out_dev = at(s["weights"]), at(o["weights"])
            a.weights_stride = s["weights"].shape[-1]
        _workspace(s, a, R.ra_attention_decode_workspace_bytes(a))
        return R.ra_attention_decode, (a,)
    if c["op"] == "evict":
        a = R.ra_kv_evict_args(
            src=cache(s["table"], s["k_pages"], s["v_pages"]), dst=cache(s["out_table"], o["k_pages"], o["v_pages"]),
            lens_dev=at(s["lens"]), weights_dev=at(s["weights"]), weights_stride=s["weights"].shape[-1],
            lens_out_dev=at(o["lens"]), kept_dev=at(o["kept"]), weights_out_dev=at(o["weights"]),
            weights_out_stride=o["weights"].shape[-1], batch=B, max_len=c["len"], budget=c["budget"],
            first=c["first"], recent=c["recent"])
        return R.ra_kv_evict, (a,)
    if c["op"] == "window":
        h, kv, dh = c["heads"], c["kv_heads"], c["head_dim"]
        a = R.ra_attention_window_args(
            q_dev=at(s["q"]), k_dev=at(s["k"]), v_dev=at(s["v"]), q_stride=h * dh, k_stride=kv * dh, v_stride=kv * dh,
            out_dev=at(o["out"]), out_stride=h * dh, lse_dev=at(o["lse"]), lens_dev=at(s["lens"]), batch=B,
            seq=c["seq"], n_heads=h, n_kv_heads=kv, head_dim=dh, window=c["window"], sinks=c["sinks"], dtype=dt,
            scale=dh ** -0.5)
        if not c["train"]:
            return R.ra_attention_window_forward, (a,)
        a.dout_dev, a.dout_stride = at(s["dout"]), h * dh
        a.dq_dev, a.dk_dev, a.dv_dev = at(o["dq"]), at(o["dk"]), at(o["dv"])
        a.dq_stride, a.dk_stride, a.dv_stride = h * dh, kv * dh, kv * dh
        _workspace(s, a, R.ra_attention_window_workspace_bytes(a))
        return _train_step, (R, a)
    a = R.ra_verify_draft_args(
        target_dev=at(s["target"]), draft_dev=at(s["draft"]), target_stride=c["vocab"], draft_stride=c["vocab"],
        tokens_dev=at(s["tokens"]), uniform_dev=at(s["uniform"]), noise_dev=at(s["noise"]),
        accepted_dev=at(o["accepted"]), out_tokens_dev=at(o["tokens"]), batch=B, n_draft=c["drafted"],
        vocab=c["vocab"], dtype=dt)
    _workspace(s, a, R.ra_verify_draft_workspace_bytes(a))
    return R.ra_verify_draft, (a,)


def _workspace(s, a, n):
    s["workspace"] = torch.zeros(max(n, 256), dtype=torch.uint8, device="cuda")
    a.workspace_dev, a.workspace_bytes = s["workspace"].data_ptr(), n


def _train_step(R, a):
    R.ra_attention_window_forward(a)
    R.ra_attention_window_backward(a)


def run(state):
    if own:
        call, arguments = state["call"]
        call(*arguments)
        return _returned(state["case"], state["outputs"])
    return _returned(state["case"], {"append": _plain_append, "decode": _plain_decode, "evict": _plain_evict,
                                     "window": _plain_window, "verify": _plain_verify}[state["case"]["op"]](
        state["case"], state))


# ---- the plain forms, in 32 bits ----------------------------------------------------------

def _turn(x, cos, sin):
    lo, hi = x.chunk(2, -1)
    return torch.cat([lo * cos - hi * sin, hi * cos + lo * sin], -1)


def _plain_append(c, s):
    B, T, h, kv, dh, page = (c[n] for n in ("batch", "new", "heads", "kv_heads", "head_dim", "page"))
    dt = DT[c["dtype"]]
    q, k, v = s["qkv"].view(B, T, h + 2 * kv, dh).split([h, kv, kv], 2)
    slot = s["lens"].long()[:, None] - T + torch.arange(T, device="cuda")
    cos, sin = s["rope"][slot][:, :, None].chunk(2, -1)
    at = s["table"].gather(1, slot // page).long()
    s["k_pages"][at, :, slot % page] = _turn(k.float(), cos, sin).to(dt)
    s["v_pages"][at, :, slot % page] = v
    return {"q": _turn(q.float(), cos, sin).to(dt), "k_pages": s["k_pages"], "v_pages": s["v_pages"]}


def _cached(pages, table):
    """[B, kv heads, slots, head dim] of a paged cache, in 32 bits."""
    return pages[table.long()].float().transpose(1, 2).flatten(2, 3)


def _seen(query, key, window, sinks):
    """Whether the token at `query` sees the one at `key`."""
    ok = key <= query
    return ok & ((query - key < window) | (key < sinks)) if window else ok


def _plain_decode(c, s):
    B, T, h, kv, dh = (c[n] for n in ("batch", "new", "heads", "kv_heads", "head_dim"))
    g = h // kv
    k, v = _cached(s["k_pages"], s["table"]), _cached(s["v_pages"], s["table"])
    n = k.shape[2]
    q = s["q"].float().view(B, T, kv, g, dh).permute(0, 2, 1, 3, 4).reshape(B, kv, T * g, dh)
    query = s["lens"].long()[:, None] - T + torch.arange(T, device="cuda")
    seen = _seen(query[:, :, None], torch.arange(n, device="cuda"), c["window"], c["sinks"])
    seen = seen[:, None, :, None].expand(B, 1, T, g, n).reshape(B, 1, T * g, n)
    p = (q @ k.transpose(2, 3) * dh ** -0.5).masked_fill(~seen, -math.inf)
    p = (p - p.amax(-1, keepdim=True)).exp()
    p = p / p.sum(-1, keepdim=True)
    out = (p @ v).view(B, kv, T, g, dh).permute(0, 2, 1, 3, 4).reshape(B, T, h, dh)
    got = {"out": out.to(DT[c["dtype"]])}
    if c["weights"]:
        got["weights"] = s["weights"] + p.sum(2)
    return got


def _plain_evict(c, s):
    B, kv, page, budget, first, recent = (c[n] for n in ("batch", "kv_heads", "page", "budget", "first", "recent"))
    lens = s["lens"].long()
    slot = torch.arange(s["weights"].shape[-1], device="cuda")
    length = lens[:, None, None]
    always = (slot < first) | (slot >= length - recent)
    # the heaviest of those between, of equal ones the lowest: a stable sort, falling
    rank = s["weights"].masked_fill(always, math.inf).masked_fill(slot >= length, -math.inf)
    order = rank.sort(dim=-1, descending=True, stable=True).indices[..., :budget]
    n = lens.clamp(max=budget)
    live = torch.arange(budget, device="cuda") < n[:, None, None]
    kept = order.masked_fill(~live, slot.numel()).sort(-1).values
    from_slot = kept.clamp(max=slot.numel() - 1)
    out = dict(s["outputs"])
    out["kept"] = kept.masked_fill(~live, -1).to(torch.int32)
    out["lens"] = n.to(torch.int32)
    out["weights"][..., :budget] = s["weights"].gather(2, from_slot).masked_fill(~live, 0.0)
    head = torch.arange(kv, device="cuda")[None, :, None]
    page_of = s["table"].long()[torch.arange(B, device="cuda")[:, None, None], from_slot // page]
    to = torch.arange(budget, device="cuda").expand(B, kv, budget)
    to_page = s["out_table"].long()[torch.arange(B, device="cuda")[:, None, None], to // page]
    mark = live.expand(B, kv, budget)[..., None]
    out["k_pages"][to_page, head, to % page] = s["k_pages"][page_of, head, from_slot % page] * mark
    out["v_pages"][to_page, head, to % page] = s["v_pages"][page_of, head, from_slot % page] * mark
    return out


def _plain_window(c, s):
    B, S, h, kv, dh = (c[n] for n in ("batch", "seq", "heads", "kv_heads", "head_dim"))
    g, scale, dt = h // kv, dh ** -0.5, DT[c["dtype"]]
    q = s["q"].float().view(B, S, kv, g, dh).permute(0, 2, 3, 1, 4)
    k, v = (s[n].float().permute(0, 2, 1, 3)[:, :, None] for n in "kv")
    at, live = torch.arange(S, device="cuda"), torch.arange(S, device="cuda") < s["lens"][:, None]
    seen = _seen(at[:, None], at, c["window"], c["sinks"]) & live[:, :, None]
    p = (q @ k.transpose(3, 4)).mul_(scale).masked_fill_(~seen[:, None, None], -math.inf)
    top = p.amax(-1, keepdim=True).clamp(min=-1e30)
    p = p.sub_(top).exp_()
    total = p.sum(-1, keepdim=True)
    p = p.div_(total.clamp(min=1e-30))
    o = p @ v
    heads = lambda t: t.permute(0, 3, 1, 2, 4).reshape(B, S, -1, dh).to(dt)  # noqa: E731
    got = {"out": heads(o)}
    if not c["train"]:
        got["lse"] = (top + total.log()).view(B, h, S)
        return got
    do = s["dout"].float().view(B, S, kv, g, dh).permute(0, 2, 3, 1, 4)
    ds = (do @ v.transpose(3, 4)).sub_((do * o).sum(-1, keepdim=True)).mul_(p)
    got["dq"] = heads(ds @ k * scale)
    got["dk"] = heads((ds.transpose(3, 4) @ q).sum(2, keepdim=True) * scale)
    got["dv"] = heads((p.transpose(3, 4) @ do).sum(2, keepdim=True))
    return got


def _plain_verify(c, s):
    B, K = c["batch"], c["drafted"]
    target, draft, tokens = s["target"], s["draft"], s["tokens"].long()
    p = target[:, :K].gather(2, tokens[..., None])[..., 0].float()
    q = draft.gather(2, tokens[..., None])[..., 0].float()
    stands = (s["uniform"] * q < p).long().cumprod(1)
    n = stands.sum(1)
    row = torch.arange(B, device="cuda")
    p = target[row, n].float()
    q = draft[row, n.clamp(max=K - 1)].float() * (n < K)[:, None]
    r = (p - q).clamp(min=0)
    r = torch.where((r > 0).any(-1, keepdim=True), r, p)
    last = (r / s["noise"]).argmax(-1)
    at = torch.arange(K + 1, device="cuda")
    padded = torch.cat([tokens, tokens.new_zeros(B, 1)], 1)
    out = torch.where(at < n[:, None], padded, torch.where(at == n[:, None], last[:, None], -1))
    return {"accepted": n.to(torch.int32), "tokens": out.to(torch.int32)}


# ---- the work of a call -------------------------------------------------------------------

def _visible(length, new, window, sinks):
    """Pairs of one of the `new` newest of `length` tokens and a token that it sees."""
    if not window:
        return new * length - new * (new - 1) // 2
    total = 0
    for i in range(length - new, length):
        inside = min(i + 1, window)
        total += inside + min(sinks, i + 1 - inside)
    return total


def work(case):
    c, es, B = case, {"f32": 4, "bf16": 2}[case["dtype"]], case["batch"]
    if c["op"] == "verify":
        return {"bytes": B * (c["vocab"] * (2 * es + 4) + c["drafted"] * (2 * es + 8) + 4 * c["drafted"] + 8),
                "flops": 3 * B * c["vocab"]}
    kv, dh = c["kv_heads"], c["head_dim"]
    if c["op"] == "append":
        rows = B * c["new"]
        return {"bytes": rows * dh * (es * 2 * (c["heads"] + 2 * kv) + 4), "flops": 3 * rows * dh * (c["heads"] + kv)}
    lens = _lens(c, c.get("new", 1))
    if c["op"] == "evict":
        kept = sum(min(n, c["budget"]) for n in lens)
        return {"bytes": kv * (4 * sum(lens) + kept * (4 * dh * es + 8)) + 8 * B, "flops": kv * sum(lens)}
    h = c["heads"]
    if c["op"] == "decode":
        T = c["new"]
        pairs = sum(_visible(n, T, c["window"], c["sinks"]) for n in lens)
        far = c["window"] + T - 1
        tokens = sum(n if not c["window"] or n <= far else far + min(c["sinks"], n - far) for n in lens)
        b = es * (2 * kv * dh * tokens + 2 * B * T * h * dh)
        return {"bytes": b + (8 * kv * sum(lens) if c["weights"] else 0), "flops": 4 * h * dh * pairs}
    S = c["seq"]
    pairs = sum(_visible(n, n, c["window"], c["sinks"]) for n in lens)
    b = es * B * S * dh * (2 * h + 2 * kv)
    if c["train"]:
        return {"bytes": b + es * B * S * dh * (3 * h + 4 * kv), "flops": 14 * h * dh * pairs}
    return {"bytes": b + 4 * B * S * h, "flops": 4 * h * dh * pairs}


# ---- the same in 64 bits ------------------------------------------------------------------

def _softmax_rows(scores, allowed):
    """Softmax of each row over its allowed places (all zero where there are none), and log-sum-exp."""
    scores = torch.where(allowed, scores, torch.full_like(scores, -math.inf))
    lse = torch.logsumexp(scores, -1, keepdim=True)
    return torch.where(allowed, torch.exp(scores - torch.nan_to_num(lse, neginf=0.0)), torch.zeros_like(scores)), lse[..., 0]


def _allowed(first, n_query, n_key, c, length=None):
    """[n_query, n_key]: which keys the queries at first, first + 1, ... see."""
    i = first + torch.arange(n_query, device="cuda").unsqueeze(1)
    j = torch.arange(n_key, device="cuda").unsqueeze(0)
    ok = j.le(i)
    if c["window"] > 0:
        ok = ok.logical_and(j.gt(i - c["window"]).logical_or(j.lt(c["sinks"])))
    if length is not None:
        ok = ok.logical_and(i.lt(length))
    return ok


def _exact_append(c, s):
    dh, h, kv, T, page = c["head_dim"], c["heads"], c["kv_heads"], c["new"], c["page"]
    x = s["qkv"].double().view(c["batch"], T, -1, dh)
    pos = (s["lens"].long().unsqueeze(1) - T) + torch.arange(T, device="cuda")
    z = torch.view_as_complex(torch.stack(s["rope"].double()[pos].chunk(2, -1), -1)).unsqueeze(2)
    pairs = torch.complex(x[..., : h + kv, : dh // 2], x[..., : h + kv, dh // 2:]) * z
    turned = torch.cat([pairs.real, pairs.imag], -1)
    got = {"q": turned[:, :, :h]}
    for name, rows in (("k_pages", turned[:, :, h:]), ("v_pages", x[:, :, h + kv:])):
        pool = torch.zeros_like(s[name], dtype=torch.float64)
        for b in range(c["batch"]):
            pool[s["table"][b].long()[pos[b] // page], :, pos[b] % page] = rows[b]
        got[name] = pool
    return got


def _exact_decode(c, s):
    T, h, kv, dh = c["new"], c["heads"], c["kv_heads"], c["head_dim"]
    out = torch.zeros((c["batch"], T, h, dh), dtype=torch.float64, device="cuda")
    weights = s["weights"].double() if c["weights"] else None
    for b, n in enumerate(s["lens"].tolist()):
        pages = s["table"][b].long()
        k, v = (s[x][pages].permute(1, 0, 2, 3).reshape(kv, -1, dh)[:, :n].double() for x in ("k_pages", "v_pages"))
        ok = _allowed(n - T, T, n, c)
        for head in range(h):
            p, _ = _softmax_rows(s["q"][b, :, head].double() @ k[head * kv // h].T / math.sqrt(dh), ok)
            out[b, :, head] = p @ v[head * kv // h]
            if weights is not None:
                weights[b, head * kv // h, :n] += p.sum(0)
    return {"out": out, "weights": weights} if c["weights"] else {"out": out}


def _exact_evict(c, s):
    got = {k: (t.double() if t.is_floating_point() else t) for k, t in _outputs(c, s).items()}
    page, budget = c["page"], c["budget"]
    got["kept"].fill_(-1)
    for b, n in enumerate(s["lens"].tolist()):
        m = min(n, budget)
        got["lens"][b] = m
        for head in range(c["kv_heads"]):
            w = s["weights"][b, head, :n]
            keep = torch.ones(n, dtype=torch.bool, device="cuda")
            if n > budget:
                middle = w[c["first"]: n - c["recent"]]
                room = budget - c["first"] - c["recent"]
                chosen = torch.zeros_like(middle, dtype=torch.bool)
                if room > 0:
                    edge = torch.topk(middle, room).values[-1]
                    chosen = middle > edge
                    equal = torch.nonzero(middle == edge)[:, 0]
                    chosen[equal[: room - int(chosen.sum())]] = True
                keep[c["first"]: n - c["recent"]] = chosen
            slots = torch.nonzero(keep)[:, 0]
            got["kept"][b, head, :m] = slots.int()
            got["weights"][b, head, :m] = w[slots].double()
            to = torch.arange(m, device="cuda")
            src, dst = s["table"][b].long()[slots // page], s["out_table"][b].long()[to // page]
            for x in ("k_pages", "v_pages"):
                got[x][dst, head, to % page] = s[x][src, head, slots % page].double()
    return got


def _exact_window(c, s):
    B, S, h, kv, dh = c["batch"], c["seq"], c["heads"], c["kv_heads"], c["head_dim"]
    zeros = lambda n: torch.zeros((B, S, n, dh), dtype=torch.float64, device="cuda")  # noqa: E731
    got = {"out": zeros(h)}
    if c["train"]:
        got.update(dq=zeros(h), dk=zeros(kv), dv=zeros(kv))
    else:
        got["lse"] = torch.zeros((B, h, S), dtype=torch.float64, device="cuda")
    for b, n in enumerate(s["lens"].tolist()):
        ok = _allowed(0, S, S, c, n)
        for head in range(h):
            e = head * kv // h
            q, k, v = s["q"][b, :, head].double(), s["k"][b, :, e].double(), s["v"][b, :, e].double()
            p, lse = _softmax_rows(q @ k.T / math.sqrt(dh), ok)
            got["out"][b, :, head] = p @ v
            if not c["train"]:
                got["lse"][b, head] = lse
                continue
            do = s["dout"][b, :, head].double()
            dp = do @ v.T
            ds = p * (dp - (p * dp).sum(-1, keepdim=True)) / math.sqrt(dh)
            got["dq"][b, :, head] = ds @ k
            got["dk"][b, :, e] += ds.T @ q
            got["dv"][b, :, e] += p.T @ do
    return got


def _exact_verify(c, s):
    K = c["drafted"]
    accepted, out = [], []
    for b in range(c["batch"]):
        p, q = s["target"][b].double(), s["draft"][b].double()
        row, n = s["tokens"][b].tolist(), 0
        while n < K and float(s["uniform"][b, n].double() * q[n, row[n]]) < float(p[n, row[n]]):
            n += 1
        left = p[n] if n == K else torch.relu(p[n] - q[n])
        if float(left.max()) <= 0.0:
            left = p[n]
        token = int(torch.argmax(left / s["noise"][b].double()))
        accepted.append(n)
        out.append(row[:n] + [token] + [-1] * (K - n))
    return {"accepted": torch.tensor(accepted, dtype=torch.int32, device="cuda"),
            "tokens": torch.tensor(out, dtype=torch.int32, device="cuda")}


def exact(case, seed):
    s = _inputs(case, seed)
    if case["op"] == "window" and case["batch"] * case["heads"] * case["seq"] ** 2 * case["head_dim"] > 1e12:
        return None  # (the longest prompt would take over 20 seconds in 64 bits)
    return {"append": _exact_append, "decode": _exact_decode, "evict": _exact_evict, "window": _exact_window,
            "verify": _exact_verify}[case["op"]](case, s)
