"""ra_kv_append and ra_kv_evict against plain implementations: what is only moved is equal, what is turned by RoPE
is within one rounding of the type (a product sum of two terms: |x c| + |y s| times 2^-23 for fp32, and 2^-8 more of
the result for bf16)."""
import math

import pytest
import torch

import operator_helpers as H
from paper_2502_19864_gb300 import ringada as R

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def built():
    import __graft_entry__
    __graft_entry__.build()


def rope_table(n, dh):
    at = torch.arange(n, dtype=torch.float64)[:, None] * 10000.0 ** (-torch.arange(dh // 2, dtype=torch.float64) * 2 / dh)
    return torch.cat([at.cos(), at.sin()], -1).float().cuda()


def turned(x, rope, pos):
    """64-bit rotation of [n, heads, dh] by the rows `pos` of the table, and its bound for fp32."""
    x = x.double()
    lo, hi = x.chunk(2, -1)
    c, s = (t[:, None] for t in rope.double()[pos].chunk(2, -1))
    size = torch.cat([lo.abs() * c.abs() + hi.abs() * s.abs(), hi.abs() * c.abs() + lo.abs() * s.abs()], -1)
    return torch.cat([lo * c - hi * s, hi * c + lo * s], -1), size * 2.0 ** -23


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("B,new,heads,kv,dh,page", [(1, 1, 2, 2, 64, 16), (3, 5, 8, 2, 128, 16), (2, 40, 16, 16, 128, 24),
                                                    (5, 1, 3, 1, 40, 7), (2, 3, 32, 4, 256, 64), (4, 130, 4, 4, 96, 1),
                                                    (2, 9, 1, 1, 8, 16)])
@pytest.mark.parametrize("positions", [False, True])
@pytest.mark.parametrize("fused", [False, True])
def test_append(dtype, B, new, heads, kv, dh, page, positions, fused):
    g = torch.Generator(device="cuda").manual_seed(1)
    dt = H.DT[dtype]
    rand = lambda *s: torch.randn(s, generator=g, device="cuda").to(dt)  # noqa: E731
    per = -(-(new + 50) // page)
    pools = [torch.full((B * per, kv, page, dh), 9.0, dtype=dt, device="cuda") for _ in "kv"]
    table = torch.randperm(B * per, generator=g, device="cuda").to(torch.int32).view(B, per)
    lens = torch.randint(0, new + 50, (B,), generator=g, device="cuda", dtype=torch.int32)  # some below `new`: padding
    lens[0] = new
    pos = lens + 11 if positions else None
    rope = rope_table(new + 70, dh)
    n = B * new
    if fused:
        buf = rand(n, (heads + 2 * kv) * dh)
        q, k, v = (t.reshape(n, -1, dh).clone() for t in buf.split([heads * dh, kv * dh, kv * dh], 1))
        ptr, es, row = buf.data_ptr(), buf.element_size(), buf.shape[1]
        where = dict(q_dev=ptr, k_dev=ptr + heads * dh * es, v_dev=ptr + (heads + kv) * dh * es, q_stride=row,
                     k_stride=row, v_stride=row, q_out_dev=ptr, q_out_stride=row)  # rotated in place
        q_out = buf[:, :heads * dh].unflatten(1, (heads, dh))
    else:
        q, k, v = rand(n, heads, dh), rand(n, kv, dh), rand(n, kv, dh)
        q_out = torch.full_like(q, 5.0)
        where = dict(q_dev=q.data_ptr(), k_dev=k.data_ptr(), v_dev=v.data_ptr(), q_stride=heads * dh, k_stride=kv * dh,
                     v_stride=kv * dh, q_out_dev=q_out.data_ptr(), q_out_stride=heads * dh)
    err = torch.zeros(1, dtype=torch.int32, device="cuda")
    a = R.ra_kv_append_args(cache=H.cache(*pools, table, err), lens_dev=lens.data_ptr(),
                            pos_dev=pos.data_ptr() if positions else None, rope_dev=rope.data_ptr(),
                            rope_len=rope.shape[0], batch=B, n_new=new, n_heads=heads, **where)
    R.ra_kv_append(a)
    torch.cuda.synchronize()
    e16 = H.E if dtype == "bf16" else 0.0
    want = [p.clone().fill_(9.0) for p in pools]
    for b in range(B):
        t = torch.arange(new, device="cuda")
        slot = int(lens[b]) - new + t
        live = slot >= 0
        p = ((int(pos[b]) if positions else int(lens[b])) - new + t).clamp(min=0)
        rows = b * new + t
        ref, tol = turned(q[rows], rope, p)
        got = q_out[rows].double()
        assert ((got - ref).abs() <= tol + e16 * ref.abs())[live].all()
        assert (got[~live] == 0).all()
        at, off = table[b].long()[slot[live] // page], slot[live] % page
        ref, tol = turned(k[rows], rope, p)
        got = pools[0][at, :, off].double()
        assert ((got - ref[live]).abs() <= tol[live] + e16 * ref[live].abs()).all()
        assert torch.equal(pools[1][at, :, off], v[rows][live])
        want[0][at, :, off] = pools[0][at, :, off]
        want[1][at, :, off] = v[rows][live]
    assert torch.equal(pools[0], want[0]) and torch.equal(pools[1], want[1])  # nothing else was written
    assert err.item() == 0


def test_append_without_rope_and_queries():
    k, v = (torch.randn(6, 2, 64, device="cuda") for _ in "kv")
    pools = [torch.zeros(4, 2, 16, 64, device="cuda") for _ in "kv"]
    table = torch.tensor([[2, 0], [1, 3]], dtype=torch.int32, device="cuda")
    lens = torch.tensor([18, 3], dtype=torch.int32, device="cuda")
    a = R.ra_kv_append_args(cache=H.cache(*pools, table), lens_dev=lens.data_ptr(), k_dev=k.data_ptr(), v_dev=v.data_ptr(),
                            k_stride=128, v_stride=128, batch=2, n_new=3)
    R.ra_kv_append(a)
    for pool, x in zip(pools, (k, v)):
        assert torch.equal(H.slots(pool, table, 0, 18)[:, 15:].transpose(0, 1), x[:3])
        assert torch.equal(H.slots(pool, table, 1, 3).transpose(0, 1), x[3:])


def test_append_reports_what_it_does_not_follow():
    k = torch.randn(3, 2, 64, device="cuda")
    pools = [torch.zeros(2, 2, 16, 64, device="cuda") for _ in "kv"]
    table = torch.tensor([[7], [0], [1]], dtype=torch.int32, device="cuda")  # page 7 is none
    lens = torch.tensor([4, 400, 3], dtype=torch.int32, device="cuda")       # 400 is past the table: the last slot
    rope = rope_table(8, 64)
    err = torch.zeros(1, dtype=torch.int32, device="cuda")
    a = R.ra_kv_append_args(cache=H.cache(*pools, table, err), lens_dev=lens.data_ptr(), k_dev=k.data_ptr(), v_dev=k.data_ptr(),
                            k_stride=128, v_stride=128, batch=3, n_new=1, rope_dev=rope.data_ptr(), rope_len=8)
    R.ra_kv_append(a)
    torch.cuda.synchronize()
    assert err.item() == R.RA_DEV_BOUNDS
    want = torch.zeros_like(pools[1])
    want[0, :, 15], want[1, :, 2] = k[1], k[2]
    assert torch.equal(pools[1], want)


# ---- eviction ------------------------------------------------------------------------------

def kept_slots(w, n, budget, first, recent):
    """The slots that stay, by the definition, one after the other: weights as (is NaN, value), lower slots first."""
    if n <= budget:
        return list(range(n))
    middle = sorted(range(first, n - recent), key=lambda i: (not math.isnan(w[i]), -w[i] if not math.isnan(w[i]) else 0.0, i))
    return sorted(list(range(first)) + middle[:budget - first - recent] + list(range(n - recent, n)))


def check_evict(dtype, lens, kv, dh, page, budget, first, recent, weights, out_page=None, pad=0):
    g = torch.Generator(device="cuda").manual_seed(2)
    dt, B, out_page = H.DT[dtype], len(lens), out_page or page
    per, out_per = max(1, -(-max(lens) // page)), -(-budget // out_page) + 1
    src = [torch.randn((B * per, kv, page, dh), generator=g, device="cuda").to(dt) for _ in "kv"]
    dst = [torch.full((B * out_per, kv, out_page, dh), 9.0, dtype=dt, device="cuda") for _ in "kv"]
    table = torch.randperm(B * per, generator=g, device="cuda").to(torch.int32).view(B, per)
    out_table = torch.randperm(B * out_per, generator=g, device="cuda").to(torch.int32).view(B, out_per)
    w = weights((B, kv, per * page + pad), g)
    lens_dev = torch.tensor(lens, dtype=torch.int32, device="cuda")
    kept = torch.full((B, kv, budget), 99, dtype=torch.int32, device="cuda")
    lens_out = torch.full((B,), 99, dtype=torch.int32, device="cuda")
    w_out = torch.full((B, kv, budget + 3), 9.0, device="cuda")
    err = torch.zeros(1, dtype=torch.int32, device="cuda")
    a = R.ra_kv_evict_args(src=H.cache(*src, table, err), dst=H.cache(*dst, out_table, err), lens_dev=lens_dev.data_ptr(),
                           weights_dev=w.data_ptr(), weights_stride=w.shape[2], lens_out_dev=lens_out.data_ptr(),
                           kept_dev=kept.data_ptr(), weights_out_dev=w_out.data_ptr(), weights_out_stride=w_out.shape[2],
                           batch=B, budget=budget, first=first, recent=recent)
    R.ra_kv_evict(a)
    torch.cuda.synchronize()
    assert err.item() == 0
    want = [d.clone().fill_(9.0) for d in dst]
    for b, n in enumerate(lens):
        stay = min(n, budget)
        assert lens_out[b].item() == stay
        for h in range(kv):
            at = kept_slots(w[b, h, :n].tolist(), n, budget, first, recent)
            assert kept[b, h].tolist() == at + [-1] * (budget - stay), (b, h)
            i = torch.tensor(at, dtype=torch.long, device="cuda")
            assert torch.equal(w_out[b, h, :stay].nan_to_num(nan=-7.0), w[b, h][i].nan_to_num(nan=-7.0))
            assert (w_out[b, h, stay:budget] == 0).all() and (w_out[b, h, budget:] == 9.0).all()
            to = torch.arange(stay, device="cuda")
            for s, d in zip(src, want):
                d[out_table[b].long()[to // out_page], h, to % out_page] = s[table[b].long()[i // page], h, i % page]
    assert torch.equal(dst[0], want[0]) and torch.equal(dst[1], want[1])


def heavy(shape, g):
    return torch.randn(shape, generator=g, device="cuda").mul_(2).exp_()


def few_values(shape, g):
    return torch.randint(0, 4, shape, generator=g, device="cuda").float() / 3


def awkward(shape, g):
    pool = torch.tensor([0.0, -0.0, math.inf, -math.inf, math.nan, -1.0, 1e-45, 1.0, -1e-45], device="cuda")
    return pool[torch.randint(0, len(pool), shape, generator=g, device="cuda")]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("weights", [heavy, few_values, awkward])
@pytest.mark.parametrize("budget,first,recent", [(64, 4, 20), (64, 0, 0), (64, 64, 0), (64, 0, 64), (64, 30, 34), (1, 0, 0),
                                                 (63, 1, 31), (200, 5, 17)])
def test_evict(dtype, weights, budget, first, recent):
    check_evict(dtype, [300, 64, 65, 63, 0, 1, 201, 199], 2, 64, 16, budget, first, recent, weights)


@pytest.mark.parametrize("dtype,kv,dh,page,out_page", [("bf16", 3, 128, 24, 16), ("f32", 1, 256, 7, 64), ("bf16", 2, 8, 16, 5),
                                                       ("f32", 2, 4, 1, 3), ("bf16", 1, 200, 64, 64)])
def test_evict_layouts(dtype, kv, dh, page, out_page):
    check_evict(dtype, [500, 100, 333], kv, dh, page, 120, 4, 40, heavy, out_page, pad=11)


def test_evict_long():
    """More slots than shared memory holds, beside shorter ones."""
    check_evict("bf16", [60000, 49153, 49152, 2000], 1, 16, 64, 5000, 4, 1000, heavy)
    check_evict("bf16", [60000], 1, 16, 64, 5000, 4, 1000, few_values)


def test_evict_of_nothing_but_equal_weights():
    check_evict("f32", [1000, 40], 2, 8, 16, 100, 0, 10, lambda shape, g: torch.zeros(shape, device="cuda"))


def test_evict_reports_bad_pages():
    src = [torch.randn(4, 1, 16, 8, device="cuda") for _ in "kv"]
    dst = [torch.zeros(1, 1, 16, 8, device="cuda") for _ in "kv"]
    table = torch.tensor([[0, 9, 2, 3]], dtype=torch.int32, device="cuda")
    out_table = torch.tensor([[0]], dtype=torch.int32, device="cuda")
    lens = torch.tensor([64], dtype=torch.int32, device="cuda")
    w = torch.zeros(1, 1, 64, device="cuda")
    w[0, 0, [3, 20, 40, 41]] = 1.0
    err = torch.zeros(1, dtype=torch.int32, device="cuda")
    kept, lens_out = (torch.zeros(n, dtype=torch.int32, device="cuda") for n in (4, 1))
    a = R.ra_kv_evict_args(src=H.cache(*src, table, err), dst=H.cache(*dst, out_table, err), lens_dev=lens.data_ptr(),
                           weights_dev=w.data_ptr(), weights_stride=64, lens_out_dev=lens_out.data_ptr(),
                           kept_dev=kept.data_ptr(), batch=1, budget=4)
    R.ra_kv_evict(a)
    torch.cuda.synchronize()
    assert kept.tolist() == [3, 20, 40, 41] and err.item() == R.RA_DEV_BOUNDS
    assert torch.equal(dst[0][0, 0, 0], src[0][0, 0, 3]) and (dst[0][0, 0, 1] == 0).all()
    assert torch.equal(dst[1][0, 0, 2], src[1][2, 0, 8])


@pytest.mark.parametrize("dtype,dh", [("f32", 4), ("f32", 12), ("f32", 20), ("f32", 252), ("bf16", 24), ("bf16", 248)])
@pytest.mark.parametrize("heads,kv", [(1, 1), (40, 8)])
def test_append_of_halves_that_no_wide_load_divides(dtype, dh, heads, kv):
    """Head dims whose halves are cut into 2 (f32) or 4 (bf16) values a thread, up to 63 a row."""
    for fused in (False, True):
        test_append(dtype, 3, 5, heads, kv, dh, 16, True, fused)


def test_evict_with_lengths_in_place():
    """lens_out may be lens: heads of a sequence whose turn comes after another head's still find its old length."""
    B, kv, page, budget, n = 96, 48, 16, 64, 160
    g = torch.Generator(device="cuda").manual_seed(3)
    src = [torch.randn((10 * B, kv, page, 8), generator=g, device="cuda") for _ in "kv"]
    dst = [torch.zeros((4 * B, kv, page, 8), device="cuda") for _ in "kv"]
    table = torch.randperm(10 * B, generator=g, device="cuda").to(torch.int32).view(B, 10)
    out_table = torch.randperm(4 * B, generator=g, device="cuda").to(torch.int32).view(B, 4)
    w = heavy((B, kv, 8192), g)  # (a long stride, for the kernel of the most threads a CTA)
    lens = torch.full((B,), n, dtype=torch.int32, device="cuda")
    lens[5], lens[6] = 30, 64
    kept = torch.full((B, kv, budget), 99, dtype=torch.int32, device="cuda")
    other = torch.full_like(kept, 99)
    new = torch.zeros_like(lens)
    a = R.ra_kv_evict_args(src=H.cache(*src, table), dst=H.cache(*dst, out_table), lens_dev=lens.data_ptr(), weights_dev=w.data_ptr(),
                           weights_stride=w.shape[2], lens_out_dev=new.data_ptr(), kept_dev=other.data_ptr(), batch=B, budget=budget,
                           first=4, recent=20)
    R.ra_kv_evict(a)
    rows = [d.clone() for d in dst]
    a.lens_out_dev, a.kept_dev = lens.data_ptr(), kept.data_ptr()
    R.ra_kv_evict(a)
    torch.cuda.synchronize()
    assert torch.equal(lens, new) and lens.tolist() == [30 if b == 5 else 64 for b in range(B)]
    assert torch.equal(kept, other) and torch.equal(dst[0], rows[0]) and torch.equal(dst[1], rows[1])
