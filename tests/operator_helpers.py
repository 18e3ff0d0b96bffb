"""Shared helpers of the tests of the decoder's answering operators: plain implementations in 64 bits, and
the bounds that the kernels' roundings give.

Bounds (element by element, against 64 bits on the same inputs).  u = 2^-24 is the fp32 rounding, e = 2^-8 the
bf16 one (eight significant bits).  A score is a sum of head_dim products, off by at most (head_dim + 2) u sum |q k| scale =: ds; an
exponential by 4 u (the instruction) and by u |s| (its argument); so a weight is off by dp = 2 ds + 2 u max|s| +
8 u relative to itself (twice: numerator and sum), and by n u more for a sum of n of them.  An output is a sum of
n products, off by n u more.  With A = sum_j p_j |v_j| the bound of an fp32 output is (dp + 2 n u) A + u |o|.
  A bf16 kernel that rounds its weights to bf16 before the product with v adds e A, and e |o| for its output.
  The decode kernel's weights enter the product in two bf16 terms, off by e^2: the output's rounding is left, and
  e |o| <= e / 2 (A + |o|), as |o| <= A."""
import math

import torch

from paper_2502_19864_gb300 import ringada as R

U, E = 2.0 ** -24, 2.0 ** -8
DT = {"f32": torch.float32, "bf16": torch.bfloat16}
RA = {"f32": R.RA_F32, "bf16": R.RA_BF16}


def seen(query, key, window, sinks):
    """[..., n_query, n_key] of slot numbers: j <= i and inside the window or among the sinks."""
    i, j = query[..., :, None], key[..., None, :]
    ok = j <= i
    return ok & ((i - j < window) | (j < sinks)) if window else ok


def attention64(q, k, v, mask, scale, dtype, e=E):
    """One head: q [m, d], k, v [n, d] (any type), mask [m, n] -> out, lse, weights and the out's bound, in 64 bits."""
    q, k, v = q.double(), k.double(), v.double()
    if k.shape[0] == 0:
        z = q.new_zeros(q.shape[0], v.shape[1])
        return z, q.new_full((q.shape[0],), -math.inf), q.new_zeros(q.shape[0], 0), z, 0.0
    s = (q @ k.T * scale).masked_fill(~mask, -math.inf)
    lse = torch.logsumexp(s, -1)
    p = torch.exp(s - torch.nan_to_num(lse, neginf=0.0)[:, None])
    p = torch.where(mask, p, torch.zeros_like(p))
    out = p @ v
    d, n = q.shape[1], k.shape[0]
    ds = (d + 2) * U * float((q.abs() @ k.abs().T).max()) * scale
    dp = 2 * ds + 2 * U * float(torch.where(mask, s.abs(), torch.zeros_like(s)).max()) + 8 * U
    e16 = e if dtype == "bf16" else 0.0
    bound = (dp + 2 * n * U + e16) * (p @ v.abs()) + (e16 + U) * out.abs() + 1e-30
    return out, lse, p, bound, dp + n * U


def cache(k_pages, v_pages, table, err=None):
    """The argument block of a paged cache; pools [n_pages, kv heads, page, head dim]."""
    return R.ra_kv_cache(k_dev=k_pages.data_ptr(), v_dev=v_pages.data_ptr(), block_table_dev=table.data_ptr(),
                         err_dev=err.data_ptr() if err is not None else None, n_pages=k_pages.shape[0],
                         max_pages=table.shape[1], page_size=k_pages.shape[2], n_kv_heads=k_pages.shape[1],
                         head_dim=k_pages.shape[3], dtype=R.RA_BF16 if k_pages.dtype == torch.bfloat16 else R.RA_F32)


def slots(pages, table, b, n):
    """[kv heads, n, head dim]: the first n slots of sequence b."""
    page = pages.shape[2]
    at = torch.arange(n, device=pages.device)
    return pages[table[b].long()[at // page], :, at % page].transpose(0, 1)


def workspace(n, device="cuda"):
    return torch.zeros(max(n, 256), dtype=torch.uint8, device=device)
