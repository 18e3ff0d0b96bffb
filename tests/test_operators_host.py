"""Refusals of the decoder's answering operators: the argument blocks are checked on the host before anything else, so
none of this needs a GPU."""
import pytest

from paper_2502_19864_gb300 import ringada as R


@pytest.fixture(scope="module", autouse=True)
def built():
    import __graft_entry__
    __graft_entry__.build()


P = 1 << 20  # an address that is aligned and never followed


def cache(**kw):
    c = dict(k_dev=P, v_dev=P, block_table_dev=P, n_pages=8, max_pages=4, page_size=16, n_kv_heads=2, head_dim=64, dtype=R.RA_BF16)
    c.update(kw)
    return R.ra_kv_cache(**c)


def append(c=None, **kw):
    a = dict(cache=c or cache(), lens_dev=P, q_dev=P, k_dev=P, v_dev=P, q_out_dev=P, q_stride=256, k_stride=128, v_stride=128,
             q_out_stride=256, rope_dev=P, rope_len=10, batch=1, n_new=1, n_heads=4)
    a.update(kw)
    return R.ra_kv_append_args(**a)


def decode(c=None, **kw):
    a = dict(cache=c or cache(), lens_dev=P, q_dev=P, q_stride=256, out_dev=P, out_stride=256, workspace_dev=P,
             workspace_bytes=1 << 40, batch=1, n_new=1, n_heads=4, scale=0.125)
    a.update(kw)
    return R.ra_attention_decode_args(**a)


def evict(src=None, dst=None, **kw):
    a = dict(src=src or cache(), dst=dst or cache(), lens_dev=P, weights_dev=P, weights_stride=64, lens_out_dev=P, kept_dev=P,
             weights_out_dev=P, weights_out_stride=32, batch=1, budget=32, first=4, recent=8)
    a.update(kw)
    return R.ra_kv_evict_args(**a)


def window(**kw):
    a = dict(q_dev=P, k_dev=P, v_dev=P, q_stride=256, k_stride=128, v_stride=128, out_dev=P, out_stride=256, lse_dev=P, dout_dev=P,
             dout_stride=256, dq_dev=P, dk_dev=P, dv_dev=P, dq_stride=256, dk_stride=128, dv_stride=128, workspace_dev=P,
             workspace_bytes=1 << 40, batch=1, seq=100, n_heads=4, n_kv_heads=2, head_dim=64, window=10, sinks=1, dtype=R.RA_BF16,
             scale=0.125)
    a.update(kw)
    return R.ra_attention_window_args(**a)


def verify(**kw):
    a = dict(target_dev=P, target_stride=100, draft_dev=P, draft_stride=100, tokens_dev=P, uniform_dev=P, noise_dev=P, accepted_dev=P,
             out_tokens_dev=P, workspace_dev=P, workspace_bytes=1 << 40, batch=2, n_draft=3, vocab=100, dtype=R.RA_BF16)
    a.update(kw)
    return R.ra_verify_draft_args(**a)


ARG, SHAPE, NOMEM = R.RA_ERR_ARG, R.RA_ERR_SHAPE, R.RA_ERR_NOMEM
CACHES = [(dict(k_dev=None), ARG), (dict(v_dev=P + 8), ARG), (dict(block_table_dev=None), ARG), (dict(dtype=7), ARG),
          (dict(n_pages=0), ARG), (dict(max_pages=0), ARG), (dict(page_size=0), ARG), (dict(n_kv_heads=0), ARG),
          (dict(head_dim=60), SHAPE), (dict(head_dim=264), SHAPE), (dict(head_dim=0), SHAPE),
          (dict(max_pages=1 << 30, page_size=16), SHAPE)]


def refused(call, args, status):
    with pytest.raises(R.RingAdaError) as e:
        call(args)
    assert e.value.status == status, (e.value, status)


@pytest.mark.parametrize("bad,status", CACHES)
def test_caches(bad, status):
    refused(R.ra_kv_append, append(cache(**bad)), status)
    refused(R.ra_attention_decode, decode(cache(**bad)), status)
    refused(R.ra_kv_evict, evict(src=cache(**bad)), status)
    refused(R.ra_kv_evict, evict(dst=cache(**bad)), status)


@pytest.mark.parametrize("bad,status", [
    (dict(lens_dev=None), ARG), (dict(k_dev=None), ARG), (dict(v_dev=P + 2), ARG), (dict(k_stride=120), SHAPE),
    (dict(v_stride=132), SHAPE), (dict(q_dev=None), ARG), (dict(q_out_dev=None), ARG), (dict(n_heads=3), ARG), (dict(n_heads=0), ARG),
    (dict(q_stride=248), SHAPE), (dict(q_out_stride=248), SHAPE), (dict(rope_len=0), ARG), (dict(rope_dev=P + 4), ARG),
    (dict(batch=-1), ARG), (dict(n_new=0), ARG)])
def test_append(bad, status):
    refused(R.ra_kv_append, append(**bad), status)


@pytest.mark.parametrize("bad,status", [
    (dict(lens_dev=None), ARG), (dict(q_dev=None), ARG), (dict(out_dev=P + 8), ARG), (dict(q_stride=255), SHAPE),
    (dict(out_stride=128), SHAPE), (dict(n_heads=5), ARG), (dict(n_new=0), ARG), (dict(window=-1), ARG), (dict(sinks=-1), ARG),
    (dict(max_len=-1), ARG), (dict(scale=0.0), ARG), (dict(scale=float("nan")), ARG), (dict(weights_in_dev=P), ARG), (dict(weights_out_dev=P, weights_stride=63), SHAPE),
    (dict(workspace_dev=None), ARG), (dict(workspace_dev=P + 128), ARG), (dict(workspace_bytes=100), NOMEM), (dict(batch=-2), ARG),
    (dict(batch=1 << 20, n_new=1 << 10), SHAPE)])
def test_decode(bad, status):
    refused(R.ra_attention_decode, decode(**bad), status)


@pytest.mark.parametrize("bad,status", [
    (dict(lens_dev=None), ARG), (dict(weights_dev=None), ARG), (dict(lens_out_dev=None), ARG), (dict(kept_dev=None), ARG),
    (dict(budget=0), ARG), (dict(first=-1), ARG), (dict(recent=-1), ARG), (dict(first=20, recent=13), ARG),
    (dict(first=(1 << 31) - 1, recent=(1 << 31) - 1), ARG), (dict(weights_stride=63), SHAPE), (dict(weights_out_stride=31), SHAPE),
    (dict(budget=65, weights_out_stride=65), SHAPE), (dict(dst=cache(n_kv_heads=1)), SHAPE), (dict(dst=cache(head_dim=128)), SHAPE),
    (dict(dst=cache(dtype=R.RA_F32)), SHAPE), (dict(batch=-1), ARG)])
def test_evict(bad, status):
    refused(R.ra_kv_evict, evict(**bad), status)


@pytest.mark.parametrize("bad,status", [
    (dict(q_dev=None), ARG), (dict(k_dev=P + 8), ARG), (dict(v_stride=64), SHAPE), (dict(out_dev=None), ARG), (dict(dtype=2), ARG),
    (dict(n_kv_heads=3), ARG), (dict(n_kv_heads=0), ARG), (dict(head_dim=96), SHAPE), (dict(head_dim=6, dtype=R.RA_F32), SHAPE),
    (dict(head_dim=132, dtype=R.RA_F32), SHAPE), (dict(window=-1), ARG), (dict(sinks=-3), ARG), (dict(seq=-1), ARG),
    (dict(scale=-1.0), ARG), (dict(scale=float("inf")), ARG),
    (dict(batch=1 << 16, seq=1 << 15), SHAPE), (dict(q_stride=258), SHAPE)])
def test_window(bad, status):
    refused(R.ra_attention_window_forward, window(**bad), status)
    refused(R.ra_attention_window_backward, window(**bad), status)


@pytest.mark.parametrize("bad,status", [
    (dict(lse_dev=None), ARG), (dict(dout_dev=None), ARG), (dict(dq_dev=None), ARG), (dict(dk_dev=P + 4), ARG), (dict(dv_stride=8), SHAPE),
    (dict(workspace_dev=None), ARG), (dict(workspace_bytes=16), NOMEM)])
def test_window_backward(bad, status):
    refused(R.ra_attention_window_backward, window(**bad), status)


@pytest.mark.parametrize("bad,status", [
    (dict(target_dev=None), ARG), (dict(draft_dev=None), ARG), (dict(tokens_dev=None), ARG), (dict(uniform_dev=None), ARG),
    (dict(noise_dev=None), ARG), (dict(accepted_dev=None), ARG), (dict(out_tokens_dev=None), ARG), (dict(vocab=0), ARG),
    (dict(n_draft=-1), ARG), (dict(dtype=5), ARG), (dict(target_stride=99), SHAPE), (dict(draft_stride=99), SHAPE),
    (dict(target_dev=P + 1), ARG), (dict(workspace_dev=None), ARG), (dict(workspace_bytes=1), NOMEM), (dict(batch=-1), ARG)])
def test_verify(bad, status):
    refused(R.ra_verify_draft, verify(**bad), status)


def test_null_blocks_and_workspaces_of_refused_ones():
    lib = R.lib()
    for call in (lib.ra_kv_append, lib.ra_attention_decode, lib.ra_kv_evict, lib.ra_attention_window_forward,
                 lib.ra_attention_window_backward, lib.ra_verify_draft):
        assert call(None, None) == ARG
    for size in (lib.ra_attention_decode_workspace_bytes, lib.ra_attention_window_workspace_bytes, lib.ra_verify_draft_workspace_bytes):
        assert size(None) == 0
    assert R.ra_attention_decode_workspace_bytes(decode(n_heads=5)) == 0
    assert R.ra_attention_decode_workspace_bytes(decode()) > 0
    assert R.ra_attention_window_workspace_bytes(window(head_dim=96)) == 0
    assert R.ra_verify_draft_workspace_bytes(verify(vocab=0)) == 0


BIG = (1 << 31) - 1
WIDE = dict(head_dim=128, n_kv_heads=1 << 25)  # 2^32 values a token


@pytest.mark.parametrize("call,args", [
    (R.ra_kv_append, append(cache(max_pages=(1 << 27) - 1))),      # slots up to the last 32-bit one: blocks of them end behind it
    (R.ra_attention_decode, decode(cache(max_pages=(1 << 27) - 1))),
    (R.ra_kv_evict, evict(dst=cache(max_pages=(1 << 27) - 1), budget=BIG - 15, weights_out_stride=BIG)),
    (R.ra_kv_evict, evict(src=cache(max_pages=(1 << 27) - 1), weights_stride=BIG)),
    (R.ra_kv_append, append(cache(**WIDE), q_dev=None, q_out_dev=None, k_stride=1 << 32, v_stride=1 << 32)),
    (R.ra_attention_decode, decode(cache(**WIDE), n_heads=1 << 25, q_stride=1 << 32, out_stride=1 << 32)),
    (R.ra_attention_decode, decode(cache(head_dim=256), q_stride=1024, out_stride=1024, n_new=1 << 25)),  # 2^33 values to zero
    (R.ra_attention_window_forward, window(n_heads=1 << 25, **WIDE, seq=1, q_stride=1 << 32, k_stride=1 << 32, v_stride=1 << 32,
                                           out_stride=1 << 32)),
    (R.ra_verify_draft, verify(n_draft=BIG)),
    (R.ra_verify_draft, verify(vocab=BIG, target_stride=BIG, draft_stride=BIG))])
def test_counts_that_32_bits_do_not_hold(call, args):
    refused(call, args, SHAPE)


def test_no_sequences():
    """A batch of none (or of sequences without tokens), whose tensors have no memory: nothing to do, and no error."""
    cache0 = cache(k_dev=None, v_dev=None, block_table_dev=None)
    nothing = dict(batch=0, lens_dev=None)
    R.ra_kv_append(append(cache0, q_dev=None, k_dev=None, v_dev=None, q_out_dev=None, **nothing))
    calls = [(R.ra_attention_decode, R.ra_attention_decode_workspace_bytes, decode(cache0, q_dev=None, out_dev=None, **nothing)),
             (R.ra_kv_evict, None, evict(cache0, cache0, weights_dev=None, lens_out_dev=None, kept_dev=None, **nothing)),
             (R.ra_verify_draft, R.ra_verify_draft_workspace_bytes, verify(batch=0, target_dev=None, draft_dev=None, tokens_dev=None,
                                                                          uniform_dev=None, noise_dev=None, accepted_dev=None,
                                                                          out_tokens_dev=None))]
    empty = dict(q_dev=None, k_dev=None, v_dev=None, out_dev=None, lse_dev=None, dout_dev=None, dq_dev=None, dk_dev=None, dv_dev=None)
    for a in (window(batch=0, **empty), window(seq=0, **empty)):
        calls += [(R.ra_attention_window_forward, R.ra_attention_window_workspace_bytes, a),
                  (R.ra_attention_window_backward, R.ra_attention_window_workspace_bytes, a)]
    for call, size, a in calls:
        call(a)
        if size:
            assert size(a) > 0  # (0 is that of a refused block)
