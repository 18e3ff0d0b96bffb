"""Refusals of the operators that train a decoder's weights: the argument blocks are checked on the host before anything
else, so none of this needs a GPU."""
import math

import pytest

from paper_2502_19864_gb300 import ringada as R

P = 1 << 20  # an address that is aligned and never followed
ARG, SHAPE, NOMEM = R.RA_ERR_ARG, R.RA_ERR_SHAPE, R.RA_ERR_NOMEM


@pytest.fixture(scope="module", autouse=True)
def built():
    import __graft_entry__
    __graft_entry__.build()


def norm(**kw):
    a = dict(x_dev=P, x_stride=64, residual_dev=P, residual_stride=64, sum_dev=P, sum_stride=64, gamma_dev=P, beta_dev=P, y_dev=P,
             y_stride=64, mean_dev=P, rstd_dev=P, dy_dev=P, dy_stride=64, dsum_dev=P, dsum_stride=64, dx_dev=P, dx_stride=64,
             dgamma_dev=P, dbeta_dev=P, workspace_dev=P, workspace_bytes=1 << 40, rows=5, hidden=64, dtype=R.RA_BF16,
             w_dtype=R.RA_BF16, eps=1e-5)
    a.update(kw)
    return R.ra_norm_args(**a)


def loss(**kw):
    a = dict(x_dev=P, x_stride=64, w_dev=P, w_stride=64, labels_dev=P, loss_dev=P, lse_dev=P, dloss_dev=P, dx_dev=P, dx_stride=64,
             dw_dev=P, dw_stride=64, workspace_dev=P, workspace_bytes=1 << 40, tokens=10, vocab=100, hidden=64, dtype=R.RA_BF16)
    a.update(kw)
    return R.ra_vocab_loss_args(**a)


def orth(**kw):
    a = dict(x_dev=P, x_stride=64, x_matrix_stride=640, out_dev=P, out_stride=64, out_matrix_stride=640, workspace_dev=P,
             workspace_bytes=1 << 40, n_matrices=2, rows=10, cols=64, steps=5, dtype=R.RA_BF16, a=1.0, b=1.0, c=1.0, eps=1e-7)
    a.update(kw)
    return R.ra_orthogonalize_args(**a)


BOTH = (R.ra_norm_forward, R.ra_norm_backward)
LOSS = (R.ra_vocab_loss_forward, R.ra_vocab_loss_backward)
CASES = [
    (BOTH, norm, dict(dtype=3), ARG), (BOTH, norm, dict(w_dtype=7), ARG), (BOTH, norm, dict(dtype=R.RA_F32), ARG),
    (BOTH, norm, dict(kind=2), ARG), (BOTH, norm, dict(rows=-1), ARG), (BOTH, norm, dict(hidden=0), ARG),
    (BOTH, norm, dict(hidden=32769, x_stride=40000), SHAPE), (BOTH, norm, dict(eps=-1.0), ARG), (BOTH, norm, dict(eps=math.inf), ARG),
    (BOTH, norm, dict(eps=math.nan), ARG), (BOTH, norm, dict(gamma_dev=P + 1), ARG), (BOTH, norm, dict(beta_dev=P + 1), ARG),
    (BOTH, norm, dict(sum_stride=63), SHAPE), (BOTH, norm, dict(sum_dev=P + 1), ARG), (BOTH, norm, dict(rstd_dev=P + 2), ARG),
    (BOTH[:1], norm, dict(x_dev=None), ARG), (BOTH[:1], norm, dict(x_stride=63), SHAPE), (BOTH[:1], norm, dict(y_dev=None), ARG),
    (BOTH[:1], norm, dict(y_stride=1), SHAPE), (BOTH[:1], norm, dict(residual_stride=63), SHAPE),
    (BOTH[1:], norm, dict(sum_dev=None), ARG), (BOTH[1:], norm, dict(rstd_dev=None), ARG), (BOTH[1:], norm, dict(mean_dev=None), ARG),
    (BOTH[1:], norm, dict(dy_dev=None), ARG), (BOTH[1:], norm, dict(dy_stride=63), SHAPE), (BOTH[1:], norm, dict(dsum_stride=63), SHAPE),
    (BOTH[1:], norm, dict(dx_stride=63), SHAPE), (BOTH[1:], norm, dict(dgamma_dev=P + 1), ARG),
    (BOTH[1:], norm, dict(dbeta_dev=P + 1), ARG), (BOTH[1:], norm, dict(workspace_dev=None), ARG),
    (BOTH[1:], norm, dict(workspace_dev=P + 16), ARG), (BOTH[1:], norm, dict(workspace_bytes=100), NOMEM),
    (LOSS, loss, dict(dtype=2), ARG), (LOSS, loss, dict(tokens=-1), ARG), (LOSS, loss, dict(vocab=0), ARG), (LOSS, loss, dict(hidden=0), ARG),
    (LOSS, loss, dict(hidden=60), SHAPE), (LOSS, loss, dict(hidden=1 << 21, x_stride=1 << 21), SHAPE), (LOSS, loss, dict(tokens=1 << 25), SHAPE),
    (LOSS, loss, dict(vocab=1 << 25), SHAPE), (LOSS, loss, dict(tokens=1 << 24, vocab=1 << 17), SHAPE),
    (LOSS, loss, dict(vocab=1 << 20, hidden=1 << 18, x_stride=1 << 18, w_stride=1 << 18, dx_stride=1 << 18, dw_stride=1 << 18), SHAPE),
    (LOSS, loss, dict(x_dev=None), ARG), (LOSS, loss, dict(x_dev=P + 2), ARG),
    (LOSS, loss, dict(x_stride=68), SHAPE), (LOSS, loss, dict(w_dev=None), ARG), (LOSS, loss, dict(w_stride=56), SHAPE),
    (LOSS, loss, dict(labels_dev=None), ARG), (LOSS, loss, dict(workspace_dev=None), ARG), (LOSS, loss, dict(workspace_bytes=1000), NOMEM),
    (LOSS[:1], loss, dict(loss_dev=None), ARG), (LOSS[1:], loss, dict(lse_dev=None), ARG), (LOSS[1:], loss, dict(dloss_dev=None), ARG),
    (LOSS[1:], loss, dict(dx_dev=P + 4), ARG), (LOSS[1:], loss, dict(dx_stride=60), SHAPE), (LOSS[1:], loss, dict(dw_stride=68), SHAPE),
    ((R.ra_orthogonalize,), orth, dict(dtype=2), ARG), ((R.ra_orthogonalize,), orth, dict(n_matrices=-1), ARG),
    ((R.ra_orthogonalize,), orth, dict(rows=0), ARG), ((R.ra_orthogonalize,), orth, dict(cols=-3), ARG), ((R.ra_orthogonalize,), orth, dict(steps=-1), ARG),
    ((R.ra_orthogonalize,), orth, dict(steps=65), SHAPE), ((R.ra_orthogonalize,), orth, dict(rows=32769), SHAPE),
    ((R.ra_orthogonalize,), orth, dict(n_matrices=65536), SHAPE), ((R.ra_orthogonalize,), orth, dict(a=math.inf), ARG),
    ((R.ra_orthogonalize,), orth, dict(c=math.nan), ARG), ((R.ra_orthogonalize,), orth, dict(eps=-1e-9), ARG),
    ((R.ra_orthogonalize,), orth, dict(x_dev=None), ARG), ((R.ra_orthogonalize,), orth, dict(out_dev=P + 1), ARG),
    ((R.ra_orthogonalize,), orth, dict(x_stride=63), SHAPE), ((R.ra_orthogonalize,), orth, dict(out_stride=63), SHAPE),
    ((R.ra_orthogonalize,), orth, dict(x_matrix_stride=639), SHAPE), ((R.ra_orthogonalize,), orth, dict(out_matrix_stride=0), SHAPE),
    ((R.ra_orthogonalize,), orth, dict(workspace_dev=None), ARG), ((R.ra_orthogonalize,), orth, dict(workspace_bytes=1000), NOMEM),
]


@pytest.mark.parametrize("calls,block,change,status", CASES)
def test_refused(calls, block, change, status):
    for call in calls:
        with pytest.raises(R.RingAdaError) as e:
            call(block(**change))
        assert e.value.status == status, call


def test_no_work():
    R.ra_norm_forward(R.ra_norm_args(hidden=8, dtype=R.RA_BF16, w_dtype=R.RA_F32))
    R.ra_norm_backward(R.ra_norm_args(hidden=8, dtype=R.RA_BF16, w_dtype=R.RA_F32))
    R.ra_vocab_loss_forward(R.ra_vocab_loss_args(vocab=8, hidden=8))
    R.ra_vocab_loss_backward(R.ra_vocab_loss_args(vocab=8, hidden=8))
    R.ra_orthogonalize(R.ra_orthogonalize_args())


def test_workspaces():
    for size, block in ((R.ra_norm_workspace_bytes, norm), (R.ra_vocab_loss_workspace_bytes, loss), (R.ra_orthogonalize_workspace_bytes, orth)):
        assert size(block()) >= 16384
        assert size(block(dtype=9)) == 0
        assert size(block(workspace_dev=None, workspace_bytes=0)) == size(block())
    # blocks of the backward alone, or the forward alone
    assert R.ra_norm_workspace_bytes(norm(x_dev=None, y_dev=None)) == R.ra_norm_workspace_bytes(norm())
    assert R.ra_norm_workspace_bytes(norm(dy_dev=None, rstd_dev=None)) == R.ra_norm_workspace_bytes(norm())
    assert R.ra_vocab_loss_workspace_bytes(loss(loss_dev=None)) == R.ra_vocab_loss_workspace_bytes(loss())
    assert 0 < R.ra_vocab_loss_workspace_bytes(loss(dloss_dev=None, lse_dev=None, dx_dev=None, dw_dev=None)) <= R.ra_vocab_loss_workspace_bytes(loss())
    for change in (dict(dx_dev=None), dict(dw_dev=None)):  # (either gradient alone takes no more)
        assert R.ra_vocab_loss_workspace_bytes(loss(**change)) == R.ra_vocab_loss_workspace_bytes(loss())


def test_matrices_side_by_side():
    side = dict(x_stride=128, x_matrix_stride=64, out_stride=130, out_matrix_stride=65)
    assert R.ra_orthogonalize_workspace_bytes(orth(**side)) >= 16384
    for wrong in (dict(x_stride=127), dict(x_matrix_stride=63), dict(out_stride=128), dict(out_matrix_stride=67)):
        assert R.ra_orthogonalize_workspace_bytes(orth(**{**side, **wrong})) == 0


def test_products_let_dependents_start_behind_the_allocation():
    """As test_tmem_order.py has it for the kernels in .cu files: the products' kernel is in a header."""
    import os
    import re
    path = os.path.join(os.path.dirname(os.path.abspath(__file__)), "..", "paper_2502_19864_gb300", "csrc", "products.cuh")
    body = re.sub(r"//[^\n]*", "", open(path).read()).split("__global__")[1]
    barrier = body.index("__syncthreads()", body.rindex("tcgen05.alloc"))
    assert body.index("pdl_trigger()") > barrier


def test_forms_of_the_tested_sizes():
    """The sizes at which the GPU tests run each form of the products do take it: the forms come from times that may be fitted anew."""
    from tests import test_gpu_orthogonalize as O
    from tests import test_gpu_vocab_loss as V
    from tests.operator_helpers import RA, orthogonalize_plan, vocab_loss_plan
    for dtype, tokens, vocab, hidden, forms in V.FORMS:
        V.check_forms(vocab_loss_plan(loss(tokens=tokens, vocab=vocab, hidden=hidden, x_stride=hidden, w_stride=hidden, dx_stride=hidden,
                                           dw_stride=hidden, dtype=RA[dtype])), forms)
    for dtype, n, rows, cols, forms in O.FORMS:
        O.check_forms(orthogonalize_plan(orth(n_matrices=n, rows=rows, cols=cols, x_stride=cols, out_stride=cols, x_matrix_stride=rows * cols,
                                              out_matrix_stride=rows * cols, dtype=RA[dtype])), forms)


def test_no_form_of_no_work():
    import ctypes as C
    out = (C.c_int32 * 17)()
    for plan, blocks in ((R.lib().ra_internal_vocab_loss_plan, (loss(tokens=0), loss(tokens=-1), loss(x_dev=None))),
                         (R.lib().ra_internal_orthogonalize_plan, (orth(n_matrices=0), orth(n_matrices=-1), orth(x_dev=None)))):
        assert plan(None, out) == ARG
        for block in blocks:
            assert plan(C.byref(block), out) == ARG
