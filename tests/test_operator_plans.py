"""How the operators beside the commit step cut rows of logits into parts, and which memory their outputs may take: on
the host, before anything is enqueued."""
import ctypes

import pytest

from paper_2609_36452_amd import binding as rpd

P = 1 << 20   # non-NULL, never dereferenced


def _r(n):
    return (n + 255) // 256 * 256


def _distill(N, V, logits=P, ls=None, grad=None, gs=None, dtype=rpd.DTYPE_BF16):
    # N <= 0 or a missing workspace end a call before it enqueues anything
    return rpd.RpdDistill(N, V, 8, dtype, rpd.DTYPE_F32, logits, ls or V, P, P, None, None, None, 1.0, P, P, grad, gs or V)


@pytest.mark.parametrize("N,V,ls,at,gs,refused", [
    (4, 100, 100, 0, 100, True),            # the logits themselves
    (4, 100, 100, 399, 100, True),          # their last element
    (4, 100, 100, 400, 100, False),         # right behind them
    (4, 100, 100, -400, 100, False),        # right in front of them
    (4, 100, 100, -399, 100, True),
    (1, 100, 100, 50, 100, True),
    (4, 100, 200, 100, 200, False),         # rows between the logits' rows
    (4, 100, 200, 300, 200, False),
    (4, 100, 200, 99, 200, True),
    (4, 100, 200, 101, 200, True),
    (4, 100, 200, 150, 200, True),
    (4, 100, 200, 100, 100, True),          # of another stride: row 1 over the logits' row 1
    (3, 100, 1000, 2100, 100, False),       # behind the logits' last element
])
@pytest.mark.parametrize("dtype", [rpd.DTYPE_BF16, rpd.DTYPE_F32])
def test_distill_refuses_a_gradient_over_the_logits(N, V, ls, at, gs, refused, dtype):
    size = 4 if dtype == rpd.DTYPE_F32 else 2
    p = _distill(N, V, ls=ls, grad=P + at * size, gs=gs, dtype=dtype)
    # a call that is not refused for its memory is for its workspace
    assert rpd.lib().rpd_distill_loss(ctypes.byref(p), None, 0, None) == (3 if refused else 1)
    assert ("logits" in rpd.last_error()) == refused and ("workspace" in rpd.last_error()) != refused


@pytest.mark.parametrize("V,parts", [(131072, 16), (262144, 32), (262145, 22), (300000, 25), (393216, 32), (393217, 49),
                                     (1 << 20, 64)])
def test_parts_of_many_rows(V, parts):
    """Parts of whole 2048 entries, at most 64 of them, doubled while they are shorter than 8192."""
    p = _distill(4000, V)
    assert rpd.lib().rpd_distill_workspace_size(ctypes.byref(p)) == _r(4000 * parts * 8)
    q = rpd.RpdVerify(2000, 1, V, rpd.DTYPE_BF16, P, 2 * V, V, None, 0, 0, P, None, P, P, 1.0, 1.0,
                      rpd.VERIFY_GREEDY, P, P, P)
    assert rpd.lib().rpd_verify_workspace_size(ctypes.byref(q)) == _r(4000 * parts * 16)
