"""Which outputs of dartree_rotary may lie where, without a GPU.  Addresses are never
dereferenced; a call that is not refused fails at its launch, as there is no device."""
import ctypes

import pytest
import torch

from paper_2608_13524_amd import dartree as D

BASE = 0x10000000
ROW, HQ, HKV, N = 256, 8, 2, 10          # bytes of a head in bf16; 2 requests of 5 rows
BAD = D.ERR_INVALID_ARG


def call(q, qs, k, ks, qo, qos, ko, kos, **kw):
    """Byte offsets and strides in heads of 128 elements."""
    p = D.RotaryParams(2, 5, HQ, HKV, 128, 128, D.ROTARY_HALF, D.BF16, 0, 0, 1.0)
    for name, value in kw.items():
        setattr(p, name, value)
    at = lambda x: BASE + x
    return D.lib().dartree_rotary(ctypes.byref(p), BASE + (1 << 24), at(q), 128 * qs, at(k), 128 * ks, at(qo), 128 * qos, at(ko), 128 * kos,
                                  None, None, None, None)


Q, K, QO, KO = 0, 0x10000, 0x20000, 0x30000


@pytest.mark.parametrize("args", [
    (Q, 8, K, 2, K, 8, KO, 2),                      # q_out over k
    (Q, 8, K, 2, QO, 8, Q, 2),                      # k_out over q
    (Q, 8, K, 2, QO, 8, QO, 2),                     # both outputs at one place
    (Q, 8, K, 2, QO, 8, QO + 9 * 8 * ROW, 2),       # k_out's first row in q_out's last
    (Q, 8, K, 2, Q + ROW, 8, KO, 2),                # a head further on than q
    (Q, 8, K, 2, Q + 8 * ROW, 8, KO, 2),            # a row further on than q
    (Q, 16, K, 2, Q + 4 * ROW, 16, KO, 2),          # in q's rows, half beside it
    (Q, 12, Q + 8 * ROW, 12, Q, 12, Q + 9 * ROW, 12),    # a fused projection: k_out half beside k
    (Q, 12, Q + 8 * ROW, 12, Q, 12, Q + 7 * ROW, 12),    # k_out over q's last head
    (Q, 12, Q + 8 * ROW, 12, QO, 12, Q + 8 * ROW + 12 * ROW, 12),   # k_out a row further on than k
    (Q, 10, Q + 8 * ROW, 10, QO, 10, QO + 7 * ROW, 10)])
def test_overlapping_outputs_are_refused(args):
    assert call(*args) == BAD


@pytest.mark.parametrize("args", [
    (Q, 8, K, 2, QO, 8, KO, 2),                                     # four tensors
    (Q, 8, K, 2, Q, 8, K, 2),                                       # in place
    (Q, 12, Q + 8 * ROW, 12, Q, 12, Q + 8 * ROW, 12),               # in place in the rows of a fused projection
    (Q, 12, Q + 8 * ROW, 12, QO, 11, QO + 8 * ROW, 11),             # into the rows of a wider tensor
    (Q, 24, Q + 8 * ROW, 24, Q + 12 * ROW, 24, Q + 20 * ROW, 24),   # beside them in the same rows
    (Q, 12, Q + 8 * ROW, 24, QO, 8, Q + 10 * ROW, 12),              # k's rows twice as far apart as k_out's
    (Q, 8, Q + N * 8 * ROW, 2, QO, 8, QO + N * 8 * ROW, 2)])        # one right behind the other
def test_outputs_apart_are_not_refused(args):
    if torch.cuda.is_available():
        pytest.skip("addresses that no device has")
    assert call(*args) == D.ERR_HIP


def test_one_row_has_no_stride():
    one = dict(batch=1, rows=1)
    assert call(Q, 8, K, 2, QO, 8, QO + 7 * ROW, 4096, **one) == BAD
    assert call(Q, 4096, K, 2, K, 8, KO, 2, **one) == BAD


def test_heads_that_are_not_there_are_not_looked_at():
    if torch.cuda.is_available():
        pytest.skip("addresses that no device has")
    assert call(Q, 8, Q, 2, Q, 8, Q, 2, heads_kv=0) == D.ERR_HIP
    assert call(K, 8, K, 2, K, 8, K, 2, heads_q=0) == D.ERR_HIP
