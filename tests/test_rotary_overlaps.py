"""Outputs of rotary positions that share memory with rows that are read, or with each other, are refused before
anything is enqueued (no GPU needed: the pointers are never read)."""

import pytest

from test_step_refusals import APPEND, APPEND_GOOD, INVALID, L, ROTARY, ROTARY_GOOD, _call  # noqa: F401

# One matrix of rows of 1024 elements of 2 bytes: q in its elements 0 to 511, k in 512 to 767, v in 768 to 1023.
X, LD = 1 << 20, 1024
Q, K, V = X, X + 2 * 512, X + 2 * 768
FAR = 1 << 24
ROTARY_ROWS = {**ROTARY_GOOD, "q": Q, "ld_q": LD, "k": K, "ld_k": LD, "T": 100, "q_out": FAR, "k_out": 2 * FAR}
APPEND_ROWS = {**APPEND_GOOD, "q": Q, "ld_q": LD, "k": K, "ld_k": LD, "v": V, "ld_v": LD, "T": 100, "q_out": FAR}
ROW, LAST = 2 * LD, 99 * 2 * LD


@pytest.mark.parametrize("changes", [
    dict(q_out=K, ld_q_out=LD), dict(q_out=Q + 16, ld_q_out=LD), dict(q_out=K - 16, ld_q_out=LD),
    dict(q_out=Q + ROW, ld_q_out=LD), dict(q_out=Q - ROW, ld_q_out=LD), dict(q_out=K + LAST + 496, ld_q_out=LD),
    dict(q_out=Q - LAST - 1008, ld_q_out=LD),
    dict(k_out=Q, ld_k_out=LD), dict(k_out=Q + 1008, ld_k_out=LD), dict(k_out=K + 3 * ROW, ld_k_out=LD),
    dict(k_out=K - 16, ld_k_out=LD), dict(k_out=FAR), dict(k_out=FAR + 1008, ld_k_out=512),
    dict(q_out=Q, ld_q_out=LD, k_out=Q + 512, ld_k_out=LD),
    # Rows of another distance, dense ones in the matrix here.
    dict(q_out=X), dict(q_out=X + 4096), dict(k_out=K + LAST + 496), dict(q_out=FAR, k_out=FAR + 2 * 512 * 99),
    # One token.
    dict(T=1, q_out=Q + 1008), dict(T=1, k_out=K - 496), dict(T=1, k_out=Q), dict(T=1, q_out=FAR, k_out=FAR + 1008),
    # Far beyond any memory.
    dict(T=(1 << 30) - 1, ld_q=1 << 62, ld_q_out=1 << 62, q_out=Q + 16),
])
def test_rotary(L, changes):  # noqa: F811
    assert _call(L.dptq_rotary, ROTARY, ROTARY_ROWS, **changes) == INVALID


@pytest.mark.parametrize("changes", [
    dict(q_out=K, ld_q_out=LD), dict(q_out=V - 1008, ld_q_out=LD), dict(q_out=V + 496, ld_q_out=LD),
    dict(q_out=Q + 16, ld_q_out=LD), dict(q_out=Q + 5 * ROW, ld_q_out=LD), dict(q_out=X), dict(q_out=V + LAST + 496),
    dict(T=1, q_out=V), dict(T=1, q_out=K - 16),
])
def test_rotary_kv8_append(L, changes):  # noqa: F811
    assert _call(L.dptq_rotary_kv8_append, APPEND, APPEND_ROWS, **changes) == INVALID
