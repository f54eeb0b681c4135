"""Rows of which there are more than 32-bit numbers can count, shares of heads included, are refused before anything is launched (no GPU
needed: the pointers are never followed)."""
import pytest

from paper_2607_27735_b200 import binding
from test_round_ops_host import P, SHAPE, _append, _kv


@pytest.mark.parametrize("n,heads", [(1 << 28, 128), ((1 << 28) + 1, 128), (1 << 30, 64), (1 << 27, 136)])
def test_too_many_rows_for_the_second_launch(n, heads):
    """(rows of one token, broadcast: a stride of 0)"""
    kv = _kv(kv_dtype=2, k_scale=P, v_scale=P, n_q_heads=heads, n_kv_heads=heads)
    assert _append(kv, q=None, out=None, n=n, kr=0, vr=0, bytes=1 << 50) == SHAPE
