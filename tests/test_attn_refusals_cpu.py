"""Calls of the attention operators that are refused before any device call, beside those
of test_attn_cpu.py."""
import pytest

import paper_2202_11836_amd as P
from test_attn_cpu import PTR, call, pytestmark, shape  # noqa: F401


@pytest.mark.parametrize("backward", [0, 1])
def test_scales_whose_base_2_form_is_infinite(backward):
    """scale * log2(e) is beyond fp32: a score of 0 would become NaN."""
    for scale in (2.36e38, 3.4e38):
        st, msg = call(backward, shape(scale=scale))
        assert st == 1 and "scale" in msg
    st, msg = call(backward, shape(scale=2.35e38), ws_bytes=0, q=None)
    assert st == 1 and "scale" not in msg  # (refused for the missing q)


def test_table_over_its_gradient():
    rp = P.RelPos(32, 128).c
    st, msg = call(1, shape(), rp, dtable=PTR["table"])
    assert st == 1 and "over an input" in msg
