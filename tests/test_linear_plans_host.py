"""Scratch of the dense layers' backward pass: what it has to hold, by the types and the activation (no GPU)."""
import ctypes as C

import pytest

import paper_2003_10735_amd as st

P, F32, BF16 = 4096, st.ST_F32, st.ST_BF16


def mat(rows, cols, dtype):
    return st.StMatrix(P, dtype, rows, cols, cols, 1)


@pytest.mark.parametrize("act,dtype,dy,terms", [(st.ST_ACT_GELU, BF16, BF16, 2), (st.ST_ACT_SILU, BF16, F32, 2), (st.ST_ACT_NONE, BF16, F32, 2),
                                                (st.ST_ACT_RELU, BF16, BF16, 1), (st.ST_ACT_GELU, F32, BF16, 1), (st.ST_ACT_NONE, BF16, BF16, 0)])
def test_scratch_holds_the_terms_of_dz(act, dtype, dy, terms):
    """A float32 result beside bfloat16 operands asks for two terms of dz, whatever dy's type: scratch has room for them, since it is made before the
    results' types are known.  (Many tokens and few channels: 32 parts of dw, 512 of db and their rounding up are less than half a term; 448
    positions of dx's contraction are not split.)"""
    m, n, k = 1 << 17, 448, 64
    nbytes = st.lib().st_linear_backward_workspace(*(C.byref(x) for x in (mat(m, k, dtype), mat(n, k, dtype), mat(m, n, dy))), act)
    dz = terms * m * n * (2 if dtype == BF16 else 4)
    assert dz <= nbytes < dz + m * n
