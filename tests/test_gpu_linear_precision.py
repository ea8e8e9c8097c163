"""Gradients of bfloat16 layers from bfloat16 gradients, with results in float32: what dz = dy act'(z) is rounded to does not show in them.

Tolerances as for the layers' other gradients: a sum of k products in float32 is within (k + 16) 2^-24 sum |a||b| (two terms of dz: 2 k), a slope within
2^-17 of dy, dz within 2^-16 of itself beside a result in float32 (two bfloat16 terms) and within 2^-8 beside one in bfloat16 (one term).
"""
import pytest

import paper_2003_10735_amd as st

from test_gpu_linear import ACTS, EPS, mm64, rand, slope64, within

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

F, B = torch.float32, torch.bfloat16
SMOOTH = ["gelu", "gelu_tanh", "silu"]


@pytest.mark.parametrize("act", SMOOTH)
@pytest.mark.parametrize("dx_type,dw_type", [(F, F), (B, F), (F, B), (None, F), (F, None)])
@pytest.mark.parametrize("m,n,k", [(1, 40, 70), (60, 100, 300), (64, 64, 2000), (700, 640, 256), (2100, 1030, 136), (2000, 2000, 1100)])
def test_results_in_float32_keep_sixteen_bits_of_dz(m, n, k, dx_type, dw_type, act):
    x, w, dy, z = rand((m, k), 1, "bf16"), rand((n, k), 2, "bf16", k ** -0.5), rand((m, n), 3, "bf16"), rand((m, n), 4, "bf16", 2.0)
    dx, dw = (None if t is None else torch.empty(s, dtype=t, device="cuda") for t, s in ((dx_type, (m, k)), (dw_type, (n, k))))
    db = torch.empty(n, device="cuda")
    st.st_linear_backward(x, w, dy, z, ACTS[act], dx, dw, db)
    dz = dy.double() * slope64(z, act)
    slope_far = 2.0 ** -17 * dy.double().abs()
    for got, a, b, length in ((dx, dz, w, n), (dw, dz.t(), x, m)):
        if got is None:
            continue
        half = 2.0 ** -16 if got.dtype == F else 2.0 ** -8
        far = slope_far + half * (dz.abs() + slope_far)
        far = far + (2 * length + 16) * EPS * (dz.abs() + far)
        assert within(got, mm64(a, b.t()), mm64(far if a is dz else far.t(), b.t().abs()))
    assert within(db, dz.sum(0), (slope_far + (m + 16) * EPS * (dz.abs() + slope_far)).sum(0))


@pytest.mark.parametrize("act", SMOOTH)
def test_gradients_added_over_frames_keep_them_too(act):
    """Four batches added into one float32 dw: errors of 2^-8 a term would be far outside."""
    m, n, k = 300, 130, 200
    dw, want, far = torch.zeros(n, k, device="cuda"), 0.0, 0.0
    for i in range(4):
        x, dy, z = rand((m, k), 10 + i, "bf16"), rand((m, n), 20 + i, "bf16"), rand((m, n), 30 + i, "bf16", 2.0)
        st.st_linear_backward(x, None, dy, z, ACTS[act], dw=dw, accumulate=i > 0)
        dz = dy.double() * slope64(z, act)
        slope_far = 2.0 ** -17 * dy.double().abs()
        off = slope_far + 2.0 ** -16 * (dz.abs() + slope_far)
        want = want + mm64(dz.t(), x.t())
        far = far + mm64((off + (2 * m + 32) * EPS * (dz.abs() + off)).t(), x.t().abs())
    assert within(dw, want, far)


@pytest.mark.parametrize("act", ["none", "relu"])
def test_dz_that_bfloat16_holds_has_one_term(act):
    """Nothing is left of it for a second term: results are the same sums, whatever their type."""
    m, n, k = 300, 136, 200
    x, w, dy, z = rand((m, k), 1, "bf16"), rand((n, k), 2, "bf16"), rand((m, n), 3, "bf16"), rand((m, n), 4, "bf16")
    both = [(torch.empty(m, k, dtype=t, device="cuda"), torch.empty(n, k, dtype=t, device="cuda")) for t in (F, B)]
    for dx, dw in both:
        st.st_linear_backward(x, w, dy, z, ACTS[act], dx, dw)
    for a, b in zip(*both):
        assert torch.equal(a.to(B), b)
