"""Every tile of the 8-bit product with remainders in all three sizes, in both directions, and that it is the tile that ran.

The numbers are checked as in test_gpu_int8_layers; which kernel ran is asked of the library's profile, so a change of the rule that
chooses tiles cannot leave one of them without a test.
"""
import pytest

import paper_2003_10735_amd as st

from test_gpu_int8_layers import DT, EPS, check_backward, check_linear, rand

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

TILES = {"int8_product_256", "int8_product_128", "int8_product_128_deep", "int8_product_64"}


def ran(call):
    """Names of the library's kernels that a call launches."""
    st.st_profile_filter(None)
    st.st_profile_reset()
    st.st_profile_enable(True)
    try:
        call()
        torch.cuda.synchronize()
        return set(st.st_profile_read())
    finally:
        st.st_profile_enable(False)
        st.st_profile_reset()


FORWARD = [("int8_product_256", 3333, 1030, 4201), ("int8_product_128", 2100, 1030, 2050), ("int8_product_128_deep", 1503, 2050, 1701),
           ("int8_product_64", 333, 1001, 1003)]
BACKWARD = [("int8_product_256", 2901, 2303, 2507), ("int8_product_128", 2003, 1100, 1701), ("int8_product_128_deep", 1301, 1103, 700),
            ("int8_product_64", 481, 203, 137)]


@pytest.mark.parametrize("tile,m,k,n", FORWARD)
@pytest.mark.parametrize("x_type,y_type,order,relu", [("bf16", "bf16", "rows", True), ("bf16", "f32", "columns", False), ("f32", "bf16", "inside", False)])
def test_forward_tiles(tile, m, k, n, x_type, y_type, order, relu):
    names = ran(lambda: check_linear(m, k, n, x_type, y_type, order, bias=not relu, relu=relu))
    assert names & TILES == {tile}, names


@pytest.mark.parametrize("tile,m,k,n", BACKWARD)
@pytest.mark.parametrize("x_type,w_type,dy_type,order,relu", [("bf16", "bf16", "bf16", "rows", True), ("f32", "f32", "f32", "columns", False)])
def test_backward_tiles(tile, m, k, n, x_type, w_type, dy_type, order, relu):
    names = ran(lambda: check_backward(m, k, n, x_type, w_type, dy_type, order, relu))
    assert names & TILES == {tile}, names


def test_every_tile_is_among_the_cases():
    assert {c[0] for c in FORWARD} == TILES == {c[0] for c in BACKWARD}


@pytest.mark.parametrize("zeros", [False, True])
def test_cells_of_large_tiles_do_not_see_each_other(zeros):
    """One value of x and one channel of w that are not zero: one row and one column of the result, wherever they lie in a tile."""
    m, k, n = 3333, 1030, 4201
    x, w = torch.zeros(m, k, device="cuda"), rand((n, k), 1)
    rows = [0, 31, 32, 127, 128, 255, 256, 3327, 3328, 3332]
    for i, r in enumerate(rows):
        x[r, (i * 131) % k] = 1.0 + i
    wq, ws = st.st_int8_quantize(w)
    out = torch.full((m, n), float("nan"), device="cuda")
    if zeros:
        wq.zero_()
    names = ran(lambda: st.st_int8_linear(x, wq, ws, out=out))
    assert "int8_product_256" in names
    want = torch.zeros(m, n, device="cuda", dtype=torch.float64)
    for i, r in enumerate(rows):
        want[r] = (1.0 + i) * wq[:, (i * 131) % k].double() * ws.double()
    assert ((out.double() - want).abs() <= 6 * EPS * want.abs()).all()


def test_more_tokens_than_a_32_bit_sum_holds_in_large_tiles():
    """The weights' gradient in parts, tiles of 256: column i of dy holds a_i, column j of x holds b_j, so that every cell of dw is its
    own product, tokens * a_i * b_j, and codes are exact."""
    m, k, n = st.ST_INT8_MAX_SUM + 1000, 3601, 3507
    a = rand((n,), 1).to(DT["bf16"])
    b = rand((k,), 2).to(DT["bf16"])
    a, b = torch.where(a == 0, torch.ones_like(a), a), torch.where(b == 0, torch.ones_like(b), b)
    x, dy = b.expand(m, k).contiguous(), a.expand(m, n).contiguous()
    dw, db = torch.empty(n, k, device="cuda"), torch.empty(n, device="cuda")
    names = ran(lambda: st.st_int8_linear_backward(x, None, dy, dw=dw, db=db))
    assert names & TILES == {"int8_product_256"} and "int8_join" in names
    want = m * a.double()[:, None] * b.double()
    assert ((dw.double() - want).abs() <= 10 * EPS * want.abs()).all()
    assert ((db.double() - m * a.double()).abs() <= 72 * EPS * m * a.double().abs()).all()
