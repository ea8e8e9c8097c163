"""One token, whose values may lie any number of elements apart: every operand is read with its own step.

A single row has no pitch, so a row of a column-ordered matrix ([1, n] with strides (1, p)), one value for all channels ([1, n] with
strides (1, 0)) and a contiguous row are all rows; what a call gives for them is bit for bit what it gives for contiguous copies."""
import pytest

import paper_2003_10735_amd as st

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

DT = {"f32": torch.float32, "bf16": torch.bfloat16}
LAYOUTS = ["contiguous", "strided", "expanded"]


def row(n, seed, dtype, layout, scale=1.0):
    """[1, n]: one of the rows of a column-ordered matrix whose other rows are NaN, or one value n times."""
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    x = (scale * torch.randn(1, n, device="cuda", generator=g)).to(DT[dtype])
    if layout == "strided":
        whole = torch.full((n, 3), float("nan"), dtype=DT[dtype], device="cuda")
        whole[:, 1] = x[0]
        x = whole.t()[1:2]
        assert x.stride() == (1, 3)
    elif layout == "expanded":
        x = x[:, :1].expand(1, n)
        assert x.stride(1) == 0
    return x


@pytest.mark.parametrize("y_layout", LAYOUTS)
@pytest.mark.parametrize("dy_layout", LAYOUTS)
@pytest.mark.parametrize("n", [2, 9, 70, 1030])
def test_mask_of_one_token(n, dy_layout, y_layout):
    k = 48
    g = torch.Generator(device="cuda")
    g.manual_seed(n)
    w = torch.randn(n, k, device="cuda", generator=g)
    for seed, dy_type, y_type in ((1, "f32", "bf16"), (2, "bf16", "f32"), (3, "f32", "f32"), (4, "bf16", "bf16")):
        x = row(k, 10 + seed, "f32", "contiguous")
        dy, y = row(n, 20 + seed, dy_type, dy_layout), row(n, 30 + seed, y_type, y_layout)
        outs = [st.st_int8_linear_backward(x, w, a, y=b, dx=torch.full_like(x, 7.0), dw=torch.full_like(w, 7.0), db=torch.full((n,), 7.0, device="cuda"))
                for a, b in ((dy, y), (dy.clone(memory_format=torch.contiguous_format), y.clone(memory_format=torch.contiguous_format)))]
        for a, b in zip(*outs):
            assert torch.isfinite(b).all() and torch.equal(a, b)
        dz = torch.where(y > 0, dy.float(), torch.zeros_like(dy.float()))
        assert torch.equal(outs[0][2], dz[0])              # one token: the sum is its value
        for i, given in enumerate((dict(dx=torch.empty_like(x)), dict(dw=torch.empty_like(w)), dict(db=torch.empty(n, device="cuda")))):
            alone = st.st_int8_linear_backward(x if i == 1 else None, w if i == 0 else None, dy, y=y, **given)
            assert torch.equal(alone[i], outs[1][i])


@pytest.mark.parametrize("layout", LAYOUTS[1:])
@pytest.mark.parametrize("k", [2, 7, 200, 5000, 40000])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_token_of_any_step(k, dtype, layout):
    x = row(k, k, dtype, layout)
    c = x.clone(memory_format=torch.contiguous_format)
    assert x.stride(1) != 1 and c.stride(1) == 1
    (q, s), (q1, s1) = st.st_int8_quantize(x), st.st_int8_quantize(c)
    assert torch.equal(q, q1) and torch.equal(s, s1)
    g = torch.Generator(device="cuda")
    g.manual_seed(k)
    wq, ws = st.st_int8_quantize(torch.randn(35, k, device="cuda", generator=g))
    assert torch.equal(st.st_int8_linear(x, wq, ws), st.st_int8_linear(c, wq, ws))
    dy, dw = row(35, 3, "f32", "contiguous"), [torch.empty(35, k, device="cuda") for _ in range(2)]
    for a, out in zip((x, c), dw):
        st.st_int8_linear_backward(a, None, dy, dw=out)
    assert torch.equal(*dw)
