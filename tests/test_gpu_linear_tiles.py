"""Every tile of the dense layers, with and without a contraction in parts, in both directions and types: results of whole numbers are exact, and the
kernel profile says that it was this tile that ran."""
import pytest

import paper_2003_10735_amd as st

from test_gpu_linear import laid, mm64, whole

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

# Sizes for which the choice of a form takes each of them, the odd ones by way of copies or of the loose tile.  (The choice goes by measured times: where
# those change, sizes have to be found again.)
CASES = [
    ("forward", "bf16", 6784, 520, 64, "product_128", False), ("forward", "bf16", 4176, 80, 4704, "product_128", True),
    ("forward", "bf16", 72, 8960, 64, "product_128_deep", False), ("forward", "bf16", 1088, 80, 8896, "product_128_deep", True),
    ("forward", "bf16", 7688, 1976, 72, "product_256", False), ("forward", "bf16", 4528, 1552, 6624, "product_256", True),
    ("forward", "bf16", 64, 64, 232, "small", False), ("forward", "bf16", 64, 64, 2648, "small", True),
    ("forward", "bf16", 64, 64, 72, "product_64", False), ("forward", "bf16", 336, 72, 4120, "product_64", True),
    ("backward", "bf16", 288, 64, 8592, "product_128", False), ("backward", "bf16", 72, 8616, 408, "product_128", True),
    ("backward", "bf16", 72, 80, 6616, "product_128_deep", False), ("backward", "bf16", 272, 8784, 136, "product_128_deep", True),
    ("backward", "bf16", 640, 704, 8920, "product_256", False), ("backward", "bf16", 920, 7512, 1000, "product_256", True),
    ("backward", "bf16", 200, 64, 64, "small", False), ("backward", "bf16", 2736, 64, 64, "small", True),
    ("backward", "bf16", 64, 64, 64, "product_64", False), ("backward", "bf16", 64, 4936, 72, "product_64", True),
    ("two terms", "bf16", 280, 72, 8408, "product_128", False), ("two terms", "bf16", 80, 4584, 528, "product_128", True),
    ("two terms", "bf16", 72, 88, 7808, "product_128_deep", False), ("two terms", "bf16", 536, 4128, 72, "product_128_deep", True),
    ("two terms", "bf16", 552, 688, 8936, "product_256", False), ("two terms", "bf16", 4568, 136, 4080, "product_256", True),
    ("two terms", "bf16", 64, 104, 64, "small", False), ("two terms", "bf16", 64, 1432, 64, "small", True),
    ("two terms", "bf16", 72, 64, 72, "product_64", False), ("two terms", "bf16", 2040, 72, 88, "product_64", True),
    ("forward", "f32", 992, 5296, 64, "product_128", False), ("forward", "f32", 6152, 104, 3264, "product_128", True),
    ("forward", "f32", 4872, 600, 64, "product_128_deep", False), ("forward", "f32", 72, 3952, 3504, "product_128_deep", True),
    ("forward", "f32", 7056, 1704, 64, "product_256", False), ("forward", "f32", 7888, 240, 6584, "product_256", True),
    ("forward", "f32", 64, 64, 64, "small", False), ("forward", "f32", 72, 72, 1024, "small", True),
    ("forward", "f32", 2112, 104, 64, "product_64", False), ("forward", "f32", 328, 72, 4144, "product_64", True),
    ("backward", "f32", 592, 208, 7408, "product_128", False), ("backward", "f32", 4872, 72, 936, "product_128", True),
    ("backward", "f32", 184, 208, 8056, "product_128_deep", False), ("backward", "f32", 936, 4992, 72, "product_128_deep", True),
    ("backward", "f32", 1024, 944, 7312, "product_256", False), ("backward", "f32", 400, 6464, 984, "product_256", True),
    ("backward", "f32", 64, 64, 64, "small", False), ("backward", "f32", 72, 1040, 64, "small", True),
    ("backward", "f32", 64, 72, 1808, "product_64", False), ("backward", "f32", 64, 8192, 80, "product_64", True),
    ("forward", "bf16", 8397, 393, 69, "product_128", False), ("forward", "bf16", 233, 2137, 5989, "product_128", True),
    ("forward", "bf16", 337, 4369, 65, "product_128_deep", False), ("forward", "bf16", 547, 451, 6181, "product_128_deep", True),
    ("forward", "bf16", 2491, 6369, 65, "product_256", False), ("forward", "bf16", 7653, 899, 6691, "product_256", True),
    ("forward", "bf16", 73, 73, 65, "small_loose", False), ("forward", "bf16", 75, 69, 2699, "small_loose", True),
    ("forward", "bf16", 67, 5653, 67, "product_64", False), ("forward", "bf16", 1077, 419, 7381, "product_64", True),
    ("backward", "bf16", 137, 129, 8277, "product_128", False), ("backward", "bf16", 69, 8141, 401, "product_128", True),
    ("backward", "bf16", 67, 65, 7075, "product_128_deep", False), ("backward", "bf16", 1123, 4497, 67, "product_128_deep", True),
    ("backward", "bf16", 817, 691, 8069, "product_256", False), ("backward", "bf16", 6131, 139, 6403, "product_256", True),
    ("backward", "bf16", 137, 65, 65, "small_loose", False), ("backward", "bf16", 65, 2821, 69, "small_loose", True),
    ("backward", "bf16", 69, 65, 65, "product_64", False), ("backward", "bf16", 69, 5019, 67, "product_64", True),
    ("two terms", "bf16", 129, 147, 8493, "product_128", False), ("two terms", "bf16", 67, 8729, 265, "product_128", True),
    ("two terms", "bf16", 73, 67, 7693, "product_128_deep", False), ("two terms", "bf16", 4105, 525, 67, "product_128_deep", True),
    ("two terms", "bf16", 843, 701, 7683, "product_256", False), ("two terms", "bf16", 5195, 3323, 131, "product_256", True),
    ("two terms", "bf16", 65, 65, 101, "small_loose", False), ("two terms", "bf16", 69, 1501, 65, "small_loose", True),
    ("two terms", "bf16", 65, 69, 67, "product_64", False), ("two terms", "bf16", 2163, 99, 75, "product_64", True),
    ("forward", "f32", 2339, 2213, 65, "product_128", False), ("forward", "f32", 1251, 617, 4051, "product_128", True),
    ("forward", "f32", 5595, 523, 65, "product_128_deep", False), ("forward", "f32", 1193, 669, 4091, "product_128_deep", True),
    ("forward", "f32", 3281, 3749, 65, "product_256", False), ("forward", "f32", 3909, 441, 6333, "product_256", True),
    ("forward", "f32", 67, 75, 69, "small_loose", False), ("forward", "f32", 73, 67, 1057, "small_loose", True),
    ("forward", "f32", 99, 4341, 65, "product_64", False), ("forward", "f32", 817, 931, 2821, "product_64", True),
    ("backward", "f32", 293, 323, 8987, "product_128", False), ("backward", "f32", 67, 4085, 1093, "product_128", True),
    ("backward", "f32", 197, 205, 6429, "product_128_deep", False), ("backward", "f32", 4723, 297, 323, "product_128_deep", True),
    ("backward", "f32", 923, 931, 7781, "product_256", False), ("backward", "f32", 8497, 129, 2517, "product_256", True),
    ("backward", "f32", 67, 69, 67, "small_loose", False), ("backward", "f32", 1065, 65, 69, "small_loose", True),
    ("backward", "f32", 69, 65, 1355, "product_64", False), ("backward", "f32", 8235, 67, 67, "product_64", True),
]


def kernels(call):
    st.st_profile_enable(True)
    st.st_profile_reset()
    call()
    torch.cuda.synchronize()
    names = set(st.st_profile_read())
    st.st_profile_enable(False)
    st.st_profile_reset()
    return names


def check_names(names, kernel, joined):
    assert {n for n in names if n.startswith(("linear_small", "linear_product", "linear_few"))} == {"linear_" + kernel}
    assert ("linear_join" in names) == joined


@pytest.mark.parametrize("order", ["rows", "columns"])
@pytest.mark.parametrize("kind,dtype,m,n,k,kernel,joined", CASES)
def test_tiles(kind, dtype, m, n, k, kernel, joined, order):
    """(Two terms: gradients of ten bits, which one bfloat16 does not hold, beside operands of -1 .. 1; all sums stay below 2^24.)"""
    most = 1 if kind == "two terms" else 2
    x, w = whole((m, k), 1, dtype, most), whole((n, k), 2, dtype, most)
    if kind == "forward":
        b, r = whole((n,), 3, "f32"), whole((m, n), 4, "bf16")
        y = torch.full((m, n), 7.0, device="cuda")
        check_names(kernels(lambda: st.st_linear(laid(x, order), laid(w, order), b, residual=r, out=y)), kernel, joined)
        assert torch.equal(y.double(), mm64(x, w) + b.double() + r.double())
        return
    dy, z = whole((m, n), 3, "f32", 700) if kind == "two terms" else whole((m, n), 3, dtype), whole((m, n), 4, "bf16")
    dz = dy.double() * (z > 0)
    dx, dw, db = torch.full((m, k), 7.0, device="cuda"), torch.ones(n, k, device="cuda"), torch.ones(n, device="cuda")
    check_names(kernels(lambda: st.st_linear_backward(laid(x, order), laid(w, order), dy, z, st.ST_ACT_RELU, dx, dw, db, accumulate=True)), kernel, joined)
    assert torch.equal(dx.double(), mm64(dz, w.t())) and torch.equal(dw.double(), mm64(dz.t(), x.t()) + 1) and torch.equal(db.double(), dz.sum(0) + 1)
