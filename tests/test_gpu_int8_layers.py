"""Dense layers in 8-bit integers against the formulas in 64 bits.

Tolerances.  A code is checked to be the nearest whole number but for the roundings of 1/a, the factor 127 and the product (three of
2^-24 on a value of at most 127: 2.3e-5) and the scale to be a/127 but for two (2^-23).  A product of known codes is checked against the
exact sum: int32 -> float32, two scales, the bias: four roundings of 2^-24 of the parts, and the result's own rounding, which is monotone:
a result lies between the roundings of the ends of the interval its unrounded value lies in.  A
whole layer is checked against the unquantised one: every operand is within half a scale (plus the above) of its value, so
|dot - exact| <= sum |da||b| + |a||db| + |da||db|.
"""
import numpy as np
import pytest

import paper_2003_10735_amd as st

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

EPS = 2.0 ** -24
DT = {"f32": torch.float32, "bf16": torch.bfloat16} if hasattr(torch, "float32") else {}
HALF = 0.5 + 3 * 127 * EPS


def rand(shape, seed, dtype="f32", scale=1.0):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return (scale * torch.randn(*shape, device="cuda", generator=g)).to(DT[dtype])


def laid(x, order):
    """The same matrix row by row, column by column, or row by row inside a wider buffer that begins one element off."""
    if order == "rows":
        return x.contiguous()
    if order == "columns":
        return x.t().contiguous().t()
    big = torch.full((x.shape[0], x.shape[1] + 3), float("nan"), dtype=x.dtype, device=x.device)
    big[:, 1:1 + x.shape[1]] = x
    return big[:, 1:1 + x.shape[1]]


def within(y, want, far):
    """Whether y can be the rounding to its type of a value at most `far` from want."""
    lo, hi = ((want + d * far).float().to(y.dtype).double() for d in (-1, 1))
    lo, hi = lo - EPS * lo.abs(), hi + EPS * hi.abs()        # (the ends' own rounding to float32)
    return ((y.double() >= lo) & (y.double() <= hi)).all()


def check_codes(x, q, s):
    x, q, s = x.double(), q.double(), s.double()[:, None]
    top = x.abs().amax(dim=1, keepdim=True)
    assert ((s - top / 127).abs() <= 2 * EPS * top / 127).all()
    assert (q.abs() <= 127).all()
    share = torch.where(top > 0, x / top * 127, torch.zeros_like(x))
    assert ((q - share).abs() <= HALF).all()


@pytest.mark.parametrize("order", ["rows", "columns", "inside"])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("rows,cols", [(1, 1), (1, 300), (3, 15), (5, 16), (64, 129), (65, 1000), (130, 1025), (7, 2049), (3, 9000), (129, 64),
                                       (1000, 40), (300, 513)])
def test_quantized_rows(rows, cols, dtype, order):
    x = rand((rows, cols), rows * 7 + cols, dtype, 3.0)
    if rows > 2:
        x[1] = 0
    pitch = st.int8_pitch(cols)
    q = torch.full((rows, pitch + 256), 77, dtype=torch.int8, device="cuda")
    q, s = st.st_int8_quantize(laid(x, order), q=q)
    check_codes(x, q[:, :cols], s)
    end = (cols + 127) // 128 * 128
    assert (q[:, cols:end] == 0).all() and (q[:, end:] == 77).all()          # zeros up to the multiple of 128, nothing behind it
    q2, s2 = st.st_int8_quantize(laid(x, order))
    assert q2.shape[1] == pitch and torch.equal(q2[:, :cols], q[:, :cols]) and torch.equal(s, s2) and (q2[:, cols:] == 0).all()


@pytest.mark.parametrize("order", ["rows", "columns"])
def test_quantized_rows_of_extreme_values(order):
    x = torch.zeros(10, 200, device="cuda")
    x[0, 5] = float("nan")
    x[1, 199] = float("inf")
    x[2, 0] = float("-inf")
    x[3, 7] = 3e38
    x[4, 9] = -1e-37                      # below 2^-119: zeros
    x[5, 3] = 2.0 ** -118
    x[6, :] = -1.0
    x[7, 0], x[7, 1] = float("inf"), float("nan")
    x[8, 11] = 1e-45
    q, s = st.st_int8_quantize(laid(x, order))
    q, s = q.cpu(), s.cpu()
    assert torch.isnan(s[[0, 1, 2, 7]]).all() and (q[[0, 1, 2, 7]] == 0).all()
    assert q[3, 7] == 127 and abs(s[3].item() * 127 / 3e38 - 1) < 1e-6
    assert (s[[4, 8, 9]] == 0).all() and (q[[4, 8, 9]] == 0).all()
    assert q[5, 3] == 127 and (q[6, :200] == -127).all()


def exact_of(q, s, wq, ws, bias, relu):
    """(y, the size of its parts) of known codes, in 64 bits."""
    k = q.shape[1]
    y = (q.double() @ wq[:, :k].double().t().contiguous()) * s.double()[:, None] * ws.double()
    size = y.abs()
    if bias is not None:
        y = y + bias.double()
        size = size + bias.double().abs()
    return (y.clamp(min=0) if relu else y), size


def weights(n, k, seed):
    """Codes with other numbers behind a row's end, which must not matter."""
    w = rand((n, k), seed, scale=0.1)
    q, s = st.st_int8_quantize(w)
    q[:, k:] = 99
    return w, q, s


def check_linear(m, k, n, x_type="f32", y_type="f32", order="rows", bias=True, relu=False):
    x = rand((m, k), m + 3 * k + 5 * n, x_type, 2.0)
    w, wq, ws = weights(n, k, k + n)
    b = rand((n,), n) if bias else None
    wide = torch.full((m, n + 5), 7.0, dtype=DT[y_type], device="cuda")
    y = st.st_int8_linear(laid(x, order), wq, ws, bias=b, relu=relu, out=wide[:, :n])
    assert (wide[:, n:] == 7.0).all()
    q, s = st.st_int8_quantize(x.contiguous())
    want, size = exact_of(q[:, :k], s, wq, ws, b, relu)
    assert within(y, want, 4 * EPS * size)
    # and the layer that is meant: float x, float weights
    xd, wd = x.double(), w.double()
    dx, dw = s.double()[:, None] * HALF, ws.double() * HALF
    far = dx * wd.abs().sum(1) + xd.abs().sum(1, keepdim=True) * dw + k * dx * dw
    true = xd @ wd.t().contiguous() + (b.double() if bias else 0)
    true = true.clamp(min=0) if relu else true
    assert within(y, true, far * (1 + 1e-6) + 4 * EPS * size)


@pytest.mark.parametrize("m", [1, 2, 5, 8, 15, 16, 17, 32, 33, 63, 64, 65, 129, 300])
@pytest.mark.parametrize("k,n", [(1, 1), (15, 3), (128, 64), (129, 65), (1000, 257)])
def test_linear_sizes(m, k, n):
    check_linear(m, k, n)


@pytest.mark.parametrize("x_type", ["f32", "bf16"])
@pytest.mark.parametrize("y_type", ["f32", "bf16"])
@pytest.mark.parametrize("order", ["rows", "columns", "inside"])
@pytest.mark.parametrize("m,k,n", [(1, 515, 130), (7, 2048, 96), (40, 4100, 50), (200, 300, 400)])
def test_linear_types_and_orders(m, k, n, x_type, y_type, order):
    check_linear(m, k, n, x_type, y_type, order, bias=order != "columns", relu=order == "rows")


@pytest.mark.parametrize("m,k,n", [(3000, 130, 4200), (1700, 300, 2000), (5000, 64, 31), (2100, 1030, 2050), (1, 9000, 5000), (16, 3000, 7001)])
def test_linear_large_tiles_and_splits(m, k, n):
    check_linear(m, k, n, "bf16", "bf16", relu=True)
    check_linear(m, k, n, "bf16", "f32", bias=False)


@pytest.mark.parametrize("k", [1, 16, 63, 64, 65, 128, 129, 250, 256, 257, 512, 513])
@pytest.mark.parametrize("n", [1, 32, 33, 120, 128, 129, 256, 257])
def test_linear_narrow_layers(k, n):
    """Around the sizes up to which a block takes a layer whole."""
    for m, x_type, y_type, order in ((65, "bf16", "f32", "rows"), (97, "f32", "bf16", "inside"), (1000, "bf16", "bf16", "rows")):
        check_linear(m, k, n, x_type, y_type, order, bias=m != 97, relu=m == 1000)


@pytest.mark.parametrize("m", [1, 2, 3, 4, 5, 7, 8, 9, 11, 16])
@pytest.mark.parametrize("k", [4, 200, 511, 512, 513, 1024, 2056, 4096, 4104, 8200, 32768, 40000])
def test_linear_few_tokens(m, k):
    """Around the sizes up to which every block quantises the tokens itself, in both types, aligned and not."""
    check_linear(m, k, 50, "bf16", "f32")
    check_linear(m, k, 17, "f32", "bf16", "inside")
    check_linear(m, k, 33, "bf16" if m % 2 else "f32", "f32", "columns")


@pytest.mark.parametrize("m", [1, 70])
def test_longest_sum_fits_32_bits(m):
    k, n = st.ST_INT8_MAX_SUM, 20
    x = torch.full((m, k), -2.0, device="cuda")
    wq = torch.full((n, st.int8_pitch(k)), -128, dtype=torch.int8, device="cuda")
    ws = torch.ones(n, device="cuda")
    y = st.st_int8_linear(x, wq, ws)
    want = 127.0 * 128 * k * 2 / 127
    assert ((y.double() - want).abs() <= 6 * EPS * want).all()


def test_linear_keeps_rows_apart():
    """A row that holds a NaN spoils itself only; a row of zeros gives the bias; a NaN passes ReLU."""
    x = rand((70, 200), 1)
    x[3, 7], x[5, 0], x[6] = float("nan"), float("inf"), 0.0
    _, wq, ws = weights(90, 200, 2)
    b = rand((90,), 3)
    y = st.st_int8_linear(x, wq, ws, bias=b, relu=True)
    assert torch.isnan(y[[3, 5]]).all() and torch.equal(y[6], b.clamp(min=0))
    keep = [i for i in range(70) if i not in (3, 5)]
    assert torch.isfinite(y[keep]).all()
    one = st.st_int8_linear(x[4:5], wq, ws, bias=b, relu=True)
    assert torch.equal(one[0], y[4])                  # however many tokens come along: exact sums
    few = st.st_int8_linear(x[:9], wq, ws, bias=b, relu=True)
    assert torch.equal(few[6:9], y[6:9]) and torch.isnan(few[[3, 5]]).all()


def test_linear_without_tokens():
    _, wq, ws = weights(5, 40, 2)
    assert st.st_int8_linear(torch.empty(0, 40, device="cuda"), wq, ws).shape == (0, 5)


def test_rows_broadcast_over_tokens():
    """One token for all rows (a stride of 0)."""
    _, wq, ws = weights(33, 40, 2)
    x = rand((1, 40), 5)
    y = st.st_int8_linear(x.expand(100, 40), wq, ws)
    assert torch.equal(y, st.st_int8_linear(x, wq, ws).expand(100, 33))


# ------------------------------------------------------------------------------------------------------------ backward
def check_backward(m, k, n, x_type, w_type, dy_type, order="rows", relu=False, dx_type=None):
    x, w = rand((m, k), 1 + m, x_type, 2.0), rand((n, k), 2 + n, w_type, 0.1)
    dy = rand((m, n), 3 + k, dy_type, 1e-3)
    y = rand((m, n), 4, "bf16") if relu else None
    dx = torch.full((m, k + 2), 7.0, dtype=DT[dx_type or x_type], device="cuda")
    dw = torch.full((n, k + 3), 7.0, device="cuda")
    db = torch.empty(n, device="cuda")
    args = [laid(t, order) for t in (x, w, dy)]
    st.st_int8_linear_backward(*args, y=None if y is None else laid(y, order), dx=dx[:, :k], dw=dw[:, :k], db=db)
    assert (dx[:, k:] == 7.0).all() and (dw[:, k:] == 7.0).all()
    dz = dy.double()
    if relu:
        dz = dz * (y > 0)
    xd, wd = x.double(), w.double()

    def scales(t, dim):
        return t.abs().amax(dim=dim) / 127

    def bound(a, b, sa, sb, length):          # a [r, length], b [c, length]
        da, db_ = sa[:, None] * HALF, sb * HALF
        return da * b.abs().sum(1) + a.abs().sum(1, keepdim=True) * db_ + length * da * db_

    want = dz @ wd
    far = bound(dz, wd.t(), scales(dz, 1), scales(wd, 0), n) + 8 * EPS * (dz.abs() @ wd.abs())
    assert within(dx[:, :k], want, far * (1 + 1e-6))
    want = dz.t().contiguous() @ xd
    far = bound(dz.t(), xd.t(), scales(dz, 0), scales(xd, 0), m) + 8 * EPS * (dz.abs().t().contiguous() @ xd.abs())
    assert ((dw[:, :k].double() - want).abs() <= far * (1 + 1e-5)).all()
    # float32 sums of 64 values and of the parts' halves, float64 above them: 64 + 8 roundings at the very most
    assert ((db.double() - dz.sum(0)).abs() <= 72 * EPS * dz.abs().sum(0)).all()
    return x, w, dy, y, dx[:, :k], dw[:, :k], db


@pytest.mark.parametrize("order", ["rows", "columns", "inside"])
@pytest.mark.parametrize("m,k,n", [(1, 1, 1), (1, 200, 70), (2, 17, 33), (63, 128, 64), (130, 65, 129), (700, 100, 30), (300, 1000, 257)])
@pytest.mark.parametrize("relu", [False, True])
def test_backward(m, k, n, order, relu):
    check_backward(m, k, n, "f32", "f32", "f32", order, relu)


@pytest.mark.parametrize("x_type", ["f32", "bf16"])
@pytest.mark.parametrize("w_type", ["f32", "bf16"])
@pytest.mark.parametrize("dy_type", ["f32", "bf16"])
def test_backward_types(x_type, w_type, dy_type):
    check_backward(260, 140, 90, x_type, w_type, dy_type, relu=True)
    check_backward(260, 140, 90, x_type, w_type, dy_type, order="columns", dx_type="f32")


def test_backward_large():
    check_backward(2300, 2200, 2100, "bf16", "bf16", "bf16", relu=True)


@pytest.mark.parametrize("order", ["rows", "columns"])
def test_many_tokens(order):
    """Backward: tiles of 128, and the weights' gradient, whose blocks would outlast the other product's, in two parts.  Forward: the same
    tiles."""
    check_backward(5930, 657, 1331, "bf16", "f32", "bf16", order, relu=True)
    check_linear(5001, 1100, 450, "bf16", "bf16", order)


def test_more_tokens_than_a_32_bit_sum_holds():
    m = st.ST_INT8_MAX_SUM + 9000
    x, dy = torch.full((m, 3), 2.0, device="cuda"), torch.full((m, 2), -3.0, device="cuda")
    dw, db = torch.empty(2, 3, device="cuda"), torch.empty(2, device="cuda")
    st.st_int8_linear_backward(x, None, dy, dw=dw, db=db)
    assert ((dw.double() + 6.0 * m).abs() <= 8 * EPS * 6 * m).all() and ((db.double() + 3.0 * m).abs() <= 4 * EPS * 3 * m).all()


def test_each_output_alone_is_the_same():
    x, w, dy, y, dx, dw, db = check_backward(333, 190, 70, "bf16", "f32", "f32", relu=True)
    a = st.st_int8_linear_backward(None, w, dy, y=y, dx=torch.empty_like(x))[0]
    b = st.st_int8_linear_backward(x, None, dy, y=y, dw=torch.empty_like(w))[1]
    c = st.st_int8_linear_backward(None, None, dy, y=y, db=torch.empty(70, device="cuda"))[2]
    assert torch.equal(a, dx) and torch.equal(b, dw) and ((c - db).abs() <= 4 * EPS * dy.abs().sum(0)).all()


def test_masked_out_rows_and_values():
    """A token whose mask leaves nothing, and infinities and NaN where the mask lets nothing through."""
    m, k, n = 40, 64, 48
    x, w, dy, y = rand((m, k), 1), rand((n, k), 2), rand((m, n), 3), rand((m, n), 4)
    y[5], y[:, 7], y[9, 3], y[11, 2] = -1.0, 0.0, -2.0, float("nan")
    clean = dy * (y > 0)
    dy[9, 3], dy[5, 1], dy[20, 7], dy[11, 2] = float("inf"), float("nan"), float("-inf"), float("nan")
    outs = [st.st_int8_linear_backward(x, w, d, y=t, dx=torch.empty_like(x), dw=torch.empty_like(w), db=torch.empty(n, device="cuda"))
            for d, t in ((dy, y), (clean, None))]
    for a, b in zip(*outs):
        assert torch.equal(a, b)
    assert (outs[0][0][5] == 0).all() and (outs[0][1][7] == 0).all() and outs[0][2][7] == 0


def test_backward_without_tokens():
    dw, db = torch.full((6, 4), 9.0, device="cuda"), torch.full((6,), 9.0, device="cuda")
    st.st_int8_linear_backward(torch.empty(0, 4, device="cuda"), rand((6, 4), 1), torch.empty(0, 6, device="cuda"),
                               dx=torch.empty(0, 4, device="cuda"), dw=dw, db=db)
    assert (dw == 0).all() and (db == 0).all()


@pytest.mark.parametrize("seed", [1, 2, 3])
def test_gradients_against_differences(seed):
    """d/dt of L(x + t u, w + t z) = sum c * relu(x w^T + b): a difference quotient in 64 bits, and the library's gradients along (u, z).
    The quantisation error is bounded as above, along the direction."""
    m, k, n = 50, 70, 40
    x, w, b, c = rand((m, k), seed), rand((n, k), seed + 10, scale=0.2), rand((n,), seed + 20), rand((m, n), seed + 30)
    u, z, e = rand((m, k), seed + 40), rand((n, k), seed + 50, scale=0.2), rand((n,), seed + 60)
    pre = x.double() @ w.double().t().contiguous() + b.double()
    y = pre.clamp(min=0).float()

    def loss(t):
        h = (x.double() + t * u.double()) @ (w.double() + t * z.double()).t().contiguous() + b.double() + t * e.double()
        return (c.double() * torch.where(y > 0, h, torch.zeros_like(h))).sum()       # (the kink stays where it is)

    t = 1e-4
    quotient = (loss(t) - loss(-t)) / (2 * t)            # exact up to t^2 terms that cancel: L is quadratic in t
    dx, dw, db = st.st_int8_linear_backward(x, w, c, y=y, dx=torch.empty_like(x), dw=torch.empty_like(w), db=torch.empty(n, device="cuda"))
    along = (dx.double() * u.double()).sum() + (dw.double() * z.double()).sum() + (db.double() * e.double()).sum()
    dz, xd, wd = c.double() * (y > 0), x.double(), w.double()
    s1, s2 = dz.abs().amax(1) / 127 * HALF, wd.abs().amax(0) / 127 * HALF
    far_x = s1[:, None] * wd.abs().sum(0) + dz.abs().sum(1, keepdim=True) * s2 + n * s1[:, None] * s2
    s3, s4 = dz.abs().amax(0) / 127 * HALF, xd.abs().amax(0) / 127 * HALF
    far_w = s3[:, None] * xd.abs().sum(0) + dz.abs().sum(0)[:, None] * s4 + m * s3[:, None] * s4
    far = (far_x * u.double().abs()).sum() + (far_w * z.double().abs()).sum() + 1e-5 * (db.double() * e.double()).abs().sum()
    assert (along - quotient).abs() <= far
    # the bound is of the size of the worst case; the errors are random, and their sum is a small part of the derivative's parts
    parts = ((dx.double() * u.double()).square().sum() + (dw.double() * z.double()).square().sum()).sqrt()
    assert (along - quotient).abs() <= 0.1 * parts


# ------------------------------------------------------------------------------------------------------------- streams
def test_other_stream_and_graph():
    x, w, dy = rand((200, 300), 1, "bf16"), rand((150, 300), 2), rand((200, 150), 3, "bf16")
    wq, ws = st.st_int8_quantize(w)
    work, back = st.new_int8_workspace(200, 150, 300), st.new_int8_workspace(200, 150, 300, backward=True)
    y = torch.empty(200, 150, device="cuda")
    outs = [torch.empty(200, 300, device="cuda"), torch.empty(150, 300, device="cuda"), torch.empty(150, device="cuda")]

    def call():
        st.st_int8_linear(x, wq, ws, out=y, workspace=work)
        st.st_int8_linear_backward(x, w, dy, dx=outs[0], dw=outs[1], db=outs[2], workspace=back)

    call()
    torch.cuda.synchronize()
    want = [t.clone() for t in [y] + outs]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        for t in [y] + outs:
            t.zero_()
        call()
    side.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(want, [y] + outs))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call()
    for i in range(3):
        x.copy_(rand((200, 300), 100 + i, "bf16"))
        for t in [y] + outs:
            t.fill_(3.0)
        graph.replay()
        torch.cuda.synchronize()
        got = [t.clone() for t in [y] + outs]
        call()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(got, [y] + outs)), i


def test_offsets_that_pass_32_bits():
    """More than 2^31 values of x, of its codes, and of the result: rows at the end are what the same rows are alone."""
    m, k, n = 40000, 60000, 17
    base = rand((8, k), 1, "bf16")
    x = base.repeat(m // 8, 1)
    _, wq, ws = weights(n, k, 2)
    y = st.st_int8_linear(x, wq, ws, out_dtype=torch.float32)
    alone = st.st_int8_linear(base, wq, ws, out_dtype=torch.float32)
    for first in (0, 35784, m - 8):          # 35784 * k is where 31 bits end
        assert torch.equal(y[first:first + 8], alone)
    q, s = st.st_int8_quantize(x)
    q1, s1 = st.st_int8_quantize(base)
    assert torch.equal(q[m - 8:], q1) and torch.equal(s[m - 8:], s1)
    del x, q
    m, n = 70000, 33000
    x = base[:, :64].contiguous().repeat(m // 8, 1)
    _, wq, ws = weights(n, 64, 3)
    y = st.st_int8_linear(x, wq, ws)
    alone = st.st_int8_linear(base[:, :64].contiguous(), wq, ws)
    for first in (0, 65072, m - 8):
        assert torch.equal(y[first:first + 8], alone)


def test_host_tensors_and_small_workspaces_are_refused():
    x, dy = rand((40, 64), 1), rand((40, 32), 2)
    w = rand((32, 64), 3)
    wq, ws = st.st_int8_quantize(w)
    small = torch.empty(256, dtype=torch.uint8, device="cuda")
    dw = torch.empty_like(w)
    calls = [lambda: st.st_int8_quantize(x.cpu()), lambda: st.st_int8_quantize(x, q=wq.new_empty((40, 64)).cpu()),
             lambda: st.st_int8_quantize(x.t(), workspace=small), lambda: st.st_int8_linear(x.cpu(), wq, ws, out=dy),
             lambda: st.st_int8_linear(x, wq.cpu(), ws), lambda: st.st_int8_linear(x, wq, ws.cpu()),
             lambda: st.st_int8_linear(x, wq, ws, bias=torch.zeros(32)), lambda: st.st_int8_linear(x, wq, ws, out=dy.cpu()),
             lambda: st.st_int8_linear(x, wq, ws, workspace=small), lambda: st.st_int8_linear_backward(x, w, dy.cpu(), dw=dw),
             lambda: st.st_int8_linear_backward(x, w, dy, dw=dw.cpu()), lambda: st.st_int8_linear_backward(x, w, dy, dw=dw, workspace=small)]
    for call in calls:
        with pytest.raises(st.StError):
            call()
