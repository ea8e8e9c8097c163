"""The norm of many gradients and clipping by it, against 64 bits.

Tolerances: the norm's squares and sums are float64, so it is the float32 nearest to the exact one but for a last place; a factor is
max_norm / norm in float64, rounded to float32 (2^-24), a result one product and its type's rounding.
"""
import math

import pytest

import paper_2003_10735_amd as st

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

EPS = 2.0 ** -24
F, B = torch.float32, torch.bfloat16


def make(sizes, types, seed=0, scale=1.0, off=1):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return [(scale * torch.randn(n + off, device="cuda", generator=g)).to(types[i % len(types)])[off:] for i, n in enumerate(sizes)]


def norm64(grads):
    return math.sqrt(sum(float(g.double().square().sum()) for g in grads))


def check(grads, outs, norm, max_norm, scale):
    want = norm64(grads) * scale
    assert abs(float(norm) - want) <= 2 * EPS * want
    c = scale * (max_norm / want if 0 < max_norm < want else 1.0)
    for g, o in zip(grads, outs):
        v = g.double() * c
        half = 2.0 ** -8 if o.dtype == B else EPS
        assert ((o.double() - v).abs() <= (half + 3 * EPS) * v.abs()).all()


SIZES = [(1,), (7, 0, 1000), (2048, 2049, 8191, 8192, 8193), tuple(range(300)), (3000001, 5, 70000), (20000000, 3)]


@pytest.mark.parametrize("out", [None, F, B])
@pytest.mark.parametrize("types", [(F,), (B,), (F, B)])
@pytest.mark.parametrize("sizes", SIZES)
def test_norm_and_clipping(sizes, types, out):
    grads = make(sizes, types)
    before = [g.clone() for g in grads]
    outs = [torch.full((n + 2,), 7.0, dtype=out, device="cuda") for n in sizes] if out else None
    tensors = st.GradTensors(grads, [o[1:1 + n] for o, n in zip(outs, sizes)] if out else None)
    norm = torch.empty(1, device="cuda")
    want = norm64(grads)
    for max_norm, scale in ((0.3 * want, 1.0), (0.0, 0.125), (0.01 * want, 0.125), (2.0 * want, 1.0)):
        if out is None:
            for g, b in zip(grads, before):
                g.copy_(b)
        st.st_grad_clip(tensors, max_norm, scale, norm, workspace=st.new_grad_workspace(tensors))
        check(before, [o[1:1 + n] for o, n in zip(outs, sizes)] if out else grads, norm, max_norm, scale)
        if out:
            assert all(torch.equal(g, b) for g, b in zip(grads, before)) and all(float(o[0]) == 7 and float(o[-1]) == 7 for o in outs)


def test_the_norm_alone():
    grads = make((5000, 31), (F, B))
    norm = torch.empty(1, device="cuda")
    array = (st.StGradTensor * 2)(*[st.StGradTensor(g.data_ptr(), None, g.numel(), st._dtype(g, ""), 0) for g in grads])
    ws = torch.empty(st.lib().st_grad_clip_workspace(array, 2), dtype=torch.uint8, device="cuda")
    before = [g.clone() for g in grads]
    assert st.lib().st_grad_clip(array, 2, 2.0, 1.0, norm.data_ptr(), ws.data_ptr(), torch.cuda.current_stream().cuda_stream) == st.ST_OK
    assert abs(float(norm) - 2 * norm64(grads)) <= 4 * EPS * float(norm) and all(torch.equal(a, b) for a, b in zip(grads, before))
    empty = st.GradTensors([torch.empty(0, device="cuda")])
    st.st_grad_clip(empty, 1.0, grad_norm=norm)
    assert float(norm) == 0.0


@pytest.mark.parametrize("value", [3e38, 1e-38, 1e-44])
def test_squares_neither_overflow_nor_vanish(value):
    g = torch.full((100,), value, device="cuda")
    want = norm64([g])
    norm, out = torch.empty(1, device="cuda"), torch.empty(100, device="cuda")
    st.st_grad_clip(st.GradTensors([g], [out]), 1.0, grad_norm=norm)
    if want > 3.4e38:
        assert math.isinf(float(norm))      # the norm is more than float32 holds, the gradients are clipped by it all the same
    else:
        assert abs(float(norm) - want) <= max(2 * EPS * want, 1e-45)
    c = min(1.0, 1.0 / want)
    assert ((out.double() - g.double() * c).abs() <= 4 * EPS * g.double() * c + 1.5e-45).all()


@pytest.mark.parametrize("bad", [float("nan"), float("inf"), float("-inf")])
def test_a_norm_that_is_not_finite_clips_nothing(bad):
    grads = make((3000, 40), (F, B))
    grads[1][7] = bad
    outs = [torch.empty_like(g) for g in grads]
    norm = torch.empty(1, device="cuda")
    st.st_grad_clip(st.GradTensors(grads, outs), 1e-3, 0.5, norm)
    assert not math.isfinite(float(norm))
    assert torch.equal(outs[0], grads[0] * 0.5) and torch.equal(torch.nan_to_num(outs[1]), torch.nan_to_num(grads[1] * 0.5))


def test_results_do_not_depend_on_the_order_of_work():
    grads = make((300000, 77, 9000), (B, F))
    outs = [torch.empty_like(g) for g in grads]
    tensors, norms = st.GradTensors(grads, outs), []
    for _ in range(5):
        norm = torch.empty(1, device="cuda")
        st.st_grad_clip(tensors, 1.0, grad_norm=norm)
        norms.append((float(norm), [o.clone() for o in outs]))
    assert all(n == norms[0][0] and all(torch.equal(a, b) for a, b in zip(o, norms[0][1])) for n, o in norms)
