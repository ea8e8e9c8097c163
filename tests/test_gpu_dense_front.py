"""A 1x1 layer trained together with the head: the 8-bit products, the head's full backward pass and the optimiser in one path."""
import numpy as np
import pytest

import paper_2003_10735_amd as st
import workloads as WL

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu


def setup(n=1, c_front=96, seed=0):
    wl = WL.small_variant(WL.WORKLOADS["720p"], n=n, h=12, w=20, c_in=64, c1=64, c2=64, steps=2, n_sites=9)
    desc = st.HeadDesc.of(wl)
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    cells = torch.randn(n * wl.h * wl.w, c_front, device="cuda", generator=g).clamp(min=0).bfloat16()
    weight = torch.randn(wl.c_in, c_front, device="cuda", generator=g) / c_front ** 0.5
    bias = torch.zeros(wl.c_in, device="cuda")
    labels = torch.from_numpy(WL.make_labels(wl)).cuda()
    head = torch.from_numpy(WL.make_head_params(wl).astype(np.float32)).cuda()
    return desc, cells, weight, bias, labels, head


@pytest.mark.parametrize("bits", [8, 32])
@pytest.mark.parametrize("n", [1, 2])
def test_training_the_layer_lowers_the_loss(bits, n):
    from paper_2003_10735_amd.dense import DenseFront
    desc, cells, weight, bias, labels, head = setup(n)
    front = DenseFront(desc, weight, bias, lr=3e-3, weight_decay=0.01, max_norm=1.0, state_bits=bits)
    losses = [float(front.step(cells, labels, head, head_lr=0.0)) for _ in range(30)]      # the head stays: what falls is the layer's doing
    assert np.isfinite(losses).all() and losses[-1] < 0.8 * losses[0], losses
    assert torch.isfinite(front.grad_norm).all()


def test_gradients_of_the_layer_follow_the_head():
    """dw and db of the first step against the head's own gradient of the features, in 64 bits: each operand of dw is within half a scale
    of its value."""
    from paper_2003_10735_amd.dense import DenseFront
    desc, cells, weight, bias, labels, head = setup()
    front = DenseFront(desc, weight, bias, lr=0.0)
    front.step(cells, labels, head, head_lr=0.0)
    g = front.feature_grad[0].reshape(desc.c_in, -1).double()            # [c, cells]
    x = cells.double()
    assert ((front.grads[1].double() - g.sum(1)).abs() <= 72 * 2.0 ** -24 * g.abs().sum(1)).all()
    sg, sx = g.abs().amax(1) / 127 * 0.501, x.abs().amax(0) / 127 * 0.501
    far = sg[:, None] * x.abs().sum(0) + g.abs().sum(1)[:, None] * sx + x.shape[0] * sg[:, None] * sx
    assert ((front.grads[0].double() - g @ x).abs() <= far * 1.001).all()
    # the features are the layer's: float products within the operands' half scales, rounded to bfloat16
    y = x @ weight.double().t().contiguous()
    sw, sr = weight.double().abs().amax(1) / 127 * 0.501, x.abs().amax(1) / 127 * 0.501
    far = sr[:, None] * weight.double().abs().sum(1) + x.abs().sum(1, keepdim=True) * sw + x.shape[1] * sr[:, None] * sw
    got = front.features.reshape(-1, desc.c_in).double()
    assert ((got - y).abs() <= far * 1.001 + 2.0 ** -8 * y.abs() + 2.0 ** -8 * far).all()
