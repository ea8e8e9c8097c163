"""A step of the trainable layer that is recorded right behind eager ones, whose count is not settled yet."""
import pytest

from paper_2003_10735_amd import dense

from test_gpu_dense_front import setup

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu


def test_a_step_recorded_right_behind_eager_ones():
    desc, cells, weight, bias, labels, head = setup()
    front = dense.DenseFront(desc, weight, bias, lr=3e-3, state_bits=32)
    for _ in range(3):
        front.step(cells, labels, head, head_lr=0.0)
    want = weight.clone()
    desc, cells, weight, bias, labels, head = setup()
    again = dense.DenseFront(desc, weight, bias, lr=3e-3, state_bits=32)
    for _ in range(2):
        again.step(cells, labels, head, head_lr=0.0)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        again.step(cells, labels, head, head_lr=0.0)
    assert again.steps == 3
    graph.replay()
    torch.cuda.synchronize()
    assert torch.equal(weight, want)
