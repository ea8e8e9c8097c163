"""Steps of the trainable layer that a norm without a finite value leaves out: the layer goes on as if they had not been."""
import pytest

import paper_2003_10735_amd as st
from paper_2003_10735_amd import dense

from test_gpu_dense_front import setup

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu


@pytest.fixture
def spoil(monkeypatch):
    """spoil.now: the weights' gradient of the next steps gets that value in one place."""
    backward = st.st_int8_linear_backward

    def call(*a, **k):
        r = backward(*a, **k)
        if call.now is not None:
            k["dw"][0, 0] = call.now
        return r

    call.now = None
    monkeypatch.setattr(dense.st, "st_int8_linear_backward", call)
    return call


def run(spoil, values, bits, max_norm=1.0):
    """Steps with the head at rest; values: None, or what spoils the step.  Returns (layer, weights behind each step)."""
    desc, cells, weight, bias, labels, head = setup()
    front = dense.DenseFront(desc, weight, bias, lr=3e-3, max_norm=max_norm, state_bits=bits)
    seen = []
    for value in values:
        spoil.now = value
        front.step(cells, labels, head, head_lr=0.0)
        seen.append(weight.clone())
    return front, seen


@pytest.mark.parametrize("bad", [float("nan"), float("inf")])
@pytest.mark.parametrize("bits", [8, 32])
def test_steps_that_are_left_out_do_not_count(spoil, bits, bad):
    """Bad steps first, in between, two in a row and last: the good ones are bit for bit the steps of a run without them, so their bias
    corrections are too."""
    front, seen = run(spoil, [bad, None, bad, bad, None, None, bad], bits)
    assert front.steps == 3
    alone, want = run(spoil, [None, None, None], bits)
    assert alone.steps == 3
    start = setup()[2]
    for got, step in zip(seen, (None, 0, 0, 0, 1, 2, 2)):
        assert torch.equal(got, start if step is None else want[step])
    for a, b in zip(front.tensors.kept[2:4], alone.tensors.kept[2:4]):
        assert all(torch.equal(x, y) for x, y in zip(a, b))


def test_without_a_clip_every_step_counts(spoil):
    front, _ = run(spoil, [None, float("nan"), None], 32, max_norm=0.0)
    assert front.steps == 3


def test_a_count_can_be_set(spoil):
    """A layer that goes on from a stored state: the count is the user's."""
    front, _ = run(spoil, [None, float("nan")], 32)
    front.steps = 10
    assert front.steps == 10


def test_a_recorded_step_is_an_eager_one(spoil):
    """A step in a graph, which has the number that follows the steps before it."""
    front, seen = run(spoil, [None, None, None], 32)
    desc, cells, weight, bias, labels, head = setup()
    again = dense.DenseFront(desc, weight, bias, lr=3e-3, state_bits=32)
    for _ in range(2):
        again.step(cells, labels, head, head_lr=0.0)
    assert again.steps == 2                       # (waits: nothing is left to be asked for while the graph is recorded)
    before = [t.clone() for t in (weight, bias, *again.tensors.kept[2], *again.tensors.kept[3])]
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        again.step(cells, labels, head, head_lr=0.0)
    for _ in range(3):
        for t, b in zip((weight, bias, *again.tensors.kept[2], *again.tensors.kept[3]), before):
            t.copy_(b)
        st.st_int8_quantize(weight, *again.quantized)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(weight, seen[2]) and again.steps == 3
