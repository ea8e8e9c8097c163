"""Steps of the trainable block whose gradients hold a value that is not finite: neither of its two lists takes them, and they do not count."""
import math

import pytest

import paper_2003_10735_amd as st
from paper_2003_10735_amd.dense import DenseBlockFront

from test_gpu_dense_block import setup

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu


def held(block):
    """What a step changes: parameters, the matrices' copies, both lists' states."""
    lists = [x for t in (block.matrices, block.biases) for x in t.kept[2:6] if x is not None]
    return [*block.params, *block.copies, *(t for x in lists for t in x)]


def spoil(block, which, value):
    """A gradient with that value in one place, or (None) as it is."""
    if value is not None:
        block.grads[which].view(-1)[0] = value


def run(values, which, bits, max_norm=1.0):
    """Steps on one key frame, the head at rest.  Returns the block and what it held behind each step."""
    desc, cells, params, labels, head = setup()
    block = DenseBlockFront(desc, *params, lr=3e-3, weight_decay=0.01, max_norm=max_norm, state_bits=bits)
    seen = [[t.clone() for t in held(block)]]
    for value in values:
        block.backward(cells, labels, head, head_lr=0.0)
        spoil(block, which, value)
        block.apply()
        seen.append([t.clone() for t in held(block)])
    return block, seen


@pytest.mark.parametrize("bad", [float("nan"), float("inf")])
@pytest.mark.parametrize("which", range(4))
@pytest.mark.parametrize("bits,max_norm", [(8, 1.0), (32, 1.0), (32, 0.0)])
def test_steps_that_are_left_out_do_not_count(bits, max_norm, which, bad):
    """Bad steps first, in between, two in a row and last, the bad value in any of the four tensors: both lists go on bit for bit as if they had
    not been, so their clipping and their bias corrections are those of a run without them."""
    block, seen = run([bad, None, bad, bad, None, None, bad], which, bits, max_norm)
    assert block.steps == 3 and not math.isfinite(float(block.grad_norm))
    alone, want = run([None, None, None], which, bits, max_norm)
    assert alone.steps == 3
    for got, step in zip(seen, (0, 0, 1, 1, 1, 2, 3, 3)):
        assert all(torch.equal(a, b) for a, b in zip(got, want[step]))
    assert not any(torch.equal(a, b) for a, b in zip(want[0][:4], want[1][:4]))      # (a step does change every parameter)


def test_a_norm_that_float32_does_not_hold():
    """Finite gradients whose norm is more than float32 holds: left out like one that is not finite, in both lists."""
    desc, cells, params, labels, head = setup()
    block = DenseBlockFront(desc, *params, lr=3e-3)
    block.backward(cells, labels, head, head_lr=0.0)
    block.grads[0].view(-1)[:4] = 3e38
    before = [t.clone() for t in held(block)]
    block.apply()
    assert math.isinf(float(block.grad_norm)) and block.steps == 0 and all(torch.equal(a, b) for a, b in zip(held(block), before))


def test_a_count_can_be_set():
    """A block that goes on from a stored state: the count is the user's."""
    block, _ = run([None, float("nan")], 2, 32)
    block.steps = 10
    assert block.steps == 10


def test_a_recorded_step_is_an_eager_one():
    """A step in a graph has the number that follows the steps before it; replayed on bad gradients it changes nothing."""
    _, seen = run([None, None, None], 0, 32)
    desc, cells, params, labels, head = setup()
    block = DenseBlockFront(desc, *params, lr=3e-3, weight_decay=0.01, state_bits=32)
    for _ in range(2):
        block.step(cells, labels, head, head_lr=0.0)
    assert block.steps == 2                       # (waits: nothing is left to be asked for while the graph is recorded)
    block.backward(cells, labels, head, head_lr=0.0)
    before, grads = [t.clone() for t in held(block)], [g.clone() for g in block.grads]
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        block.apply()
    for bad in (None, float("nan"), None, float("inf"), None):
        for t, b in zip((*held(block), *block.grads), (*before, *grads)):
            t.copy_(b)
        spoil(block, 3, bad)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(held(block), before if bad is not None else seen[3])) and block.steps == 3


@pytest.mark.parametrize("bad", [None, float("nan")])
def test_a_step_recorded_right_behind_eager_ones(bad):
    """The count of the eager steps is settled while the graph is recorded."""
    values = [None, bad, None]
    block, seen = run(values, 1, 32)
    desc, cells, params, labels, head = setup()
    again = DenseBlockFront(desc, *params, lr=3e-3, weight_decay=0.01, state_bits=32)
    for value in values[:2]:
        again.backward(cells, labels, head, head_lr=0.0)
        spoil(again, 1, value)
        again.apply()
    again.frames = 1
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        again.apply()
    again.backward(cells, labels, head, head_lr=0.0)
    before, grads = [t.clone() for t in held(again)], [g.clone() for g in again.grads]
    for _ in range(3):
        for t, b in zip((*held(again), *again.grads), (*before, *grads)):
            t.copy_(b)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(held(again), seen[3])) and again.steps == block.steps == (3 if bad is None else 2)
