"""Calls on a stream that is not the current one, without a workspace: what they make themselves is that stream's."""
import pytest

import paper_2003_10735_amd as st

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu


def on_stream(t, stream):
    """Whether the allocator keeps the tensor's memory for that stream."""
    for seg in torch.cuda.memory.memory_snapshot():
        if seg["address"] <= t.data_ptr() < seg["address"] + seg["total_size"]:
            return seg["stream"] == stream.cuda_stream
    raise AssertionError("no segment holds the tensor")


def rand(*shape, seed=0):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return torch.randn(*shape, device="cuda", generator=g)


def test_results_and_scratch_belong_to_the_given_stream():
    """The current stream's allocator is kept busy with tensors of the scratch's sizes behind every call: none of them may reach it."""
    x, w, dy = rand(700, 600, seed=1), rand(900, 600, seed=2), rand(700, 900, seed=3)
    torch.cuda.synchronize()

    def calls(stream):
        wq, ws = st.st_int8_quantize(w, stream=stream)
        yield wq, ws
        yield st.st_int8_quantize(x.t(), stream=stream)
        yield st.st_int8_linear(x, wq, ws, stream=stream),
        dx, dw, db = torch.empty_like(x), torch.empty_like(w), torch.empty(900, device="cuda")
        yield st.st_int8_linear_backward(x, w, dy, dx=dx, dw=dw, db=db, stream=stream)
        params = [w.clone()]
        torch.cuda.synchronize()
        t = st.AdamWTensors(params, [dw], **st.new_adamw_state(params, 8))
        torch.cuda.synchronize()
        st.st_adamw_step(t, 1, 0.1, max_norm=1.0, stream=stream)
        yield tuple(params)
        state = t.kept
        yield st.st_adamw_state(state[2][0], state[4][0], state[3][0], state[5][0], stream=stream)

    want = []
    for out in calls(None):
        torch.cuda.synchronize()
        want.append([t.clone() for t in out])
    sizes = [st.lib().st_int8_linear_workspace(700, 900, 600), st.lib().st_int8_linear_backward_workspace(700, 900, 600),
             st.lib().st_int8_quantize_workspace(600, 700), 4096]
    torch.cuda.empty_cache()
    side, got = torch.cuda.Stream(), []
    for out in calls(side):
        for n in sizes:
            torch.full((n,), 255, dtype=torch.uint8, device="cuda")
        side.synchronize()
        torch.cuda.synchronize()
        got.append(out)
    for i, (a, b) in enumerate(zip(want, got)):
        assert all(torch.equal(s, t) for s, t in zip(a, b)), i
    for i in (0, 1, 2, 5):                       # results that the calls made
        assert all(on_stream(t, side) for t in got[i]), i
    used = sum(seg["total_size"] for seg in torch.cuda.memory.memory_snapshot() if seg["stream"] == side.cuda_stream)
    assert used >= sum(t.nbytes for i in (0, 1, 2, 5) for t in got[i]) + max(sizes)
