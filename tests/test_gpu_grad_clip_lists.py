"""Clipping of long lists: the norm's parts are added once, not once in every block of every launch."""
import pytest

import paper_2003_10735_amd as st

from test_gpu_grad_clip import check, make

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

F, B = torch.float32, torch.bfloat16


def launches(call):
    st.st_profile_enable(True)
    st.st_profile_reset()
    call()
    torch.cuda.synchronize()
    names = {name: count for name, (count, _) in st.st_profile_read().items()}
    st.st_profile_enable(False)
    st.st_profile_reset()
    return names


@pytest.mark.parametrize("out", [None, F])
@pytest.mark.parametrize("count", [130, 1000, 2048, 5000])
def test_many_tensors(count, out):
    """A part a tensor here: where many launches would read many parts, one launch adds them for all that follow."""
    sizes = [1 + i * 7 % 1500 for i in range(count)]
    grads = make(sizes, (F, B))
    before = [g.clone() for g in grads]
    outs = [torch.full((n,), 7.0, dtype=out, device="cuda") for n in sizes] if out else None
    tensors, norm = st.GradTensors(grads, outs), torch.empty(1, device="cuda")
    ws = st.new_grad_workspace(tensors)
    names = launches(lambda: st.st_grad_clip(tensors, 1.0, 0.5, norm, workspace=ws))
    check(before, outs if out else grads, norm, 1.0, 0.5)
    pieces = -(-count // 120)
    assert names["clip_squares"] == names["clip_scale"] == pieces and names.get("clip_norm", 0) == (1 if pieces * count > 1 << 14 else 0)


def test_the_norm_alone_of_many_tensors():
    grads = make([1 + i % 300 for i in range(3000)], (B, F))
    array = (st.StGradTensor * 3000)(*[st.StGradTensor(g.data_ptr(), None, g.numel(), st._dtype(g, ""), 0) for g in grads])
    ws, norm = torch.empty(st.lib().st_grad_clip_workspace(array, 3000), dtype=torch.uint8, device="cuda"), torch.empty(1, device="cuda")
    names = launches(lambda: st.lib().st_grad_clip(array, 3000, 1.0, 1.0, norm.data_ptr(), ws.data_ptr(), torch.cuda.current_stream().cuda_stream))
    check(grads, [], norm, 0.0, 1.0)
    assert names == {"clip_squares": 25, "clip_scale": 1}       # (one block reads the parts)


def test_two_lists_on_one_scratch():
    """A short list behind a long one on the same scratch, and the long one again: neither sees the other's norm."""
    long, short = make([64] * 3000, (F,)), make([50, 60], (F,), seed=1, scale=100.0)
    outs = [[torch.empty_like(g) for g in grads] for grads in (long, short)]
    lists, norms = [st.GradTensors(g, o) for g, o in zip((long, short), outs)], torch.empty(2, device="cuda")
    ws = st.new_grad_workspace(lists[0])
    for i in (0, 1, 0, 1, 0):
        st.st_grad_clip(lists[i], 1.0, 1.0, norms[i:i + 1], workspace=ws)
        check((long, short)[i], outs[i], norms[i], 1.0, 1.0)
