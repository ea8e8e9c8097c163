"""The norm's parts are added by the step's own blocks in short lists and by a launch before it in long ones: both give the same."""
import pytest

import paper_2003_10735_amd as st

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("bits,tile", [(8, 2048), (32, 1024)])
def test_same_step_by_either_way_of_adding_the_norm(bits, tile):
    """A tensor of zeros, whose gradients are zeros, beside the others: it adds tiles and nothing to the norm, so what the others get is bit
    for bit the same however long it is."""
    sizes, got = [70001, 300, 5000], {}
    for more in (1, 1900 * tile, 2100 * tile, 6000 * tile):
        g = torch.Generator(device="cuda")
        g.manual_seed(5)
        params = [torch.randn(n, device="cuda", generator=g) for n in sizes]
        grads = [torch.randn(n, device="cuda", generator=g) for n in sizes]
        params.append(torch.zeros(more, device="cuda"))
        grads.append(torch.zeros(more, device="cuda"))
        state = st.new_adamw_state(params, bits)
        t = st.AdamWTensors(params, grads, **state)
        norm = torch.empty(1, device="cuda")
        st.st_profile_reset()
        st.st_profile_enable(True)
        try:
            st.st_adamw_step(t, 1, 1e-2, max_norm=0.5, grad_norm=norm)
            torch.cuda.synchronize()
            launched = "grad_norm" in st.st_profile_read()
        finally:
            st.st_profile_enable(False)
            st.st_profile_reset()
        want = sum(x.double().square().sum() for x in grads).sqrt()
        assert abs(norm.item() - want.item()) <= 1e-6 * want.item()
        assert not params[-1].any() and not state["m"][-1].any() and not state["v"][-1].any()
        got.setdefault(launched, []).append([norm.clone(), *params[:3], *state["m"][:3], *state["v"][:3]])
    assert set(got) == {False, True}
    every = got[False] + got[True]
    for other in every[1:]:
        assert all(torch.equal(a, b) for a, b in zip(every[0], other))
