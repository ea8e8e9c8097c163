"""Dense layers whose matrices are parts of one buffer: neighbours that do not overlap are computed, what overlaps is refused."""
import pytest

import paper_2003_10735_amd as st

from test_gpu_linear import mm64, whole

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("m,n,k", [(1, 40, 72), (7, 40, 72), (300, 136, 200), (1100, 520, 264)])
def test_columns_of_one_buffer(m, n, k, dtype):
    """x, y, z and r side by side in one buffer's columns, dy, dx too; the weights and their gradient in another's; the residual in place."""
    big, other = whole((m, 2 * k + 4 * n), 1, dtype), whole((n, 2 * k + 1), 2, dtype)
    x, y, z, r, dy, dx = big.split([k, n, n, n, n, k], dim=1)
    w, dw, db = other[:, :k], other[:, k:2 * k], torch.empty(n, device="cuda")
    want = mm64(x, w)
    rest = x.clone(), r.clone(), dy.clone(), w.clone()
    st.st_linear(x, w, residual=r, pre=z, out=y)
    T = y.dtype
    assert torch.equal(z, want.to(T)) and torch.equal(y, (want + r.double()).to(T))
    st.st_linear(x, w, residual=y, out=y)
    st.st_linear_backward(x, w, dy, dx=dx, dw=dw, db=db)
    assert torch.equal(dx, mm64(dy, w.t()).to(T)) and torch.equal(dw, mm64(dy.t(), x.t()).to(T)) and torch.equal(db.double(), dy.double().sum(0))
    assert all(torch.equal(a, b) for a, b in zip((x, r, dy, w), rest))


def test_what_overlaps_is_refused():
    m, n, k = 30, 24, 40
    x, w, dy = whole((m, k), 1, "f32"), whole((n, k), 2, "f32"), whole((m, n), 3, "f32")
    big = torch.zeros(m, 100, device="cuda")
    flat = torch.zeros(2000, device="cuda")
    v = flat[:n * k].view(n, k)
    before = x.clone(), w.clone(), dy.clone()
    for call in (lambda: st.st_linear(x, w, out=x[:, :n]), lambda: st.st_linear(x, w, out=x.view(-1)[5:5 + m * n].view(m, n)),
                 lambda: st.st_linear(x, w, pre=big[:, :n], out=big[:, n - 1:2 * n - 1]), lambda: st.st_linear(x, w, residual=big[:, 1:1 + n], out=big[:, :n]),
                 lambda: st.st_linear(x, w, w[0, :n], out=w.view(-1)[:m * n].view(m, n)),
                 lambda: st.st_linear_backward(x, w, dy, dx=x, dw=big.view(-1)[:n * k].view(n, k)),      # (x is read for dw alone)
                 lambda: st.st_linear_backward(None, v, dy, dx=flat[100:100 + m * k].view(m, k)),
                 lambda: st.st_linear_backward(x, None, dy, dw=w, db=w[0, :n]),
                 lambda: st.st_linear_backward(x, w, dy, dw=big.view(-1)[:n * k].view(n, k), db=big[0, :n])):
        with pytest.raises(st.StError) as e:
            call()
        assert e.value.status == st.ST_ERR_ARG
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip((x, w, dy), before)) and not big.any() and not flat.any()
