"""What a dense layer writes overlaps nothing that it reads or writes beside it: such calls are refused before any work is enqueued (no GPU)."""
import ctypes as C
import os
import random
import subprocess

import pytest

import paper_2003_10735_amd as st

torch = pytest.importorskip("torch")
# (the addresses are made up: a call that got through on a machine with a GPU would write there)
no_gpu = pytest.mark.skipif(torch.cuda.is_available(), reason="addresses that are not there")

F32, BF16 = st.ST_F32, st.ST_BF16
M, N, K = 6, 8, 16
X, W, Y, R, Z, B, DY, DX, DW, DB, WS = (i << 30 for i in range(1, 12))      # places far apart, of which a test moves one


def mat(data, rows, cols, rs=None, cs=1, dtype=F32):
    return st.StMatrix(data, dtype, rows, cols, cols if rs is None else rs, cs)


def forward(x=mat(X, M, K), w=mat(W, N, K), y=Y, pitch=N, dtype=F32, **o):
    opts = dict(bias=B, residual=R, residual_pitch=N, pre=Z, pre_pitch=N)
    opts.update(o)
    return st.lib().st_linear(C.byref(x), C.byref(w), C.byref(st.StLinearOpts(**opts)), y, dtype, pitch, WS, 1 << 28, None)


@no_gpu
@pytest.mark.parametrize("kw", [
    dict(y=X), dict(y=X + M * K * 4 - 4), dict(y=X - M * N * 4 + 4), dict(y=W + 4), dict(y=B + 28), dict(y=Z + 4 * N), dict(pre=Y), dict(pre=X + 8), dict(pre=W), dict(pre=B),
    dict(pre=R), dict(residual=Y + 4), dict(residual=Y - 4 * N), dict(residual=Y, pre=Y + 4),
    # slices of one buffer with rows of 40 values: columns 0 .. 15 are x
    dict(x=mat(X, M, K, rs=40), y=X + 15 * 4, pitch=40), dict(x=mat(X, M, K, rs=40), y=X + 33 * 4, pitch=40), dict(x=mat(X, M, K, rs=40), y=X + (40 * 3 - 7) * 4, pitch=40),
    dict(x=mat(X, M, K, rs=40), pre=X + 44, pre_pitch=40), dict(x=mat(X, M, K, rs=40), y=X + 12 * 4), dict(x=mat(X, M, K, rs=1, cs=M), y=X + M * (K - 1) * 4),
    dict(x=mat(X, M, K, dtype=BF16), w=mat(W, N, K, dtype=BF16), y=X + M * K * 2 - 4), dict(y=Y, pre=Y + 8, dtype=BF16, pitch=N, pre_dtype=BF16),
    dict(x=mat(X, M, K, rs=0), y=X + 60),
])
def test_forward_refuses(kw):
    assert forward(**kw) == st.ST_ERR_ARG


def backward(x=mat(X, M, K), w=mat(W, N, K), dy=mat(DY, M, N), pre=mat(Z, M, N), act=st.ST_ACT_SILU, **g):
    fields = dict(dx=DX, dx_pitch=K, dx_dtype=F32, dw=DW, dw_pitch=K, dw_dtype=F32, db=DB)
    fields.update(g)
    return st.lib().st_linear_backward(C.byref(x), C.byref(w), C.byref(dy), C.byref(pre), act, C.byref(st.StLinearGrads(**fields)), WS, 1 << 28, None)


@no_gpu
@pytest.mark.parametrize("kw", [
    dict(dx=X), dict(dx=W), dict(dx=DY), dict(dx=Z), dict(dx=DW + 4), dict(dx=DB - 4), dict(dw=X), dict(dw=W + 8), dict(dw=DY), dict(dw=Z), dict(dw=DB), dict(dw=DW, accumulate=1, db=DW),
    dict(db=X), dict(db=W), dict(db=DY + 4), dict(db=Z), dict(dy=mat(DX, M, N, rs=1, cs=M)), dict(dx=DY, dx_dtype=BF16), dict(dx=None, dw=None, db=DY), dict(dx=None, dw=X),
    dict(dw=None, dx=W), dict(dx=W + 4 * 12, dx_pitch=20, w=mat(W, N, K, rs=20)),
])
def test_backward_refuses(kw):
    assert backward(**kw) == st.ST_ERR_ARG


SOURCE = """
#include "st_overlap.hpp"
extern "C" int overlap(const long long* v) { return st::overlap(st::Runs{(uint64_t)v[0], v[1], v[2], v[3]}, st::Runs{(uint64_t)v[4], v[5], v[6], v[7]}); }
"""


@pytest.fixture(scope="module")
def overlap(tmp_path_factory):
    where = tmp_path_factory.mktemp("overlap")
    (where / "o.cpp").write_text(SOURCE)
    csrc = os.path.join(os.path.dirname(st.__file__), "csrc")
    subprocess.run(["g++", "-std=c++17", "-O1", "-shared", "-fPIC", "-I", csrc, str(where / "o.cpp"), "-o", str(where / "o.so")], check=True)
    f = C.CDLL(str(where / "o.so")).overlap
    return lambda *v: bool(f((C.c_longlong * 8)(*v)))


def touched(at, count, n, pitch):
    return {at + i * pitch + j for i in range(count) for j in range(n)}


def test_runs_overlap_where_they_have_a_byte_in_common(overlap):
    """Every answer against the bytes themselves; two different pitches are the one case that may be taken as apart."""
    rng = random.Random(1)
    seen = {True: 0, False: 0}
    for i in range(40000):
        a = [100 + rng.randint(0, 60), rng.randint(1, 6), rng.randint(1, 9), rng.randint(0, 14)]
        b = [100 + rng.randint(0, 60), rng.randint(1, 6), rng.randint(1, 9), a[3] if i % 2 else rng.randint(0, 14)]
        want = bool(touched(*a) & touched(*b))
        strided = [r[1] > 1 and r[3] > r[2] for r in (a, b)]
        if all(strided) and a[3] != b[3]:
            assert not overlap(*a, *b) or want, (a, b)
        else:
            assert overlap(*a, *b) == want == overlap(*b, *a), (a, b)
            seen[want] += 1
    assert min(seen.values()) > 5000


def test_runs_far_apart_do_not_pass_64_bits(overlap):
    far, most = 1 << 39, (1 << 24) - 1
    assert not overlap(1 << 46, most, 64, far, (1 << 46) + 64, most, 64, far) and overlap(1 << 46, most, 64, far, (1 << 46) + 63, most, 64, far)
    assert overlap(1 << 46, most, 64, far, (1 << 46) + 5 * far, 1, 1, 0) and not overlap(1 << 46, most, 64, far, (1 << 46) + 5 * far - 1, 1, 1, 0)
