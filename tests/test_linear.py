"""The product with bias, activation and residual, and its gradients, against the definition in 64 bits."""
import ctypes
import math

import numpy as np
import pytest
import torch

import paper_2407_13726_b200 as dastac
from paper_2407_13726_b200 import binding

gpu = pytest.mark.gpu
ACTS = [dastac.ACT_NONE, dastac.ACT_RELU, dastac.ACT_SIGMOID, dastac.ACT_SILU, dastac.ACT_GELU]
_erf = np.vectorize(math.erf, otypes=[np.float64])


def _sig(z):
    return np.where(z >= 0, 1 / (1 + np.exp(-np.abs(z))), np.exp(-np.abs(z)) / (1 + np.exp(-np.abs(z))))


def _f(act, z):
    if act == dastac.ACT_RELU:
        return np.maximum(z, 0)
    if act == dastac.ACT_SIGMOID:
        return _sig(z)
    if act == dastac.ACT_SILU:
        return z * _sig(z)
    if act == dastac.ACT_GELU:
        return 0.5 * z * (1 + _erf(z / math.sqrt(2)))
    return z


def _slope(act, z):
    if act == dastac.ACT_RELU:
        return (z > 0).astype(np.float64)
    if act == dastac.ACT_SIGMOID:
        return _sig(z) * _sig(-z)
    if act == dastac.ACT_SILU:
        return _sig(z) * (1 + z * _sig(-z))
    if act == dastac.ACT_GELU:
        return 0.5 * (1 + _erf(z / math.sqrt(2))) + z * np.exp(-z * z / 2) / math.sqrt(2 * math.pi)
    return np.ones_like(z)


def _sum_error(k):
    """Bound of the fp32 accumulation relative to the sum of |terms|: sums of 16 exact products join a running
    sum one after the other, each step off by at most an ulp (2^-23), and a few more for a split contraction."""
    return (k / 16 + 16) * 2.0 ** -23


# half an ulp of bf16, and of fp32 with the arithmetic of bias, activation and residual
BF16, EPI = 2.0 ** -8, 2.0 ** -20


def _check(out, ref, bound, what, norm):
    """Every element within its bound, and the 2-norm of the error within `norm` of the result's."""
    out = out.detach().float().cpu().double().numpy()
    assert out.shape == ref.shape and np.isfinite(out).all(), what
    over = (np.abs(out - ref) / (bound + 1e-30)).max(initial=0.0)
    assert over <= 1.0, f"{what}: {over:.3g} times the bound"
    assert np.linalg.norm(out - ref) <= norm * np.linalg.norm(ref) + 1e-30, what


def _norm(dtype, k):
    # one rounding to bf16 is off by at most half an ulp, 2^-8 of the value
    return 2.0 ** -8 if dtype == torch.bfloat16 else 4 * _sum_error(k)


def _place(t, layout):
    """The same matrix with another pitch or base; what lies between the rows is NaN."""
    M, K = t.shape
    if layout == "plain":
        return t
    extra, base = {"pitch16": (16, 0), "odd_pitch": (3, 0), "odd_base": (8, 1)}[layout]
    big = torch.full((M * (K + extra) + base + 8,), float("nan"), dtype=t.dtype, device=t.device)
    v = big[base:base + M * (K + extra)].view(M, K + extra)[:, :K]
    v.copy_(t)
    return v


def _rand(gen, *s, scale=1.0, dtype=torch.bfloat16):
    return (torch.randn(*s, generator=gen) * scale).to(dtype).cuda()


def _np(t):
    return t.float().cpu().double().numpy()


def _ws(n):
    return torch.randint(0, 255, (n,), dtype=torch.uint8, device="cuda") if n else None


def _forward(M, N, K, act, dtype, bias=True, residual=True, keep=True, layout="plain", out_layout="plain", seed=0):
    gen = torch.Generator().manual_seed(seed + M + 3 * N + 7 * K)
    x, w = _place(_rand(gen, M, K), layout), _place(_rand(gen, N, K, scale=max(K, 1) ** -0.5), layout)
    b = _rand(gen, N, dtype=torch.float32) if bias else None
    r = _place(_rand(gen, M, N, dtype=dtype), out_layout) if residual else None
    y = _place(torch.zeros(M, N, dtype=dtype, device="cuda"), out_layout)
    z = _place(torch.zeros(M, N, dtype=torch.bfloat16, device="cuda"), out_layout) if keep else None
    err = torch.zeros(1, dtype=torch.int32, device="cuda")
    dastac.linear_forward(x, w, y, bias=b, act=act, residual=r, z=z, workspace=_ws(dastac.linear_workspace(x, w)), err_word=err)
    assert int(err.item()) == 0
    X, W = _np(x), _np(w)
    Z = X @ W.T + (_np(b) if bias else 0)
    R = _np(r) if residual else 0
    Y = _f(act, Z) + R
    ez = _sum_error(K) * (np.abs(X) @ np.abs(W).T) + EPI * (np.abs(Z) + 1)
    ey = 1.2 * ez + EPI * (np.abs(Y) + np.abs(R) + 1)   # the activations' slopes are below 1.2
    _check(y, Y, ey + (BF16 * (np.abs(Y) + ey) if dtype == torch.bfloat16 else 0), "y", _norm(dtype, K))
    if keep:
        _check(z, Z, ez + BF16 * (np.abs(Z) + ez), "z", _norm(torch.bfloat16, K))


@gpu
@pytest.mark.parametrize("K,N", [(64, 128), (8, 8), (1, 1), (72, 130), (63, 65), (1000, 257), (520, 363), (4096, 40)])
@pytest.mark.parametrize("M", [1, 2, 16, 17, 33, 65, 128, 129, 256, 300])
def test_forward_sizes(M, K, N):
    _forward(M, N, K, dastac.ACT_SILU, torch.bfloat16)


@gpu
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16], ids=["f32", "bf16"])
@pytest.mark.parametrize("act", ACTS)
@pytest.mark.parametrize("M", [5, 200])
def test_forward_activations(M, act, dtype):
    _forward(M, 200, 192, act, dtype)
    _forward(M, 131, 200, act, dtype, bias=False, residual=False, keep=False)


@gpu
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16], ids=["f32", "bf16"])
@pytest.mark.parametrize("out_layout", ["plain", "odd_pitch", "odd_base"])
@pytest.mark.parametrize("layout", ["plain", "pitch16", "odd_pitch", "odd_base"])
@pytest.mark.parametrize("M", [9, 140])
def test_forward_strides(M, layout, out_layout, dtype):
    _forward(M, 150, 136, dastac.ACT_GELU, dtype, layout=layout, out_layout=out_layout)


@gpu
def test_forward_many_tiles_and_splits():
    _forward(2300, 2600, 200, dastac.ACT_RELU, torch.bfloat16)          # more tiles than clusters
    _forward(3, 19000, 64, dastac.ACT_NONE, torch.float32)              # more tiles than multiprocessors
    _forward(20, 300, 8192, dastac.ACT_NONE, torch.float32)             # a contraction split eight ways
    _forward(100, 1000, 2048, dastac.ACT_SIGMOID, torch.float32)


@gpu
@pytest.mark.parametrize("M", [3, 150])
def test_forward_residual_in_place_and_no_inner(M):
    gen = torch.Generator().manual_seed(1)
    x, w, y = _rand(gen, M, 96), _rand(gen, 80, 96, scale=0.1), _rand(gen, M, 80)
    r = _np(y)
    dastac.linear_forward(x, w, y, residual=y)
    ref = _np(x) @ _np(w).T + r
    _check(y, ref, _sum_error(96) * (np.abs(_np(x)) @ np.abs(_np(w)).T) + EPI * (np.abs(ref) + np.abs(r)) + BF16 * np.abs(ref) * 1.01, "y", BF16)
    b = _rand(gen, 80, dtype=torch.float32)
    y = dastac.linear_forward(x[:, :0], w[:, :0], bias=b, act=dastac.ACT_RELU)
    assert torch.equal(y, torch.relu(b).bfloat16().expand(M, 80))
    assert dastac.linear_forward(x[:0], w).shape == (0, 80) and dastac.linear_forward(x, w[:0]).shape == (M, 0)


@gpu
@pytest.mark.parametrize("M", [4, 200])
def test_what_is_not_finite_stays_in_its_row(M):
    gen = torch.Generator().manual_seed(2)
    x, w = _rand(gen, M, 200), _rand(gen, 300, 200)
    clean = dastac.linear_forward(x, w)
    x[1], w[7] = float("nan"), float("inf")
    dirty = dastac.linear_forward(x, w)
    rows, cols = torch.arange(M, device="cuda") != 1, torch.arange(300, device="cuda") != 7
    assert torch.equal(clean[rows][:, cols], dirty[rows][:, cols])
    assert dirty[1].isnan().all() and not dirty[:, 7].isfinite().any()


@gpu
def test_same_bits_every_time():
    gen = torch.Generator().manual_seed(3)
    for M, N, K in [(7, 500, 4096), (600, 700, 512)]:
        x, w = _rand(gen, M, K), _rand(gen, N, K)
        first = dastac.linear_forward(x, w, torch.empty(M, N, device="cuda"))
        for _ in range(4):
            assert torch.equal(first, dastac.linear_forward(x, w, torch.empty(M, N, device="cuda")))


# ---- the kernel on pairs of CTAs, which takes products of many tiles ----------------------------------------------

def _torch_f(act, z):
    if act == dastac.ACT_RELU:
        return z.clamp(min=0)
    if act == dastac.ACT_SIGMOID:
        return torch.sigmoid(z)
    if act == dastac.ACT_SILU:
        return z * torch.sigmoid(z)
    if act == dastac.ACT_GELU:
        return 0.5 * z * (1 + torch.erf(z / math.sqrt(2)))
    return z


def _kernel_of(x, w, y, act, b, r, z):
    """The library's choice for this call."""
    ptr, pitch = (lambda t: 0 if t is None else t.data_ptr()), (lambda t: 0 if t is None else t.stride(0))
    which = ctypes.c_int32(-1)
    a = binding._LinearArgs(M=x.shape[0], N=w.shape[0], K=x.shape[1], act=act, y_dtype=int(y.dtype == torch.bfloat16), x=ptr(x), ldx=pitch(x),
                            w=ptr(w), ldw=pitch(w), bias=ptr(b), residual=ptr(r), ldr=pitch(r), y=ptr(y), ldy=pitch(y), z=ptr(z), ldz=pitch(z))
    assert binding._lib.dastac_linear_forward_kernel(a, ctypes.byref(which)) == 0
    return which.value


def _forward_on_pairs(M, N, K, act, dtype, full=True, layout="plain", out_layout="plain", in_place=False):
    gen = torch.Generator().manual_seed(M + 3 * N + 7 * K)
    x, w = _place(_rand(gen, M, K), layout), _place(_rand(gen, N, K, scale=max(K, 1) ** -0.5), layout)
    b = _rand(gen, N, dtype=torch.float32) if full else None
    r = _place(_rand(gen, M, N, dtype=dtype), out_layout) if full else None
    y = r if in_place else _place(torch.full((M, N), float("nan"), dtype=dtype, device="cuda"), out_layout)
    z = _place(torch.full((M, N), float("nan"), dtype=torch.bfloat16, device="cuda"), out_layout) if full else None
    assert _kernel_of(x, w, y, act, b, r, z) == 2
    X, W = x.double(), w.double()
    Z = X @ W.T + (b.double() if full else 0)
    R = r.double().clone() if full else torch.zeros_like(Z)
    err = torch.zeros(1, dtype=torch.int32, device="cuda")
    dastac.linear_forward(x, w, y, bias=b, act=act, residual=r, z=z, workspace=_ws(dastac.linear_workspace(x, w)), err_word=err)
    assert int(err.item()) == 0
    Y = _torch_f(act, Z) + R
    ez = _sum_error(K) * (X.abs() @ W.abs().T) + EPI * (Z.abs() + 1)
    ey = 1.2 * ez + EPI * (Y.abs() + R.abs() + 1)
    results = [(y, Y, ey, dtype)] + ([(z, Z, ez, torch.bfloat16)] if full else [])
    for out, ref, e, t in results:
        bound = e + (BF16 * (ref.abs() + e) if t == torch.bfloat16 else 0)
        over = float(((out.double() - ref).abs() / (bound + 1e-30)).max())   # NaN, where nothing was written, fails as well
        assert over <= 1.0, over
        assert float((out.double() - ref).norm()) <= _norm(t, K) * float(ref.norm())
    return x, w, y


@gpu
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16], ids=["f32", "bf16"])
@pytest.mark.parametrize("act", ACTS)
@pytest.mark.parametrize("N", [1504, 1500, 1501])    # rows of whole 16 bytes, of whole pairs (bf16), of neither
def test_pairs_activations(N, act, dtype):
    _forward_on_pairs(1701, N, 136, act, dtype)
    _forward_on_pairs(1701, N, 136, act, dtype, full=False)


@gpu
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16], ids=["f32", "bf16"])
@pytest.mark.parametrize("layout,out_layout", [("pitch16", "pitch16"), ("odd_pitch", "odd_pitch"), ("odd_base", "odd_base"), ("plain", "odd_base")])
@pytest.mark.parametrize("M,N,K", [(1700, 1512, 72), (2305, 2568, 72), (2305, 2568, 2200)])   # the last two: more tiles than pairs of CTAs
def test_pairs_strides_and_several_tiles_a_pair(M, N, K, layout, out_layout, dtype):
    _forward_on_pairs(M, N, K, dastac.ACT_GELU, dtype, layout=layout, out_layout=out_layout)


@gpu
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16], ids=["f32", "bf16"])
@pytest.mark.parametrize("K", [0, 1, 64, 65, 512, 513, 1024, 1100, 2048, 2049])   # around the parts of an fp32 sum
@pytest.mark.parametrize("out_layout", ["plain", "odd_pitch"])
def test_pairs_lengths_and_residual_in_place(K, out_layout, dtype):
    _forward_on_pairs(2305, 2568, K, dastac.ACT_SIGMOID, dtype, out_layout=out_layout, in_place=True)


@gpu
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16], ids=["f32", "bf16"])
def test_pairs_keep_what_is_not_finite_and_the_same_bits(dtype):
    x, w, first = _forward_on_pairs(2305, 2568, 1100, dastac.ACT_NONE, dtype, full=False)
    ws = _ws(dastac.linear_workspace(x, w))
    for _ in range(4):
        assert torch.equal(first, dastac.linear_forward(x, w, torch.empty_like(first), workspace=ws))
    x[1000], w[7] = float("nan"), float("inf")
    dirty = dastac.linear_forward(x, w, torch.empty_like(first), workspace=ws)
    rows, cols = torch.arange(2305, device="cuda") != 1000, torch.arange(2568, device="cuda") != 7
    assert torch.equal(first[rows][:, cols], dirty[rows][:, cols])
    assert dirty[1000].isnan().all() and not dirty[:, 7].isfinite().any()


def _backward(M, N, K, act, dw_dtype=torch.bfloat16, accumulate=False, layout="plain", out_layout="plain", want="xwb"):
    gen = torch.Generator().manual_seed(11 + M + 3 * N + 7 * K)
    x, w, dy = (_place(t, layout) for t in (_rand(gen, M, K), _rand(gen, N, K, scale=max(K, 1) ** -0.5), _rand(gen, M, N)))
    z = _place(_rand(gen, M, N, scale=1.5), layout) if act != dastac.ACT_NONE else None
    dx = _place(torch.full((M, K), float("nan"), dtype=torch.bfloat16, device="cuda"), out_layout) if "x" in want else None
    dw0, db0 = _rand(gen, N, K, dtype=dw_dtype), _rand(gen, N, dtype=torch.float32)
    dw = _place(dw0.clone(), out_layout) if "w" in want else None
    db = db0.clone() if "b" in want else None
    err = torch.zeros(1, dtype=torch.int32, device="cuda")
    dastac.linear_backward(dy, x, w, act=act, z=z, dx=dx, dw=dw, db=db, accumulate=accumulate,
                           workspace=_ws(dastac.linear_backward_workspace(dy, x, w, act)), err_word=err)
    assert int(err.item()) == 0
    X, W, dZ = _np(x), _np(w), _np(dy) * (_slope(act, _np(z)) if z is not None else 1.0)
    round_z = 0.0 if act == dastac.ACT_NONE else BF16   # dZ as an operand
    # a slope is a sum of terms of order one, good to EPI whatever its own size
    slope_err = EPI * np.abs(_np(dy))
    two = 2.0 ** -7 + EPI                                # two roundings to bf16, one after the other
    start = 1.0 if accumulate else 0.0
    if dx is not None:
        ref, size = dZ @ W, np.abs(dZ) @ np.abs(W)
        e = (_sum_error(N) + EPI + round_z) * size + slope_err @ np.abs(W)
        _check(dx, ref, e + BF16 * (np.abs(ref) + e), "dx", two)
    if dw is not None:
        ref, size = dZ.T @ X + start * _np(dw0), np.abs(dZ).T @ np.abs(X) + start * np.abs(_np(dw0))
        e = (_sum_error(M) + EPI + round_z) * size + slope_err.T @ np.abs(X)
        exact = act == dastac.ACT_NONE and dw_dtype == torch.float32
        _check(dw, ref, e + (BF16 * (np.abs(ref) + e) if dw_dtype == torch.bfloat16 else 0), "dw",
               4 * _sum_error(M) if exact else two)
    if db is not None:
        ref, size = dZ.sum(0) + start * _np(db0), np.abs(dZ).sum(0) + start * np.abs(_np(db0))
        # 8 rows a thread, 8 partial sums, one sum a block of 64 rows, eight sums of those
        _check(db, ref, (EPI + (M / 512 + 24) * 2.0 ** -24) * size + slope_err.sum(0), "db", 1e-4)


@gpu
@pytest.mark.parametrize("act", ACTS)
@pytest.mark.parametrize("M,N,K", [(1, 1, 1), (1, 128, 64), (7, 40, 130), (64, 64, 64), (130, 257, 72), (300, 363, 520), (257, 1000, 63)])
def test_backward_sizes(M, N, K, act):
    _backward(M, N, K, act)


@gpu
@pytest.mark.parametrize("layout,out_layout", [("pitch16", "plain"), ("odd_pitch", "odd_pitch"), ("odd_base", "odd_base"), ("plain", "odd_pitch")])
@pytest.mark.parametrize("act", [dastac.ACT_NONE, dastac.ACT_SILU])
@pytest.mark.parametrize("M", [20, 200])
def test_backward_strides(M, act, layout, out_layout):
    _backward(M, 136, 200, act, layout=layout, out_layout=out_layout)
    _backward(M, 136, 200, act, torch.float32, layout=layout, out_layout=out_layout)


@gpu
@pytest.mark.parametrize("want", ["x", "w", "b", "xb", "wb", "xwb"])
@pytest.mark.parametrize("act", [dastac.ACT_NONE, dastac.ACT_GELU])
def test_backward_parts_and_accumulation(act, want):
    _backward(150, 264, 192, act, torch.float32, accumulate=True, want=want)
    _backward(150, 264, 192, act, torch.bfloat16, want=want)


@gpu
def test_backward_many_tiles():
    _backward(2100, 2600, 1100, dastac.ACT_SILU)


@gpu
def test_backward_empty_extents():
    bf = dict(dtype=torch.bfloat16, device="cuda")
    x, w, dy = torch.ones(0, 16, **bf), torch.ones(24, 16, **bf), torch.ones(0, 24, **bf)
    dw, db = torch.ones(24, 16, device="cuda"), torch.ones(24, device="cuda")
    dastac.linear_backward(dy, x, w, dw=dw, db=db, accumulate=True)
    assert (dw == 1).all() and (db == 1).all()
    dastac.linear_backward(dy, x, w, dw=dw, db=db)
    assert (dw == 0).all() and (db == 0).all()
    dx = torch.ones(8, 16, **bf)
    dastac.linear_backward(torch.ones(8, 0, **bf), torch.ones(8, 16, **bf), torch.ones(0, 16, **bf), dx=dx)
    assert (dx == 0).all()


@gpu
def test_backward_empty_extents_and_one_row_of_any_pitch():
    """A (1, K) tensor made from a column has a pitch of 1, which says nothing for a single row."""
    bf = dict(dtype=torch.bfloat16, device="cuda")
    dx = torch.ones(16, 1, **bf).t()
    dastac.linear_backward(torch.ones(1, 0, **bf), torch.ones(1, 16, **bf), torch.ones(0, 16, **bf), dx=dx)
    assert dx.stride() == (1, 1) and (dx == 0).all()
    for dw in (torch.ones(16, 1, device="cuda").t(), torch.ones(16, 1, **bf).t()):
        db = torch.ones(1, device="cuda")
        dastac.linear_backward(torch.ones(0, 1, **bf), torch.ones(0, 16, **bf), torch.ones(1, 16, **bf), dw=dw, db=db)
        assert (dw == 0).all() and (db == 0).all()


# An fp32 result is a sum of parts, each of at most 64 sums of 16 products that join an accumulator one after the other.
# The accumulator is cut off rather than rounded: half an ulp (2^-24) each in the mean, of a sum that grows with the root of
# the number of terms, 2/3 of its final size in the mean.  The parts and what follows are rounded to nearest.
FOLDED = 64 * 2 / 3 * 2.0 ** -24 + 2.0 ** -22


@gpu
@pytest.mark.parametrize("M,N,K", [(600, 600, 8192), (2600, 2600, 8192), (2600, 2600, 2100), (2600, 130, 16384), (100, 19000, 8192), (1, 5000, 8192)])
def test_fp32_results_of_long_sums(M, N, K):
    """The same accuracy for many tiles as for few, and for any length."""
    gen = torch.Generator().manual_seed(M + N)
    x, w = _rand(gen, M, K), _rand(gen, N, K)
    y = dastac.linear_forward(x, w, torch.empty(M, N, device="cuda"), workspace=_ws(dastac.linear_workspace(x, w)))
    ref = x.double() @ w.double().T
    assert float((y - ref).norm()) <= FOLDED * float(ref.norm())
    dy, xs, dw = _rand(gen, K, M), _rand(gen, K, N), torch.empty(M, N, device="cuda")   # the sum is over the K rows here
    unused = torch.empty(M, N, dtype=torch.bfloat16, device="cuda")
    dastac.linear_backward(dy, xs, unused, dw=dw, workspace=_ws(dastac.linear_backward_workspace(dy, xs, unused)))
    ref = dy.double().T @ xs.double()
    assert float((dw - ref).norm()) <= FOLDED * float(ref.norm())


@gpu
@pytest.mark.parametrize("act", ACTS[1:])
@pytest.mark.parametrize("M,N,K,layout", [(1, 8, 8, "plain"), (300, 130, 72, "odd_pitch"), (2000, 264, 200, "plain"), (700, 2600, 1100, "plain")])
def test_fp32_weight_gradient_behind_an_activation(M, N, K, layout, act):
    """dZ has more bits than one bf16 number; an fp32 dW is as good as two of them (2^-16 of each term, and as much of the
    result, the terms' errors being independent)."""
    gen = torch.Generator().manual_seed(M + act)
    x, w, dy = (_place(t, layout) for t in (_rand(gen, M, K), _rand(gen, N, K), _rand(gen, M, N)))
    z = _place(_rand(gen, M, N, scale=1.5), layout)
    start = _rand(gen, N, K, dtype=torch.float32)
    for accumulate in (False, True):
        dx, dw = torch.empty(M, K, dtype=torch.bfloat16, device="cuda"), start.clone()
        dastac.linear_backward(dy, x, w, act=act, z=z, dx=dx, dw=dw, accumulate=accumulate,
                               workspace=_ws(dastac.linear_backward_workspace(dy, x, w, act)))
        X, dZ = _np(x), _np(dy) * _slope(act, _np(z))
        ref, size = dZ.T @ X + accumulate * _np(start), np.abs(dZ).T @ np.abs(X) + accumulate * np.abs(_np(start))
        bound = (_sum_error(M) + EPI + 2.0 ** -16) * size + EPI * np.abs(_np(dy)).T @ np.abs(X)
        # a slope is good to EPI whatever its own size: relative to dY, which is 4 times dZ or less in the 2-norm
        _check(dw, ref, bound, "dw", 2.0 ** -16 + FOLDED + 4 * EPI)
    # a bf16 dW, and one that does without the second part, ask for less (relu's dZ has none)
    half = dastac.linear_backward_workspace(dy, x, w, act, dw_dtype=torch.bfloat16)
    assert half == dastac.linear_backward_workspace(dy, x, w, act, round_dz=True)
    assert (half < dastac.linear_backward_workspace(dy, x, w, act)) == (act != dastac.ACT_RELU)
    coarse, bf16 = torch.empty(N, K, device="cuda"), torch.empty(N, K, dtype=torch.bfloat16, device="cuda")
    dastac.linear_backward(dy, x, w, act=act, z=z, dx=dx, dw=coarse, round_dz=True, workspace=_ws(half))
    dastac.linear_backward(dy, x, w, act=act, z=z, dx=dx, dw=bf16, workspace=_ws(half))
    for dw in (coarse, bf16):
        assert float((dw.double().cpu() - torch.from_numpy(dZ.T @ X)).norm()) <= 2.0 ** -7 * float(np.linalg.norm(dZ.T @ X))


@gpu
def test_infinite_gradients_stay_infinite_in_an_fp32_weight_gradient():
    gen = torch.Generator().manual_seed(8)
    x, w, dy, z = _rand(gen, 200, 40), _rand(gen, 48, 40), _rand(gen, 200, 48), _rand(gen, 200, 48)
    grads = []
    for bad in (1.0, float("inf")):
        dy[3, 5], z[3, 5] = bad, 1.0
        dw = torch.empty(48, 40, device="cuda")
        dastac.linear_backward(dy, x, w, act=dastac.ACT_SILU, z=z, dw=dw, workspace=_ws(dastac.linear_backward_workspace(dy, x, w, dastac.ACT_SILU)))
        grads.append(dw)
    others = torch.arange(48, device="cuda") != 5
    assert torch.equal(grads[0][others], grads[1][others])
    assert torch.equal(grads[1][5], torch.sign(x[3].float()) * float("inf"))


@gpu
@pytest.mark.parametrize("act", ACTS[1:])
def test_gradients_against_differences(act):
    """<gradient, direction> against central differences of the 64-bit forward pass.  The kept preactivation is
    a rounded one, so the differences are taken of f around it: z enters as x w^T + (z - x w^T)."""
    gen = torch.Generator().manual_seed(5)
    M, N, K = 140, 40, 72
    x, w, dy, z = _rand(gen, M, K), _rand(gen, N, K, scale=K ** -0.5), _rand(gen, M, N), _rand(gen, M, N)
    z = torch.where(z.abs() < 0.01, torch.full_like(z, 0.5), z)   # relu: no kink within a step
    dx, dw, db = torch.empty(M, K, dtype=torch.bfloat16, device="cuda"), torch.empty(N, K, device="cuda"), torch.empty(N, device="cuda")
    dastac.linear_backward(dy, x, w, act=act, z=z, dx=dx, dw=dw, db=db, workspace=_ws(dastac.linear_backward_workspace(dy, x, w, act)))
    X, W, G, B = _np(x), _np(w), _np(dy), np.zeros(N)
    rest = _np(z) - X @ W.T
    loss = lambda a, b, c: (_f(act, a @ b.T + c + rest) * G).sum()  # noqa: E731
    rng = np.random.default_rng(0)
    for k, grad in enumerate((dx, dw, db)):
        g = _np(grad)
        v = rng.standard_normal(g.shape)
        up, down = [X, W, B], [X, W, B]
        up[k], down[k] = up[k] + 1e-5 * v, down[k] - 1e-5 * v
        want = (loss(*up) - loss(*down)) / 2e-5
        # dZ and dx are rounded to bf16: independent errors of 2^-8 of each term
        assert abs((g * v).sum() - want) <= 2.0 ** -8 * np.abs(g * v).sum()


# ---- refusals (no GPU) -------------------------------------------------------------------------------------------

def _args(**k):
    v = dict(M=200, N=64, K=72, act=0, y_dtype=1, dw_dtype=1, accumulate=0, x=256, ldx=72, w=256, ldw=72, y=256, ldy=64, z=256, ldz=64,
             dy=256, lddy=64, dx=256, lddx=72, dw=256, lddw=72, db=256)
    v.update(k)
    return binding._LinearArgs(**v)


def test_refusals_do_not_launch():
    before = dastac.launch_count()
    lib, n = binding._lib, ctypes.c_size_t()
    fwd = lambda **k: lib.dastac_linear_forward(_args(**k), None, 0, None, None)  # noqa: E731
    bwd = lambda **k: lib.dastac_linear_backward(_args(**k), None, 0, None, None)  # noqa: E731
    both = [(dict(M=-1), 1), (dict(N=-1), 1), (dict(K=-1), 1), (dict(act=5), 1), (dict(act=-1), 1), (dict(M=2 ** 30 + 1), 6),
            (dict(x=None), 1), (dict(w=None), 1), (dict(ldx=71), 4), (dict(ldw=71), 4), (dict(x=257), 5), (dict(w=255), 5)]
    for k, status in both + [(dict(y=None), 1), (dict(ldy=63), 4), (dict(y=257), 5), (dict(y_dtype=2), 3), (dict(residual=256, ldr=63), 4),
                             (dict(z=256, ldz=60), 4), (dict(bias=258), 5), (dict(y_dtype=0, y=258), 5),
                             (dict(ldx=73), 7), (dict(w=258), 7)]:           # needs a copy, no workspace
        assert fwd(**k) == status, k
    for k, status in both + [(dict(dy=None), 1), (dict(lddy=63), 4), (dict(act=3, z=None), 1), (dict(act=3, ldz=63), 4), (dict(dx=257), 5),
                             (dict(lddx=71), 4), (dict(dw_dtype=2), 3), (dict(accumulate=1), 3), (dict(db=258), 5),
                             (dict(), 7), (dict(act=1), 7), (dict(M=2 ** 22, ldx=72), 7)]:
        assert bwd(**k) == status, k
    assert lib.dastac_linear_forward_workspace(_args(), ctypes.byref(n)) == 0 and n.value == 0
    assert lib.dastac_linear_forward_workspace(_args(ldx=73), ctypes.byref(n)) == 0 and n.value == 256 * 113   # 200 x 72 x 2 rounded up
    assert lib.dastac_linear_backward_workspace(_args(), ctypes.byref(n)) == 0 and n.value > 0
    assert lib.dastac_linear_forward_workspace(_args(), None) == 1 and lib.dastac_linear_forward_workspace(None, ctypes.byref(n)) == 1
    assert lib.dastac_linear_forward(_args(ldx=73), 8, 1 << 20, None, None) == 7                       # misaligned workspace
    assert dastac.launch_count() == before


def test_kernel_query_refuses_what_the_call_refuses():
    lib, which = binding._lib, ctypes.c_int32(-1)
    assert lib.dastac_linear_forward_kernel(_args(M=0), ctypes.byref(which)) == 0 and which.value == 0
    assert lib.dastac_linear_forward_kernel(_args(), None) == 1 and lib.dastac_linear_forward_kernel(None, ctypes.byref(which)) == 1
    assert lib.dastac_linear_forward_kernel(_args(ldx=71), ctypes.byref(which)) == 4


def test_binding_checks_tensors():
    x, w = torch.zeros(2, 8, dtype=torch.bfloat16), torch.zeros(4, 8, dtype=torch.bfloat16)
    with pytest.raises(AssertionError):
        dastac.linear_forward(x, w)    # not on a GPU: there is no other code path
