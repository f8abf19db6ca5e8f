"""4-bit weights: the quantizer's codes, exponents and values against the
definition, and products with them against 64-bit sums over the same weights.

Tolerances: a product's terms are exact (8 bits times 2, a part at a time) and
summed in 32 bits, at most 2^-23 of the running sum lost per step of 32 rows
and part, per wavefront and per term inside a step (a chain of D / 32 parts, 32
terms, 8 wavefronts), then one rounding to the output's type."""
import math

import numpy as np
import pytest
import torch

import paper_2207_05808_amd as mdn
from paper_2207_05808_amd import _lib

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
GRID = np.array([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0])
PARTS = {torch.bfloat16: 1, torch.float16: 2, torch.float32: 3}


def quantized(B):
    """(codes [D][M], exponents [G][M], values [D][M]) from the definition, in
    64 bits on the host."""
    B = B.double().cpu().numpy()
    D, M = B.shape
    G = -(-D // 32)
    W = np.zeros((G * 32, M))
    W[:D] = B
    a = np.abs(W).reshape(G, 32, M).max(1)
    e = np.full((G, M), -120)
    for k in range(-120, 126):   # the smallest k with a <= 6 * 2^k
        e = np.where((a > 6.0 * 2.0 ** (k - 1)) & (k > -120), k, e)
    t = np.abs(W) / np.repeat(2.0 ** e, 32, 0)
    d = np.abs(t[..., None] - GRID)
    d[..., 1::2] = np.nextafter(d[..., 1::2], np.inf)   # ties to the even code
    q = d.argmin(-1)
    s = np.where(W < 0, -1.0, 1.0)
    return np.where((W < 0) & (q > 0), q + 8, q)[:D], e, (s * GRID[q] * np.repeat(2.0 ** e, 32, 0))[:D]


def unpacked(w):
    """(codes [D][M], exponents [G][M]) of packed weights, by the header's indices."""
    c, x = w.codes.cpu().numpy(), w.exps.cpu().numpy()
    d, m = np.arange(w.D)[:, None], np.arange(w.M)[None, :]
    r = d % 128
    lane = 16 * (r % 32 // 8) + m % 16
    byte = c[m // 16, d // 128, lane, 4 * (r // 32) + r % 8 // 2]
    g = np.arange(-(-w.D // 32))[:, None]
    return (byte >> (4 * (d % 2))) & 15, x[m // 16, g // 4, m % 16, g % 4].astype(int) - 127


def rand(shape, seed, dtype=torch.float32):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    return torch.randn(*shape, generator=g, device=DEV).to(dtype)


@pytest.mark.parametrize("D,M", [(1, 1), (32, 16), (31, 17), (33, 15), (128, 16), (129, 33), (300, 100), (1024, 260)])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16, torch.float16])
@pytest.mark.parametrize("order", ["dm", "md", "strided"])
def test_quantize(D, M, dtype, order):
    B = rand((D, M), D + M, dtype)
    B = B * torch.exp2(torch.randint(-8, 5, (1, M), device=DEV).to(dtype))   # columns of different size
    if order == "md":
        B = B.t().contiguous().t()
    if order == "strided":
        big = torch.zeros((2 * D, 3 * M), dtype=dtype, device=DEV)
        big[::2, ::3] = B
        B = big[::2, ::3]
    w = mdn.quantize_w4(B)
    q, e, v = quantized(B)
    gq, ge = unpacked(w)
    assert np.array_equal(gq, q) and np.array_equal(ge, e)
    assert np.array_equal(mdn.dequantize_w4(w).double().cpu().numpy(), v)
    assert np.array_equal(mdn.dequantize_w4(w, dtype=torch.float32).double().cpu().numpy(), v)
    # past the matrix: code 0, exponent 0
    full = mdn.W4Weights(w.codes, w.exps, w.codes.shape[1] * 128, w.codes.shape[0] * 16)
    fq, fe = unpacked(full)
    assert not fq[D:].any() and not fq[:, M:].any() and not fe[:, M:].any() and not fe[-(-D // 32):].any()


def test_quantize_edges():
    """Every tie and both sides of it, the largest and smallest groups, zeros
    of both signs, and groups that are not finite."""
    t = np.array([0, 0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0, 6.0], dtype=np.float32)
    col = np.concatenate([t, np.nextafter(t[1:], np.float32(9)), np.nextafter(t[1:], np.float32(0))])
    col = np.minimum(col, 6)                        # 25 values
    cols = [np.concatenate([col, -col[:7]])]        # one group at e = 0
    cols += [cols[0] * np.float32(2.0 ** k) for k in (-118, -100, 20, 124, 125)]
    cols += [np.full(32, 3e38, np.float32), np.full(32, 1e-44, np.float32), np.full(32, -0.0, np.float32), np.full(32, np.finfo(np.float32).max, np.float32)]
    B = torch.from_numpy(np.stack(cols, 1).astype(np.float32)).to(DEV)
    w = mdn.quantize_w4(B)
    q, e, v = quantized(B)
    gq, ge = unpacked(w)
    assert np.array_equal(ge, e) and np.array_equal(gq, q)
    assert np.array_equal(mdn.dequantize_w4(w, dtype=torch.float32).double().cpu().numpy(), v)
    for bad in (math.inf, -math.inf, math.nan):
        B = rand((96, 5), 1)
        B[40, 2] = bad
        v = mdn.dequantize_w4(mdn.quantize_w4(B))
        nan = torch.zeros((96, 5), dtype=torch.bool, device=DEV)
        nan[32:64, 2] = True
        assert torch.equal(v.isnan(), nan)
        assert torch.isfinite(v[~nan]).all()


def reference(A, w, bias, act):
    W = mdn.dequantize_w4(w, dtype=torch.float32).double()
    y = A.double() @ W
    size = A.double().abs() @ W.abs()
    if bias is not None and act != "none":
        y, size = y + bias.double(), size + bias.double().abs()
    steps = A.shape[1] / 32 * PARTS[A.dtype] + 32 + 8 + 2
    return y, size * steps * 2.0 ** -23


def check(A, w, bias, act, out_dtype=None):
    y = mdn.matmul_w4(A, w, col_bias=bias, act=act, out_dtype=out_dtype)
    ref, tol = reference(A, w, bias, act)
    if act == "softmax":
        z, dz = ref, tol.amax(1, keepdim=True)
        ref = torch.softmax(z, 1)
        rel = 2 * dz + ((z - z.amax(1, keepdim=True)).abs() + A.shape[0] * 0 + w.M + 5) * 2.0 ** -24
        tol = ref * rel + 2.0 ** -126
    else:
        if act == "relu":
            ref = torch.relu(ref)
        tol = tol + ref.abs() * torch.finfo(y.dtype).eps / 2
    assert y.shape == ref.shape
    err = (y.double() - ref).abs()
    assert bool((err <= tol).all()), float((err / tol.clamp(min=1e-300)).max())
    return y


@pytest.mark.parametrize("N", [1, 2, 15, 16, 17, 33, 64, 65, 200, 513, 1537])
@pytest.mark.parametrize("D,M", [(1, 1), (64, 10), (127, 31), (512, 100), (1000, 257), (4100, 48)])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16, torch.float32])
def test_matmul(N, D, M, dtype):
    w = mdn.quantize_w4(rand((D, M), 3))
    check(rand((N, D), 4, dtype), w, None, "none")


@pytest.mark.parametrize("N,D,M", [(2500, 128, 5000), (3000, 321, 4099), (1600, 64, 30003), (12000, 4000, 40)])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16, torch.float32])
def test_many_rows(N, D, M, dtype):
    """More tiles than compute units, and fp32 rows whose parts are made in two
    turns; with the caller's workspace (dirty) and with none at all, which takes
    the kernel of few rows."""
    w = mdn.quantize_w4(rand((D, M), 3) * D ** -0.5)
    A, bias = rand((N, D), 4, dtype), rand((M,), 5)
    y = check(A, w, bias, "relu")
    ws = torch.full((mdn.matmul_w4_workspace_bytes(A, M) + 255,), 255, dtype=torch.uint8, device=DEV)
    assert torch.equal(mdn.matmul_w4(A, w, col_bias=bias, act="relu", workspace=ws), y)
    with pytest.raises(ValueError):
        mdn.matmul_w4(A, w, workspace=ws[:1000])
    z = mdn.matmul_w4(A, w, col_bias=bias, act="relu", out_dtype=torch.float32)
    none = torch.empty_like(z)
    st = _lib.lib().maddness_matmul_w4(A.data_ptr(), {torch.float32: 0, torch.bfloat16: 1, torch.float16: 2}[dtype], N, D, D, w.codes.data_ptr(),
                                       w.exps.data_ptr(), M, bias.data_ptr(), 2, none.data_ptr(), 0, None, 0, torch.cuda.current_stream().cuda_stream)
    assert st == 0
    assert torch.allclose(none, z, rtol=1e-4, atol=1e-4)
    few = torch.cat([mdn.matmul_w4(A[n:n + 64], w, col_bias=bias, act="relu", out_dtype=torch.float32) for n in (0, 64, N - 64)])
    many = torch.cat([z[:128], z[N - 64:]])
    assert torch.allclose(many, few, rtol=1e-4, atol=1e-4)


@pytest.mark.parametrize("dtype", [torch.float16, torch.bfloat16])
def test_exponents_far_apart(dtype):
    """Groups of one column 30 octaves apart, columns of the largest and the
    smallest exponents: exact weights all the same."""
    D, M = 128, 300
    B = rand((D, M), 3)
    B[32:64] *= 2.0 ** -30
    B[:, 10] *= 2.0 ** 100
    B[:, 11] *= 2.0 ** -80
    B[:, 12] = 0.0
    w = mdn.quantize_w4(B)
    A = rand((1700, D), 4, dtype)
    A[:, :32] = 0
    A[:, 64:] = 0     # only the small groups are left
    W = mdn.dequantize_w4(w, dtype=torch.float32).double()
    for rows in (A, A[:300], A[:9]):
        y = mdn.matmul_w4(rows, w, out_dtype=torch.float32).double()
        ref, size = rows.double() @ W, rows.double().abs() @ W.abs()
        assert bool(((y - ref).abs() <= size * 70 * 2.0 ** -23).all())


@pytest.mark.parametrize("N,D,M", [(1, 256, 130), (5, 300, 7), (70, 129, 1003), (300, 512, 512), (40, 700, 9000), (100, 200, 20000), (130, 257, 45000)])
@pytest.mark.parametrize("act", ["bias", "relu", "softmax"])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_layer_output(N, D, M, act, dtype):
    w = mdn.quantize_w4(rand((D, M), 3) * D ** -0.5)
    A, bias = rand((N, D), 4, dtype), rand((M,), 5)
    check(A, w, bias, act, torch.float32)
    if act != "softmax":
        check(A, w, bias, act)
    check(A, w, None, act, torch.float32)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16, torch.float32])
@pytest.mark.parametrize("N", [3, 150])
def test_strides_and_sentinels(dtype, N):
    """Rows of any stride and alignment; what lies around A (NaN) is not read
    into the result, what lies behind y is left as it was."""
    D, M = 515, 77
    w = mdn.quantize_w4(rand((D, M), 3))
    for pad, off in ((0, 0), (1, 1), (8, 0), (13, 5)):
        big = torch.full((N + 1, D + pad + off), math.nan, dtype=dtype, device=DEV)
        big[:N, off:off + D] = rand((N, D), 4, dtype)
        A = big[:N, off:off + D]
        got = check(A, w, None, "none")
        store = torch.full((N * M + 64,), 7.0, dtype=dtype, device=DEV)
        y = store[:N * M].view(N, M)
        assert mdn.matmul_w4(A, w, y_out=y) is y
        assert torch.equal(y, got) and bool((store[N * M:] == 7.0).all())


def test_wide_rows_softmax_and_switched_off_columns():
    M = 70001
    w = mdn.quantize_w4(rand((64, M), 3))
    bias = rand((M,), 5)
    bias[M // 2:] = -math.inf
    bias[5] = torch.finfo(torch.float32).min
    A = rand((2, 64), 4)
    p = mdn.matmul_w4(A, w, col_bias=bias, act="softmax")
    z = A.double() @ mdn.dequantize_w4(w, dtype=torch.float32).double() + bias.double()
    ref = torch.softmax(z, 1)
    assert not p[:, M // 2:].any() and not p[:, 5].any()
    assert float(((p.double() - ref).abs() / ref.clamp(min=1e-30)).amax()) < (M + 100) * 2.0 ** -23
    assert torch.allclose(p.double().sum(1), torch.ones(2, device=DEV, dtype=torch.float64), atol=1e-4)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16, torch.float32])
def test_values_that_are_not_finite(dtype):
    """An infinite activation gives the infinity that its weight's sign says
    (NaN for a zero weight), a NaN only its own row; a NaN group its columns."""
    D, M = 200, 40
    B = rand((D, M), 3)
    B[7, 9] = 0.0
    w = mdn.quantize_w4(B)
    W = mdn.dequantize_w4(w, dtype=torch.float32)
    for N in (4, 90, 600, 1700):
        A = rand((N, D), 4, dtype)
        A[1, 7] = math.inf
        A[2, 100] = math.nan
        y = mdn.matmul_w4(A, w, out_dtype=torch.float32)
        want = torch.sign(W[7]) * math.inf
        want[W[7] == 0] = math.nan
        assert torch.equal(torch.nan_to_num(y[1], nan=5.0), torch.nan_to_num(want, nan=5.0))
        assert y[2].isnan().all() and torch.isfinite(y[0]).all() and torch.isfinite(y[3:]).all()
    big = torch.full((1, D), torch.finfo(dtype).max, dtype=dtype, device=DEV)   # (every part stays finite)
    half = mdn.quantize_w4(torch.full((D, 1), 2.0 ** -20, device=DEV))
    check(big, half, None, "none", torch.float32)
    B[150, 3] = math.nan
    for N in (4, 300, 1700):
        y = mdn.matmul_w4(rand((N, D), 4, dtype), mdn.quantize_w4(B))
        assert y[:, 3].isnan().all() and torch.isfinite(y[:, 4:]).all()


def test_refusals():
    w = mdn.quantize_w4(rand((64, 20), 3))
    A = rand((4, 64), 4, torch.bfloat16)
    with pytest.raises(ValueError):
        mdn.matmul_w4(rand((4, 63), 4), w)
    with pytest.raises(ValueError):
        mdn.matmul_w4(rand((64, 4), 4).t(), w)                # columns not dense
    with pytest.raises(ValueError):
        mdn.matmul_w4(A[:1].expand(4, 64), w)                 # overlapping rows
    with pytest.raises(ValueError):
        mdn.matmul_w4(A, w._replace(M=33))
    with pytest.raises(ValueError):
        mdn.matmul_w4(A, w._replace(D=200))
    with pytest.raises(ValueError):
        mdn.matmul_w4(A, w, act="gelu")
    with pytest.raises(ValueError):
        mdn.matmul_w4(A, w, col_bias=rand((19,), 1))
    with pytest.raises(TypeError):
        mdn.matmul_w4(A, w, out_dtype=torch.float16)
    with pytest.raises(TypeError):
        mdn.matmul_w4(A, w, act="softmax", out_dtype=torch.bfloat16)
    with pytest.raises(TypeError):
        mdn.matmul_w4(A.double(), w)
    with pytest.raises(ValueError):
        mdn.matmul_w4(A, w, y_out=torch.empty((4, 21), dtype=torch.bfloat16, device=DEV))
    with pytest.raises(mdn.MaddnessError):
        mdn.matmul_w4(A, w, act=7)
    with pytest.raises(TypeError):
        mdn.dequantize_w4(w, dtype=torch.float16)
    with pytest.raises(ValueError):
        mdn.quantize_w4(torch.empty((0, 4), device=DEV))
    assert mdn.matmul_w4(A[:0], w).shape == (0, 20)
