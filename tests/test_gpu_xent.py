"""Softmax cross entropy without logits, and its gradient, against 64 bits.

Tolerances count roundings.  Logits: terms are exact (bf16) or lose 2^-24 each
(fp32 in parts), sums lose at most 2^-23 of the running size per step of 16 k
and part product and per term of a step.  lse: the logits' error, the sums of
exponentials (at most 300 steps and the logits' range, 2^-23 each).  Gradients:
G's relative error from its exponent, half a step of bf16 where G is rounded to
it, the two products as above, one rounding of the result."""
import math

import pytest
import torch

import paper_2207_05808_amd as mdn

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
U = 2.0 ** -23
CHAIN = {torch.bfloat16: 1, torch.float32: 6}


def rand(shape, seed, dtype=torch.float32):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    return torch.randn(*shape, generator=g, device=DEV).to(dtype)


def problem(N, D, M, dtype, md, bias=True, seed=1):
    B = (rand((M, D), seed) * D ** -0.5).to(dtype)
    B = B.t() if md else B.t().contiguous()
    A = rand((N, D), seed + 1, dtype) * 3
    g = torch.Generator(device=DEV)
    g.manual_seed(seed + 2)
    target = torch.randint(0, M, (N,), generator=g, device=DEV)
    target[::5] = -100 if N > 1 else target[::5]
    b = rand((M,), seed + 3) if bias else None
    gl = torch.rand((N,), generator=g, device=DEV) / N
    return A, B, target, b, gl


def steps(K, dtype):
    return K / 16 * CHAIN[dtype] + 16 + 2


def logits64(A, B, b):
    """(z, how far a logit may be off)"""
    z, size = A.double() @ B.double(), A.double().abs() @ B.double().abs()
    if b is not None:
        z, size = z + b.double(), size + torch.nan_to_num(b.double().abs(), posinf=0.0)
    return z, size * steps(A.shape[1], A.dtype) * U


def loss64(z, target):
    M = z.shape[1]
    live = (target >= 0) & (target < M)
    lse = torch.logsumexp(z, 1)
    zt = z.gather(1, torch.where(live, target, 0)[:, None])[:, 0]
    return torch.where(live, torch.where(lse == -math.inf, math.inf, lse - zt), 0.0), lse, live


def close(x, ref, tol):
    same = torch.nan_to_num(x.double(), posinf=9e99, neginf=-9e99) == torch.nan_to_num(ref, posinf=9e99, neginf=-9e99)
    ok = same | ((x.double() - ref).abs() <= tol)
    assert bool(ok.all()), float(((x.double() - ref).abs() / tol)[~ok].max())


def lse_tol(z, dz, lse):
    reach = torch.where(torch.isfinite(z), z.amax(1, keepdim=True) - z, 0.0).clamp(max=100).amax(1)
    return dz.amax(1) + (300 + 2 * reach) * U + lse.abs().nan_to_num(posinf=0.0) * U


def check_forward(A, B, target, b, **kw):
    loss, lse = mdn.linear_xent(A, B, target, col_bias=b, **kw)
    z, dz = logits64(A, B, b)
    rloss, rlse, live = loss64(z, target)
    tol = lse_tol(z, dz, rlse)
    close(lse, rlse, tol)
    close(loss, rloss, tol + dz.amax(1) + z.abs().nan_to_num(posinf=0.0).amax(1) * U)
    return loss, lse


def grads64(A, B, target, b, gl, lse):
    """Gradients for this lse, and how far each may be off."""
    z, dz = logits64(A, B, b)
    M = z.shape[1]
    live = (target >= 0) & (target < M) & (lse > -math.inf)
    x = z - torch.where(live, lse.double(), 0.0)[:, None]
    p = torch.where(live[:, None], torch.exp(x), 0.0)
    g = torch.where(live, gl.double(), 0.0)[:, None]
    G = p.clone()
    G[live, target[live]] -= 1.0
    G = G * g
    dG = g.abs() * (p * (dz + (2 * x.abs().nan_to_num(posinf=0.0) + 8) * U) + (G.abs() / g.abs().clamp(min=1e-300)) * U)
    db, ddb = G.sum(0), dG.sum(0) + G.abs().sum(0) * (A.shape[0] / 32 + 40) * U
    half = torch.finfo(A.dtype).eps / 2
    if A.dtype != torch.float32:
        dG = dG + G.abs() * half
    Ad, Bd = A.double(), B.double()
    dA, dB = G @ Bd.t(), Ad.t() @ G
    tA = dG @ Bd.abs().t() + (G.abs() @ Bd.abs().t()) * steps(M, A.dtype) * U + dA.abs() * half
    tB = Ad.abs().t() @ dG + (Ad.abs().t() @ G.abs()) * steps(A.shape[0], A.dtype) * U + dB.abs() * half
    tiny = 2.0 ** -120
    return (dA, tA + tiny), (dB, tB + tiny), (db, ddb + tiny)


def check_grad(A, B, target, b, gl, lse, **kw):
    got = mdn.linear_xent_grad(A, B, target, lse, gl, col_bias=b, **kw)
    for x, (ref, tol) in zip(got, grads64(A, B, target, b, gl, lse)):
        assert x.shape == ref.shape
        close(x, ref, tol)
    return got


SHAPES = [(1, 1, 1), (1, 64, 300), (3, 24, 10), (32, 100, 129), (33, 257, 1000), (100, 512, 100), (130, 64, 2001), (257, 136, 520),
          (64, 1000, 65), (2000, 72, 40)]


@pytest.mark.parametrize("N,D,M", SHAPES)
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("md", [False, True])
def test_forward_and_gradient(N, D, M, dtype, md):
    A, B, target, b, gl = problem(N, D, M, dtype, md, bias=(N + M) % 2 == 0)
    _, lse = check_forward(A, B, target, b)
    dA, dB, _ = check_grad(A, B, target, b, gl, lse)
    assert dA.is_contiguous() and dB.t().is_contiguous() == (md or D == 1 or M == 1) and dA.dtype == dB.dtype == dtype
    dead = (target < 0)
    assert not dA[dead].any()


@pytest.mark.parametrize("N,D,M,dtype,md", [(700, 200, 5000, torch.bfloat16, True), (700, 200, 5000, torch.bfloat16, False),
                                            (5000, 48, 9000, torch.bfloat16, False), (4200, 40, 9001, torch.float32, True),
                                            (40, 96, 70001, torch.bfloat16, False), (9000, 264, 4100, torch.bfloat16, True),
                                            (600, 600, 25001, torch.bfloat16, False), (600, 601, 25001, torch.bfloat16, True),
                                            (600, 616, 25000, torch.bfloat16, True), (520, 600, 30011, torch.bfloat16, True), (600, 601, 25001, torch.bfloat16, False),
                                            (700, 75, 9001, torch.float32, False), (700, 75, 9001, torch.float32, True),
                                            (9000, 1032, 30001, torch.bfloat16, False), (9001, 1000, 30000, torch.bfloat16, True)])
def test_larger(N, D, M, dtype, md):
    """More tiles than the card has compute units, whole 16-byte rows and odd
    ones, long sums split, and (9000 rows) the outputs in several pieces."""
    A, B, target, b, gl = problem(N, D, M, dtype, md)
    _, lse = check_forward(A, B, target, b)
    check_grad(A, B, target, b, gl, lse)


def test_pieces_are_used():
    """The sizes above do take several pieces: the workspace is below all of G."""
    assert mdn.linear_xent_grad_workspace_bytes(9000, 264, 41000, torch.bfloat16) < 9000 * 41000 * 2
    A, B, target, b, gl = problem(9000, 32, 17000, torch.bfloat16, True)
    _, lse = check_forward(A, B, target, b)
    check_grad(A, B, target, b, gl, lse)


def test_gradient_against_differences():
    """Central differences of the loss this library computes (fp32; the step
    moves a loss of about 3 by 1e-2, its own rounding is below 1e-5)."""
    A, B, target, b, gl = problem(6, 20, 30, torch.float32, False)
    gl = gl * 0 + 1.0
    _, lse = mdn.linear_xent(A, B, target, col_bias=b)
    dA, dB, db = mdn.linear_xent_grad(A, B, target, lse, gl, col_bias=b)
    h = 2.0 ** -6
    total = lambda *a: float(mdn.linear_xent(a[0], a[1], target, col_bias=a[2])[0].double().sum())  # noqa: E731
    for t, d in ((0, dA), (1, dB), (2, db)):
        for at in ((1, 3), (2, 7), (4, 19)):
            at = at if t < 2 else at[1:]
            args = [A, B, b]
            ends = []
            for s in (h, -h):
                moved = [x.clone() for x in args]
                moved[t][at] += s
                ends.append(total(*moved))
            want = (ends[0] - ends[1]) / (2 * h)
            # third derivative of a sum of 6 log-sum-exps of logits moved by |x| h <= 12 h: below 6 * 12^3 h^2 / 6
            assert abs(want - float(d[at])) <= 12.0 ** 3 * h * h / 10 + 6e-5 / h


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_masks(dtype):
    """Outputs switched off by -inf or the type's lowest value, a target among
    them, rows without a target (also past M), a row of which nothing is left."""
    N, D, M = 70, 64, 333
    A, B, target, b, gl = problem(N, D, M, dtype, False)
    target[:] = torch.arange(N, device=DEV) % 100
    target[3], target[4], target[5], target[6] = -1, M, M + 10 ** 12, -(2 ** 62)
    b[200:] = -math.inf
    b[150:160] = torch.finfo(torch.float32).min
    b[20] = -math.inf
    loss, lse = check_forward(A, B, target, b)
    assert loss[20] == math.inf and not loss[3:7].any()
    gl[20] = 0.0   # (its loss is infinite)
    dA, dB, db = check_grad(A, B, target, b, gl, lse)
    assert not dA[3:7].any() and not dB[:, 200:].any() and not db[200:].any() and not dB[:, 20].any()
    b[:] = -math.inf
    loss, lse = mdn.linear_xent(A, B, target, col_bias=b)
    assert bool((lse == -math.inf).all()) and not loss[3:7].any() and bool((loss[7:] == math.inf).all())
    for x in mdn.linear_xent_grad(A, B, target, lse, gl, col_bias=b):
        assert not x.any()
    b[:] = torch.finfo(torch.float32).min
    z, _ = logits64(A * 0, B, b)
    loss, lse = mdn.linear_xent(A * 0, B, target, col_bias=b)
    assert torch.allclose(lse.double(), torch.logsumexp(z, 1), rtol=1e-6)


def test_large_and_small_logits():
    """Logits of hundreds (no overflow) and losses near zero."""
    A, B, target, b, gl = problem(50, 64, 200, torch.float32, True)
    A = A * 60
    _, lse = check_forward(A, B, target, b)
    check_grad(A, B, target, b, gl, lse)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_strides_sentinels_and_repeats(dtype):
    """Rows of A of any stride and alignment among NaN, outputs among
    sentinels, workspace the caller's and dirty: the same bits every time."""
    N, D, M = 77, 130, 501
    A0, B, target, b, gl = problem(N, D, M, dtype, False)
    first = None
    for pad, off in ((0, 0), (1, 1), (6, 0), (21, 9)):
        big = torch.full((N + 1, D + pad + off), math.nan, dtype=dtype, device=DEV)
        big[:N, off:off + D] = A0
        A = big[:N, off:off + D]
        ws = torch.full((mdn.linear_xent_workspace_bytes(N, D, M, dtype) + 255,), 255, dtype=torch.uint8, device=DEV)
        wg = torch.full((mdn.linear_xent_grad_workspace_bytes(N, D, M, dtype) + 255,), 255, dtype=torch.uint8, device=DEV)
        bufs = [torch.full((n + 99,), 7.0, dtype=t, device=DEV) for n, t in ((N, torch.float32), (N, torch.float32), (N * D, dtype), (D * M, dtype), (M, torch.float32))]
        loss, lse = mdn.linear_xent(A, B, target, col_bias=b, loss_out=bufs[0][:N], lse_out=bufs[1][:N], workspace=ws)
        dA, dB, db = mdn.linear_xent_grad(A, B, target, lse, gl, col_bias=b, dA_out=bufs[2][:N * D].view(N, D),
                                          dB_out=bufs[3][:D * M].view(D, M), dbias_out=bufs[4][:M], workspace=wg)
        for t, n in zip(bufs, (N, N, N * D, D * M, M)):
            assert bool((t[n:] == 7.0).all())
        out = [t.clone() for t in (loss, lse, dA, dB, db)]
        assert all(torch.isfinite(t).all() for t in out)
        if first is None:
            first = out
            check_forward(A, B, target, b)
            check_grad(A, B, target, b, gl, lse)
        assert all(torch.equal(x, y) for x, y in zip(first, out))


def test_no_rows():
    A, B = torch.empty((0, 16), device=DEV), rand((16, 40), 1)
    t = torch.empty((0,), dtype=torch.int64, device=DEV)
    loss, lse = mdn.linear_xent(A, B, t)
    assert loss.shape == lse.shape == (0,)
    dA, dB, db = mdn.linear_xent_grad(A, B, t, lse, loss)
    assert dA.shape == (0, 16) and dB.shape == (16, 40) and not dB.any() and not db.any()


def test_refusals():
    A, B, target, b, gl = problem(8, 16, 40, torch.float32, False)
    lse = gl.clone()
    bad = [lambda: mdn.linear_xent(A, B[:, ::2], target), lambda: mdn.linear_xent(A, B[:15], target),
           lambda: mdn.linear_xent(A, B, target[:7]), lambda: mdn.linear_xent(A, B, target, col_bias=b[:3]),
           lambda: mdn.linear_xent(A.t().contiguous().t(), B, target), lambda: mdn.linear_xent(A[:1].expand(8, 16), B, target),
           lambda: mdn.linear_xent(A, B, target, workspace=torch.empty(8, dtype=torch.uint8, device=DEV)),
           lambda: mdn.linear_xent(A, B, target, loss_out=torch.empty(9, device=DEV)),
           lambda: mdn.linear_xent(A, B, target.cpu()), lambda: mdn.linear_xent_grad(A, B, target, lse[:4], gl),
           lambda: mdn.linear_xent_grad(A, B, target, lse, gl[:4]),
           lambda: mdn.linear_xent_grad(A, B, target, lse, gl, dB_out=torch.empty((40, 16), device=DEV).t()),
           lambda: mdn.linear_xent(A, B, target, workspace=torch.empty(1 << 20, dtype=torch.uint8))]
    for call in bad:
        with pytest.raises(ValueError):
            call()
    for call in (lambda: mdn.linear_xent(A.half(), B.half(), target), lambda: mdn.linear_xent(A, B.bfloat16(), target),
                 lambda: mdn.linear_xent(A, B, target.int()), lambda: mdn.linear_xent_grad(A, B, target, lse.double(), gl)):
        with pytest.raises(TypeError):
            call()
