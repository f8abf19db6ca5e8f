"""The output layer's C entry points on the host: bad arguments are rejected
before any HIP call, sizes of workspaces and packed weights are what the header
says (no GPU needed, nothing is launched)."""
import ctypes

import pytest
import torch

import paper_2207_05808_amd as mdn

FAKE, NULL = ctypes.c_void_p(0x10000), None   # never dereferenced


def at(n):
    return ctypes.c_void_p(0x10000 + n)


@pytest.fixture(scope="module")
def L():
    from paper_2207_05808_amd import _lib
    return _lib.lib()


def rejects(fn, good, changes):
    for where, value, status in changes:
        args = list(good)
        args[where] = value
        assert fn(*args) == status, (where, value)


def test_packed_sizes(L):
    assert L.maddness_w4_code_bytes(1, 1) == 1024 and L.maddness_w4_exponent_bytes(1, 1) == 64
    assert L.maddness_w4_code_bytes(128, 16) == 1024
    assert L.maddness_w4_code_bytes(129, 17) == 4096 and L.maddness_w4_exponent_bytes(129, 17) == 256
    assert L.maddness_w4_code_bytes(1 << 20, 1 << 20) == 1 << 39
    for D, M in ((0, 4), (4, 0), (-1, 4)):
        assert L.maddness_w4_code_bytes(D, M) == -1 and L.maddness_w4_exponent_bytes(D, M) == -1


def test_quantize_rejects(L):
    #       B dtype D  M  sd sm codes exps stream
    good = [FAKE, 0, 64, 16, 16, 1, FAKE, FAKE, NULL]
    rejects(L.maddness_quantize_w4, good, [
        (0, NULL, 1), (1, -1, 1), (1, 3, 1), (2, 0, 1), (3, 0, 1), (4, -1, 1), (5, -1, 1), (6, NULL, 1), (7, NULL, 1),
        (0, at(2), 1), (6, at(8), 1), (7, at(2), 1), (2, (1 << 31) - 100, 3), (3, (1 << 31) - 100, 3)])
    good = [FAKE, FAKE, 64, 16, FAKE, 1, NULL]
    rejects(L.maddness_dequantize_w4, good, [
        (0, NULL, 1), (1, NULL, 1), (2, 0, 1), (3, -3, 1), (4, NULL, 1), (5, 2, 1), (5, -1, 1), (0, at(4), 1), (1, at(1), 1), (4, at(1), 1), (2, (1 << 31) - 1, 3), (3, (1 << 31) - 1, 3)])


def test_matmul_rejects(L):
    #       A  dtype N  D   lda codes exps M  bias act y  ydtype ws bytes stream
    good = [FAKE, 1, 10, 64, 64, FAKE, FAKE, 16, NULL, 0, FAKE, 1, NULL, 0, NULL]
    rejects(L.maddness_matmul_w4, good, [
        (0, NULL, 1), (1, 3, 1), (1, -1, 1), (2, -1, 1), (3, 0, 1), (4, 63, 1), (5, NULL, 1), (6, NULL, 1), (7, 0, 1), (9, 4, 1), (9, -1, 1),
        (10, NULL, 1), (11, 2, 1), (0, at(1), 1), (5, at(8), 1), (6, at(2), 1), (8, at(2), 1), (10, at(1), 1), (7, (1 << 31) - 1, 3)])
    rejects(L.maddness_matmul_w4, good, [(9, 3, 1)])   # a softmax in 16 bits
    assert L.maddness_matmul_w4(NULL, 1, 0, 64, 64, NULL, NULL, 16, NULL, 0, NULL, 1, NULL, 0, NULL) == 0
    size = L.maddness_matmul_w4_workspace_bytes(FAKE, 1, 4000, 64, 64, 512)
    assert size > 0
    many = [FAKE, 1, 4000, 64, 64, FAKE, FAKE, 512, NULL, 0, FAKE, 1, FAKE, size, NULL]
    rejects(L.maddness_matmul_w4, many, [(12, at(64), 1), (13, size - 1, 1), (13, 0, 1)])
    Q = L.maddness_matmul_w4_workspace_bytes
    assert Q(FAKE, 1, 1, 64, 64, 512) == 0 and Q(NULL, 0, 0, 64, 64, 512) == 0
    for bad in ((FAKE, 3, 10, 64, 64, 512), (FAKE, 1, -1, 64, 64, 512), (FAKE, 1, 10, 0, 64, 512), (FAKE, 1, 10, 64, 63, 512), (FAKE, 1, 10, 64, 64, 0)):
        assert Q(*bad) == -1


def test_xent_rejects(L):
    size = L.maddness_linear_xent_workspace_bytes(10, 64, 100, 1)
    assert size > 0
    #       A  dtype N  D   lda B  M  first bias target loss lse ws bytes stream
    good = [FAKE, 1, 10, 64, 64, FAKE, 100, 0, NULL, FAKE, FAKE, FAKE, FAKE, size, NULL]
    rejects(L.maddness_linear_xent, good, [
        (0, NULL, 1), (1, 2, 1), (1, -1, 1), (2, -1, 1), (2, 1 << 31, 3), (3, 0, 1), (4, 63, 1), (5, NULL, 1), (6, 0, 1), (7, 2, 1),
        (8, at(1), 1), (9, NULL, 1), (9, at(4), 1), (10, NULL, 1), (11, NULL, 1), (12, NULL, 1), (12, at(128), 1), (13, size - 1, 1),
        (0, at(1), 1), (5, at(1), 1), (10, at(2), 1), (11, at(2), 1)])
    assert L.maddness_linear_xent(NULL, 1, 0, 64, 64, FAKE, 100, 0, NULL, NULL, NULL, NULL, NULL, 0, NULL) == 0


def test_xent_grad_rejects(L):
    size = L.maddness_linear_xent_grad_workspace_bytes(10, 64, 100, 0)
    assert size > 0
    #       A  dtype N  D   lda B  M  first bias target lse g dA dB db ws bytes stream
    good = [FAKE, 0, 10, 64, 64, FAKE, 100, 1, NULL, FAKE, FAKE, FAKE, FAKE, FAKE, FAKE, FAKE, size, NULL]
    rejects(L.maddness_linear_xent_grad, good, [
        (0, NULL, 1), (1, 2, 1), (2, -1, 1), (2, 1 << 31, 3), (3, 0, 1), (4, 63, 1), (5, NULL, 1), (6, 0, 1), (7, -1, 1), (8, at(2), 1),
        (9, NULL, 1), (10, NULL, 1), (11, NULL, 1), (12, NULL, 1), (13, NULL, 1), (14, NULL, 1), (15, NULL, 1), (15, at(64), 1),
        (16, size - 1, 1), (10, at(2), 1), (11, at(1), 1), (12, at(2), 1), (13, at(2), 1), (14, at(2), 1)])


def test_xent_workspace(L):
    """The gradient's workspace stays far below the logits of a large
    vocabulary, and out of range sizes are refused."""
    N, D, M = 8192, 4096, 131072
    assert L.maddness_linear_xent_grad_workspace_bytes(N, D, M, 1) < N * M * 4 // 8
    for f in (L.maddness_linear_xent_workspace_bytes, L.maddness_linear_xent_grad_workspace_bytes):
        assert f(0, 8, 8, 0) > 0 and f((1 << 31) - 1, 8, 8, 0) > 0
        for bad in ((-1, 8, 8, 0), (1 << 31, 8, 8, 0), (8, 0, 8, 0), (8, 8, 0, 0), (8, 8, 8, 2), (8, 8, 8, -1)):
            assert f(*bad) == -1
    with pytest.raises(mdn.MaddnessError):
        mdn.linear_xent_workspace_bytes(8, 8, 8, torch.float16)


def test_binding_refuses_host_tensors_and_types():
    A, B, t = torch.zeros(4, 8), torch.zeros(8, 6), torch.zeros(4, dtype=torch.int64)
    v = torch.zeros(4)
    for call in (lambda: mdn.quantize_w4(B), lambda: mdn.linear_xent(A, B, t), lambda: mdn.linear_xent_grad(A, B, t, v, v)):
        with pytest.raises(ValueError, match="device"):
            call()
    for call in (lambda: mdn.quantize_w4(B.double()), lambda: mdn.quantize_w4([1.0]), lambda: mdn.linear_xent(A.half(), B.half(), t),
                 lambda: mdn.matmul_w4(A.int(), None), lambda: mdn.dequantize_w4((1, 2, 3, 4))):
        with pytest.raises(TypeError):
            call()
