"""The output layer's operators as they are used together: gradient steps on
its weights, the weights quantized, single rows answered; on streams of the
caller's, in captured graphs, and several calls at once."""
import pytest
import torch

import paper_2207_05808_amd as mdn

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def rand(shape, seed, dtype=torch.float32):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    return torch.randn(*shape, generator=g, device=DEV).to(dtype)


def layer(N=300, D=200, M=1000, dtype=torch.bfloat16):
    A, B = rand((N, D), 1, dtype), (rand((D, M), 2) * D ** -0.5).to(dtype)
    return A, B, torch.randint(0, M, (N,), device=DEV), rand((M,), 3) * 0.1


def step(A, B, target, b, eta):
    loss, lse = mdn.linear_xent(A, B, target, col_bias=b)
    g = torch.full_like(lse, 1.0 / len(lse))
    dA, dB, db = mdn.linear_xent_grad(A, B, target, lse, g, col_bias=b)
    return loss, dA, B - eta * dB, b - eta * db


def test_train_quantize_answer():
    """Three gradient steps in fp32 follow the same steps in 64 bits; the
    trained weights, quantized, give the probabilities of the quantized layer."""
    A, B, target, b = layer(dtype=torch.float32)
    B64, b64 = B.double(), b.double()
    for _ in range(3):
        loss, dA, B, b = step(A, B, target, b, 2.0)
        z = A.double() @ B64 + b64
        G = torch.softmax(z, 1)
        rloss = torch.logsumexp(z, 1) - z.gather(1, target[:, None])[:, 0]
        G[torch.arange(len(target)), target] -= 1.0
        G /= len(target)
        rdA = G @ B64.t()
        B64, b64 = B64 - 2.0 * (A.double().t() @ G), b64 - 2.0 * G.sum(0)
        # a chain of 6 * 200 / 16 part products and 16 terms, sizes below 40, 2^-23 each, three steps
        assert float((loss.double() - rloss).abs().max()) < 40 * 100 * 2.0 ** -23 * 3
        assert float((dA.double() - rdA).abs().max()) < 1e-3 * float(rdA.abs().max())
    assert float((B.double() - B64).abs().max()) < 1e-4
    w = mdn.quantize_w4(B)
    W = mdn.dequantize_w4(w, dtype=torch.float32)
    for n in (0, 7, 299):
        p = mdn.matmul_w4(A[n:n + 1], w, col_bias=b, act="softmax")
        ref = torch.softmax(A[n:n + 1].double() @ W.double() + b.double(), 1)
        assert float(((p.double() - ref) / ref).abs().max()) < (2 * 40 * 100 + 1000 + 30) * 2.0 ** -23
    every = mdn.matmul_w4(A, w, col_bias=b, act="softmax")
    assert torch.equal(every.argmax(1)[:3], torch.cat([mdn.matmul_w4(A[n:n + 1], w, col_bias=b, act="softmax") for n in range(3)]).argmax(1))


def test_caller_streams():
    """Every call on a stream that is not the current one gives the same bits,
    two at once on two streams too (each with its own workspace)."""
    A, B, target, b = layer()
    loss, dA, B1, b1 = step(A, B, target, b, 0.5)
    w = mdn.quantize_w4(B)
    y = mdn.matmul_w4(A, w, col_bias=b)
    streams = [torch.cuda.Stream() for _ in range(2)]
    torch.cuda.synchronize()
    for _ in range(4):
        out = []
        for s in streams:
            l, e = mdn.linear_xent(A, B, target, col_bias=b, stream=s)
            with torch.cuda.stream(s):
                g = torch.full_like(e, 1.0 / len(e))
                out.append((l, *mdn.linear_xent_grad(A, B, target, e, g, col_bias=b)))
            q = mdn.quantize_w4(B, stream=s)
            out[-1] += (mdn.matmul_w4(A, q, col_bias=b, stream=s), q.codes, q.exps)
        torch.cuda.synchronize()
        for l, da, dB, db, yy, c, x in out:
            assert torch.equal(l, loss) and torch.equal(da, dA) and torch.equal(yy, y)
            assert torch.equal(B - 0.5 * dB, B1) and torch.equal(b - 0.5 * db, b1)
            assert torch.equal(c, w.codes) and torch.equal(x, w.exps)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_captured(dtype):
    """A training step and an answer captured in a graph, replayed on new
    inputs with the program's own work between the replays."""
    A, B, target, b = layer(dtype=dtype)
    w = mdn.quantize_w4(B)

    def work():
        loss, lse = mdn.linear_xent(A, B, target, col_bias=b)
        g = torch.full_like(lse, 1.0 / len(lse))
        return (loss, *mdn.linear_xent_grad(A, B, target, lse, g, col_bias=b), mdn.matmul_w4(A, w, col_bias=b, act="relu"),
                mdn.matmul_w4(A[:1], w, col_bias=b, act="softmax"))

    s = torch.cuda.Stream()
    with torch.cuda.stream(s):
        work()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        held = work()
    for k in range(4):
        A.copy_(rand(A.shape, 20 + k, dtype))
        target.copy_(torch.randint(0, B.shape[1], target.shape, device=DEV))
        graph.replay()
        torch.cuda.synchronize()
        for x, y in zip(held, work()):
            assert torch.equal(x, y)
        torch.cuda.synchronize()


def test_two_graphs_share_a_workspace():
    """Two captured calls that name the same workspace, replayed one after the
    other on one stream."""
    A, B, target, b = layer()
    A2 = rand((150, 200), 9, torch.bfloat16)
    size = max(mdn.linear_xent_grad_workspace_bytes(n, 200, 1000, torch.bfloat16) for n in (300, 150)) + 255
    ws = torch.empty((size,), dtype=torch.uint8, device=DEV)
    calls = []
    for a, t in ((A, target), (A2, target[:150].clone())):
        _, lse = mdn.linear_xent(a, B, t, col_bias=b)
        g = torch.full_like(lse, 0.25)
        calls.append((a, t, lse, g))
    want = [mdn.linear_xent_grad(a, B, t, lse, g, col_bias=b) for a, t, lse, g in calls]
    graphs = []
    for a, t, lse, g in calls:
        mdn.linear_xent_grad(a, B, t, lse, g, col_bias=b, workspace=ws)
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            out = mdn.linear_xent_grad(a, B, t, lse, g, col_bias=b, workspace=ws)
        graphs.append((graph, out))
    for _ in range(3):
        for graph, _ in graphs:
            graph.replay()
        torch.cuda.synchronize()
        for (_, out), ref in zip(graphs, want):
            assert all(torch.equal(x, y) for x, y in zip(out, ref))
