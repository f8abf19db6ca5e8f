"""What the output layer's operators are timed on: softmax cross entropy over a
large set of outputs without keeping the logits (with its gradient), and
products with 4-bit block floating point weights (with their quantizer).

`run` computes a pass in plain torch, in 32 bits, or with this framework's
kernels where `own` is set; `exact` computes it from the definition in 64
bits.  Inputs are drawn on the GPU: activations that lean towards their
target's weight column (as those of a partly trained layer do), weights of
variance 1 / D, a share of rows without a target, and vocabularies padded with
columns that a bias of -inf switches off.
"""
from __future__ import annotations

import math

import torch

own = False

GROUP = 32                       # rows of one weight column that share a scale
KB, MB = 128, 16                 # rows and columns of a block of packed weights
VALUES = (0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0, -0.0, -0.5, -1.0, -1.5, -2.0, -3.0, -4.0, -6.0)
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
BYTES = {"f32": 4, "bf16": 2, "f16": 2}
ROWS = 1024                      # rows per block of the 64-bit references


def _w4(name, N, D, M, type, act="none", out="same", pad=0):
    return {"name": name, "kind": "w4", "N": N, "D": D, "M": M, "type": type, "act": act, "out": out, "pad": pad}


def _quant(name, D, M, type, layout="dm"):
    return {"name": name, "kind": "quant", "D": D, "M": M, "type": type, "layout": layout}


def _xent(name, kind, N, D, M, type, layout="dm", bias=True, off=0):
    return {"name": name, "kind": kind, "N": N, "D": D, "M": M, "type": type, "layout": layout, "bias": bias, "off": off}


def listed():
    return [
        # one token through a wide layer 1024 -> 4096 with bias and ReLU: the smallest call, where latency counts
        _w4("w4_token_wide", 1, 1024, 4096, "bf16", act="relu"),
        # one token through an output layer of 65536 classes, logits in fp32: all of the weights are read once
        _w4("w4_token_head", 1, 4096, 65536, "bf16", out="f32"),
        # an odd serving batch of fp32 rows (the framework's own activations), odd sizes, class probabilities
        _w4("w4_batch_softmax", 37, 1000, 1003, "f32", act="softmax", out="f32"),
        # a prompt of 4096 tokens in half precision through a wide layer: bound by the products
        _w4("w4_prompt", 4096, 4096, 8192, "f16", act="relu"),
        # the wide layer's weights, quantized once for serving
        _quant("quant_wide", 1024, 4096, "f32"),
        # an output layer kept as one row per class, quantized for serving
        _quant("quant_head", 4096, 65536, "bf16", layout="md"),
        # a 100-class classifier on 512 features over a test set of 10000 images, in fp32
        _xent("xent_classifier", "xent", 10000, 512, 100, "f32"),
        # a small evaluation batch over an odd vocabulary, some of it switched off, odd rows
        _xent("xent_small_batch", "xent", 63, 1024, 50001, "bf16", off=241),
        # a training batch over a large vocabulary stored one row per class: the largest forward pass
        _xent("xent_vocabulary", "xent", 8192, 4096, 131072, "bf16", layout="md", bias=False),
        # the classifier's gradient step, in fp32
        _xent("grad_classifier", "grad", 10000, 512, 100, "f32"),
        # a ragged training batch over an odd vocabulary
        _xent("grad_odd", "grad", 1999, 1024, 50001, "bf16", off=241),
        # the large vocabulary's gradients: the largest case
        _xent("grad_vocabulary", "grad", 8192, 2048, 131072, "bf16", layout="md", bias=False),
    ]


def _log(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    kind = rng.choice(["w4", "w4", "w4", "quant", "xent", "xent", "grad", "grad"])
    if kind == "w4":
        act = rng.choice(["none", "bias", "relu", "softmax"])
        c = _w4("", rng.choice([1, 1, 2, 7, 16, _log(rng, 1, 4096), _log(rng, 17, 4096)]), _log(rng, 33, 4096),
                _log(rng, 10, 65536), rng.choice(["bf16", "bf16", "f16", "f32"]), act=act,
                out="f32" if act == "softmax" else rng.choice(["same", "f32"]), pad=rng.choice([0, 0, 3, 8]))
        c["N"] = max(1, min(c["N"], 4096 * 4096 * 8192 // (c["D"] * c["M"])))
    elif kind == "quant":
        c = _quant("", _log(rng, 33, 4096), _log(rng, 10, 65536), rng.choice(["f32", "bf16", "f16"]), rng.choice(["dm", "md"]))
    else:
        even = rng.random() < 0.5
        D, M = _log(rng, 24, 4096 if kind == "xent" else 2048), _log(rng, 10, 131072)
        if even:
            D, M = (D + 7) // 8 * 8, (M + 7) // 8 * 8
        bias = rng.random() < 0.6
        type = rng.choice(["bf16", "bf16", "f32"])
        N = _log(rng, 1, 8192 if type == "bf16" else 4096)
        if type == "f32":
            M = min(M, 50000)
        c = _xent("", kind, N, D, M, type, rng.choice(["dm", "md"]), bias, rng.choice([0, M // 50]) if bias else 0)
    c.pop("name", None)
    return c


# ------------------------------------------------------------------ inputs


def _gen(seed, k):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed * 1000003 + k)
    return g


def _randn(g, *shape):
    return torch.randn(*shape, generator=g, device="cuda", dtype=torch.float32)


def _weights(case, seed):
    """B [D][M]: in memory as it stands ("dm") or one row per column of B ("md")."""
    D, M, t = case["D"], case["M"], TYPES[case["type"]]
    if case.get("layout") == "md":
        return (_randn(_gen(seed, 1), M, D) * D ** -0.5).to(t).t()
    return (_randn(_gen(seed, 1), D, M) * D ** -0.5).to(t)


def _exponents(B):
    """(e [G][M] int32, B [G][32][M] padded with zeros): the smallest e in
    [-120, 125] with max |B| <= 6 2^e over each group."""
    D, M = B.shape
    G = -(-D // GROUP)
    W = torch.zeros((G * GROUP, M), device=B.device, dtype=torch.float32)
    W[:D] = B
    W = W.view(G, GROUP, M)
    m, x = torch.frexp(W.abs().amax(1))
    e = (x - 2 - (m <= 0.75).to(torch.int32)).clamp(-120, 125)
    return torch.where(m == 0, -120, e).to(torch.int32), W


def _codes(B):
    """4-bit codes [G][32][M] (sign in bit 3) and exponents [G][M]."""
    e, W = _exponents(B)
    t = torch.ldexp(W.abs().double(), -e[:, None, :]).float()
    q = (t > 0.25).to(torch.uint8)
    for edge, up in ((0.75, True), (1.25, False), (1.75, True), (2.5, False), (3.5, True), (5.0, False)):
        q += t >= edge if up else t > edge       # a tie goes to the even code
    return torch.where((W < 0) & (q > 0), q + 8, q), e


def _pack(B):
    """The packed weights as the layer keeps them: bytes [Mb][Kb][64][16] and
    biased exponents [Mb][Kb][16][4].  Lane l of a block holds column l % 16;
    nibble i of its word j is row 32 j + 8 (l // 16) + i of the block."""
    D, M = B.shape
    q, e = _codes(B)
    G = q.shape[0]
    nk, nm = -(-D // KB), -(-M // MB)
    Q = torch.zeros((nk * 4, GROUP, nm * MB), device=B.device, dtype=torch.uint8)
    E = torch.full((nk * 4, nm * MB), 127, device=B.device, dtype=torch.uint8)
    Q[:G, :, :M] = q
    E[:G, :M] = (e + 127).to(torch.uint8)
    Q = Q.view(nk, 4, 4, 4, 2, nm, MB).permute(5, 0, 2, 6, 1, 3, 4)   # [Mb][Kb][quarter][column][word][byte][nibble]
    packed = (Q[..., 0] | (Q[..., 1] << 4)).reshape(nm, nk, 64, 16).contiguous()
    return packed, E.view(nk, 4, nm, MB).permute(2, 0, 3, 1).contiguous()


def prepare(case, seed):
    if case["kind"] == "quant":
        return {"case": case, "B": _weights(case, seed)}
    N, D, M, t = case["N"], case["D"], case["M"], TYPES[case["type"]]
    if case["kind"] == "w4":
        packed, exps = _pack(_weights({**case, "type": "f32"}, seed))
        A = _randn(_gen(seed, 2), N, D + case["pad"]).to(t)[:, :D]
        bias = None if case["act"] == "none" else _randn(_gen(seed, 3), M) * 0.1
        return {"case": case, "A": A, "packed": packed, "exps": exps, "bias": bias,
                "table": torch.tensor(VALUES, device="cuda", dtype=torch.float32)}
    B = _weights(case, seed)
    live = M - case["off"]
    target = torch.randint(0, live, (N,), generator=_gen(seed, 4), device="cuda")
    lean = torch.rand((N, 1), generator=_gen(seed, 5), device="cuda") * 8
    A = (_randn(_gen(seed, 2), N, D) + lean * B[:, target].t().float()).to(t)
    target = torch.where(torch.rand((N,), generator=_gen(seed, 6), device="cuda") < 0.05, -100, target)
    bias = None
    if case["bias"]:
        bias = _randn(_gen(seed, 3), M) * 0.1
        bias[live:] = -math.inf
    state = {"case": case, "A": A, "B": B, "target": target, "bias": bias}
    if case["kind"] == "grad":
        state["lse"] = torch.logsumexp(_logits(state), dim=1)
        state["gloss"] = torch.full((N,), 1.0 / N, device="cuda") * (0.5 + torch.rand((N,), generator=_gen(seed, 7), device="cuda"))
    return state


# ------------------------------------------------------------------ passes


def _logits(s):
    z = s["A"].float() @ s["B"].float()
    return z if s["bias"] is None else z + s["bias"]


def _plain_quant(s):
    q, e = _codes(s["B"])
    D, M = s["B"].shape
    v = torch.tensor(VALUES, device="cuda", dtype=torch.float32)[q.int()]
    return torch.ldexp(v, e[:, None, :]).view(-1, M)[:D].to(torch.bfloat16)


def _plain_w4(s):
    c, packed, exps = s["case"], s["packed"], s["exps"]
    nm, nk = packed.shape[:2]
    v = s["table"][torch.stack((packed & 15, packed >> 4), dim=-1).int()]          # [Mb][Kb][64][16][2]
    v = v.view(nm, nk, 4, 16, 4, 8) * torch.exp2(exps.float() - 127).view(nm, nk, 1, 16, 4, 1)
    W = v.permute(1, 4, 2, 5, 0, 3).reshape(nk * KB, nm * MB)[:c["D"], :c["M"]]
    y = s["A"].float() @ W
    if s["bias"] is not None:
        y = y + s["bias"]
    if c["act"] == "relu":
        y = torch.clamp(y, min=0)
    if c["act"] == "softmax":
        y = torch.exp(y - y.amax(1, keepdim=True))
        y = y / y.sum(1, keepdim=True)
    return y.to(torch.float32 if c["out"] == "f32" else s["A"].dtype)


def _target_of(s):
    live = (s["target"] >= 0) & (s["target"] < s["case"]["M"])
    return live, torch.where(live, s["target"], 0)


def _plain_xent(s):
    z = _logits(s)
    live, t = _target_of(s)
    top = z.amax(1)
    lse = top + torch.log(torch.exp(z - top[:, None]).sum(1))
    return torch.where(live, lse - z.gather(1, t[:, None])[:, 0], 0.0), lse


def _plain_grad(s):
    live, t = _target_of(s)
    g = torch.where(live, s["gloss"], 0.0)[:, None]
    G = torch.exp(_logits(s) - s["lse"][:, None]) * g
    G.scatter_add_(1, t[:, None], -g)
    dA, dB = G @ s["B"].float().t(), s["A"].float().t() @ G
    return dA.to(s["A"].dtype), dB.to(s["B"].dtype), G.sum(0)


def _own(s):
    import paper_2207_05808_amd as mdn
    c = s["case"]
    if c["kind"] == "quant":
        return mdn.dequantize_w4(mdn.quantize_w4(s["B"]))
    if c["kind"] == "w4":
        w = mdn.W4Weights(s["packed"], s["exps"], c["D"], c["M"])
        return mdn.matmul_w4(s["A"], w, col_bias=s["bias"], act=c["act"], out_dtype=torch.float32 if c["out"] == "f32" else None)
    if c["kind"] == "xent":
        return mdn.linear_xent(s["A"], s["B"], s["target"], col_bias=s["bias"])
    return mdn.linear_xent_grad(s["A"], s["B"], s["target"], s["lse"], s["gloss"], col_bias=s["bias"])


def run(state):
    if own:
        return _own(state)
    return {"quant": _plain_quant, "w4": _plain_w4, "xent": _plain_xent, "grad": _plain_grad}[state["case"]["kind"]](state)


# ------------------------------------------------------------------ what a pass cannot do without


def work(case):
    D, M = case["D"], case["M"]
    b = BYTES[case["type"]]
    packed = D * M / 2 + D * M / GROUP
    if case["kind"] == "quant":
        return {"bytes": D * M * b + packed + D * M * 2, "flops": D * M}
    N = case["N"]
    if case["kind"] == "w4":
        y = N * M * (4 if case["out"] == "f32" else b)
        return {"bytes": packed + N * D * b + y + (0 if case["act"] == "none" else 4 * M), "flops": 2 * N * D * M}
    ins = N * D * b + D * M * b + N * 8 + (4 * M if case["bias"] else 0)
    if case["kind"] == "xent":
        return {"bytes": ins + N * 8, "flops": 2 * N * D * M}
    return {"bytes": ins + N * 8 + N * D * b + D * M * b + 4 * M, "flops": 6 * N * D * M}


# ------------------------------------------------------------------ the definition in 64 bits


def _exact_weights(case, seed):
    """The quantized weights in 64 bits: each the nearest point of the grid to
    B, found by distance (ties to the even code), scaled by its group."""
    B = _weights(case, seed).double()
    D, M = B.shape
    W = torch.zeros((-(-D // GROUP) * GROUP, M), device="cuda", dtype=torch.float64)
    W[:D] = B
    top = W.view(-1, GROUP, M).abs().amax(1)
    e = torch.ceil(torch.log2(torch.clamp(top, min=2.0 ** -140) / 6.0)).clamp(-120, 125)
    e = torch.where((top <= 6.0 * torch.exp2(e - 1)) & (e > -120), e - 1, e)
    e = torch.where((top > 6.0 * torch.exp2(e)) & (e < 125), e + 1, e)
    scale = torch.exp2(e).repeat_interleave(GROUP, 0)
    t = W.abs() / scale
    best, code = torch.full_like(t, math.inf), torch.zeros_like(t)
    for k in (0, 2, 4, 6, 1, 3, 5, 7):           # the even codes first: a tie stays there
        d = (t - VALUES[k]).abs()
        code = torch.where(d < best, VALUES[k], code)
        best = torch.minimum(best, d)
    return (torch.sign(W) * code * scale)[:D]


def _exact_rows(s):
    """Blocks of rows: (rows, their A in 64 bits, logits in 64 bits)."""
    B = s["B"].double()
    bias = None if s["bias"] is None else s["bias"].double()
    for r in range(0, s["A"].shape[0], ROWS):
        a = s["A"][r:r + ROWS].double()
        z = a @ B
        yield slice(r, r + ROWS), a, z if bias is None else z.add_(bias), B


def exact(case, seed):
    if case["kind"] == "quant":
        return _exact_weights(case, seed)
    s = prepare(case, seed)
    if case["kind"] == "w4":
        y = s["A"].double() @ _exact_weights({**case, "type": "f32"}, seed)
        if s["bias"] is not None:
            y = y + s["bias"].double()
        if case["act"] == "relu":
            y = torch.relu(y)
        return torch.softmax(y, 1) if case["act"] == "softmax" else y
    out = []
    if case["kind"] == "xent":
        for rows, _, z, _ in _exact_rows(s):
            t = s["target"][rows]
            lse = torch.logsumexp(z, 1)
            live = (t >= 0) & (t < case["M"])
            out.append((torch.where(live, lse - z.gather(1, torch.where(live, t, 0)[:, None])[:, 0], 0.0), lse))
        return torch.cat([o[0] for o in out]), torch.cat([o[1] for o in out])
    dB = torch.zeros((case["D"], case["M"]), device="cuda", dtype=torch.float64)
    db = torch.zeros((case["M"],), device="cuda", dtype=torch.float64)
    for rows, a, z, B in _exact_rows(s):
        t = s["target"][rows]
        live = (t >= 0) & (t < case["M"])
        g = torch.where(live, s["gloss"][rows].double(), 0.0)
        z.sub_(s["lse"][rows].double()[:, None]).exp_()
        z[live, t[live]] -= 1.0
        z.mul_(g[:, None])
        out.append(z @ B.t())
        dB.addmm_(a.t(), z)
        db.add_(z.sum(0))
    return torch.cat(out), dB, db
