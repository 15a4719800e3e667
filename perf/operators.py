"""The timed cases of the 8-bit floating point operators: what a program that serves a transformer's MLP layers has them
do, from one token to a long prompt.

    gemm   Y = X W^T + bias of two e4m3 matrices, X with a scale for each 1 x 128 block, W for each 128 x 128
    quant  floats -> e4m3 codes and block scales, with an activation function and the product of a gated MLP before them
    norm   norm after a block, gate, residual sum, norm before the next block, the result as floats or as e4m3 codes

    listed()             the cases, each a dict of plain values with a name
    draw(rng)            one more case from the same ranges
    prepare(case, seed)  what the program holds before the call
    run(state)           one pass; the operators in their plain form, or, with `own`, this library's
    exact(case, seed)    the same outputs from the definition, in 64 bits
    work(case)           bytes and operations the pass cannot do without

e4m3: 1 sign, 4 exponent (bias 7) and 3 mantissa bits, largest value 448, no infinities.  A block with largest magnitude a
has the scale s = max(a / 448, 2^-126) (1 if a is 0) and the codes e4m3(v * (1 / s)), rounded to nearest even.
"""
from __future__ import annotations

import math

import torch

own = False

BLOCK = 128
DTYPES = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
BYTES = {"f32": 4, "f16": 2, "bf16": 2}
E4M3 = torch.float8_e4m3fn


def _gemm(M, N, K, out="bf16", bias=False):
    return dict(kind="gemm", M=M, N=N, K=K, out=out, bias=bias)


def _quant(M, K, dtype="bf16", act="none", mul=False, rows=1):
    return dict(kind="quant", M=M, K=K, dtype=dtype, act=act, mul=mul, rows=rows)


def _norm(M, D, dtype="bf16", stream="bf16", post="rms", pre="rms", gate="none", out="fp8"):
    return dict(kind="norm", M=M, D=D, dtype=dtype, stream=stream, post=post, pre=pre, gate=gate, out=out)


def listed():
    return [
        # one token through a projection: the weights are the traffic, latency counts
        dict(_gemm(1, 4096, 4096), name="gemm_1x4096x4096"),
        # a small batch of decoding steps through a wide layer
        dict(_gemm(24, 8192, 8192), name="gemm_24x8192x8192"),
        # one image's tokens, sizes that fit no tile or block, fp32 out with a bias
        dict(_gemm(197, 1000, 2008, out="f32", bias=True), name="gemm_197x1000x2008"),
        # a short prompt, or the tokens of a few hundred users
        dict(_gemm(512, 8192, 4096), name="gemm_512x8192x4096"),
        # a long prompt
        dict(_gemm(8192, 8192, 8192), name="gemm_8192x8192x8192"),
        # one token's activations on their way into a layer
        dict(_quant(1, 8192), name="quant_1x8192"),
        # the gated product between the two layers of an MLP, a long prompt
        dict(_quant(16384, 8192, act="silu", mul=True), name="quant_silu_16384x8192"),
        # the activation function of an ungated MLP, odd sizes
        dict(_quant(1009, 5003, dtype="f16", act="gelu"), name="quant_gelu_1009x5003"),
        # weights on their way in
        dict(_quant(8192, 8192, dtype="f32", rows=128), name="quant_weights_8192x8192"),
        # one token between two blocks
        dict(_norm(1, 4096), name="norm_1x4096"),
        # a long prompt between two blocks, codes for the next layer
        dict(_norm(16384, 4096), name="norm_16384x4096"),
        # the tokens of eight images with a gate of each image's own, layer norms, fp32 stream
        dict(_norm(1576, 768, dtype="f32", stream="f32", post="none", pre="layer", gate="group", out="float"), name="norm_layer_1576x768"),
    ]


# ---- more cases of the same ranges ---------------------------------------------------------------------------

MOST_FLOPS, MOST_ELEMENTS = 2.0 * 8192 ** 3, 16384 * 8192


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["gemm", "gemm", "gemm", "quant", "quant", "norm", "norm"])
    dtype = rng.choice(["bf16", "bf16", "f16", "f32"])
    while True:
        if kind == "gemm":
            c = _gemm(_log(rng, 1, 8192), _log(rng, 100, 8192), _log(rng, 100, 8192), out=dtype, bias=rng.random() < 0.3)
            if rng.random() < 0.5:       # half of them sizes that layers have
                c["N"], c["K"] = max(128, c["N"] // 128 * 128), max(128, c["K"] // 128 * 128)
            fits = 2.0 * c["M"] * c["N"] * c["K"] <= MOST_FLOPS
        elif kind == "quant":
            c = _quant(_log(rng, 1, 16384), _log(rng, 100, 16384), dtype=dtype, act=rng.choice(["none", "silu", "gelu", "gelu_tanh", "relu"]),
                       mul=rng.random() < 0.4, rows=1)
            if rng.random() < 0.25:
                c.update(act="none", mul=False, rows=128)
            if rng.random() < 0.5:
                c["K"] = max(128, c["K"] // 128 * 128)
            fits = c["M"] * c["K"] * (1 + c["mul"]) * BYTES[dtype] <= MOST_ELEMENTS * 4
        else:
            c = _norm(_log(rng, 1, 16384), _log(rng, 100, 16384), dtype=dtype, stream=rng.choice([dtype, "f32"]),
                      post=rng.choice(["rms", "layer", "none"]), pre=rng.choice(["rms", "layer"]),
                      gate=rng.choice(["none", "channel", "group", "token"]), out=rng.choice(["fp8", "fp8", "float"]))
            if rng.random() < 0.5:
                c["D"] = max(128, c["D"] // 128 * 128)
            fits = c["M"] * c["D"] * BYTES[dtype] <= MOST_ELEMENTS
        if fits:
            return c


# ---- inputs ----------------------------------------------------------------------------------------------------

def _activations(gen, M, D, dtype):
    """Unit variance with a spread between channels and a few channels that stand out, as hidden states have them."""
    x = torch.randn(M, D, generator=gen, device="cuda")
    x *= torch.exp(0.5 * torch.randn(D, generator=gen, device="cuda"))
    x[:, torch.randint(0, D, (max(1, D // 500),), generator=gen, device="cuda")] *= 20.0
    return x.to(dtype)


def _blocks(n):
    return -(-n // BLOCK)


def _gate_rows(case):
    """Tokens that share a row of the gate."""
    return {"channel": case["M"], "group": 197, "token": 1}[case["gate"]]


def prepare(case, seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(int(seed))
    if own:
        import paper_2506_17870_amd as nq
    s = dict(case=case)
    if own:
        s["nq"], s["dt"] = nq, _dt(nq, case["out"] if case["kind"] == "gemm" else case["dtype"])
    if case["kind"] == "gemm":
        M, N, K = case["M"], case["N"], case["K"]
        ld = -(-K // 16) * 16                       # rows start on 16 bytes
        for name, rows, block_rows in (("x", M, 1), ("w", N, BLOCK)):
            nb = rows if block_rows == 1 else _blocks(rows)
            # codes as the quantiser leaves them: the largest of a block near 448, the others a normal distribution
            q = torch.zeros(rows, ld, dtype=E4M3, device="cuda")
            q[:, :K] = (torch.randn(rows, K, generator=gen, device="cuda") * 130).clamp_(-448, 448).to(E4M3)
            scale = (torch.randn(_blocks(K), nb, generator=gen, device="cuda") * 0.4).exp_() * ((1.0 if name == "x" else K ** -0.5) / 130)
            s[name + "q"], s[name + "s"] = q, scale
        s["bias"] = torch.randn(N, generator=gen, device="cuda") if case["bias"] else None
        s["result"] = s["y"] = torch.empty(M, N, dtype=DTYPES[case["out"]], device="cuda")
        if own:
            s["x"], s["w"] = nq.make_fp8(s["xq"], K, s["xs"].t()), nq.make_fp8(s["wq"], K, s["ws"].t(), BLOCK)
    elif case["kind"] == "quant":
        M, K, t = case["M"], case["K"], DTYPES[case["dtype"]]
        s["x"] = _activations(gen, M, K, t) if case["rows"] == 1 else (torch.randn(M, K, generator=gen, device="cuda") * 0.02).to(t)
        s["mul"] = torch.randn(M, K, generator=gen, device="cuda").to(t) if case["mul"] else None
        s["result"] = _output_codes(s, M, K, case["rows"])
        if own:
            s["act"] = {"none": nq.NQ_ACT_NONE, "relu": nq.NQ_ACT_RELU, "silu": nq.NQ_ACT_SILU, "gelu": nq.NQ_ACT_GELU, "gelu_tanh": nq.NQ_ACT_GELU_TANH}[case["act"]]
            s["out"] = nq.make_fp8(s["q"], K, s["scale"].t(), case["rows"])
    else:
        M, D, t = case["M"], case["D"], DTYPES[case["dtype"]]
        s["h"] = (_activations(gen, M, D, torch.float32) * 4).to(DTYPES[case["stream"]])
        s["y"] = _activations(gen, M, D, t)
        vector = lambda shift: shift + 0.2 * torch.randn(D, generator=gen, device="cuda")  # noqa: E731
        s["post_w"], s["post_b"], s["pre_w"], s["pre_b"] = vector(1.0), vector(0.0), vector(1.0), vector(0.0)
        s["gate"] = (0.5 + 0.3 * torch.randn(-(-M // _gate_rows(case)), D, generator=gen, device="cuda")).to(t) if case["gate"] != "none" else None
        s["h_out"] = torch.empty_like(s["h"])
        if case["out"] == "fp8":
            x = _output_codes(s, M, D, 1)
        else:
            x = s["x"] = torch.empty(M, D, dtype=t, device="cuda")
        s["result"] = {"h": s["h_out"], "x": x}
        if own:
            kind = {"none": nq.NQ_NORM_NONE, "rms": nq.NQ_NORM_RMS, "layer": nq.NQ_NORM_LAYER}
            norm = lambda k, w, b: nq.make_norm(kind[k], EPS, w if k != "none" else None, b if k == "layer" else None)  # noqa: E731
            s["out"] = nq.make_fp8(s["q"], D, s["scale"].t()) if case["out"] == "fp8" else None
            s["job"] = nq.make_block_norm(s["h"], _dt(nq, case["stream"]), D, s["y"], s["dt"], D,
                                          s["gate"], D, _gate_rows(case) if case["gate"] != "none" else 0, RESIDUAL, BRANCH,
                                          norm(case["post"], s["post_w"], s["post_b"]), norm(case["pre"], s["pre_w"], s["pre_b"]),
                                          s["h_out"], D, s.get("x"), D, s["out"])
    return s


EPS, RESIDUAL, BRANCH = 1e-5, 1.0, 0.7


def _dt(nq, name):
    return {"f32": nq.NQ_DT_F32, "f16": nq.NQ_DT_F16, "bf16": nq.NQ_DT_BF16}[name]


def _output_codes(s, M, K, rows):
    s["q"] = torch.zeros(M, -(-K // 16) * 16, dtype=E4M3, device="cuda")
    s["scale"] = torch.empty(_blocks(K), M if rows == 1 else _blocks(M), device="cuda")
    return {"q": s["q"][:, :K], "scale": s["scale"]}


# ---- one pass --------------------------------------------------------------------------------------------------

def run(s):
    case = s["case"]
    if own:
        return _run_own(case, s)
    return {"gemm": _plain_gemm, "quant": _plain_quant, "norm": _plain_norm}[case["kind"]](case, s)


def _run_own(case, s):
    nq = s["nq"]
    if case["kind"] == "gemm":
        nq.nq_gemm_fp8(s["x"], s["w"], s["bias"], s["y"], s["dt"], case["N"])
    elif case["kind"] == "quant":
        nq.nq_quantize_fp8(s["x"], s["dt"], case["K"], s["mul"], case["K"], s["act"], s["out"])
    else:
        nq.nq_block_norm(s["job"], case["M"], case["D"])
    return s["result"]


def _spread(scale, K):
    """Scales [blocks of columns][rows] -> one for each column, [rows][K]."""
    return scale.t().repeat_interleave(BLOCK, 1)[:, :K]


def _plain_gemm(case, s):
    N, K = case["N"], case["K"]
    x = s["xq"][:, :K].float() * _spread(s["xs"], K)
    w = s["wq"][:, :K].float() * _spread(s["ws"], K).repeat_interleave(BLOCK, 0)[:N]
    y = x @ w.t()
    if s["bias"] is not None:
        y = y + s["bias"]
    return y.to(DTYPES[case["out"]])


def _codes(v, rows):
    """fp32 [M][K] -> codes [M][K] and scales [blocks of columns][rows or blocks of rows]."""
    M, K = v.shape
    pad_rows = 0 if rows == 1 else -M % rows
    t = torch.nn.functional.pad(v, (0, -K % BLOCK, 0, pad_rows)).view((M + pad_rows) // rows, rows, _blocks(K), BLOCK)
    a = t.abs().amax(dim=(1, 3), keepdim=True)
    scale = torch.where(a == 0, 1.0, (a / 448).clamp(min=2.0 ** -126))
    q = (t * (1 / scale)).to(E4M3).view(M + pad_rows, -1)[:M, :K]
    return q, scale[:, 0, :, 0].t()


def _plain_quant(case, s):
    v = s["x"].float()
    if case["act"] == "relu":
        v = torch.where(v < 0, 0.0, v)
    elif case["act"] == "silu":
        v = v / (1 + (-v).exp())
    elif case["act"] == "gelu":
        v = 0.5 * v * (1 + (v * math.sqrt(0.5)).erf())
    elif case["act"] == "gelu_tanh":
        v = 0.5 * v * (1 + (math.sqrt(2 / math.pi) * (v + 0.044715 * v * v * v)).tanh())
    if case["mul"]:
        v = v * s["mul"].float()
    q, scale = _codes(v, case["rows"])
    return {"q": q, "scale": scale}


def _plain_of_norm(kind, v, w, b):
    if kind == "none":
        return v
    if kind == "rms":
        return v * (v.square().mean(-1, keepdim=True) + EPS).rsqrt() * w
    v = v - v.mean(-1, keepdim=True)
    return v * (v.square().mean(-1, keepdim=True) + EPS).rsqrt() * w + b


def _plain_norm(case, s):
    p = _plain_of_norm(case["post"], s["y"].float(), s["post_w"], s["post_b"])
    if s["gate"] is not None:
        p = p * s["gate"].float().repeat_interleave(_gate_rows(case), 0)[:case["M"]]
    h = RESIDUAL * s["h"].float() + BRANCH * p
    x = _plain_of_norm(case["pre"], h, s["pre_w"], s["pre_b"])
    if case["out"] == "fp8":
        q, scale = _codes(x, 1)
        x = {"q": q, "scale": scale}
    else:
        x = x.to(DTYPES[case["dtype"]])
    return {"h": h.to(DTYPES[case["stream"]]), "x": x}


# ---- the definition in 64 bits ---------------------------------------------------------------------------------

def _exact_codes(v, rows):
    """The value of every code and the scales, block by block of columns."""
    M, K = v.shape
    q, scales = torch.empty_like(v), []
    of_row = torch.arange(M, device=v.device) // rows
    for at in range(0, K, BLOCK):
        t = v[:, at:at + BLOCK]
        a = torch.zeros(int(of_row[-1]) + 1, dtype=v.dtype, device=v.device).index_reduce_(0, of_row, t.abs().max(1).values, "amax")
        scale = torch.where(a > 0, torch.maximum(a / 448, torch.full_like(a, 2.0 ** -126)), torch.ones_like(a))
        t = t / scale[of_row][:, None]
        # spacing of the values: 2^-9 below 2^-6, 2^(e - 3) from 2^e on
        step = torch.exp2(torch.floor(torch.log2(t.abs().clamp(min=2.0 ** -6))) - 3)
        q[:, at:at + BLOCK] = (t / step).round() * step
        scales.append(scale)
    return {"q": q, "scale": torch.stack(scales)}


def _exact_of_norm(kind, v, w, b):
    if kind == "none":
        return v
    mean = v.sum(1, keepdim=True) / v.shape[1] if kind == "layer" else 0.0
    var = ((v - mean) ** 2).sum(1, keepdim=True) / v.shape[1]
    return (v - mean) / torch.sqrt(var + EPS) * w.double() + (b.double() if kind == "layer" else 0.0)


def exact(case, seed):
    s = prepare(case, seed)
    if case["kind"] == "gemm":
        N, K = case["N"], case["K"]
        y = torch.zeros(case["M"], N, dtype=torch.float64, device="cuda")
        if s["bias"] is not None:
            y += s["bias"].double()
        of_row = torch.arange(N, device="cuda") // BLOCK
        for b in range(_blocks(K)):
            cols = slice(b * BLOCK, min(K, b * BLOCK + BLOCK))
            w = s["wq"][:, cols].double() * s["ws"][b].double()[of_row][:, None]
            y.addmm_(s["xq"][:, cols].double() * s["xs"][b].double()[:, None], w.t())
        return y
    if case["kind"] == "quant":
        v = s["x"].double()
        if case["act"] == "relu":
            v = v.clamp(min=0)
        elif case["act"] == "silu":
            v = v * torch.sigmoid(v)
        elif case["act"] == "gelu":
            v = v * torch.special.ndtr(v)
        elif case["act"] == "gelu_tanh":
            v = v * torch.sigmoid(2 * math.sqrt(2 / math.pi) * (v + 0.044715 * v ** 3))
        if case["mul"]:
            v = v * s["mul"].double()
        return _exact_codes(v, case["rows"])
    p = _exact_of_norm(case["post"], s["y"].double(), s["post_w"], s["post_b"])
    if s["gate"] is not None:
        p = p * s["gate"].double()[torch.arange(case["M"], device="cuda") // _gate_rows(case)]
    h = RESIDUAL * s["h"].double() + BRANCH * p
    x = _exact_of_norm(case["pre"], h, s["pre_w"], s["pre_b"])
    return {"h": h, "x": _exact_codes(x, 1) if case["out"] == "fp8" else x}


def work(case):
    if case["kind"] == "gemm":
        M, N, K = case["M"], case["N"], case["K"]
        scales = _blocks(K) * (M + _blocks(N)) * 4
        return {"bytes": M * K + N * K + scales + M * N * BYTES[case["out"]] + (4 * N if case["bias"] else 0), "flops": 2 * M * N * K}
    if case["kind"] == "quant":
        M, K = case["M"], case["K"]
        scales = _blocks(K) * (M if case["rows"] == 1 else _blocks(M)) * 4
        return {"bytes": M * K * BYTES[case["dtype"]] * (1 + case["mul"]) + M * K + scales, "flops": 4 * M * K}
    M, D = case["M"], case["D"]
    t, h = BYTES[case["dtype"]], BYTES[case["stream"]]
    gate = 0 if case["gate"] == "none" else -(-M // _gate_rows(case)) * D * t
    vectors = 4 * D * sum({"none": 0, "rms": 1, "layer": 2}[case[k]] for k in ("post", "pre"))
    out = M * D + 4 * M * _blocks(D) if case["out"] == "fp8" else M * D * t
    return {"bytes": M * D * (t + 2 * h) + gate + vectors + out, "flops": 12 * M * D}
