"""The quantiser's activation functions against 64 bits, relative to their results.

A block of one element has the scale |f(v)| / 448, so a matrix of one column shows the function to a unit of fp32.  In units of
u = 2^-23 of the result, a step rounded to nearest costs 1/2, the hardware's exponential and reciprocal 1:
  SiLU       8: the exponential squared 2 1/2, its correction 1/2 and 2 for the constant at an exponent of 126, 1 + w 1/2, the reciprocal 1,
             two products 1.  Below -87 exp(v) is subnormal: 64, and |v| 2^-148.
  GELU       8 for reciprocal, polynomial (1.3 by its fit), exponential and products; the exponent v^2 / (2 ln 2) is the result of two
             rounded products and a constant's 0.22 of half a unit: 1.11 u ln 2 times it, 0.6 v^2.
  GELU_TANH  8, and the exponent 2.3 |v| + 0.103 |v|^3 by four roundings and two constants: 1.2 for each unit of it.
Results below 2^-126 may have any size below it (GELU) or are off by half a unit of the smallest number for each product."""
import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu

U = 2.0 ** -23
SMALL = 2.0 ** -126


@pytest.fixture(scope="module")
def nq():
    import paper_2506_17870_amd as nq
    return nq


def codes_of(q):
    return q.view(torch.float8_e4m3fn).double().cpu().numpy()


def values(dtype):
    """Every 16-bit number, or many fp32 ones, from 2^-20 to 110 in magnitude; some far beyond."""
    if dtype == torch.float32:
        r = np.random.default_rng(1)
        v = np.concatenate([r.uniform(-110, 110, 100000), r.uniform(-6, 6, 100000), np.exp(r.uniform(np.log(2.0 ** -20), np.log(110), 50000)),
                            -np.exp(r.uniform(np.log(2.0 ** -20), np.log(110), 50000))])
        t = torch.from_numpy(v.astype(np.float32))
    else:
        t = torch.arange(-32768, 32768, dtype=torch.int32).to(torch.int16).view(dtype)
        t = t[torch.isfinite(t) & (t.abs() >= 2.0 ** -20) & (t.abs() <= 110)]
    far = torch.tensor([0.0, -0.0, 200.0, -200.0, 5000.0, -5000.0, 60000.0, -60000.0]).to(dtype)
    return torch.cat([t, far])


def exact(act, v):
    t = torch.from_numpy(v)
    if act == "silu":
        f = t / (1 + torch.exp(-t))
    elif act == "gelu":
        f = 0.5 * t * torch.special.erfc(-t * 0.5 ** 0.5)
    else:
        f = t / (1 + torch.exp(-2 * (2 / torch.pi) ** 0.5 * (t + 0.044715 * t ** 3)))
    return f.numpy()


def allowed(act, v, f):
    z = np.abs(v)
    if act == "silu":
        return np.where(v < -87, 64, 8) * U * np.abs(f) + np.where(v < -87, z * 2.0 ** -148, 0)
    if act == "gelu":
        return np.where(np.abs(f) < SMALL, np.abs(f), (8 + 0.6 * np.minimum(v, 0) ** 2) * U * np.abs(f))
    return (8 + np.where(v < 0, 1.2 * (2.31 * z + 0.103 * z ** 3), 0)) * U * np.abs(f) + z * 2.0 ** -148


@pytest.mark.parametrize("dtype", [torch.float32, torch.float16, torch.bfloat16])
@pytest.mark.parametrize("act", ["silu", "gelu", "gelu_tanh"])
def test_one_value_to_a_block(nq, act, dtype):
    t = values(dtype)
    q, scale = torch.zeros(t.numel(), 1, dtype=torch.uint8, device="cuda"), torch.zeros(t.numel(), 1, device="cuda")
    code = {"silu": nq.NQ_ACT_SILU, "gelu": nq.NQ_ACT_GELU, "gelu_tanh": nq.NQ_ACT_GELU_TANH}[act]
    dt = {torch.float32: nq.NQ_DT_F32, torch.float16: nq.NQ_DT_F16, torch.bfloat16: nq.NQ_DT_BF16}[dtype]
    nq.nq_quantize_fp8(t.cuda().view(-1, 1), dt, 1, None, 0, code, nq.make_fp8(q, 1, scale))
    v = t.double().numpy()
    f, s, c = exact(act, v), scale.double().cpu().numpy()[:, 0], codes_of(q)[:, 0]
    off = allowed(act, v, f)
    by_scale = np.abs(f) >= 449 * SMALL                        # (the smallest scale is 2^-126: below that the code tells)
    assert (np.abs(s * 448 - np.abs(f)) <= off + U * np.abs(f))[by_scale].all()
    assert (c == np.sign(f) * 448)[by_scale].all()
    half = 2.0 ** (np.floor(np.log2(np.maximum(np.abs(f) / SMALL * (1 + 2.0 ** -10), 2.0 ** -6))) - 4) * SMALL
    assert (np.abs(c * s - f) <= off + half * (1 + 2.0 ** -10))[~by_scale].all()


@pytest.mark.parametrize("dtype", [torch.float32, torch.float16, torch.bfloat16])
@pytest.mark.parametrize("act", ["silu", "gelu", "gelu_tanh"])
@pytest.mark.parametrize("block_rows", [1, 128])
def test_blocks_of_negative_values(nq, act, dtype, block_rows):
    """Blocks whose every value is in the tail: the largest is the block's scale, the others its codes."""
    M, K = 256, 384
    g = torch.Generator().manual_seed(7)
    t = torch.cat([-(lo + (hi - lo) * torch.rand(M, 128, generator=g)) for lo, hi in ((2, 5), (5, 8), (8, 10))], 1).to(dtype)
    m = nq.Fp8Matrix(M, K, block_rows)
    code = {"silu": nq.NQ_ACT_SILU, "gelu": nq.NQ_ACT_GELU, "gelu_tanh": nq.NQ_ACT_GELU_TANH}[act]
    dt = {torch.float32: nq.NQ_DT_F32, torch.float16: nq.NQ_DT_F16, torch.bfloat16: nq.NQ_DT_BF16}[dtype]
    nq.nq_quantize_fp8(t.cuda(), dt, K, None, 0, code, m.desc)
    v = t.double().numpy()
    f, c = exact(act, v), codes_of(m.q)
    off = allowed(act, v, f)
    s = m.scale.t().double().cpu().numpy().repeat(block_rows, 0).repeat(128, 1)
    of_block = lambda a: a.reshape(M // block_rows, block_rows, K // 128, 128).max((1, 3)).repeat(block_rows, 0).repeat(128, 1)  # noqa: E731
    largest, off_largest = of_block(np.abs(f)), of_block(off)
    assert (np.abs(s * 448 - largest) <= off_largest + U * largest).all()
    half = 2.0 ** (np.floor(np.log2(np.maximum(np.abs(f) / s * (1 + 2.0 ** -10), 2.0 ** -6))) - 4)
    assert (np.abs(c * s - f) <= s * half * (1 + 2.0 ** -10) + off + 4 * U * np.abs(f)).all()


@pytest.mark.parametrize("act", ["SILU", "GELU", "GELU_TANH"])
def test_not_finite(nq, act):
    """An infinite or missing input leaves a scale that is not finite, whatever its sign; its neighbours' blocks do not see it."""
    x = torch.ones(8, 1)
    x[:6, 0] = torch.tensor([float("inf"), 1.0, float("-inf"), 2.0, float("nan"), -3.0])
    for dtype, dt in ((torch.float32, nq.NQ_DT_F32), (torch.float16, nq.NQ_DT_F16), (torch.bfloat16, nq.NQ_DT_BF16)):
        m = nq.Fp8Matrix(8, 1)
        nq.nq_quantize_fp8(x.to(dtype).cuda(), dt, 1, None, 0, getattr(nq, "NQ_ACT_" + act), m.desc)
        finite = torch.isfinite(m.scale[0]).tolist()
        assert finite == [False, True, False, True, False, True, True, True] and m.scale[0, 0] == float("inf") and torch.isnan(m.scale[0, 4])
