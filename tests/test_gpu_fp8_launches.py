"""The fp8 calls on sizes that need more than one dispatch, against calls on slices of them."""
import pytest
import torch

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def nq():
    import paper_2506_17870_amd as nq
    return nq


@pytest.mark.parametrize("rows,block_rows,dtype", [((1 << 28) + 300, 1, torch.bfloat16), ((1 << 29) + 300, 128, torch.float32)])
def test_quantise_many_rows(nq, rows, block_rows, dtype):
    """One column: more blocks than one dispatch can have threads for."""
    dt = nq.NQ_DT_BF16 if dtype == torch.bfloat16 else nq.NQ_DT_F32
    x = torch.empty(rows, 1, dtype=dtype, device="cuda").normal_()
    q, scale = torch.zeros(rows, 1, dtype=torch.uint8, device="cuda"), torch.zeros(-(-rows // block_rows), 1, device="cuda")
    nq.nq_quantize_fp8(x, dt, 1, None, 0, nq.NQ_ACT_NONE, nq.make_fp8(q, 1, scale, block_rows))
    torch.cuda.synchronize()
    assert bool((scale > 0).all())
    for at in [0] + [(i << 27) - 256 for i in range(1, (rows >> 27) + 1)] + [(rows - 500) // 128 * 128]:
        part = slice(at, min(rows, at + 512))
        pq, ps = torch.zeros_like(q[part]), torch.zeros(-(-q[part].shape[0] // block_rows), 1, device="cuda")
        nq.nq_quantize_fp8(x[part], dt, 1, None, 0, nq.NQ_ACT_NONE, nq.make_fp8(pq, 1, ps, block_rows))
        assert torch.equal(q[part], pq) and torch.equal(scale[part.start // block_rows:-(-part.stop // block_rows)], ps), at


@pytest.mark.parametrize("M,N,ld", [(1, 1 << 30, 1), (2, (1 << 22) + 1000, 16), (3, (1 << 21) + 77, 3), ((1 << 18) + 300, 2000, 16)])
def test_product_of_many_outputs(nq, M, N, ld):
    """More tiles than one dispatch can have threads for, over the weights' rows and over the tokens, with scales and biases of their own."""
    x, w = (torch.randint(0, 120, (n, ld), dtype=torch.uint8, device="cuda") for n in (M, N))
    xs = torch.rand(M, 1, device="cuda") + 0.5
    ws = torch.rand(-(-N // 128), 1, device="cuda") * 2.0 ** -8 + 2.0 ** -8
    bias = torch.rand(N, device="cuda")
    y = torch.empty(M, N, dtype=torch.float16, device="cuda")
    nq.nq_gemm_fp8(nq.make_fp8(x, 1, xs), nq.make_fp8(w, 1, ws, 128), bias, y, nq.NQ_DT_F16, N)
    value = lambda q: q[:, 0].view(torch.float8_e4m3fn).float()  # noqa: E731
    step = max(128, (1 << 28) // M // 128 * 128)
    for at in range(0, N, step):                               # (one product and a sum: the nearest f16 but for fp32 roundings)
        n = min(step, N - at)
        scale = ws[at // 128:-(-(at + n) // 128)].repeat_interleave(128, 0)[:n, 0]
        want = (value(x) * xs[:, 0])[:, None] * (value(w[at:at + n]) * scale)[None] + bias[at:at + n]
        assert bool(((y[:, at:at + n].float() - want).abs() <= 2.0 ** -10 * want + 2.0 ** -25).all()), at
