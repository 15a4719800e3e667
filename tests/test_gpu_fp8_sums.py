"""The e4m3 product where its terms cancel or one of them stands out, output by output against 64 bits.

fp32 outputs: the terms are whole numbers under 2^24 with scales of 1, so every sum is exact.  16-bit outputs: the fp8 matrix instructions cut a
product off at 2^-14 of the largest one added with it, so an output is off by that much of each block's largest product for each of the
block's products, at most, and by half a unit of its type (2^-11, 2^-8; the smallest f16 numbers are 2^-24 apart)."""
import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def nq():
    import paper_2506_17870_amd as nq
    return nq


def operands(kind, M, N, K):
    """Whole numbers that e4m3 holds: normally spread; with a pair of products of 448 * 448 that cancel in every block; with one column far above
    the others."""
    r = np.random.default_rng(K)
    x, w = r.integers(-15, 16, (M, K)), r.integers(-15, 16, (N, K))
    if kind == "cancels":
        x[:, 3::64], w[:, 3::64] = 448, 448 * r.choice([-1, 1], (N, 1))
        x[:, 40::64], w[:, 40::64] = -448, w[:, 3::64][:, :w[:, 40::64].shape[1]]
        if x[:, 3::64].shape[1] > x[:, 40::64].shape[1]:      # (no partner in the last block)
            x[:, 3::64][:, -1] = 0
    if kind == "stands out":
        x[:, 7], w[:, 7] = 448 * r.choice([-1, 1], M), 208
    return x.astype(np.float64), w.astype(np.float64)


@pytest.mark.parametrize("kind", ["spread", "cancels", "stands out"])
@pytest.mark.parametrize("M,N,K", [(1, 64, 128), (16, 130, 300), (70, 200, 513), (300, 140, 1000), (40, 70, 77)])
@pytest.mark.parametrize("aligned", [True, False])
def test_products_that_cancel(nq, kind, M, N, K, aligned):
    x, w = operands(kind, M, N, K)
    ld = -(-K // 16) * 16 if aligned else K + (K % 16 == 0)

    def matrix(v, block_rows):
        q = torch.zeros(v.shape[0], ld, dtype=torch.uint8, device="cuda")
        q[:, :K] = torch.from_numpy(v).to(torch.float32).to(torch.float8_e4m3fn).view(torch.uint8).cuda()
        assert np.array_equal(q[:, :K].contiguous().view(torch.float8_e4m3fn).double().cpu().numpy(), v)
        return nq.make_fp8(q, K, torch.ones(-(-v.shape[0] // block_rows), -(-K // 128), device="cuda"), block_rows)

    xm, wm, want = matrix(x, 1), matrix(w, 128), x @ w.T
    largest = np.zeros_like(want)
    for b in range(0, K, 128):
        n = min(128, K - b)
        largest += n * 2.0 ** -14 * np.abs(x[:, None, b:b + n] * w[None, :, b:b + n]).max(2)
    for dtype, dt, unit in ((torch.float32, nq.NQ_DT_F32, 0.0), (torch.float16, nq.NQ_DT_F16, 2.0 ** -11), (torch.bfloat16, nq.NQ_DT_BF16, 2.0 ** -8)):
        y = torch.empty(M, N, dtype=dtype, device="cuda")
        nq.nq_gemm_fp8(xm, wm, None, y, dt, N)
        got = y.double().cpu().numpy()
        if dtype == torch.float32:
            assert np.array_equal(got, want)
        elif dtype == torch.bfloat16 or np.abs(want).max() < 65000:
            assert (np.abs(got - want) <= largest + unit * (np.abs(want) + largest) + 2.0 ** -25).all()
