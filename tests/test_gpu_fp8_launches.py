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
