"""The e4m3 product in every tile form, each asserted to be the one that ran."""
import pytest
from fp8_forms import ANY_BYTE, FORMS
from test_gpu_fp8 import check_gemm

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def nq():
    import paper_2506_17870_amd as nq
    return nq


@pytest.mark.parametrize("out,form", [(out, form) for out in ("f32", "f16", "bf16") for form in FORMS["f32" if out == "f32" else "16 bits"]])
def test_form(nq, out, form):
    for M, N, K in FORMS["f32" if out == "f32" else "16 bits"][form]:
        ld = dict(ld=-(-K // 16) * 16)
        check_gemm(nq, M, N, K, out=out, exact=True, seed=K, x_kw=ld, w_kw=ld)
        assert nq.nq_profile_last_kernel() == (12, form)
        check_gemm(nq, M, N, K, out=out, bias=True, seed=K + 1, x_kw=dict(by_row=True, **ld), w_kw=ld)


@pytest.mark.parametrize("out", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("variant", ANY_BYTE)
def test_rows_on_any_byte(nq, out, variant):
    for M, N, K in ANY_BYTE[variant]:
        check_gemm(nq, M, N, K, out=out, exact=True, seed=K)
        assert nq.nq_profile_last_kernel() == (12, variant)


def test_time_stamps(nq):
    """The events around a product's dispatch: more time for more work, none left for the next call."""
    import torch
    ms = {}
    for n in (256, 4096):
        x, w = nq.Fp8Matrix(n, n), nq.Fp8Matrix(n, n, 128)
        y = torch.empty(n, n, dtype=torch.bfloat16, device="cuda")
        start, stop = nq.nq_event_create(), nq.nq_event_create()
        for _ in range(3):
            nq.nq_profile_next_launch(start, stop)
            nq.nq_gemm_fp8(x.desc, w.desc, None, y, nq.NQ_DT_BF16, n)
            nq.nq_gemm_fp8(x.desc, w.desc, None, y, nq.NQ_DT_BF16, n)
            torch.cuda.synchronize()
        ms[n] = nq.nq_event_elapsed_ms(start, stop)
        nq.nq_event_destroy(start), nq.nq_event_destroy(stop)
    assert 0 < ms[256] < ms[4096] < 10
