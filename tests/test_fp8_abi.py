"""CPU checks of the fp8 entry points: what is refused, with which status, before anything touches a GPU, through the binding's
extension and through ctypes alike."""
import ctypes
import os

import pytest
import torch

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
A = 0x1000                                       # an address nobody reads


@pytest.fixture(scope="module")
def nq():
    if not os.path.exists(os.path.join(ROOT, "paper_2506_17870_amd", "libnq.so")):
        from paper_2506_17870_amd import build
        build.build()
    import paper_2506_17870_amd as nq
    return nq


def fp8(nq, rows=4, cols=256, ld=None, block_rows=1, q=A, scale=A, row_step=1, col_step=4):
    return nq.nq_fp8(q, rows, cols, cols if ld is None else ld, scale, row_step, col_step, block_rows, 0)


def status(nq, name, *args):
    """The status of a call through the binding, after the same through ctypes."""
    as_c = [ctypes.byref(a) if isinstance(a, ctypes.Structure) else a for a in args]
    st = getattr(nq.binding._lib, name)(*as_c, 0)
    try:
        getattr(nq, name)(*args, stream=0)
    except nq.NQError as e:
        assert e.status == st and name in str(e)
    else:
        assert st == nq.NQ_OK
    return st


BAD_MATRIX = [(dict(rows=-1), "NQ_ERR_INVALID_ARG"), (dict(cols=-1), "NQ_ERR_INVALID_ARG"), (dict(block_rows=0), "NQ_ERR_INVALID_ARG"),
              (dict(block_rows=64), "NQ_ERR_INVALID_ARG"), (dict(ld=255), "NQ_ERR_SHAPE"), (dict(cols=65537), "NQ_ERR_SHAPE"),
              (dict(rows=1 << 41), "NQ_ERR_SHAPE"), (dict(ld=1 << 21), "NQ_ERR_SHAPE"), (dict(q=None), "NQ_ERR_INVALID_ARG"),
              (dict(scale=None), "NQ_ERR_INVALID_ARG"), (dict(scale=A + 2), "NQ_ERR_ALIGN"), (dict(row_step=-1), "NQ_ERR_INVALID_ARG"),
              (dict(col_step=-1), "NQ_ERR_INVALID_ARG"), (dict(row_step=1 << 21), "NQ_ERR_SHAPE"), (dict(col_step=1 << 41), "NQ_ERR_SHAPE")]


@pytest.mark.parametrize("kw,want", BAD_MATRIX)
def test_matrix_descriptor(nq, kw, want):
    want = getattr(nq, want)
    assert status(nq, "nq_quantize_fp8", A, 0, 1 << 20, None, 0, 0, fp8(nq, **kw)) == want
    assert status(nq, "nq_gemm_fp8", fp8(nq, **kw), fp8(nq, block_rows=128), None, A, 0, 4) == want
    assert status(nq, "nq_gemm_fp8", fp8(nq), fp8(nq, **{"block_rows": 128, **kw}), None, A, 0, 4) == want


def test_quantise(nq):
    q = fp8(nq)
    call = lambda x=A, dtype=0, ldx=256, mul=None, ldmul=0, act=0, q=q: status(nq, "nq_quantize_fp8", x, dtype, ldx, mul, ldmul, act, q)  # noqa: E731
    assert call(dtype=3) == call(dtype=-1) == call(act=5) == call(act=-1) == call(x=None) == nq.NQ_ERR_INVALID_ARG
    assert call(ldx=255) == call(mul=A, ldmul=255) == call(ldx=(1 << 32) + 1) == nq.NQ_ERR_SHAPE
    assert call(x=A + 2) == call(dtype=2, x=A + 1) == call(mul=A + 1, ldmul=256) == nq.NQ_ERR_ALIGN
    assert call(q=fp8(nq, rows=0, q=None, scale=None)) == call(q=fp8(nq, cols=0, q=None, scale=None), x=None) == nq.NQ_OK


def test_gemm(nq):
    x, w = fp8(nq), fp8(nq, rows=8, block_rows=128)
    call = lambda x=x, w=w, bias=None, y=A, dtype=0, ldy=8: status(nq, "nq_gemm_fp8", x, w, bias, y, dtype, ldy)  # noqa: E731
    assert call(dtype=3) == call(dtype=-1) == call(y=None) == nq.NQ_ERR_INVALID_ARG
    assert call(x=w) == call(w=x) == nq.NQ_ERR_UNSUPPORTED
    assert call(w=fp8(nq, cols=128, block_rows=128)) == call(ldy=7) == call(w=fp8(nq, rows=1 << 31, block_rows=128), ldy=1 << 31) == nq.NQ_ERR_SHAPE
    assert call(y=A + 2) == call(dtype=1, y=A + 1) == call(bias=A + 2) == nq.NQ_ERR_ALIGN
    assert call(x=fp8(nq, rows=0, q=None, scale=None)) == call(w=fp8(nq, rows=0, q=None, scale=None, block_rows=128), y=None) == nq.NQ_OK


def test_block_norm(nq):
    def call(M=4, D=256, h=A, h_dtype=0, ldh=256, y=A, dtype=0, ldy=256, gate=None, ldgate=0, gate_rows=0, post=None, pre=None, h_out=A, ldho=256,
             x=None, ldx=0, q=None):
        norm = nq.make_norm(nq.NQ_NORM_RMS)
        job = nq.make_block_norm(h, h_dtype, ldh, y, dtype, ldy, gate, ldgate, gate_rows, 1.0, 1.0, post or norm, pre or norm, h_out, ldho, x, ldx, q)
        return status(nq, "nq_block_norm", job, M, D)

    assert call(M=-1) == call(D=0) == call(dtype=3) == call(h_dtype=-1) == call(h=None) == nq.NQ_ERR_INVALID_ARG
    assert call(post=nq.make_norm(3)) == call(pre=nq.make_norm(-1)) == call(gate=A, ldgate=256) == nq.NQ_ERR_INVALID_ARG
    assert call(dtype=0, h_dtype=1) == call(dtype=1, h_dtype=2) == call(q=fp8(nq, block_rows=128)) == nq.NQ_ERR_UNSUPPORTED
    assert call(D=nq.NQ_NORM_MAX_D + 1) == call(ldh=255) == call(ldy=255) == call(gate=A, ldgate=255, gate_rows=1) == nq.NQ_ERR_SHAPE
    assert call(ldho=255) == call(x=A, ldx=255) == call(q=fp8(nq, rows=5)) == call(q=fp8(nq, cols=128)) == nq.NQ_ERR_SHAPE
    assert call(h=A + 2) == call(y=A + 2) == call(x=A + 1, ldx=256) == call(post=nq.make_norm(1, 1e-5, A + 2)) == nq.NQ_ERR_ALIGN
    assert call(pre=nq.make_norm(2, 1e-5, None, A + 1)) == nq.NQ_ERR_ALIGN
    assert call(M=0) == call(M=0, h=None, y=None) == call(h_out=None) == nq.NQ_OK
    assert nq.binding._lib.nq_block_norm(None, 4, 4, 0) == nq.NQ_ERR_INVALID_ARG


def test_descriptors_from_tensors(nq):
    q, s = torch.zeros(5, 304, dtype=torch.uint8), torch.ones(3, 5)
    d = nq.make_fp8(q, 300, s.t())
    assert (d.d_q, d.rows, d.cols, d.ld, d.d_scale, d.scale_row_step, d.scale_col_step, d.block_rows) == (q.data_ptr(), 5, 300, 304, s.data_ptr(), 1, 5, 1)
    d = nq.make_fp8(q[:, :300], 300, torch.ones(1, 3), 128)
    assert (d.ld, d.block_rows, d.scale_col_step) == (304, 128, 1)
    for bad in (lambda: nq.make_fp8(q, 305, s.t()), lambda: nq.make_fp8(q.t(), 5, torch.ones(304, 1)), lambda: nq.make_fp8(q, 300, s),
                lambda: nq.make_fp8(q.short(), 300, s.t()), lambda: nq.make_fp8(q, 300, s.t().double())):
        with pytest.raises(ValueError):
            bad()
    with pytest.raises(AssertionError):             # a column of a matrix is no row
        nq.nq_gemm_fp8(fp8(nq, rows=0), fp8(nq, rows=0, block_rows=128), None, torch.zeros(4, 6).t(), 0, 4, stream=0)
    m = nq.Fp8Matrix(7, 130, 128, device="cpu")
    assert m.q.shape == (7, 144) and m.scale.shape == (2, 1) and (m.desc.ld, m.desc.cols) == (144, 130)
