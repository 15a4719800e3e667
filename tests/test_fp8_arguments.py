"""CPU checks of the tensors that the fp8 descriptors and owners are made of: types and lengths that do not fit are refused before an
address is taken of them, bare addresses are left alone."""
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


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16, torch.float64, torch.int32])
def test_norm_vectors_are_fp32(nq, dtype):
    v = torch.ones(64, dtype=dtype)
    for bad in (dict(d_weight=v), dict(d_bias=v)):
        with pytest.raises(ValueError, match="fp32"):
            nq.make_norm(nq.NQ_NORM_LAYER, 1e-5, **bad)
    nq.make_norm(nq.NQ_NORM_LAYER, 1e-5, torch.ones(64), torch.ones(64))
    nq.make_norm(nq.NQ_NORM_LAYER, 1e-5, A, None)


def job(nq, post=None, pre=None, gate=None, ldgate=0, gate_rows=0, **kw):
    none = nq.make_norm(nq.NQ_NORM_NONE)
    args = dict(d_h=A, h_dtype=nq.NQ_DT_F32, d_y=A, dtype=nq.NQ_DT_BF16, d_h_out=A, d_x=A)
    args.update(kw)
    return nq.make_block_norm(args["d_h"], args["h_dtype"], 64, args["d_y"], args["dtype"], 64, gate, ldgate, gate_rows, 1.0, 1.0, post or none,
                              pre or none, args["d_h_out"], 64, args["d_x"], 64)


def test_norm_vectors_are_as_long_as_a_row(nq):
    rms = lambda n: nq.make_norm(nq.NQ_NORM_RMS, 1e-5, torch.ones(n))  # noqa: E731
    layer = lambda w, b: nq.make_norm(nq.NQ_NORM_LAYER, 1e-5, torch.ones(w), torch.ones(b))  # noqa: E731
    for j in (job(nq, post=rms(63)), job(nq, pre=rms(63)), job(nq, post=rms(64), pre=layer(64, 63)), job(nq, pre=layer(63, 64))):
        with pytest.raises(ValueError, match="64 columns"):
            nq.nq_block_norm(j, 0, 64, stream=0)
        nq.nq_block_norm(j, 0, 63, stream=0)                 # (no rows: nothing is read)
    nq.nq_block_norm(job(nq, post=rms(64), pre=rms(65)), 0, 64, stream=0)


def test_block_norm_types(nq):
    t = lambda dtype: torch.zeros(4, 64, dtype=dtype)  # noqa: E731
    bf, f32 = torch.bfloat16, torch.float32
    for bad in (dict(gate=t(f32), ldgate=64, gate_rows=1), dict(d_h=t(bf)), dict(d_h_out=t(bf)), dict(d_y=t(f32)), dict(d_x=t(torch.float16))):
        with pytest.raises(ValueError, match="is of"):
            job(nq, **bad)
    job(nq, gate=t(bf), ldgate=64, gate_rows=1, d_h=t(f32), d_h_out=t(f32), d_y=t(bf), d_x=t(bf))


def test_gate_has_its_rows(nq):
    """Row m reads row m / gate_rows of the gate; what its storage holds behind the view counts."""
    g = torch.zeros(3, 64, dtype=torch.bfloat16)
    call = lambda M, gate, ld, rows, D=64: nq.nq_block_norm(job(nq, gate=gate, ldgate=ld, gate_rows=rows, d_h_out=None, d_x=None), M, D, stream=0)  # noqa: E731
    for M, gate, ld, rows in ((4, g, 64, 1), (7, g, 64, 2), (10, g[1:], 64, 4), (3, g, 65, 1), (2, g[0, :63], 193, 1)):
        with pytest.raises(ValueError, match="gate"):
            call(M, gate, ld, rows)
    for M, gate, ld, rows in ((3, g, 64, 1), (6, g, 64, 2), (8, g[1:], 64, 4), (3, g[0], 64, 1), (3, g.view(-1), 64, 1), (1000, g, 64, 1000), (4, A, 64, 1)):
        call(M, gate, ld, rows)                              # (no output is asked for: nothing is read)


def test_bias_of_the_product(nq):
    x = nq.nq_fp8(A, 0, 128, 128, A, 1, 1, 1, 0)
    w = nq.nq_fp8(A, 8, 128, 128, A, 1, 1, 128, 0)
    for bad in (torch.zeros(8, dtype=torch.bfloat16), torch.zeros(8, dtype=torch.float64), torch.zeros(7)):
        with pytest.raises(ValueError, match="d_bias"):
            nq.nq_gemm_fp8(x, w, bad, A, nq.NQ_DT_F32, 8, stream=0)
    for good in (torch.zeros(8), torch.zeros(9), A, None):
        nq.nq_gemm_fp8(x, w, good, A, nq.NQ_DT_F32, 8, stream=0)

def test_layers_of_the_mlp(nq):
    from paper_2506_17870_amd.fp8_mlp import Fp8Mlp
    good = dict(up=torch.zeros(128, 64), down=torch.zeros(64, 128), pre=torch.ones(64))
    for bad in (dict(pre=torch.ones(64, dtype=torch.bfloat16)), dict(post=torch.ones(64, dtype=torch.float16)), dict(pre=torch.ones(63)),
                dict(post=torch.ones(1, 64)), dict(gate=torch.ones(64)), dict(gate=torch.ones(63, dtype=torch.bfloat16))):
        with pytest.raises(ValueError, match=next(iter(bad))):
            Fp8Mlp([dict(good, **bad)], dtype=torch.bfloat16)


def test_input_of_the_mlp(nq):
    """A stream of another width is refused, not spread over the columns."""
    from paper_2506_17870_amd.fp8_mlp import Fp8Mlp
    mlp = Fp8Mlp.__new__(Fp8Mlp)
    mlp.layers = [dict(D=64)]
    for bad in (torch.zeros(4, 1), torch.zeros(4, 63), torch.zeros(64), torch.zeros(4, 64, 1)):
        with pytest.raises(ValueError, match="64"):
            mlp.forward(bad)
