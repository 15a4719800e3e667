"""The fp8 owners on streams other than the current one: nothing is ordered by a synchronisation of the test's own, and the streams
are kept busy, so that work which is not ordered by the code comes out in the wrong order."""
import pytest
import torch

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def nq():
    import paper_2506_17870_amd as nq
    return nq


@pytest.fixture(scope="module")
def busy():
    """Some milliseconds of work on the current stream, enqueued at once."""
    a, b = torch.ones(8192, 8192, dtype=torch.bfloat16, device="cuda"), torch.empty(8192, 8192, dtype=torch.bfloat16, device="cuda")
    torch.mm(a, a, out=b)
    torch.cuda.synchronize()

    def work(stream=None):
        with torch.cuda.stream(stream or torch.cuda.current_stream()):
            for _ in range(20):
                torch.mm(a, a, out=b)
    return work


def same(got, want):
    return torch.equal(got.q, want.q) and torch.equal(got.scale, want.scale)


@pytest.mark.parametrize("raw", [False, True])
@pytest.mark.parametrize("block_rows", [1, 128])
def test_fills_come_before_the_codes(nq, busy, raw, block_rows):
    w = torch.randn(300, 520, device="cuda")
    want = nq.Fp8Matrix.from_float(w, block_rows)
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    busy()
    got = nq.Fp8Matrix.from_float(w, block_rows, side.cuda_stream if raw else side)
    torch.cuda.synchronize()
    assert same(got, want) and want.q.any()


def test_floats_are_kept_until_they_are_read(nq, busy):
    w = torch.randn(1024, 1024, device="cuda")
    want = nq.Fp8Matrix.from_float(w)
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    busy(side)
    got = nq.Fp8Matrix.from_float(w.clone(), stream=side)
    others = [torch.full_like(w, 7.0) for _ in range(4)]         # (on the current stream, which does not wait)
    torch.cuda.synchronize()
    assert same(got, want) and len(others) == 4


def mlp_layers(n=2, D=256, F=512):
    g = torch.Generator(device="cuda").manual_seed(3)
    r = lambda *s: torch.randn(*s, generator=g, device="cuda")  # noqa: E731
    return [dict(up=r(2 * F, D) * D ** -0.5, down=r(D, F) * F ** -0.5, pre=1 + 0.1 * r(D), post=1 + 0.1 * r(D)) for _ in range(n)]


def stream_of(tokens, D=256, seed=5):
    return torch.randn(tokens, D, generator=torch.Generator(device="cuda").manual_seed(seed), device="cuda").to(torch.bfloat16)


def test_forward_takes_a_raw_handle(nq):
    from paper_2506_17870_amd.fp8_mlp import Fp8Mlp
    mlp, h, side = Fp8Mlp(mlp_layers()).allocate(9), stream_of(9), torch.cuda.Stream()
    want = mlp.forward(h).clone()
    torch.cuda.synchronize()
    got = mlp.forward(h, side.cuda_stream)
    side.synchronize()
    assert torch.equal(got, want)
