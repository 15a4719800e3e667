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


@pytest.mark.parametrize("raw", [False, True])
def test_floats_are_kept_until_they_are_read(nq, busy, raw):
    w = torch.randn(1024, 1024, device="cuda")
    want = nq.Fp8Matrix.from_float(w)
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    busy(side)
    got = nq.Fp8Matrix.from_float(w.clone(), stream=side.cuda_stream if raw else side)
    others = [torch.full_like(w, 7.0) for _ in range(4)]
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


@pytest.mark.parametrize("raw", [False, True])
def test_passes_in_order_on_any_stream(nq, busy, raw):
    """Weights quantised behind a busy stream, then passes of one and of another token count, each on another stream at once."""
    from paper_2506_17870_amd.fp8_mlp import Fp8Mlp
    layers, hs = mlp_layers(), [stream_of(t, seed=t) for t in (12, 40, 40, 12)]
    wants = [Fp8Mlp(layers).forward(h).clone() for h in hs]
    sides = [torch.cuda.Stream() for _ in range(2)]
    for first in (0, 1):                                     # (the allocator has memory to hand out again from the second time on)
        torch.cuda.synchronize()
        busy()
        mlp, got = Fp8Mlp(layers), []
        for i, h in enumerate(hs):
            side = sides[(i + first) % 2]
            if i == 1:
                busy(side)                                   # the next pass, on the other stream, has to wait for this one
            got.append(mlp.forward(h, side.cuda_stream if raw else side))
        got.append(mlp.forward(hs[0]))
        torch.cuda.synchronize()
        for i in (0, 2, 4):                                  # (the others' buffer is overwritten by the pass behind them)
            assert torch.equal(got[i], (wants + wants[:1])[i]), (first, i)


@pytest.mark.parametrize("raw", [False, True])
def test_buffers_are_kept_until_the_pass_is_done(nq, busy, raw):
    from paper_2506_17870_amd.fp8_mlp import Fp8Mlp
    layers, a, b = mlp_layers(), stream_of(40), stream_of(12)
    mlp, side = Fp8Mlp(layers).allocate(40), torch.cuda.Stream()
    want = mlp.forward(a).clone()
    torch.cuda.synchronize()
    busy(side)
    kept = mlp.forward(a, side.cuda_stream if raw else side)          # (its buffer lives on with this name, the others do not)
    mlp.forward(b)                                                    # another token count, on the current stream
    others = [torch.full((n,), 9, dtype=torch.uint8, device="cuda") for n in (40 * 512, 40 * 1024 * 2, 40 * 256 * 2, 40 * 256, 640, 320, 512) * 3]
    torch.cuda.synchronize()
    assert torch.equal(kept, want) and len(others) == 21


def test_a_graph_keeps_its_buffers(nq):
    """Passes with other token counts between the replays: the graph's memory stays its own, and so does everybody else's."""
    from paper_2506_17870_amd.fp8_mlp import Fp8Mlp
    layers = mlp_layers()
    mlp, eager = Fp8Mlp(layers).allocate(12), Fp8Mlp(layers)
    mlp.run()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        mlp.run()
    h12 = mlp.h
    for i, tokens in enumerate((40, 12, 3, 40)):
        other = stream_of(tokens, seed=i)
        assert torch.equal(mlp.forward(other), eager.forward(other))
        others = [torch.full((n,), 9, dtype=torch.uint8, device="cuda") for n in (12 * 512, 12 * 1024 * 2, 12 * 256 * 2, 12 * 256, 96, 192) * 3]
        h12.copy_(stream_of(12, seed=100 + i))
        g.replay()
        torch.cuda.synchronize()
        assert torch.equal(h12, eager.forward(stream_of(12, seed=100 + i))), i
        assert all(bool((t == 9).all()) for t in others), i
    assert mlp.allocate(12).h is h12 and mlp.tokens == 12


def test_no_tokens(nq):
    from paper_2506_17870_amd.fp8_mlp import Fp8Mlp
    mlp = Fp8Mlp(mlp_layers())
    want = mlp.forward(stream_of(3)).clone()
    assert mlp.forward(stream_of(0)).shape == (0, 256) and torch.equal(mlp.forward(stream_of(3)), want)


def test_memory_of_a_pass_by_handle_is_the_current_streams(nq):
    """A handle may be destroyed after its work: nothing that outlives a pass on one is asked for or kept under it."""
    from paper_2506_17870_amd.fp8_mlp import Fp8Mlp
    mlp, side = Fp8Mlp(mlp_layers()), torch.cuda.Stream()
    for tokens in (5, 9):
        mlp.forward(stream_of(tokens), side.cuda_stream)
        torch.cuda.synchronize()
        assert mlp._home.cuda_stream == torch.cuda.current_stream().cuda_stream and side.cuda_stream not in mlp._recorded
        assert all(event is not None for handle, (_, event) in mlp._after.items() if handle == side.cuda_stream)
