"""The MLP blocks on the fp8 operators against the same blocks in 64 bits without any quantisation.

Rounding a normally distributed value to e4m3 (3 mantissa bits) errs by 2^-4 / sqrt(3) of it at most and 2.6 % in the mean square; a
product of two such matrices by sqrt(2) times that, 3.7 %, and the second layer adds its own two to what it is handed: under 8 %
of the branch for a block, and sqrt(blocks) times that where the blocks' errors are independent."""
import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def nq():
    import paper_2506_17870_amd as nq
    return nq


def layers(n, D, F, gated, post, gate, seed=0):
    g = torch.Generator().manual_seed(seed)
    r = lambda *s: torch.randn(*s, generator=g)  # noqa: E731
    out = []
    for _ in range(n):
        L = dict(up=r(2 * F if gated else F, D) * D ** -0.5, down=r(D, F) * F ** -0.5 * 2, pre=1 + 0.1 * r(D))
        if post:
            L["post"] = 1 + 0.1 * r(D)
        if gate:
            L["gate"] = (0.5 + 0.1 * r(D)).to(torch.bfloat16)
        out.append(L)
    return out


def rms64(v, w):
    return v / np.sqrt((v ** 2).mean(1, keepdims=True) + 1e-5) * w.double().numpy()


def blocks64(ls, h, gated, silu, rs, bs):
    branch, prev = None, None
    for L in ls + [None]:
        if branch is not None:
            p = rms64(branch, prev["post"]) if "post" in prev else branch
            h = rs * h + bs * (prev["gate"].double().numpy() if "gate" in prev else 1.0) * p
        if L is None:
            return h
        F = L["down"].shape[1]
        y = rms64(h, L["pre"]) @ L["up"].double().numpy().T
        v = y[:, :F]
        v = v / (1 + np.exp(-v)) if silu else torch.nn.functional.gelu(torch.from_numpy(v)).numpy()
        branch, prev = (v * y[:, F:] if gated else v) @ L["down"].double().numpy().T, L


@pytest.mark.parametrize("tokens", [1, 7, 300])
@pytest.mark.parametrize("gated,post,gate,D,F", [(True, True, False, 512, 1024), (False, False, False, 768, 1000), (True, True, True, 200, 333)])
def test_against_64_bits(nq, tokens, gated, post, gate, D, F):
    from paper_2506_17870_amd.fp8_mlp import Fp8Mlp
    ls = layers(3, D, F, gated, post, gate, seed=D + tokens)
    cu = [{k: v.cuda() for k, v in L.items()} for L in ls]
    mlp = Fp8Mlp(cu, nq.NQ_ACT_SILU if gated else nq.NQ_ACT_GELU, torch.bfloat16, torch.float32, branch_scale=0.8)
    h = torch.randn(tokens, D, generator=torch.Generator().manual_seed(1)) * 2
    got = mlp.forward(h.cuda()).double().cpu().numpy()
    want = blocks64(ls, h.double().numpy(), gated, gated, 1.0, 0.8)
    moved = np.linalg.norm(want - h.double().numpy())
    assert np.linalg.norm(got - want) <= 0.08 * 3 ** 0.5 * moved


def test_on_another_stream_and_from_a_graph(nq):
    from paper_2506_17870_amd.fp8_mlp import Fp8Mlp
    cu = [{k: v.cuda() for k, v in L.items()} for L in layers(2, 256, 512, True, True, True)]
    mlp = Fp8Mlp(cu).allocate(12)
    h = torch.randn(12, 256, device="cuda").to(torch.bfloat16)
    want = mlp.forward(h).clone()
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    got = mlp.forward(h, side)
    side.synchronize()
    assert torch.equal(got, want)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        mlp.run()
    for i in range(4):
        h.normal_()
        want = mlp.forward(h).clone()
        mlp.h.copy_(h)
        g.replay()
        torch.cuda.synchronize()
        assert torch.equal(mlp.h, want), i


def test_shapes_that_do_not_fit(nq):
    from paper_2506_17870_amd.fp8_mlp import Fp8Mlp
    a, b = layers(1, 256, 512, True, False, False)[0], layers(1, 128, 512, True, False, False)[0]
    cu = lambda L: {k: v.cuda() for k, v in L.items()}  # noqa: E731
    with pytest.raises(ValueError):
        Fp8Mlp([cu(dict(a, up=b["up"]))])
    with pytest.raises(ValueError):
        Fp8Mlp([cu(a), cu(b)])
