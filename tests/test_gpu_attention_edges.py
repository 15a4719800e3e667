"""The attention operators on the GPU at values and places where the definition is easily lost: infinities and NaN that a row sees, values whose squares
are too small, begins outside the rows, memory that another stream fills."""
import pytest
import torch

import attention_reference as ref
from test_gpu_attention import BF16, E4M3, F16, F32, TokenCase, begins, check_prompt, dt, randn, run_prompt
from test_gpu_attention_use import run_dealt

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def nq():
    import paper_2506_17870_amd as nq
    assert torch.cuda.is_available()
    return nq


def check_reached(got, o, bound, reached, what=""):
    """got against (o, bound) in finite columns, not finite (infinite or NaN, which is left open) in those that a value that is not finite reaches."""
    assert not torch.isfinite(got[reached]).any(), f"{what}: a value that is seen has no part"
    ref.check(torch.where(reached, torch.zeros_like(got), got), torch.where(reached, 0.0, o), bound, what)


def check_seen(got, q, k, v, q_begin, k_begin, Hq, Hkv, D, dtype, causal, scale, heads, sequences):
    qb, kb = q_begin.tolist(), k_begin.tolist()
    for s in sequences:
        n, m = qb[s + 1] - qb[s], kb[s + 1] - kb[s]
        seen = torch.ones(n, m, dtype=torch.bool)
        if causal:
            seen = torch.arange(m)[None] <= torch.arange(n)[:, None] + (m - n)
        for h in heads:
            g = h // (Hq // Hkv)
            part = lambda x, b, i: x[b[s]:b[s + 1], i * D:i * D + D].double()  # noqa: E731
            value = part(v, kb, g)
            bad = ~torch.isfinite(value)
            o, bound = ref.attention(part(q, qb, h), part(k, kb, g), value.masked_fill(bad, 0.0), scale, seen, dtype, True)
            check_reached(got[qb[s]:qb[s + 1], h * D:h * D + D], o, bound, seen.double() @ bad.double() > 0, f"sequence {s} head {h}")


# ---- values that are not finite, in keys that every row sees --------------------------------------------------------

SEEN = [  # rows, keys, sequences, Hq, Hkv, D, dtype, causal, elements between rows: each form with the value in the last keys, which do not fill their tile
    (197, 197, 1, 3, 3, 64, F16, False, 0),
    (197, 197, 1, 3, 3, 128, BF16, False, 0),
    (197, 197, 1, 100, 1, 64, BF16, False, 0),
    (197, 197, 1, 100, 1, 128, F16, False, 4),
    (60, 60, 1, 2, 1, 96, BF16, False, 0),
    (70, 133, 1, 2, 1, 256, F16, False, 0),
    (70, 133, 1, 2, 1, 256, BF16, False, 4),
    (50, 50, 20, 8, 2, 64, F16, False, 0),
    (50, 50, 20, 8, 2, 128, BF16, False, 4),
    (30, 30, 40, 8, 4, 192, BF16, False, 0),
    (1, 1, 1, 1, 1, 64, BF16, True, 0),
    (1, 77, 1, 2, 2, 128, F16, True, 0),
    (1, 77, 1, 2, 2, 128, BF16, True, 4),
    (1, 1000, 1, 2, 1, 72, BF16, True, 0),
    (33, 33, 20, 8, 2, 128, BF16, True, 0),
    (33, 300, 1, 2, 1, 64, F16, True, 0),
    (129, 129, 1, 2, 1, 64, BF16, True, 0),
    (129, 150, 1, 2, 1, 128, F16, True, 4),
    (129, 170, 1, 2, 2, 256, BF16, True, 0),
    (33, 33, 20, 16, 2, 256, F16, True, 0),
    (1, 17, 300, 2, 1, 256, F16, True, 0),
]


def seen_inputs(seed, n, m, S, Hq, Hkv, D, dtype):
    q, k, v = (randn(seed + i, *s) for i, s in enumerate(((S * n, Hq * D), (S * m, Hkv * D), (S * m, Hkv * D))))
    for s in range(S):                                             # in other columns of each sequence
        last, c = (s + 1) * m - 1, 8 * (s % 4)
        v[last, c + 1], v[last, c + 2], v[last, c + 4] = float("inf"), -float("inf"), float("nan")
        v[s * m + m // 2, c + 5] = float("inf")
    return (x.to(dtype) for x in (q, k, v))


@pytest.mark.parametrize("case", SEEN, ids=lambda c: "-".join(str(x).replace("torch.", "") for x in c))
def test_prompt_values_that_every_row_sees(nq, case):
    n, m, S, Hq, Hkv, D, dtype, causal, gap = case
    q, k, v = seen_inputs(500, n, m, S, Hq, Hkv, D, dtype)
    q_begin, k_begin = begins([n] * S), begins([m] * S)
    got = run_prompt(nq, q, k, v, q_begin, k_begin, S, Hq, Hkv, D, dtype, causal, 0.1, gap)[0].cpu()
    check_seen(got, q, k, v, q_begin, k_begin, Hq, Hkv, D, dtype, causal, 0.1, {0, Hq - 1}, {0, S // 2, S - 1})


@pytest.mark.parametrize("n,m,D,causal", [(1, 9001, 64, True), (33, 3000, 128, True), (40, 3001, 96, False), (100, 1500, 72, False), (129, 1100, 128, True), (70, 2060, 256, False),
                                          (129, 1100, 192, True)])
def test_prompt_dealt_values_that_every_row_sees(nq, n, m, D, causal):
    q, k, v = seen_inputs(510, n, m, 1, 2, 1, D, BF16)
    got = run_dealt(nq, q, k, v, begins([n]), begins([m]), 2, 1, D, BF16, causal, 0.1)
    check_seen(got, q, k, v, begins([n]), begins([m]), 2, 1, D, BF16, causal, 0.1, {0, 1}, {0})


def hidden_weight(c, n, what, cached):
    """The first half of sequence 0's keys with scores some thousand below the others' or of -inf, a value of theirs with infinities and a NaN: the columns that are
    not finite."""
    slots = c.table[0, torch.arange(n) // c.page].long() * c.page + torch.arange(n) % c.page
    at = (slots // c.page).cuda(), (slots % c.page).cuda()
    first = torch.arange(n) < n // 2
    k, v, ks, vs = c.tensors
    x = torch.zeros(n, 1, c.D)
    x[:, 0, 0] = torch.where(first, -float("inf") if what == "-inf" else -60.0, 60.0)
    c.keys[0] = x.double()
    token = n // 4                                                 # (in a piece without others, where there are pieces)
    reached = torch.zeros(c.D, dtype=torch.bool)
    if cached == E4M3:
        k.view(torch.uint8)[at] = x.to(E4M3).view(torch.uint8).cuda()
        ks[at] = 1.0
        v.view(torch.uint8)[at[0][token], at[1][token], 0, 3] = 0x7f                        # NaN
        reached[3] = True
    else:
        k[at] = x.to(cached).cuda()
        for column, value in ((3, float("inf")), (4, -float("inf")), (6, float("nan"))):
            v[at[0][token], at[1][token], 0, column] = value
            reached[column] = True
    c.values[0][token, 0, reached] = 0.0
    c.q = torch.zeros_like(c.q)
    c.q.view(-1, c.Hq, c.D)[:, :, 0] = 16.0
    c.scale = 1.0
    return reached


@pytest.mark.parametrize("what", ["low", "-inf"])
@pytest.mark.parametrize("dtype,cached", [(BF16, BF16), (F16, F16), (BF16, E4M3)])
@pytest.mark.parametrize("lengths,D", [([2500], 64), ([1000], 128), ([3000, 40], 72), ([90], 64), ([1500] + [1] * 1030, 64), ([5000], 256)])
def test_token_values_without_weight(nq, lengths, D, dtype, cached, what):
    """A value that is not finite makes its column not finite however little weight its token has, in a sequence of one piece (short, or in a call of
    more than 1024) as in one of many."""
    if what == "-inf" and cached == E4M3:
        cached_what = "low"                                        # (e4m3 has no infinities)
    else:
        cached_what = what
    c = TokenCase(nq, lengths, None, 2, 1, D, dtype, cached, 16, "head", seed=520)
    reached = hidden_weight(c, lengths[0], cached_what, cached)[None]
    job = c.job()
    assert (job.workspace_bytes > 0) == (lengths[0] > 128 and len(lengths) <= 1024)
    nq.nq_attention_token(job)
    got = c.out.cpu()
    for h in range(2):
        o, bound = ref.attention(c.q[:1, :D].double(), c.keys[0][:, 0], c.values[0][:, 0], 1.0, torch.ones(1, lengths[0], dtype=torch.bool), dtype, False)
        check_reached(got[:1, h * D:(h + 1) * D], o, bound, reached, f"head {h}")
    assert torch.isfinite(got[1:]).all()


# ---- begins outside the rows ------------------------------------------------------------------------------------------

@pytest.mark.parametrize("Hq,D,keys,gap", [(1, 64, 200, 0), (1, 256, None, 4), (2, 128, 200, 0), (1, 256, 200, 0), (1, 64, 200, 4), (3, 64, None, 0)])
@pytest.mark.parametrize("ahead", [[-200], [-700, -300, -200], [-2 ** 31]])
def test_many_sequences_that_begin_outside(nq, ahead, Hq, D, keys, gap):
    """More sequences than are ordered by their keys, the first ones beginning in front of the rows, the last ending behind them: what lies inside is right
    in each row."""
    S, T = 300, 599
    inside = [300] + [300 + i for i in range(1, S - len(ahead))]
    q_begin = torch.tensor(ahead + inside + [10 ** 9], dtype=torch.int32)
    assert len(q_begin) == S + 1
    K = keys * S if keys else T
    k_begin = begins([keys] * S) if keys else None
    q, k, v = (randn(540 + i, rows, Hq * D).to(BF16) for i, rows in enumerate((T, K, K)))
    got = run_prompt(nq, q, k, v, q_begin, k_begin, S, Hq, Hq, D, BF16, True, 0.1, gap)[0].cpu()
    check_prompt(got, q, k, v, q_begin.clamp(0, T), k_begin, Hq, Hq, D, BF16, True, 0.1)


# ---- norms of small values ------------------------------------------------------------------------------------------

@pytest.mark.parametrize("kind", ["rms", "layer"])
@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("D", [64, 72, 128, 256])
@pytest.mark.parametrize("eps", [0.0, 2.0 ** -140])
def test_norms_of_small_values(nq, D, dtype, kind, eps):
    """Heads whose squares are below the normal numbers, without anything to speak of added under the root: their norm is as any other's.
    Off by what attention_reference.norm counts, and by the squares' lost bits: each of a head's D squares and additions, and the mean, are off by half a step of the
    smallest value, 2^-150, so the mean by 2^-149 and its root's reciprocal by 2^-150 / mean of itself (and a little of second order)."""
    T, H, page = 6, 3, 4
    x = randn(560, T, H, D) * torch.tensor([1.0, 1e-15, 1e-18, 1e-19, 1e-20, 1e-21])[:, None, None]
    x = x.to(dtype)
    w, b = 1 + 0.2 * randn(561, D), 0.3 * randn(562, D) if kind == "layer" else None
    norm = nq.make_norm(nq.NQ_NORM_LAYER if kind == "layer" else nq.NQ_NORM_RMS, eps, w.cuda(), b.cuda() if b is not None else None)
    d = x.reshape(T, H * D).cuda()
    q_out, k_out = (torch.full_like(d, 7.0) for _ in range(2))
    cache = nq.KvCache(2, page, H, D, E4M3)
    torch.cuda.synchronize()
    nq.nq_head_norm(nq.make_head_norm(d, H * D, d, H * D, None, 0, dt(nq, dtype), H, H, D, norm, norm, None, 0, 0, None, q_out, H * D, k_out, H * D, cache.desc,
                                      torch.arange(T).cuda()), T)
    back = torch.empty(T, H * D, device="cuda")
    nq.nq_cache_read(cache.desc, torch.arange(T).cuda(), T, back, H * D, None, 0, nq.NQ_DT_F32)
    x = x.double()
    y, off = ref.norm(kind, x, w.double(), None if b is None else b.double(), eps)
    c = x - x.mean(-1, keepdim=True) if kind == "layer" else x
    unbiased = y if b is None else y - b.double()
    off = off + unbiased.abs() * 1.01 * 2.0 ** -150 / ((c * c).mean(-1, keepdim=True) + eps)
    y, off, codes = y.reshape(T, -1), off.reshape(T, -1), ref.codes_bound(y, off).reshape(T, -1)
    for out in (q_out, k_out):
        ref.check(out, y, y.abs() * ref.half_step(dtype) * (1 + 2 ** -8) + 2 * off + ref.tiny(dtype))
    ref.check(back, y, codes)


# ---- a scale of 0 ------------------------------------------------------------------------------------------------------

@pytest.mark.parametrize("n,m,S,H,D,gap,dealt", [(40, 90, 1, 2, 136, 0, False), (150, 150, 1, 2, 128, 0, False), (150, 150, 1, 2, 64, 4, False), (30, 300, 1, 2, 64, 0, False),
                                                 (20, 20, 40, 8, 128, 0, False), (20, 2000, 1, 2, 64, 0, True), (130, 2100, 1, 2, 128, 0, True)])
@pytest.mark.parametrize("dtype", [F16, BF16])
def test_prompt_scale_of_zero(nq, dtype, n, m, S, H, D, gap, dealt):
    """0 times a query that is not finite is NaN, and so are its scores and its row; the other rows are the mean of what they see."""
    q, k, v = (randn(580 + i, rows, H * D) for i, rows in enumerate((S * n, S * m, S * m)))
    q[3, 5], q[7, 6], q[11, 7] = float("inf"), -float("inf"), float("nan")
    bad = torch.zeros(S * n, dtype=torch.bool)
    bad[[3, 7, 11]] = True
    q, k, v = (x.to(dtype) for x in (q, k, v))
    q_begin, k_begin = begins([n] * S), begins([m] * S)
    if dealt:
        got = run_dealt(nq, q, k, v, q_begin, k_begin, H, H, D, dtype, True, 0.0)
    else:
        got = run_prompt(nq, q, k, v, q_begin, k_begin, S, H, H, D, dtype, True, 0.0, gap)[0].cpu()
    assert torch.isnan(got[bad, :D]).all()
    q[bad], got[bad, :D] = 0.0, 0.0
    clean = check_prompt_rows(got, q, k, v, q_begin, k_begin, H, D, dtype)
    assert clean == S * n * H - 3


def check_prompt_rows(got, q, k, v, q_begin, k_begin, H, D, dtype):
    """Each row but those of zeros against the mean; how many there were."""
    count = 0
    for s in range(len(q_begin) - 1):
        a, b, c, d = (int(x) for x in (q_begin[s], q_begin[s + 1], k_begin[s], k_begin[s + 1]))
        seen = torch.arange(d - c)[None] <= torch.arange(b - a)[:, None] + (d - c) - (b - a)
        for h in range(H):
            part = lambda x, i, j: x[i:j, h * D:(h + 1) * D].double()  # noqa: E731
            o, bound = ref.attention(part(q, a, b), part(k, c, d), part(v, c, d), 0.0, seen, dtype, True)
            rows = ~(got[a:b, h * D:(h + 1) * D] == 0).all(-1)
            ref.check(got[a:b, h * D:(h + 1) * D][rows], o[rows], bound[rows], f"sequence {s} head {h}")
            count += int(rows.sum())
    return count


# ---- memory that another stream fills ------------------------------------------------------------------------------------

@pytest.mark.parametrize("raw", [False, True])
@pytest.mark.parametrize("cached", [BF16, E4M3])
def test_a_new_cache_on_another_stream(nq, cached, raw):
    """A cache made behind a busy stream and written on another at once holds what was written, zeros where nothing was."""
    a, b = torch.ones(8192, 8192, dtype=BF16, device="cuda"), torch.empty(8192, 8192, dtype=BF16, device="cuda")
    T, H, D, page, pages = 700, 8, 128, 16, 600
    d, slot = randn(600, T, H * D).to(BF16).cuda(), torch.randperm(page * pages, generator=torch.Generator().manual_seed(1))[:T].cuda()
    none, side = nq.make_norm(nq.NQ_NORM_NONE), torch.cuda.Stream()

    def write(cache, stream):
        nq.nq_head_norm(nq.make_head_norm(None, 0, d, H * D, d, H * D, nq.NQ_DT_BF16, H, H, D, none, none, None, 0, 0, None, None, 0, None, 0, cache.desc, slot), T, stream)

    want = nq.KvCache(pages, page, H, D, cached)
    torch.cuda.synchronize()
    write(want, None)
    torch.cuda.synchronize()
    for _ in range(10):
        torch.mm(a, a, out=b)
    got = nq.KvCache(pages, page, H, D, cached)
    write(got, side.cuda_stream if raw else side)
    torch.cuda.synchronize()
    for x, y in zip((got.k, got.v, got.k_scale, got.v_scale), (want.k, want.v, want.k_scale, want.v_scale)):
        if x is not None:
            x, y = (t.view(torch.uint8) if t.dtype == E4M3 else t for t in (x, y))
            assert torch.equal(x, y) and y.any()


def test_a_cache_made_in_a_capture(nq):
    """There the graph fills the pages, each time, ahead of the captured calls that write them."""
    T, H, D = 40, 2, 64
    d, none, cache = randn(610, T, H * D).to(BF16).cuda(), nq.make_norm(nq.NQ_NORM_NONE), []
    slot, back = torch.arange(T).cuda(), torch.zeros(2, T + 8, H * D, dtype=BF16, device="cuda")
    rows = torch.arange(T + 8).cuda()

    def work():
        cache[:] = [nq.KvCache(3, 16, H, D, BF16)]
        nq.nq_head_norm(nq.make_head_norm(None, 0, d, H * D, d, H * D, nq.NQ_DT_BF16, H, H, D, none, none, None, 0, 0, None, None, 0, None, 0, cache[0].desc, slot), T)
        nq.nq_cache_read(cache[0].desc, rows, T + 8, back[0], H * D, back[1], H * D, nq.NQ_DT_BF16)

    work()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        work()
    for i in range(3):
        back.fill_(9.0)
        slot.copy_(torch.randperm(T + 8, generator=torch.Generator().manual_seed(i))[:T])
        graph.replay()
        torch.cuda.synchronize()
        want = torch.zeros(T + 8, H * D, dtype=BF16, device="cuda")
        want[slot] = d
        assert torch.equal(back[0], want) and torch.equal(back[1], want)
        d.copy_(randn(611 + i, T, H * D))
