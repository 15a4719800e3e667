"""The attention operators on the GPU against 64 bits on the CPU (attention_reference.py, with what each result may be off by)."""
import math
import random

import pytest
import torch

import attention_reference as ref

pytestmark = pytest.mark.gpu

F16, BF16, F32, E4M3 = torch.float16, torch.bfloat16, torch.float32, torch.float8_e4m3fn


@pytest.fixture(scope="module")
def nq():
    import paper_2506_17870_amd as nq
    assert torch.cuda.is_available()
    return nq


def dt(nq, dtype):
    return {F32: nq.NQ_DT_F32, F16: nq.NQ_DT_F16, BF16: nq.NQ_DT_BF16}[dtype]


def randn(seed, *shape):
    return torch.randn(*shape, generator=torch.Generator().manual_seed(seed))


def rows_on_device(x, ld, start=0, fill=float("nan")):
    """x [T][width] on the device, rows ld elements apart from element `start` on, `fill` between them; a view [T][width]."""
    T, width = x.shape
    memory = torch.full((start + max(T, 1) * ld + 8,), fill, dtype=x.dtype, device="cuda")
    view = memory[start:start + T * ld].view(T, ld)[:, :width]
    view.copy_(x)
    return view


def values_of(codes, scale):
    return codes.view(torch.uint8).cpu().view(E4M3).double() * scale.double().cpu()[..., None]


def pool(nq, pages, page, heads, dim, dtype, order, poison=True):
    """A cache with every byte of its pages set to something that would show."""
    shape = (pages, heads, page, dim) if order == "head" else (pages, page, heads, dim)
    seen = lambda t: t.transpose(1, 2) if order == "head" else t  # noqa: E731
    bad = 0x7f if dtype == E4M3 else float("nan")
    make = lambda: seen(torch.full(shape, bad if poison else 0, dtype=torch.uint8 if dtype == E4M3 else dtype, device="cuda"))  # noqa: E731
    k, v = make(), make()
    ks, vs = (seen(torch.full(shape[:3], float("nan") if poison else 1.0, device="cuda")) for _ in range(2)) if dtype == E4M3 else (None, None)
    if dtype == E4M3:
        k, v = k.view(E4M3), v.view(E4M3)
    return k, v, ks, vs, nq.make_kv_cache(k, v, ks, vs)


# ---- heads into the cache ----------------------------------------------------------------------------------------

HEADS = [  # T, Hq, Hkv, D, dtype, norm, rotary, pairs, cache, page, order, extra elements between rows, first element
    (1, 32, 8, 128, BF16, "rms", 128, "halves", E4M3, 16, "head", 0, 0),
    (3, 1, 1, 8, F16, "layer", 8, "halves", F16, 1, "token", 3, 1),
    (70, 12, 12, 80, F16, "layer", 40, "neighbours", F16, 24, "token", 8, 0),
    (33, 6, 2, 72, BF16, "rms", 36, "halves", BF16, 7, "head", 5, 3),
    (19, 4, 2, 96, F32, "rms", 90, "halves", E4M3, 16, "token", 0, 0),
    (5, 16, 1, 256, BF16, "layer", 256, "neighbours", E4M3, 32, "head", 0, 0),
    (600, 5, 5, 64, BF16, "none", 64, "halves", BF16, 64, "head", 0, 0),
    (517, 7, 1, 192, F32, "none", 0, "halves", F16, 100, "head", 1, 1),
    (2, 64, 16, 40, F16, "rms", 2, "neighbours", E4M3, 16, "head", 0, 0),
    (1, 1, 1, 16, BF16, "rms", 0, "halves", None, 0, "head", 0, 0),
]


def head_inputs(seed, T, Hq, Hkv, D, dtype):
    spread = lambda H: torch.exp(0.5 * randn(seed + 7, H * D))  # noqa: E731
    return tuple((randn(seed + i, T, H * D) * spread(H)).to(dtype) for i, H in enumerate((Hq, Hkv, Hkv)))


@pytest.mark.parametrize("case", HEADS, ids=lambda c: "-".join(str(x).replace("torch.", "") for x in c))
def test_head_norm(nq, case):
    T, Hq, Hkv, D, dtype, norm, rotary, pairs, cached, page, order, gap, start = case
    q, k, v = head_inputs(11, T, Hq, Hkv, D, dtype)
    if T > 4:
        k[3] = 0                                               # a block of zeros has the scale 1
        v[3] = 0
    w = {n: (1 + 0.2 * randn(21 + i, D)) for i, n in enumerate("qk")}
    b = {n: 0.3 * randn(31 + i, D) for i, n in enumerate("qk")} if norm == "layer" else {}
    freq = torch.tensor([10000.0 ** (-2 * i / max(rotary, 1)) for i in range(rotary // 2)])
    rng = random.Random(T)
    position = torch.tensor([rng.choice([0, 1, 77, 4095, 131071, 1000003, -5, 2 ** 31 - 1]) for _ in range(T)], dtype=torch.int32)
    dq, dk, dv = (rows_on_device(x, x.shape[1] + gap, start) for x in (q, k, v))
    kind = {"none": nq.NQ_NORM_NONE, "rms": nq.NQ_NORM_RMS, "layer": nq.NQ_NORM_LAYER}[norm]
    norms = [nq.make_norm(kind, 1e-6, w[n].cuda() if norm != "none" else None, b[n].cuda() if n in b else None) for n in "qk"]
    q_out, k_out = (rows_on_device(torch.zeros(T, x.shape[1], dtype=dtype), x.shape[1] + gap, start, fill=7.0) for x in (q, k))
    cache = slot = None
    if cached:
        pages = T // page + 3
        ck, cv, ks, vs, cache = pool(nq, pages, page, Hkv, D, cached, order)
        slots = rng.sample(range(pages * page), T)
        for i in range(2, T, 9):
            slots[i] = rng.choice([-1, -2 ** 40, pages * page, 2 ** 45])
        slot = torch.tensor(slots).cuda()
    job = nq.make_head_norm(dq, q.shape[1] + gap, dk, k.shape[1] + gap, dv, k.shape[1] + gap, dt(nq, dtype), Hq, Hkv, D, *norms, freq.cuda() if rotary else None,
                            rotary, nq.NQ_PAIRS_HALVES if pairs == "halves" else nq.NQ_PAIRS_NEIGHBOURS, position.cuda() if rotary else None,
                            q_out, q.shape[1] + gap, k_out, k.shape[1] + gap, cache, slot)
    nq.nq_head_norm(job, T)
    torch.cuda.synchronize()
    want = {}
    for n, x, out in (("q", q, q_out), ("k", k, k_out)):
        y, off = ref.norm(norm, x.double().view(T, -1, D), w[n].double(), b[n].double() if n in b else None, 1e-6)
        want[n] = ref.rotate(y, off, position, freq, rotary, pairs)
        y, off = (z.reshape(T, -1) for z in want[n])
        ref.check(out, y, y.abs() * ref.half_step(dtype) * (1 + 2 ** -8) + 2 * off + ref.tiny(dtype), n)
        if start or gap:                                       # what lies before and between the rows is nobody's
            assert (torch.as_strided(out, (start,), (1,), 0) == 7).all() and (torch.as_strided(out, (T - 1, gap), (out.stride(0), 1), start + x.shape[1]) == 7).all()
    if not cached:
        return
    live = [i for i in range(T) if 0 <= slots[i] < pages * page]
    at = torch.tensor([slots[i] for i in live])
    touched = torch.zeros(pages * page, dtype=torch.bool)
    touched[at] = True
    touched = touched.view(pages, page)
    vx = v.double().view(T, Hkv, D)
    for n, got, scale, (y, off) in (("k", ck, ks, want["k"]), ("v", cv, vs, (vx, torch.zeros_like(vx)))):
        y, off = y[live], off[live]
        raw = got.view(torch.uint8) if cached == E4M3 else got
        raw = raw.cpu()
        rest = raw[~touched]
        assert (rest == 0x7f).all() if cached == E4M3 else torch.isnan(rest).all(), "a token that is not the call's has changed"
        if cached == E4M3:
            values, s = values_of(got, scale)[at // page, at % page], scale.cpu()[at // page, at % page].double()
            a = y.abs().amax(-1)
            ref.check(s, torch.where(a == 0, 1.0, a / 448), a / 448 * 4 * ref.U + off.amax(-1) / 448 * 2, n + " scale")
            ref.check(values, y, ref.codes_bound(y, off) + 1e-300, n)
            assert torch.isnan(scale.cpu()[~touched]).all()
            if n == "v":                                       # nothing before the quantiser: the codes that its definition names
                x = v.float().view(T, Hkv, D)[live]
                m = x.abs().amax(-1, keepdim=True)
                sc = torch.where(m == 0, torch.ones(()), (m / 448).clamp(min=2.0 ** -126))
                assert torch.equal((x * (1 / sc)).to(E4M3).view(torch.uint8), raw[at // page, at % page])
        else:
            bound = y.abs() * ref.half_step(cached) * (1 + 2 ** -8) + 2 * off + ref.tiny(cached)
            ref.check(got.cpu()[at // page, at % page], y, bound, n)
            if n == "v":
                assert torch.equal(v.view(T, Hkv, D)[live].float().to(cached), raw[at // page, at % page])


def test_head_norm_in_place_and_in_parts(nq):
    """Outputs over the inputs; queries alone, keys alone; equal bits to the whole call's."""
    T, Hq, Hkv, D = 37, 6, 2, 128
    q, k, v = head_inputs(3, T, Hq, Hkv, D, BF16)
    freq, position = torch.rand(64).cuda(), torch.arange(T, dtype=torch.int32).cuda() * 1000
    norm = nq.make_norm(nq.NQ_NORM_RMS, 1e-5, torch.rand(D).cuda())
    qkv = torch.cat([q, k, v], 1).cuda()
    ld = qkv.shape[1]
    parts = qkv[:, :Hq * D], qkv[:, Hq * D:(Hq + Hkv) * D], qkv[:, (Hq + Hkv) * D:]

    def call(q, k, v, q_out, k_out, cache, slot):
        job = nq.make_head_norm(q, ld, k, ld, v, ld, nq.NQ_DT_BF16, Hq, Hkv, D, norm, norm, freq, D, 0, position, q_out, ld, k_out, ld, cache, slot)
        nq.nq_head_norm(job, T)

    slot = torch.randperm(48)[:T].cuda()
    whole = torch.empty_like(qkv)
    one = pool(nq, 3, 16, Hkv, D, E4M3, "head", poison=False)
    call(*parts, whole[:, :Hq * D], whole[:, Hq * D:], one[4], slot)
    two = pool(nq, 3, 16, Hkv, D, E4M3, "head", poison=False)
    call(None, parts[1], None, None, None, two[4], slot)
    call(None, None, parts[2], None, None, two[4], slot)
    for a, b in zip(one[:4], two[:4]):
        assert torch.equal(a.view(torch.uint8) if a.dtype == E4M3 else a, b.view(torch.uint8) if b.dtype == E4M3 else b)
    call(parts[0], parts[1], None, parts[0], parts[1], None, None)
    assert torch.equal(qkv[:, :(Hq + Hkv) * D], whole[:, :(Hq + Hkv) * D]) and torch.equal(qkv[:, (Hq + Hkv) * D:].cpu(), v)


def test_far_positions(nq):
    """The angle of a position past 2^30 is the one of the position modulo whole turns."""
    T, D = 64, 64
    freq = (torch.rand(D // 2, generator=torch.Generator().manual_seed(1)) * 2 ** -4)
    position = torch.randint(2 ** 30, 2 ** 31 - 1, (T,), generator=torch.Generator().manual_seed(2), dtype=torch.int32)
    x = torch.ones(T, D)
    out = torch.empty(T, D, device="cuda")
    none = nq.make_norm(nq.NQ_NORM_NONE)
    nq.nq_head_norm(nq.make_head_norm(x.cuda(), D, None, 0, None, 0, nq.NQ_DT_F32, 1, 1, D, none, none, freq.cuda(), D, 1, position.cuda(), out, D, None, 0), T)
    want, off = ref.rotate(x.double()[:, None], torch.zeros(T, 1, D, dtype=torch.float64), position, freq, D, "neighbours")
    ref.check(out, want[:, 0], off[:, 0] + want[:, 0].abs() * ref.U)


def test_values_that_are_not_finite(nq):
    """A head with a NaN or an infinity: its row of the cache is not finite, its neighbours are as ever."""
    T, H, D = 4, 2, 64
    x = randn(5, T, H * D)
    x[1, 3], x[2, 70] = float("nan"), float("inf")
    none = nq.make_norm(nq.NQ_NORM_NONE)
    k, v, ks, vs, cache = pool(nq, 1, 4, H, D, E4M3, "token")
    d = x.to(BF16).cuda()
    nq.nq_head_norm(nq.make_head_norm(None, 0, d, H * D, d, H * D, nq.NQ_DT_BF16, H, H, D, none, none, None, 0, 0, None, None, 0, None, 0, cache,
                                      torch.arange(T).cuda()), T)
    out = torch.empty(T, H * D, device="cuda")
    nq.nq_cache_read(cache, torch.arange(T).cuda(), T, None, 0, out, H * D, nq.NQ_DT_F32)
    bad = torch.zeros(T, H, dtype=torch.bool)
    bad[1, 0] = bad[2, 1] = True
    got = out.cpu().view(T, H, D)
    assert torch.isfinite(got[~bad]).all() and not torch.isfinite(got[bad]).all(-1).any()


# ---- rows back ---------------------------------------------------------------------------------------------------

@pytest.mark.parametrize("cached", [F16, BF16, E4M3])
@pytest.mark.parametrize("T,H,D,page,order,dtype", [(1, 1, 8, 1, "head", F32), (45, 12, 64, 16, "token", F16), (130, 3, 80, 24, "head", BF16), (33, 8, 128, 16, "head", BF16),
                                                  (9, 2, 256, 100, "token", F32), (700, 1, 136, 7, "head", F16)])
def test_cache_read(nq, T, H, D, page, order, dtype, cached):
    pages = T // page + 2
    k, v, ks, vs, cache = pool(nq, pages, page, H, D, cached, order, poison=False)
    for i, (t, s) in enumerate(((k, ks), (v, vs))):
        x = randn(40 + i, *t.shape) * (100 if cached == E4M3 else 1)
        t.copy_(x.to(cached)) if cached != E4M3 else t.view(torch.uint8).copy_(x.to(E4M3).view(torch.uint8))
        if s is not None:
            s.copy_(randn(50 + i, *s.shape).exp())
    slots = torch.randint(0, pages * page, (T,), generator=torch.Generator().manual_seed(T))
    missing = torch.zeros(T, dtype=torch.bool)
    if T > 2:
        slots[1], slots[T - 1] = -1, pages * page
        missing[1] = missing[T - 1] = True
    gap = 3 if D == 80 else 0
    outs = [rows_on_device(torch.zeros(T, H * D, dtype=dtype), H * D + gap, gap, fill=9.0) for _ in range(2)]
    nq.nq_cache_read(cache, slots.cuda(), T, outs[0], H * D + gap, outs[1], H * D + gap, dt(nq, dtype))
    at = slots.clamp(0, pages * page - 1)
    for out, t, s in zip(outs, (k, v), (ks, vs)):
        x = (t.view(torch.uint8).cpu().view(E4M3) if cached == E4M3 else t.cpu()).float()
        if s is not None:
            x = x * s.cpu()[..., None]
        want = x[at // page, at % page].reshape(T, -1).to(dtype)
        want[missing] = 0
        assert torch.equal(out.cpu(), want)
        if gap:
            assert (torch.as_strided(out, (T - 1, gap), (H * D + gap, 1), out.storage_offset() + H * D) == 9).all()


# ---- whole prompts -----------------------------------------------------------------------------------------------

PROMPT = [  # query lengths, key lengths or None, Hq, Hkv, D, dtype, causal, scale, extra elements between rows
    ([1], None, 1, 1, 64, BF16, True, 0.125, 0),
    ([33], None, 4, 1, 128, BF16, True, 0.1, 0),
    ([197, 197], None, 3, 3, 64, F16, False, 0.125, 0),
    ([5, 0, 130, 1, 64, 257], None, 4, 2, 128, BF16, True, 0.09, 0),
    ([7, 40, 1, 129], [50, 40, 300, 131], 2, 1, 96, F16, True, 0.1, 8),
    ([60, 9, 0, 3], [20, 0, 5, 3], 2, 2, 64, BF16, True, 0.125, 0),
    ([60, 9], [20, 0], 2, 2, 40, F16, False, 0.2, 4),
    ([150], None, 3, 1, 72, BF16, True, -0.1, 3),
    ([65, 31], None, 2, 1, 192, F16, True, 0.07, 0),
    ([70, 129], [133, 200], 2, 1, 256, BF16, True, 0.06, 0),
    ([40], [90], 2, 1, 136, BF16, False, 0.0, 0),
    ([515], None, 2, 2, 128, F16, True, 0.2, 0),
    ([2, 700], [2, 1300], 1, 1, 64, BF16, True, 0.15, 0),
    ([1100, 300, 5], None, 32, 8, 64, BF16, True, 0.15, 0),
    ([1030], None, 40, 4, 96, F16, False, 0.1, 0),
    ([130, 900], [130, 1111], 32, 8, 128, F16, True, 0.1, 0),
    ([300] * 70, None, 2, 2, 64, BF16, True, 0.1, 0),
    ([7 * i % 60 for i in range(300)], [11 * i % 90 for i in range(300)], 1, 1, 64, BF16, True, 0.1, 0),
]


def begins(lengths, first=0):
    at = [first]
    for n in lengths:
        at.append(at[-1] + n)
    return torch.tensor(at, dtype=torch.int32)


def run_prompt(nq, q, k, v, q_begin, k_begin, S, Hq, Hkv, D, dtype, causal, scale, gap=0, out=None, stream=None):
    lds = [x.shape[1] + gap for x in (q, k, v)]
    dq, dk, dv = (rows_on_device(x, ld, gap) for x, ld in zip((q, k, v), lds))
    out = rows_on_device(torch.full_like(q, 5.0), lds[0], gap, fill=5.0) if out is None else out
    job = nq.make_attention_prompt(dq, lds[0], dk, lds[1], dv, lds[2], out, lds[0], q_begin.cuda(), k_begin.cuda() if k_begin is not None else None, S,
                                   q.shape[0], k.shape[0], dt(nq, dtype), Hq, Hkv, D, causal, scale)
    nq.nq_attention_prompt(job, stream)
    return out, job


def check_prompt(got, q, k, v, q_begin, k_begin, Hq, Hkv, D, dtype, causal, scale, what=""):
    qb, kb = q_begin.tolist(), (q_begin if k_begin is None else k_begin).tolist()
    for s in range(len(qb) - 1):
        n, m = qb[s + 1] - qb[s], kb[s + 1] - kb[s]
        seen = torch.ones(n, m, dtype=torch.bool)
        if causal:
            seen = torch.arange(m)[None] <= torch.arange(n)[:, None] + (m - n)
        for h in range(Hq):
            g = h // (Hq // Hkv)
            part = lambda x, b, i: x[b[s]:b[s + 1], i * D:i * D + D].double()  # noqa: E731
            o, bound = ref.attention(part(q, qb, h), part(k, kb, g), part(v, kb, g), scale, seen, dtype, True)
            ref.check(got[qb[s]:qb[s + 1], h * D:h * D + D], o, bound, f"{what} sequence {s} head {h}")


@pytest.mark.parametrize("case", PROMPT, ids=lambda c: "-".join(str(x).replace("torch.", "").replace(" ", "")[:40] for x in c))
def test_attention_prompt(nq, case):
    lengths, keys, Hq, Hkv, D, dtype, causal, scale, gap = case
    first, behind = (3, 5) if len(lengths) > 1 else (0, 0)
    q_begin, k_begin = begins(lengths, first), begins(keys) if keys else None
    T, K = int(q_begin[-1]) + behind, int(k_begin[-1]) + 1 if keys else int(q_begin[-1]) + behind
    q, k, v = (randn(60 + i, *s) for i, s in enumerate(((T, Hq * D), (K, Hkv * D), (K, Hkv * D))))
    q = q * 2
    for x, b in ((q, q_begin), (k, q_begin if k_begin is None else k_begin), (v, q_begin if k_begin is None else k_begin)):
        x[:int(b[0])] = float("nan")                           # rows of no sequence
        x[int(b[-1]):] = float("inf")
    q, k, v = (x.to(dtype) for x in (q, k, v))
    out, _ = run_prompt(nq, q, k, v, q_begin, k_begin, len(lengths), Hq, Hkv, D, dtype, causal, scale, gap)
    got = out.cpu()
    check_prompt(got, q, k, v, q_begin, k_begin, Hq, Hkv, D, dtype, causal, scale)
    assert (got[:first] == 5).all() and (got[int(q_begin[-1]):] == 5).all(), "rows of no sequence have changed"
    if gap:
        assert (torch.as_strided(out, (T - 1, gap), (out.stride(0), 1), out.storage_offset() + Hq * D) == 5).all()


@pytest.mark.parametrize("dtype", [F16, BF16])
@pytest.mark.parametrize("D,heads,gap", [(64, 1, 0), (128, 1, 0), (256, 1, 0), (64, 140, 0), (128, 140, 0), (128, 1, 4), (64, 140, 4)])
def test_prompt_values_that_are_not_finite(nq, dtype, D, heads, gap):
    """Keys and values that a row does not see do not reach it, whatever they are; those that it sees do.  Many heads and few: both ways to divide the
    work; rows on 16 bytes and not."""
    n = 150
    one = [randn(70 + i, n, D) for i in range(3)]
    q, k, v = (x.clone() for x in one)
    v[70, 5], v[71, 6], v[72, 7] = float("inf"), -float("inf"), float("nan")
    v[130] = float("nan")
    k[100, 0] = float("nan")
    q, k, v = (x.to(dtype) for x in (q, k, v))
    wide = lambda x: x.repeat(1, heads)  # noqa: E731
    some = {0, heads - 1}
    got = run_prompt(nq, wide(q), k, v, begins([n]), None, 1, heads, 1, D, dtype, True, 0.1, gap)[0].cpu()
    for h in some:
        part = got[:, h * D:(h + 1) * D]
        check_prompt(part[:100], q[:100], k[:100], v[:100], begins([100]), None, 1, 1, D, dtype, True, 0.1)
        assert torch.isnan(part[100:]).all()
    k[100] = 0
    got = run_prompt(nq, wide(q), k, v, begins([n]), None, 1, heads, 1, D, dtype, True, 0.1, gap)[0].cpu()
    for h in some:
        check_prompt(got[:, h * D:(h + 1) * D], q, k, v, begins([n]), None, 1, 1, D, dtype, True, 0.1)


def test_prompt_scores_of_no_weight(nq):
    """Scores of -inf: without weight beside others, NaN if there are no others, as the definition has it."""
    n, D = 40, 64
    q, k, v = torch.ones(n, D), randn(80, n, D) * 0.1, randn(81, n, D)
    k[:7, 0] = -float("inf")
    q, k, v = (x.to(BF16) for x in (q, k, v))
    out, _ = run_prompt(nq, q, k, v, begins([n]), None, 1, 1, 1, D, BF16, True, 0.1)
    got = out.cpu()
    assert torch.isnan(got[:7]).all()
    seen = (torch.arange(n)[None] <= torch.arange(n)[:, None])[7:] & (torch.arange(n) >= 7)[None]
    k[:7] = 0
    o, bound = ref.attention(q[7:].double(), k.double(), v.double(), 0.1, seen, BF16, True)
    ref.check(got[7:], o, bound)


def test_prompt_large_scores(nq):
    """Scores up to thousands, growing and falling along the keys: the running maximum's every turn."""
    n, D = 300, 64
    q, v = torch.ones(n, D), randn(82, n, D)
    k = (torch.cat([torch.linspace(-60, 60, 150), torch.linspace(60, -60, 150)]))[:, None].expand(n, D)
    for dtype in (F16, BF16):
        a, b, c = (x.to(dtype) for x in (q, k, v))
        for scale in (1.0, -1.0):
            out, _ = run_prompt(nq, a, b, c, begins([n]), None, 1, 1, 1, D, dtype, True, scale)
            check_prompt(out.cpu(), a, b, c, begins([n]), None, 1, 1, D, dtype, True, scale)


def test_prompt_equal_calls_give_equal_bits(nq):
    q, k, v = (randn(90 + i, 333, 4 * 128).to(BF16) for i in range(3))
    outs = [run_prompt(nq, q, k, v, begins([100, 233]), None, 2, 4, 4, 128, BF16, True, 0.1)[0].cpu() for _ in range(3)]
    assert torch.equal(outs[0], outs[1]) and torch.equal(outs[0], outs[2])


# ---- one token over the cache --------------------------------------------------------------------------------------

TOKEN = [  # lengths, longest or None, Hq, Hkv, D, dtype, cache, page, order
    ([1], None, 1, 1, 64, BF16, BF16, 16, "head"),
    ([0, 1, 2, 31, 32, 33, 517], None, 8, 2, 128, BF16, E4M3, 16, "head"),
    ([100, 0, 1000], 4000, 12, 12, 64, F16, F16, 24, "token"),
    ([4001], None, 32, 8, 128, BF16, E4M3, 16, "head"),
    ([3000, 5, 1999], None, 16, 1, 128, F16, E4M3, 32, "token"),
    ([900, 333], None, 40, 2, 128, BF16, BF16, 64, "head"),
    ([700, 129], None, 6, 2, 256, F16, F16, 16, "head"),
    ([700, 129], None, 4, 4, 256, BF16, E4M3, 128, "head"),
    ([300, 77], None, 4, 2, 72, BF16, E4M3, 1, "head"),
    ([300, 77, 128], None, 5, 1, 96, F16, F16, 100, "token"),
    ([200], None, 3, 1, 192, BF16, E4M3, 7, "head"),
    ([50, 513], None, 2, 1, 8, F16, E4M3, 16, "head"),
    ([64] * 130, None, 2, 2, 64, BF16, E4M3, 16, "head"),
    ([128, 2047], None, 9, 3, 248, BF16, BF16, 48, "head"),
    ([i * 37 % 900 + (1500 if i % 23 == 0 else 0) for i in range(70)], None, 2, 1, 64, BF16, E4M3, 16, "head"),
    ([i * 53 % 400 for i in range(150)] + [5000] + [i * 31 % 300 for i in range(160)], None, 1, 1, 64, F16, F16, 16, "token"),
    ([3] * 1030 + [700], None, 1, 1, 16, BF16, E4M3, 16, "head"),
    ([20000], None, 1, 1, 64, BF16, BF16, 16, "head"),
    ([640, 500], None, 2, 1, 80, BF16, BF16, 16, "head"),
]


class TokenCase:
    """A filled cache and the queries; pages in a random order, the cache's other tokens NaN."""

    def __init__(self, nq, lengths, longest, Hq, Hkv, D, dtype, cached, page, order, seed=100):
        self.nq, self.lengths, self.longest = nq, lengths, longest or max(lengths)
        self.Hq, self.Hkv, self.D, self.dtype, self.cached, self.page = Hq, Hkv, D, dtype, cached, page
        used = [-(-n // page) for n in lengths]
        pages = sum(used) + 2
        k, v, ks, vs, self.cache = pool(nq, pages, page, Hkv, D, cached, order)
        self.tensors = k, v, ks, vs
        free = list(range(pages))
        random.Random(seed).shuffle(free)
        self.table = torch.full((len(lengths), max(-(-self.longest // page), 1)), -1, dtype=torch.int32)
        self.keys, self.values = [], []
        host = [t.cpu() if t is None or t.dtype != E4M3 else t.view(torch.uint8).cpu() for t in (k, v)]
        scales = [None if s is None else s.cpu() for s in (ks, vs)]
        for i, n in enumerate(lengths):
            mine = [free.pop() for _ in range(used[i])]
            self.table[i, :used[i]] = torch.tensor(mine, dtype=torch.int32)
            at = torch.tensor(mine, dtype=torch.int64)[torch.arange(n) // page] if n else torch.zeros(0, dtype=torch.int64)
            place = torch.arange(n) % page
            for which, keep in ((0, self.keys), (1, self.values)):
                x = randn(seed + 10 * i + which, n, Hkv, D)
                if cached == E4M3:
                    s = (0.5 + randn(seed + 10 * i + which + 5, n, Hkv).abs()) / 100
                    c = (x * 100).clamp(-448, 448).to(E4M3)
                    host[which][at, place] = c.view(torch.uint8)
                    scales[which][at, place] = s
                    keep.append(c.double() * s.double()[..., None])
                else:
                    host[which][at, place] = x.to(cached)
                    keep.append(x.to(cached).double())
        for t, x in zip((k, v), host):
            (t.view(torch.uint8) if cached == E4M3 else t).copy_(x)
        for t, x in zip((ks, vs), scales):
            if t is not None:
                t.copy_(x)
        self.q = (randn(seed + 3, len(lengths), Hq * D) * 2).to(dtype)
        self.scale = D ** -0.5

    def job(self, q=None, length=None, table=None, sequences=None, gap=0, out=None):
        nq, S, width = self.nq, sequences or len(self.lengths), self.Hq * self.D
        need = nq.nq_attention_token_workspace_bytes(S, self.Hq, self.Hkv, self.D, self.longest)
        self.workspace = torch.full((need,), 0xff, dtype=torch.uint8, device="cuda")       # (NaN, wherever it is read before it is written)
        dq = rows_on_device(self.q if q is None else q, width + gap, gap)
        self.out = rows_on_device(torch.full((S, width), 5.0, dtype=self.dtype), width + gap, gap, fill=5.0) if out is None else out
        self.d_length = torch.tensor(self.lengths, dtype=torch.int32).cuda() if length is None else length
        self.d_table = self.table.cuda() if table is None else table
        return nq.make_attention_token(dq, width + gap, self.out, width + gap, self.cache, self.d_table, self.d_length, S, self.longest, dt(nq, self.dtype), self.Hq,
                                       self.scale, self.workspace)

    def check(self, got, scale=None, keep=None):
        for i, n in enumerate(self.lengths):
            for h in range(self.Hq):
                g = h // (self.Hq // self.Hkv)
                k, v = self.keys[i][:, g], self.values[i][:, g]
                seen = torch.ones(1, n, dtype=torch.bool) if keep is None else keep[i][None]
                o, bound = ref.attention(self.q[i:i + 1, h * self.D:(h + 1) * self.D].double(), k, v, self.scale if scale is None else scale, seen, self.dtype, False)
                ref.check(got[i:i + 1, h * self.D:(h + 1) * self.D], o, bound, f"sequence {i} ({n}) head {h}")


@pytest.mark.parametrize("case", TOKEN, ids=lambda c: "-".join(str(x).replace("torch.", "").replace(" ", "")[:40] for x in c))
def test_attention_token(nq, case):
    c = TokenCase(nq, *case)
    gap = 3 if c.D == 72 else 0
    job = c.job(gap=gap)
    nq.nq_attention_token(job)
    first = c.out.cpu()
    c.check(first)
    c.out.fill_(5.0)
    nq.nq_attention_token(job)
    assert torch.equal(c.out.cpu(), first), "equal calls give equal bits"


@pytest.mark.parametrize("page", [16, 24])
def test_token_pages_that_are_not_there(nq, page):
    """Tokens of pages that the cache does not have are left out; a sequence of none but those is 0."""
    c = TokenCase(nq, [1000, 40, 90], None, 4, 2, 64, BF16, E4M3, page, "head")
    keep = [torch.ones(n, dtype=torch.bool) for n in c.lengths]
    pages = c.cache.pages
    for i, p, name in ((0, 0, -1), (0, 7, pages), (0, 30, -2 ** 31), (2, 1, 2 ** 31 - 1)):
        c.table[i, p] = name
        keep[i][p * page:(p + 1) * page] = False
    c.table[1] = -7
    keep[1][:] = False
    nq.nq_attention_token(c.job())
    got = c.out.cpu()
    c.check(got, keep=keep)
    assert (got[1] == 0).all()


def test_token_lengths_out_of_range(nq):
    """Lengths below 0 count as 0, above max_length as max_length."""
    c = TokenCase(nq, [0, 300], None, 2, 1, 64, F16, F16, 16, "head")
    nq.nq_attention_token(c.job(length=torch.tensor([-5, 2 ** 31 - 1], dtype=torch.int32).cuda()))
    c.check(c.out.cpu())


def test_token_scores_of_no_weight(nq):
    """Keys with scores of -inf have no weight; NaN where there are no others.  Scores of thousands either way."""
    c = TokenCase(nq, [600, 40], None, 2, 1, 64, BF16, BF16, 16, "head")
    k = c.tensors[0]
    c.q = torch.ones_like(c.q)
    slots = c.table[0, torch.arange(600) // 16].long() * 16 + torch.arange(600) % 16
    flat = lambda t, s: t[s // 16, s % 16]  # noqa: E731
    keep = [torch.ones(600, dtype=torch.bool), torch.ones(40, dtype=torch.bool)]
    keep[0][100:400] = False
    for s in slots[100:400].tolist():
        k[s // 16, s % 16, 0, 0] = -float("inf")
    other = c.table[1, torch.arange(40) // 16].long() * 16 + torch.arange(40) % 16
    for s in other.tolist():
        k[s // 16, s % 16, 0, 3] = -float("inf")
    nq.nq_attention_token(c.job())
    got = c.out.cpu()
    assert torch.isnan(got[1]).all()
    c.lengths, c.keys, c.values, c.q = [600], c.keys[:1], c.values[:1], c.q[:1]
    c.check(got[:1], keep=keep)


@pytest.mark.parametrize("cached", [BF16, E4M3])
def test_token_split_and_whole(nq, cached):
    """The same sequences alone, with others and in another order of their batch: each within its bound."""
    lengths = [2500, 1, 800, 0, 129]
    c = TokenCase(nq, lengths, None, 8, 2, 128, BF16, cached, 16, "head")
    nq.nq_attention_token(c.job())
    c.check(c.out.cpu())
    for i in (0, 2):
        d = c.job(q=c.q[i:i + 1], length=torch.tensor(lengths[i:i + 1], dtype=torch.int32).cuda(), table=c.table[i:i + 1].cuda(), sequences=1)
        nq.nq_attention_token(d)
        alone = c.out.cpu()
        for h in range(8):
            o, bound = ref.attention(c.q[i:i + 1, h * 128:(h + 1) * 128].double(), c.keys[i][:, h // 4], c.values[i][:, h // 4], c.scale,
                                     torch.ones(1, lengths[i], dtype=torch.bool), BF16, False)
            ref.check(alone[:, h * 128:(h + 1) * 128], o, bound)


def test_small_probabilities_add_up(nq):
    """One key with most of the weight and 8191 with 2^-20 of it each: what they add is 2^-7 of the result, and none of it is lost."""
    n, D = 8192, 64
    for dtype, cached in ((F16, F16), (BF16, BF16), (F16, E4M3)):
        c = TokenCase(nq, [n], None, 1, 1, D, dtype, cached, 16, "head")
        k, v, ks, vs = c.tensors
        slots = (c.table[0, torch.arange(n) // 16].long() * 16 + torch.arange(n) % 16).cuda()
        x = torch.zeros(n, 1, D)
        x[0, 0, 0] = 1.0
        y = torch.full((n, 1, D), 1.0)
        y[0] = 0.0
        for t, z, s in ((k, x, ks), (v, y, vs)):
            if cached == E4M3:
                t.view(torch.uint8)[slots // 16, slots % 16] = z.to(E4M3).view(torch.uint8).cuda()
                s[slots // 16, slots % 16] = 1.0
            else:
                t[slots // 16, slots % 16] = z.to(cached).cuda()
        c.keys, c.values = [x.double()], [y.double()]
        c.q = torch.zeros(1, D, dtype=dtype)
        c.q[0, 0] = 20.0
        c.scale = math.log(2.0)
        nq.nq_attention_token(c.job())
        c.check(c.out.cpu())
