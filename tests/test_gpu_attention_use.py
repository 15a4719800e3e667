"""The attention operators as a program uses them: together, captured and replayed, on several streams, behind and ahead of the 8-bit floating
point layers."""
import pytest
import torch

import attention_reference as ref
from test_gpu_attention import BF16, E4M3, F16, TokenCase, begins, check_prompt, dt, pool, randn, run_prompt, values_of

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def nq():
    import paper_2506_17870_amd as nq
    assert torch.cuda.is_available()
    return nq


class Layer:
    """The attention of one layer: one projection's rows in, its cache, its buffers."""

    def __init__(self, nq, tokens, sequences, longest, Hq=8, Hkv=2, D=128, dtype=BF16, cached=E4M3, page=16):
        self.nq, self.Hq, self.Hkv, self.D, self.dtype, self.page, self.longest = nq, Hq, Hkv, D, dtype, page, longest
        self.pages = -(-longest // page) * sequences
        self.cache = nq.KvCache(self.pages, page, Hkv, D, cached)
        self.table = torch.randperm(self.pages, generator=torch.Generator().manual_seed(1)).view(sequences, -1).to(torch.int32)
        self.d_table = self.table.cuda()
        self.w = [1 + 0.2 * randn(2 + i, D) for i in range(2)]
        self.freq = torch.tensor([10000.0 ** (-2 * i / D) for i in range(D // 2)])
        self.norms = [nq.make_norm(nq.NQ_NORM_RMS, 1e-6, w.cuda()) for w in self.w]
        self.d_freq, self.width = self.freq.cuda(), (Hq + 2 * Hkv) * D
        self.qkv = torch.zeros(tokens, self.width, dtype=dtype, device="cuda")
        self.position = torch.zeros(tokens, dtype=torch.int32, device="cuda")
        self.slot = torch.full((tokens,), -1, dtype=torch.int64, device="cuda")
        self.q, self.o = (torch.zeros(tokens, Hq * D, dtype=dtype, device="cuda") for _ in range(2))
        self.k = torch.zeros(tokens, Hkv * D, dtype=dtype, device="cuda")
        q, k, v = (self.qkv[:, a * D:b * D] for a, b in ((0, Hq), (Hq, Hq + Hkv), (Hq + Hkv, Hq + 2 * Hkv)))
        self.heads = nq.make_head_norm(q, self.width, k, self.width, v, self.width, dt(nq, dtype), Hq, Hkv, D, *self.norms, self.d_freq, D, nq.NQ_PAIRS_HALVES,
                                       self.position, self.q, Hq * D, self.k, Hkv * D, self.cache.desc, self.slot)
        self.v = v

    def slots(self, sequence, first, count):
        at = torch.arange(first, first + count)
        return self.table[sequence, at // self.page].long() * self.page + at % self.page

    def put(self, x, position, slot):
        n = x.shape[0]
        self.qkv[:n].copy_(x)
        self.position[:n].copy_(position)
        self.slot[:n].copy_(slot)
        return n

    def of_the_inputs(self, x, position):
        """q, k, v in 64 bits of rows of the projection."""
        T, D = x.shape[0], self.D
        y = x.double().view(T, -1, D)
        parts = []
        for h0, h1, w in ((0, self.Hq, self.w[0]), (self.Hq, self.Hq + self.Hkv, self.w[1])):
            n, off = ref.norm("rms", y[:, h0:h1], w.double(), None, 1e-6)
            parts.append(ref.rotate(n, off, position, self.freq, D, "halves")[0])
        return (*parts, y[:, self.Hq + self.Hkv:])


def test_prompts_then_tokens(nq):
    """Two prompts through heads, cache and prompt attention, then tokens one at a time through heads, cache and token attention: every output
    against attention in 64 bits over what the caches hold."""
    lengths, more = [37, 150], 4
    L = Layer(nq, sum(lengths), 2, 200)
    D, Hq, Hkv = L.D, L.Hq, L.Hkv
    x = randn(5, sum(lengths), L.width).to(BF16)
    position = torch.cat([torch.arange(n) for n in lengths])
    n = L.put(x, position, torch.cat([L.slots(i, 0, m) for i, m in enumerate(lengths)]))
    nq.nq_head_norm(L.heads, n)
    begin = begins(lengths).cuda()
    nq.nq_attention_prompt(nq.make_attention_prompt(L.q, Hq * D, L.k, Hkv * D, L.v, L.width, L.o, Hq * D, begin, None, 2, n, n, dt(nq, BF16), Hq, Hkv, D, True, D ** -0.5))
    q, k, v = L.of_the_inputs(x, position)
    # (queries and keys are rounded to bf16 on their way: the oracle takes the rounded ones)
    check_prompt(L.o.cpu(), L.q.cpu(), L.k.cpu(), x[:, (Hq + Hkv) * D:], begins(lengths), None, Hq, Hkv, D, BF16, True, D ** -0.5)
    assert (L.q.cpu().double().view(n, Hq, D) - q).abs().max() <= 2 ** -7 * q.abs().max()
    need = nq.nq_attention_token_workspace_bytes(2, Hq, Hkv, D, L.longest)
    workspace = torch.empty(need, dtype=torch.uint8, device="cuda")
    length = torch.zeros(2, dtype=torch.int32, device="cuda")
    job = nq.make_attention_token(L.q[:2], Hq * D, L.o[:2], Hq * D, L.cache.desc, L.d_table, length, 2, L.longest, dt(nq, BF16), Hq, D ** -0.5, workspace)
    for step in range(more):
        now = torch.tensor([m + step for m in lengths])
        y = randn(50 + step, 2, L.width).to(BF16)
        L.put(y, now.to(torch.int32), torch.cat([L.slots(i, int(now[i]), 1) for i in range(2)]))
        nq.nq_head_norm(L.heads, 2)
        length.copy_(now + 1)
        nq.nq_attention_token(job)
        got = L.o[:2].cpu()
        kept = [values_of(t, s) for t, s in ((L.cache.k, L.cache.k_scale), (L.cache.v, L.cache.v_scale))]
        for i in range(2):
            s = L.slots(i, 0, int(now[i]) + 1)
            kk, vv = (c[s // L.page, s % L.page] for c in kept)
            for h in range(Hq):
                o, bound = ref.attention(L.q[i:i + 1, h * D:(h + 1) * D].cpu().double(), kk[:, h // (Hq // Hkv)], vv[:, h // (Hq // Hkv)], D ** -0.5,
                                         torch.ones(1, len(s), dtype=torch.bool), BF16, False)
                ref.check(got[i:i + 1, h * D:(h + 1) * D], o, bound, f"step {step} sequence {i} head {h}")


def test_a_prompt_behind_its_cached_prefix(nq):
    """A second prompt of a conversation: the cached keys and values back as floats, its own behind them, and attention over both."""
    D, Hkv, Hq, prefix, own = 64, 2, 4, 75, 40
    k, v, ks, vs, cache = pool(nq, 8, 16, Hkv, D, E4M3, "head", poison=False)
    none = nq.make_norm(nq.NQ_NORM_NONE)
    x = randn(7, prefix, 2 * Hkv * D).to(F16).cuda()
    slot = torch.randperm(128, generator=torch.Generator().manual_seed(3))[:prefix].cuda()
    half = Hkv * D
    nq.nq_head_norm(nq.make_head_norm(None, 0, x, 2 * half, x[:, half:], 2 * half, nq.NQ_DT_F16, Hkv, Hkv, D, none, none, None, 0, 0, None, None, 0, None, 0, cache, slot), prefix)
    keys, values = (torch.zeros(prefix + own, half, dtype=F16, device="cuda") for _ in range(2))
    nq.nq_cache_read(cache, slot, prefix, keys, half, values, half, nq.NQ_DT_F16)
    keys[prefix:], values[prefix:] = randn(8, own, half).to(F16), randn(9, own, half).to(F16)
    back = values_of(k, ks).reshape(-1, Hkv, D)[slot.cpu()].reshape(prefix, half)
    assert torch.equal(keys[:prefix].cpu(), back.float().to(F16))
    q = (randn(10, own, Hq * D) * 2).to(F16)
    out, _ = run_prompt(nq, q, keys.cpu(), values.cpu(), begins([own]), begins([prefix + own]), 1, Hq, Hkv, D, F16, True, 0.125)
    check_prompt(out.cpu(), q, keys.cpu(), values.cpu(), begins([own]), begins([prefix + own]), Hq, Hkv, D, F16, True, 0.125)


def test_between_the_fp8_layers(nq):
    """One token's whole attention block: fp8 projection, heads, cache, attention, codes, fp8 projection back; each stage takes what the last left on
    the device, and the block's output is the 64-bit product of the attention's."""
    Hq, Hkv, D, width = 4, 2, 64, 256
    L = Layer(nq, 3, 3, 64, Hq, Hkv, D)
    x = randn(20, 3, width).to(BF16).cuda()
    up, down = (nq.Fp8Matrix.from_float((randn(21 + i, *s) * 0.1).to(BF16).cuda()) for i, s in enumerate(((L.width, width), (width, Hq * D))))
    codes, back = nq.Fp8Matrix.from_float(x, 1), nq.Fp8Matrix(3, Hq * D)
    y = torch.empty(3, width, device="cuda")
    nq.nq_gemm_fp8(codes.desc, up.desc, None, L.qkv, nq.NQ_DT_BF16, L.width)
    L.position.copy_(torch.arange(3, dtype=torch.int32))
    L.slot.copy_(torch.cat([L.slots(i, 0, 1) for i in range(3)]))
    nq.nq_head_norm(L.heads, 3)
    length = torch.ones(3, dtype=torch.int32, device="cuda")
    nq.nq_attention_token(nq.make_attention_token(L.q, Hq * D, L.o, Hq * D, L.cache.desc, L.d_table, length, 3, 64, nq.NQ_DT_BF16, Hq, 0.125,
                                                  torch.empty(nq.nq_attention_token_workspace_bytes(3, Hq, Hkv, D, 64), dtype=torch.uint8, device="cuda")))
    nq.nq_quantize_fp8(L.o, nq.NQ_DT_BF16, Hq * D, None, 0, nq.NQ_ACT_NONE, back.desc)
    nq.nq_gemm_fp8(back.desc, down.desc, None, y, nq.NQ_DT_F32, width)
    # a token that sees only itself gets its own value, as the cache holds it
    kept = values_of(L.cache.v, L.cache.v_scale)
    s = torch.cat([L.slots(i, 0, 1) for i in range(3)])
    own = kept[s // L.page, s % L.page].repeat_interleave(Hq // Hkv, 1).reshape(3, Hq * D)
    assert torch.equal(L.o.cpu(), own.float().to(BF16))
    spread = lambda m, rows: m.q.view(E4M3)[:, :m.cols].cpu().double() * m.scale.cpu().double().t().repeat_interleave(128, 1)[:, :m.cols].repeat_interleave(rows, 0)[:m.rows]  # noqa: E731
    a, b = spread(back, 1), spread(down, 128)
    want = a @ b.t()
    bound = (a.abs() @ b.abs().t()) * 300 * ref.U
    assert ((y.cpu().double() - want).abs() <= bound).all()


def test_captured_and_replayed(nq):
    """Heads, cache, prompt, rows back and token attention in one graph, replayed on new inputs, lengths, tables and slots, with eager work and
    synchronisations between: each replay gives the bits of the eager calls."""
    L = Layer(nq, 6, 3, 3000, Hq=4, Hkv=2, D=64)
    Hq, Hkv, D = 4, 2, 64
    for t in (L.cache.k, L.cache.v):
        t.view(torch.uint8).copy_((randn(1, *t.shape) * 50).to(E4M3).view(torch.uint8))
    for t in (L.cache.k_scale, L.cache.v_scale):
        t.copy_(randn(2, *t.shape).abs() * 0.02)
    begin, length = torch.tensor([0, 2, 6], dtype=torch.int32).cuda(), torch.tensor([5, 2999, 700], dtype=torch.int32).cuda()
    op, back_k, back_v = torch.zeros_like(L.o), torch.zeros(6, Hkv * D, device="cuda"), torch.zeros(6, Hkv * D, device="cuda")
    need = nq.nq_attention_token_workspace_bytes(3, Hq, Hkv, D, 3000)
    assert need > 0
    workspace = torch.empty(need, dtype=torch.uint8, device="cuda")
    prompt = nq.make_attention_prompt(L.q, Hq * D, L.k, Hkv * D, L.v, L.width, op, Hq * D, begin, None, 2, 6, 6, nq.NQ_DT_BF16, Hq, Hkv, D, True, 0.1)
    token = nq.make_attention_token(L.q[:3], Hq * D, L.o[:3], Hq * D, L.cache.desc, L.d_table, length, 3, 3000, nq.NQ_DT_BF16, Hq, 0.125, workspace)

    def calls():
        nq.nq_head_norm(L.heads, 6)
        nq.nq_attention_prompt(prompt)
        nq.nq_cache_read(L.cache.desc, L.slot, 6, back_k, Hkv * D, back_v, Hkv * D, nq.NQ_DT_F32)
        nq.nq_attention_token(token)

    L.put(randn(3, 6, L.width).to(BF16), torch.arange(6, dtype=torch.int32), torch.arange(6))
    calls()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        calls()
    outs = (L.q, L.k, op, back_k, back_v, L.o)
    for i in range(5):
        L.put(randn(30 + i, 6, L.width).to(BF16), torch.arange(6, dtype=torch.int32) * 1000 * i, torch.randperm(500, generator=torch.Generator().manual_seed(i))[:6] - int(i == 2))
        length.copy_(torch.tensor([[5, 2999, 700], [0, 1, 3000], [3000, 3000, 3000], [31, 129, 2], [0, 0, 0]][i], dtype=torch.int32))
        begin.copy_(torch.tensor([[0, 2, 6], [0, 6, 6], [0, 0, 5], [1, 3, 6], [0, 3, 6]][i], dtype=torch.int32))
        L.d_table.copy_(L.table.roll(i, 0))
        op.zero_()
        graph.replay()
        torch.cuda.synchronize()
        got = [t.clone() for t in outs]
        workspace.fill_(0xff)
        op.zero_()
        calls()
        torch.cuda.synchronize()
        for a, b in zip(got, outs):
            assert torch.equal(a, b), i


def test_streams(nq):
    """Calls on streams of their own at the same time, each with its workspace, give the bits of the same calls one after the other; a stream as an
    object and as a raw handle."""
    cases = [TokenCase(nq, [2000 + 100 * i, 30 * i, 900], None, 8, 2, 128, BF16, c, 16, "head", seed=200 + i) for i, c in enumerate((E4M3, BF16, E4M3))]
    jobs = [c.job() for c in cases]
    keep = [(c.out, c.workspace, c.d_table, c.d_length) for c in cases]
    want = []
    for job, (out, *_) in zip(jobs, keep):
        nq.nq_attention_token(job)
        torch.cuda.synchronize()
        want.append(out.clone())
    streams = [torch.cuda.Stream() for _ in jobs]
    for _ in range(5):
        for out, *_ in keep:
            out.fill_(3.0)
        for s in streams:
            s.wait_stream(torch.cuda.current_stream())
        for i, (job, s) in enumerate(zip(jobs, streams)):
            nq.nq_attention_token(job, s if i % 2 else s.cuda_stream)
        torch.cuda.synchronize()
        for (out, *_), w in zip(keep, want):
            assert torch.equal(out, w)
    q, k, v = (randn(300 + i, 200, 256).to(F16) for i in range(3))
    alone, job = run_prompt(nq, q, k, v, begins([200]), None, 1, 4, 4, 64, F16, True, 0.1)
    first = alone.clone()
    alone.fill_(0)
    streams[0].wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(streams[0]):
        nq.nq_attention_prompt(job)
    streams[0].synchronize()
    assert torch.equal(alone, first)


def test_bad_begins_are_cut_off(nq):
    """Begins outside the rows: what lies inside is right, nothing outside is read or written."""
    q, k, v = (randn(400 + i, 100, 128).to(BF16) for i in range(3))
    out, _ = run_prompt(nq, q, k, v, torch.tensor([-7, 50, 1000000000], dtype=torch.int32), torch.tensor([-2 ** 31, 50, 2 ** 31 - 1], dtype=torch.int32), 2, 2, 2, 64, BF16, True, 0.1)
    check_prompt(out.cpu(), q, k, v, torch.tensor([0, 50, 100]), None, 2, 2, 64, BF16, True, 0.1)
    out, _ = run_prompt(nq, q, k, v, torch.tensor([60, 20, 90], dtype=torch.int32), None, 2, 2, 2, 64, BF16, True, 0.1)
    got = out.cpu()
    assert (got[:20] == 5).all() and (got[90:] == 5).all()


@pytest.mark.parametrize("cached", [F16, BF16, E4M3])
def test_a_cache_on_any_byte(nq, cached):
    """Steps and first elements that are no multiple of 16 bytes, scales all over the place; written, read back and attended over."""
    H, D, page, pages, n = 2, 64, 5, 9, 43
    step, es = H * (D + 3) + 1, 1 if cached == E4M3 else 2
    raw = [torch.zeros(pages * page * step + 8, dtype=torch.uint8 if es == 1 else cached, device="cuda") for _ in range(2)]
    views = [torch.as_strided(t, (pages, page, H, D), (page * step, step, D + 3, 1), 3) for t in raw]
    scales = [torch.zeros(pages * page * H * 3 + 2, device="cuda") for _ in range(2)] if cached == E4M3 else [None, None]
    sviews = [torch.as_strided(t, (pages, page, H), (3 * page * H, 3, 3 * page), 1) if t is not None else None for t in scales]
    cache = nq.make_kv_cache(*views, *sviews)
    dtype = F16 if cached == F16 else BF16
    x = randn(9, n, 2 * H * D).to(dtype).cuda()
    none = nq.make_norm(nq.NQ_NORM_NONE)
    table = torch.randperm(pages, generator=torch.Generator().manual_seed(4)).to(torch.int32)
    at = torch.arange(n)
    slot = (table[at // page].long() * page + at % page).cuda()
    nq.nq_head_norm(nq.make_head_norm(None, 0, x, 2 * H * D, x[:, H * D:], 2 * H * D, dt(nq, dtype), H, H, D, none, none, None, 0, 0, None, None, 0, None, 0, cache, slot), n)
    back = [torch.zeros(n, H * D, device="cuda") for _ in range(2)]
    nq.nq_cache_read(cache, slot, n, back[0], H * D, back[1], H * D, nq.NQ_DT_F32)
    for b, y in zip(back, (x[:, :H * D], x[:, H * D:])):
        y = y.double().cpu().view(n, H, D)
        bound = ref.codes_bound(y, torch.zeros_like(y)) if cached == E4M3 else y.abs() * ref.half_step(cached)
        ref.check(b.view(n, H, D), y, bound + 1e-30)
    q = randn(10, 1, 4 * D).to(dtype)
    out = torch.zeros(1, 4 * D, dtype=dtype, device="cuda")
    length = torch.tensor([n], dtype=torch.int32).cuda()
    nq.nq_attention_token(nq.make_attention_token(q.cuda(), 4 * D, out, 4 * D, cache, table[None].cuda(), length, 1, n, dt(nq, dtype), 4, -0.3))
    k, v = (b.cpu().double().view(n, H, D) for b in back)
    for h in range(4):
        o, bound = ref.attention(q[:, h * D:(h + 1) * D].double(), k[:, h // 2], v[:, h // 2], -0.3, torch.ones(1, n, dtype=torch.bool), dtype, False)
        ref.check(out[:, h * D:(h + 1) * D].cpu(), o, bound)
    for t in raw:                                  # between the heads, and before the first: nobody's
        assert (t[:3] == 0).all() and (torch.as_strided(t, (pages * page, H - 1, 3), (step, D + 3, 1), 3 + D) == 0).all()


@pytest.mark.parametrize("cached", [BF16, E4M3])
def test_one_long_sequence_among_many(nq, cached):
    """More sequences than the card needs to be full, one of them long, so that it is split all the same; some empty."""
    lengths = [(i * 37) % 150 for i in range(200)]
    lengths[70], lengths[199] = 9000, 1500
    case = TokenCase(nq, lengths, None, 6, 6, 16, BF16, cached, 16, "head", seed=77)
    job = case.job()
    assert job.workspace_bytes > 0
    nq.nq_attention_token(job)
    case.check(case.out.cpu())


def test_more_threads_than_32_bits_count(nq):
    """65535 sequences of 512 key heads: 2^33 threads in one launch.  A sequence of one token gets that token's value, an empty one zeros."""
    S, H, D = 65535, 512, 8
    k, v = (randn(40 + i, 3, 1, H, D).to(F16).cuda() for i in range(2))
    table = (torch.arange(S, dtype=torch.int32, device="cuda") % 3)[:, None].contiguous()
    length = (torch.arange(S, device="cuda") % 2).to(torch.int32)
    q = torch.ones(S, H * D, dtype=F16, device="cuda")
    o = torch.full((S, H * D), 7.0, dtype=F16, device="cuda")
    nq.nq_attention_token(nq.make_attention_token(q, H * D, o, H * D, nq.make_kv_cache(k, v), table, length, S, 1, nq.NQ_DT_F16, H, 0.3))
    for i in range(3):
        want = v[i].reshape(1, H * D)
        mine = o[i::3]
        there = length[i::3, None] > 0
        assert torch.equal(mine, torch.where(there, want, torch.zeros_like(want)))


@pytest.mark.parametrize("cached", [BF16, E4M3])
def test_a_cache_past_32_bits(nq, cached):
    """Two pages 2^32 elements apart, heads and tokens far apart within them."""
    H, D, page, n, dtype = 2, 64, 32, 60, BF16
    step, head = (1 << 32) + 64, 1 << 24
    size = step + head + page * D
    raw = [torch.empty(size, dtype=torch.uint8 if cached == E4M3 else cached, device="cuda") for _ in range(2)]
    views = [torch.as_strided(t, (2, page, H, D), (step, D, head, 1)) for t in raw]
    scales = [torch.ones(2, page, H, device="cuda") for _ in range(2)] if cached == E4M3 else [None, None]
    cache = nq.make_kv_cache(*views, *scales)
    x = randn(9, n, 2 * H * D).to(dtype).cuda()
    none = nq.make_norm(nq.NQ_NORM_NONE)
    at = torch.arange(n)
    slot = ((1 - at // page) * page + at % page).cuda()                # the second page first
    nq.nq_head_norm(nq.make_head_norm(None, 0, x, 2 * H * D, x[:, H * D:], 2 * H * D, dt(nq, dtype), H, H, D, none, none, None, 0, 0, None, None, 0, None, 0, cache, slot), n)
    back = [torch.zeros(n, H * D, device="cuda") for _ in range(2)]
    nq.nq_cache_read(cache, slot, n, back[0], H * D, back[1], H * D, nq.NQ_DT_F32)
    for b, y in zip(back, (x[:, :H * D], x[:, H * D:])):
        y = y.double().cpu().view(n, H, D)
        bound = ref.codes_bound(y, torch.zeros_like(y)) if cached == E4M3 else torch.zeros_like(y)
        ref.check(b.view(n, H, D), y, bound)
    q = randn(10, 1, 4 * D).to(dtype)
    out = torch.zeros(1, 4 * D, dtype=dtype, device="cuda")
    table, length = torch.tensor([[1, 0]], dtype=torch.int32).cuda(), torch.tensor([n], dtype=torch.int32).cuda()
    nq.nq_attention_token(nq.make_attention_token(q.cuda(), 4 * D, out, 4 * D, cache, table, length, 1, n, dt(nq, dtype), 4, 0.2))
    k, v = (b.cpu().double().view(n, H, D) for b in back)
    for h in range(4):
        o, bound = ref.attention(q[:, h * D:(h + 1) * D].double(), k[:, h // 2], v[:, h // 2], 0.2, torch.ones(1, n, dtype=torch.bool), dtype, False)
        ref.check(out[:, h * D:(h + 1) * D].cpu(), o, bound)


@pytest.mark.parametrize("ld,rows", [(1 << 22, 1100), ((1 << 24) + 8, 290)])
def test_prompt_rows_past_32_bits(nq, ld, rows):
    """Rows whose offsets pass 2^32 elements, below and above the step up to which tiles travel by direct loads."""
    H, D = 2, 64
    width = H * D
    store, to = (torch.empty((rows - 1) * ld + 3 * width, dtype=BF16, device="cuda") for _ in range(2))
    assert (rows - 1) * ld > 1 << 32
    parts = [torch.as_strided(store, (rows, width), (ld, 1), i * width) for i in range(3)]
    host = [randn(60 + i, rows, width).to(BF16) for i in range(3)]
    for p, x in zip(parts, host):
        p.copy_(x)
    out = torch.as_strided(to, (rows, width), (ld, 1))
    lengths = [rows - 150, 150]
    begin = begins(lengths).cuda()
    nq.nq_attention_prompt(nq.make_attention_prompt(parts[0], ld, parts[1], ld, parts[2], ld, out, ld, begin, None, 2, rows, rows, nq.NQ_DT_BF16, H, H, D, True, 0.125))
    check_prompt(out.cpu(), *host, begins(lengths), None, H, H, D, BF16, True, 0.125)


SHORT = [
    # lengths, keys, Hq, Hkv, D, dtype, causal, scale, gap
    ([1 + 5 * i % 40 for i in range(50)], None, 12, 3, 128, BF16, True, 0.1, 0),
    ([i % 23 for i in range(300)], None, 4, 4, 64, F16, True, 0.15, 0),
    ([5 * i % 37 for i in range(90)], [7 * i % 150 for i in range(90)], 8, 2, 96, BF16, True, -0.1, 0),
    ([33 + i % 31 for i in range(20)], None, 8, 2, 128, F16, False, 0.1, 0),
    ([200] + [3] * 60, [200] + [100] * 60, 9, 3, 72, F16, False, 0.1, 4),
    ([2, 17, 0, 30], [90, 17, 8, 31], 2, 1, 128, F16, True, 0.1, 3),
    ([1 + 7 * i % 33 for i in range(30)], [40 + i for i in range(30)], 10, 5, 192, BF16, True, 0.08, 0),
    ([1 + 7 * i % 33 for i in range(70)], None, 4, 1, 256, F16, True, 0.08, 0),
    ([1 + 7 * i % 33 for i in range(70)], None, 4, 1, 256, BF16, False, 0.0, 4),
]


@pytest.mark.parametrize("case", SHORT, ids=lambda c: f"{len(c[0])}-{c[2]}-{c[3]}-{c[4]}-{c[8]}")
def test_many_short_prompts(nq, case):
    """Sequences of a few rows, some of more than a tile, some over more keys than a step; rows of no sequence in front and behind."""
    lengths, keys, Hq, Hkv, D, dtype, causal, scale, gap = case
    q_begin, k_begin = begins(lengths, 3), begins(keys) if keys else None
    T = int(q_begin[-1]) + 40
    K = int(k_begin[-1]) if keys else T
    q, k, v = (randn(160 + i, *s).to(dtype) for i, s in enumerate(((T, Hq * D), (K, Hkv * D), (K, Hkv * D))))
    out, _ = run_prompt(nq, q, k, v, q_begin, k_begin, len(lengths), Hq, Hkv, D, dtype, causal, scale, gap)
    got = out.cpu()
    check_prompt(got, q, k, v, q_begin, k_begin, Hq, Hkv, D, dtype, causal, scale)
    assert (got[:3] == 5).all() and (got[int(q_begin[-1]):] == 5).all(), "rows of no sequence have changed"


@pytest.mark.parametrize("D,gap", [(64, 0), (128, 0), (256, 0), (72, 4)])
def test_short_prompts_with_values_that_are_not_finite(nq, D, gap):
    """As for long ones: what a row does not see does not reach it."""
    n, S, H = 24, 60, 6
    q, k, v = (randn(170 + i, n, D) for i in range(3))
    v[7, 5], v[9, 6], v[11, 7] = float("inf"), -float("inf"), float("nan")
    v[20] = float("nan")
    k[15, 0] = float("nan")
    q, k, v = (x.to(BF16) for x in (q, k, v))
    many = lambda x, h: x.repeat(S, h)  # noqa: E731
    got = run_prompt(nq, many(q, H), many(k, 1), many(v, 1), begins([n] * S), None, S, H, 1, D, BF16, True, 0.1, gap)[0].cpu()
    for s, h in ((0, 0), (33, 2), (S - 1, H - 1)):
        part = got[s * n:(s + 1) * n, h * D:(h + 1) * D]
        check_prompt(part[:15], q[:15], k[:15], v[:15], begins([15]), None, 1, 1, D, BF16, True, 0.1)
        assert torch.isnan(part[15:]).all()


DEALT = [
    # rows, keys, Hq, Hkv, D, dtype, causal, scale
    ([16], [4016], 32, 8, 128, BF16, True, 0.1),
    ([1], [9000], 2, 1, 64, F16, True, 0.2),
    ([40, 0, 30], [2000, 1500, 3000], 4, 2, 96, BF16, True, -0.1),
    ([100], [5000], 6, 2, 72, F16, False, 0.1),
    ([300], [4100], 4, 1, 128, BF16, True, 0.1),
    ([129, 50], [3000, 20], 2, 2, 64, F16, True, 0.1),
    ([70], [2048], 2, 1, 256, BF16, True, 0.08),
    ([20, 9, 60], [1500, 1600, 0], 2, 2, 192, F16, False, 0.08),
    ([700], [700], 1, 1, 80, BF16, True, 0.1),
    ([1100], [1100], 2, 1, 128, F16, True, 0.0),
    ([1500], [1500], 1, 1, 80, BF16, True, 0.1),
]


def run_dealt(nq, q, k, v, q_begin, k_begin, Hq, Hkv, D, dtype, causal, scale):
    S, T, K = len(q_begin) - 1, q.shape[0], k.shape[0]
    need = nq.nq_attention_prompt_workspace_bytes(S, T, K, Hq, Hkv, D)
    assert need > 0 or K < 1024 * S, "not split"                # (fewer keys than two pieces have: one workgroup all the same)
    workspace = torch.full((need + 64,), 0xff, dtype=torch.uint8, device="cuda")         # (NaN, wherever it is read before it is written)
    out = torch.full((T, Hq * D), 5.0, dtype=dtype, device="cuda")
    job = nq.make_attention_prompt(q.cuda(), Hq * D, k.cuda(), Hkv * D, v.cuda(), Hkv * D, out, Hq * D, q_begin.cuda(), k_begin.cuda(), S, T, K,
                                   dt(nq, dtype), Hq, Hkv, D, causal, scale, workspace[:need])
    nq.nq_attention_prompt(job)
    got = out.cpu()
    assert (workspace[need:] == 0xff).all()
    nq.nq_attention_prompt(job)
    assert torch.equal(out.cpu().view(torch.int16), got.view(torch.int16)), "equal calls differ"
    return got


@pytest.mark.parametrize("case", DEALT, ids=lambda c: f"{c[0]}-{c[1]}-{c[2]}-{c[3]}-{c[4]}".replace(" ", ""))
def test_keys_dealt_to_workgroups(nq, case):
    rows, keys, Hq, Hkv, D, dtype, causal, scale = case
    q_begin, k_begin = begins(rows, 2), begins(keys, 1)
    T, K = int(q_begin[-1]) + 3, int(k_begin[-1]) + 1
    q, k, v = (randn(180 + i, *s).to(dtype) for i, s in enumerate(((T, Hq * D), (K, Hkv * D), (K, Hkv * D))))
    got = run_dealt(nq, q, k, v, q_begin, k_begin, Hq, Hkv, D, dtype, causal, scale)
    check_prompt(got, q, k, v, q_begin, k_begin, Hq, Hkv, D, dtype, causal, scale)
    assert (got[:2] == 5).all() and (got[T - 3:] == 5).all(), "rows of no sequence have changed"


@pytest.mark.parametrize("n,D", [(150, 64), (30, 128), (150, 128), (150, 256)])
def test_keys_dealt_with_values_that_are_not_finite(nq, n, D):
    """What a row does not see does not reach it, in whichever piece it lies."""
    K, H = 2300, 2
    q, k, v = (randn(190 + i, m, D) for i, m in enumerate((n, K, K)))
    a = K - n                                                  # row i sees the keys up to a + i
    v[a + 7, 5], v[a + 9, 6], v[a + 11, 7] = float("inf"), -float("inf"), float("nan")
    v[a + 20] = float("nan")
    k[a + 15, 0] = float("nan")
    q, k, v = (x.to(BF16) for x in (q, k, v))
    got = run_dealt(nq, q.repeat(1, H), k, v, begins([n]), begins([K]), H, 1, D, BF16, True, 0.1)
    for h in range(H):
        part = got[:, h * D:(h + 1) * D]
        check_prompt(part[:15], q[:15], k[:a + 15], v[:a + 15], begins([15]), begins([a + 15]), 1, 1, D, BF16, True, 0.1)
        assert torch.isnan(part[15:]).all()


def test_keys_dealt_scores_of_no_weight(nq):
    """Pieces whose every score is -inf weigh nothing beside others; without others the row is NaN, and 0 where it sees no key at all."""
    D, K = 64, 2500
    q, k, v = torch.ones(40, D), randn(200, K, D) * 0.1, randn(201, K, D)
    k[:1800, 0] = -float("inf")
    q, k, v = (x.to(BF16) for x in (q, k, v))
    got = run_dealt(nq, q, k, v, begins([20, 20]), torch.tensor([0, 1500, 2500], dtype=torch.int32), 1, 1, D, BF16, False, 0.1)
    assert torch.isnan(got[:20]).all()
    o, bound = ref.attention(q[20:].double(), k[1800:].double(), v[1800:].double(), 0.1, torch.ones(20, 700, dtype=torch.bool), BF16, True)
    ref.check(got[20:], o, bound)
    got = run_dealt(nq, q, k[1800:].repeat(5, 1), v[1800:].repeat(5, 1), begins([39, 1]), torch.tensor([0, 0, 3000], dtype=torch.int32), 1, 1, D, BF16, False, 0.1)
    assert (got[:39] == 0).all() and torch.isfinite(got[39]).all()


def test_keys_dealt_captured(nq):
    """A split call in a graph, replayed on other lengths with eager work on the same workspace between: each replay gives the bits of the eager call."""
    H, D, T, K = 4, 128, 60, 4000
    q, k, v = (randn(210 + i, n, H * D).to(BF16).cuda() for i, n in enumerate((T, K, K)))
    out = torch.zeros(T, H * D, dtype=BF16, device="cuda")
    q_begin, k_begin = (torch.tensor(x, dtype=torch.int32, device="cuda") for x in ([0, 20, 60], [0, 1000, 4000]))
    workspace = torch.empty(nq.nq_attention_prompt_workspace_bytes(2, T, K, H, H, D), dtype=torch.uint8, device="cuda")
    assert workspace.numel() > 0
    job = nq.make_attention_prompt(q, H * D, k, H * D, v, H * D, out, H * D, q_begin, k_begin, 2, T, K, nq.NQ_DT_BF16, H, H, D, True, 0.1, workspace)
    nq.nq_attention_prompt(job)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        nq.nq_attention_prompt(job)
    for a, b in (([0, 20, 60], [0, 1000, 4000]), ([0, 0, 60], [0, 3000, 3500]), ([5, 50, 55], [0, 10, 4000]), ([0, 60, 60], [0, 4000, 4000])):
        q_begin.copy_(torch.tensor(a, dtype=torch.int32))
        k_begin.copy_(torch.tensor(b, dtype=torch.int32))
        out.fill_(9.0)
        graph.replay()
        torch.cuda.synchronize()
        got = out.clone()
        workspace.fill_(0xff)
        out.fill_(9.0)
        nq.nq_attention_prompt(job)
        torch.cuda.synchronize()
        assert torch.equal(out, got), (a, b)
        check_prompt(got.cpu(), q.cpu(), k.cpu(), v.cpu(), torch.tensor(a), torch.tensor(b), H, H, D, BF16, True, 0.1)
