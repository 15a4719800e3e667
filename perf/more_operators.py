"""The timed cases of the attention operators: what a program that serves transformers has them do, from one token to a long prompt.

    heads   norms of the queries' and the keys' heads, position rotation, keys and values into a paged cache
    read    rows of such a cache back as floats
    prompt  attention over whole prompts: packed sequences of different lengths, grouped heads, causal or not, keys ahead of the queries
    token   attention of one new token for each sequence over the paged cache

    listed()             the cases, each a dict of plain values with a name
    draw(rng)            one more case from the same ranges
    prepare(case, seed)  what the program holds before the call
    run(state)           one pass; the operators in their plain form, or, with `own`, this library's
    exact(case, seed)    the same outputs from the definition, in 64 bits
    work(case)           bytes and operations the pass cannot do without

A cache holds pages of `page` tokens; slot = page number * page + place in the page.  In e4m3 (1 sign, 4 exponent and 3 mantissa bits, largest
value 448) each head of a token has the scale s = max(a / 448, 2^-126) of its largest magnitude a (1 if a is 0) and the codes
e4m3(v * (1 / s)), rounded to nearest even.
"""
from __future__ import annotations

import math
import random

import torch

own = False

DTYPES = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16, "e4m3": torch.float8_e4m3fn}
BYTES = {"f32": 4, "f16": 2, "bf16": 2, "e4m3": 1}
EPS = 1e-6


def _heads(T, Hq=32, Hkv=8, D=128, dtype="bf16", norm="rms", rotary=None, pairs="halves", cache="e4m3", page=16, order="head", far=8192):
    return dict(kind="heads", T=T, Hq=Hq, Hkv=Hkv, D=D, dtype=dtype, norm=norm, rotary=D if rotary is None else rotary, pairs=pairs,
                cache=cache, page=page, order=order, far=far)


def _read(T, Hkv=8, D=128, dtype="bf16", cache="e4m3", page=16, order="head"):
    return dict(kind="read", T=T, Hkv=Hkv, D=D, dtype=dtype, cache=cache, page=page, order=order)


def _prompt(S, longest, Hq=32, Hkv=8, D=128, dtype="bf16", causal=True, ragged=False, prefix=0):
    return dict(kind="prompt", S=S, longest=longest, Hq=Hq, Hkv=Hkv, D=D, dtype=dtype, causal=causal, ragged=ragged, prefix=prefix)


def _token(S, longest, Hq=32, Hkv=8, D=128, dtype="bf16", cache="e4m3", page=16, order="head", ragged=True):
    return dict(kind="token", S=S, longest=longest, Hq=Hq, Hkv=Hkv, D=D, dtype=dtype, cache=cache, page=page, order=order, ragged=ragged)


def listed():
    return [
        # one new token between the projections and the attention: latency counts
        dict(_heads(1), name="heads_1"),
        # a prompt of an odd length, heads as wide as no tile, half of each rotated by neighbours, layer norms, floats in the cache
        dict(_heads(1009, 12, 12, 80, dtype="f16", norm="layer", rotary=40, pairs="neighbours", cache="f16", page=24, order="token"), name="heads_odd_1009"),
        # a long prompt
        dict(_heads(16384, far=131072), name="heads_16384"),
        # a short cached prefix ahead of a prompt
        dict(_read(45, 12, 64, dtype="f16", cache="f16"), name="read_45"),
        # the caches of some thousand-token conversations, each about to get another prompt
        dict(_read(32768), name="read_32768"),
        # one short question
        dict(_prompt(1, 33), name="prompt_33"),
        # the tokens of eight images, all of which see each other
        dict(_prompt(8, 197, 12, 12, 64, dtype="f16", causal=False), name="prompt_images_8x197"),
        # prompts of different lengths packed behind each other, part of them after a cached prefix
        dict(_prompt(24, 1500, ragged=True, prefix=700), name="prompt_packed_24"),
        # one long prompt
        dict(_prompt(1, 8192), name="prompt_8192"),
        # one conversation's next token
        dict(_token(1, 517), name="token_1x517"),
        # the next tokens of a batch of conversations of all lengths
        dict(_token(96, 4096), name="token_96x4096"),
        # a few very long ones, a cache of floats
        dict(_token(4, 65536, cache="bf16", page=64, ragged=False), name="token_4x65536"),
    ]


# ---- more cases of the same ranges ---------------------------------------------------------------------------

MOST = {"heads": 16384 * 48 * 128, "read": 32768 * 8 * 128, "prompt": 0.5 * 8192 * 8192 * 32 * 128, "token": 4 * 65536 * 8 * 128}


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["heads", "read", "prompt", "prompt", "token", "token"])
    while True:
        Hkv, group = rng.choice([1, 2, 4, 8, 8, 12, 16]), rng.choice([1, 1, 2, 4, 4, 6, 8, 16])
        D, dtype = rng.choice([64, 64, 72, 80, 96, 128, 128, 128, 192, 256]), rng.choice(["bf16", "bf16", "f16"])
        page, order = rng.choice([1, 16, 16, 24, 32, 64, 100, 128, 256]), rng.choice(["head", "head", "token"])
        if Hkv * group > 64:
            continue
        cache = rng.choice(["e4m3", "e4m3", dtype])
        if kind == "heads":
            c = _heads(_log(rng, 1, 16384), Hkv * group, Hkv, D, rng.choice([dtype, dtype, "f32"]), rng.choice(["rms", "rms", "layer", "none"]),
                       rng.choice([D, D, D // 2, 0]), rng.choice(["halves", "halves", "neighbours"]), cache, page, order, _log(rng, 16384, 1000000))
            cost = c["T"] * (c["Hq"] + 2 * c["Hkv"]) * D
        elif kind == "read":
            c = _read(_log(rng, 1, 32768), Hkv, D, rng.choice([dtype, dtype, "f32"]), cache, page, order)
            cost = c["T"] * Hkv * D
        elif kind == "prompt":
            c = _prompt(_log(rng, 1, 64), _log(rng, 1, 8192), Hkv * group, Hkv, D, dtype, rng.random() < 0.8, rng.random() < 0.7,
                        rng.choice([0, 0, _log(rng, 1, 4096)]))
            Lq, Lk = c["longest"], c["longest"] + c["prefix"]
            cost = c["S"] * Lq * Lk * c["Hq"] * D * (0.5 if c["causal"] and not c["prefix"] else 1.0)
        else:
            c = _token(_log(rng, 1, 256), _log(rng, 1, 65536), Hkv * group, Hkv, D, dtype, cache, page, order, rng.random() < 0.7)
            cost = c["S"] * c["longest"] * Hkv * D
        if cost <= MOST[kind]:
            return c


def _lengths(case, least=1):
    """How long each sequence is: all alike, or spread over the logarithm, the longest of them at a place of its own."""
    if not case.get("ragged"):
        return [case["longest"]] * case["S"]
    rng = random.Random(case["S"] * 70001 + case["longest"])
    got = [_log(rng, max(least, case["longest"] / 64), case["longest"]) for _ in range(case["S"])]
    got[rng.randrange(case["S"])] = case["longest"]
    return got


def _prefixes(case):
    """Keys that come ahead of a prompt's own: nothing, or for every second sequence some."""
    rng = random.Random(case["S"] * 131 + case["prefix"])
    return [rng.randint(1, case["prefix"]) if case["prefix"] and i % 2 == 0 else 0 for i in range(case["S"])]


# ---- inputs ----------------------------------------------------------------------------------------------------

def _begins(lengths):
    at = [0]
    for n in lengths:
        at.append(at[-1] + n)
    return at


def _pool(s, case, pages, gen=None):
    """The memory of a cache of `pages` pages as [pages][page][heads][D] views, empty or (with gen) full of what was written before."""
    Hkv, D, page = case["Hkv"], case["D"], case["page"]
    by_head = case["order"] == "head"
    shape = (pages, Hkv, page, D) if by_head else (pages, page, Hkv, D)
    seen = lambda t: t.transpose(1, 2) if by_head else t  # noqa: E731
    for name in ("k", "v"):
        if gen is None:
            t = torch.zeros(shape, device="cuda")
        else:
            t = torch.randn(shape, generator=gen, device="cuda")
        if case["cache"] == "e4m3":
            t = (t * 130).clamp_(-448, 448)
            scale = torch.ones(shape[:3], device="cuda")
            if gen is not None:
                scale = (torch.randn(shape[:3], generator=gen, device="cuda") * 0.3).exp_() / 130
            s[name + "_scale"] = seen(scale)
        else:
            s[name + "_scale"] = None
        s[name + "_cache"] = seen(t.to(DTYPES[case["cache"]]))


def prepare(case, seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(int(seed))
    randn = lambda *shape: torch.randn(*shape, generator=gen, device="cuda")  # noqa: E731
    s = dict(case=case)
    D, Hkv, t = case["D"], case["Hkv"], DTYPES[case["dtype"]]
    if case["kind"] == "heads":
        T, Hq = case["T"], case["Hq"]
        # what one projection gives: queries, keys and values of a token behind each other, channels of different size
        x = randn(T, (Hq + 2 * Hkv) * D) * torch.exp(0.5 * randn((Hq + 2 * Hkv) * D))
        s["qkv"] = x.to(t)
        vector = lambda shift: shift + 0.2 * randn(D)  # noqa: E731
        for n in ("q", "k"):
            s[n + "_w"], s[n + "_b"] = (vector(1.0), vector(0.0) if case["norm"] == "layer" else None) if case["norm"] != "none" else (None, None)
        half = case["rotary"] // 2
        s["freq"] = torch.tensor([10000.0 ** (-i / half) for i in range(half)], device="cuda") if half else None
        s["position"] = torch.randint(0, case["far"], (T,), generator=gen, device="cuda", dtype=torch.int32)
        pages = T // case["page"] + 2
        _pool(s, case, pages)
        # slots of the batch's tokens all over the cache; the last of a padded batch have none
        s["slot"] = torch.randperm(pages * case["page"], generator=gen, device="cuda")[:T].contiguous()
        s["slot"][T - T // 16:] = -1
        s["q"] = torch.empty(T, Hq * D, dtype=t, device="cuda")
        s["result"] = {"q": s["q"], "k": s["k_cache"], "v": s["v_cache"], "k_scale": s["k_scale"], "v_scale": s["v_scale"]}
    elif case["kind"] == "read":
        T = case["T"]
        pages = T // case["page"] + 2
        _pool(s, case, pages, gen)
        # whole pages of a conversation behind each other, as its table names them
        order = torch.randperm(pages, generator=gen, device="cuda")
        at = torch.arange(T, device="cuda")
        s["slot"] = order[at // case["page"]] * case["page"] + at % case["page"]
        s["k"], s["v"] = (torch.empty(T, Hkv * D, dtype=t, device="cuda") for _ in range(2))
        s["result"] = {"k": s["k"], "v": s["v"]}
    elif case["kind"] == "prompt":
        Hq, lengths = case["Hq"], _lengths(case)
        before = _prefixes(case)
        keys = [a + b for a, b in zip(lengths, before)]
        s["longest_key"], s["scale"] = max(keys), D ** -0.5
        q_begin, k_begin = _begins(lengths), _begins(keys)
        s["q_rows"], s["k_rows"] = q_begin[-1], k_begin[-1]
        s["q_begin"], s["k_begin"] = (torch.tensor(b, dtype=torch.int32, device="cuda") for b in (q_begin, k_begin))
        # queries and keys after their norms, sharp enough that some keys stand out
        s["q"] = (randn(s["q_rows"], Hq * D) * 1.5).to(t)
        s["k"], s["v"] = randn(s["k_rows"], Hkv * D).to(t), randn(s["k_rows"], Hkv * D).to(t)
        s["result"] = s["o"] = torch.empty(s["q_rows"], Hq * D, dtype=t, device="cuda")
    else:
        Hq, lengths = case["Hq"], _lengths(case)
        S, page = case["S"], case["page"]
        used = [-(-n // page) for n in lengths]
        _pool(s, case, sum(used) + 1, gen)
        s["scale"] = D ** -0.5
        s["length"] = torch.tensor(lengths, dtype=torch.int32, device="cuda")
        # pages in the order in which they were free; what a row does not use names no page
        order = torch.randperm(sum(used) + 1, generator=gen, device="cuda").to(torch.int32)
        s["table"] = torch.full((S, max(used)), -1, dtype=torch.int32, device="cuda")
        at = 0
        for i, n in enumerate(used):
            s["table"][i, :n] = order[at:at + n]
            at += n
        s["q"] = (randn(S, Hq * D) * 1.5).to(t)
        s["result"] = s["o"] = torch.empty(S, Hq * D, dtype=t, device="cuda")
    if own:
        _prepare_own(case, s)
    return s


def _prepare_own(case, s):
    """The library's descriptors and workspace, which a program makes once for its buffers."""
    import paper_2506_17870_amd as nq
    s["nq"] = nq
    D, Hkv, dt = case["D"], case["Hkv"], {"f32": nq.NQ_DT_F32, "f16": nq.NQ_DT_F16, "bf16": nq.NQ_DT_BF16}[case["dtype"]]
    s["dt"] = dt
    if "k_cache" in s:
        s["cache"] = nq.make_kv_cache(s["k_cache"], s["v_cache"], s["k_scale"], s["v_scale"])
    if case["kind"] == "heads":
        Hq = case["Hq"]
        q, k, v = (s["qkv"][:, a * D:b * D] for a, b in ((0, Hq), (Hq, Hq + Hkv), (Hq + Hkv, Hq + 2 * Hkv)))
        kind = {"none": nq.NQ_NORM_NONE, "rms": nq.NQ_NORM_RMS, "layer": nq.NQ_NORM_LAYER}[case["norm"]]
        pairs = nq.NQ_PAIRS_HALVES if case["pairs"] == "halves" else nq.NQ_PAIRS_NEIGHBOURS
        ld = (Hq + 2 * Hkv) * D
        s["job"] = nq.make_head_norm(q, ld, k, ld, v, ld, dt, Hq, Hkv, D, nq.make_norm(kind, EPS, s["q_w"], s["q_b"]),
                                     nq.make_norm(kind, EPS, s["k_w"], s["k_b"]), s["freq"], case["rotary"], pairs, s["position"],
                                     s["q"], Hq * D, None, 0, s["cache"], s["slot"])
    elif case["kind"] == "prompt":
        Hq = case["Hq"]
        s["job"] = nq.make_attention_prompt(s["q"], Hq * D, s["k"], Hkv * D, s["v"], Hkv * D, s["o"], Hq * D, s["q_begin"], s["k_begin"],
                                            case["S"], s["q_rows"], s["k_rows"], dt, Hq, Hkv, D, case["causal"], s["scale"])
    elif case["kind"] == "token":
        Hq = case["Hq"]
        need = nq.nq_attention_token_workspace_bytes(case["S"], Hq, Hkv, D, case["longest"])
        s["workspace"] = torch.empty(need, dtype=torch.uint8, device="cuda")
        s["job"] = nq.make_attention_token(s["q"], Hq * D, s["o"], Hq * D, s["cache"], s["table"], s["length"], case["S"], case["longest"],
                                           dt, Hq, s["scale"], s["workspace"])


# ---- one pass --------------------------------------------------------------------------------------------------

def run(s):
    case = s["case"]
    if own:
        return _run_own(case, s)
    return {"heads": _plain_heads, "read": _plain_read, "prompt": _plain_prompt, "token": _plain_token}[case["kind"]](case, s)


def _run_own(case, s):
    nq = s["nq"]
    if case["kind"] == "heads":
        nq.nq_head_norm(s["job"], case["T"])
    elif case["kind"] == "read":
        nq.nq_cache_read(s["cache"], s["slot"], case["T"], s["k"], case["Hkv"] * case["D"], s["v"], case["Hkv"] * case["D"], s["dt"])
    elif case["kind"] == "prompt":
        nq.nq_attention_prompt(s["job"])
    else:
        nq.nq_attention_token(s["job"])
    return s["result"]


def _plain_norm(kind, v, w, b):
    if kind == "none":
        return v
    if kind == "rms":
        return v * (v.square().mean(-1, keepdim=True) + EPS).rsqrt() * w
    v = v - v.mean(-1, keepdim=True)
    return v * (v.square().mean(-1, keepdim=True) + EPS).rsqrt() * w + b


def _plain_rotate(case, v, cos, sin):
    """v [T][heads][D], cos and sin [T][1][half the rotated columns]."""
    half, rotary = case["rotary"] // 2, case["rotary"]
    if not rotary:
        return v
    if case["pairs"] == "halves":
        a, b = v[..., :half], v[..., half:rotary]
        r = torch.cat([a * cos - b * sin, b * cos + a * sin], -1)
    else:
        a, b = v[..., 0:rotary:2], v[..., 1:rotary:2]
        r = torch.stack([a * cos - b * sin, b * cos + a * sin], -1).flatten(-2)
    return torch.cat([r, v[..., rotary:]], -1)


def _plain_write(case, s, name, v, live):
    """v fp32 [T][heads][D] into the slots; those of no token are written nowhere."""
    page, slot = case["page"], s["slot"][:live]
    v = v[:live]
    if case["cache"] == "e4m3":
        a = v.abs().amax(-1, keepdim=True)
        scale = torch.where(a == 0, 1.0, (a / 448).clamp(min=2.0 ** -126))
        s[name + "_scale"][slot // page, slot % page] = scale[..., 0]
        s[name + "_cache"].view(torch.uint8)[slot // page, slot % page] = (v * (1 / scale)).to(DTYPES["e4m3"]).view(torch.uint8)
    else:
        s[name + "_cache"][slot // page, slot % page] = v.to(DTYPES[case["cache"]])


def _plain_heads(case, s):
    T, Hq, Hkv, D = case["T"], case["Hq"], case["Hkv"], case["D"]
    x = s["qkv"].view(T, Hq + 2 * Hkv, D)
    live = T - T // 16
    cos = sin = None
    if case["rotary"]:
        angle = s["position"].double()[:, None, None] * s["freq"].double()      # (fp32 loses the angles of far positions)
        cos, sin = angle.cos().float(), angle.sin().float()
    q = _plain_rotate(case, _plain_norm(case["norm"], x[:, :Hq].float(), s["q_w"], s["q_b"]), cos, sin)
    k = _plain_rotate(case, _plain_norm(case["norm"], x[:, Hq:Hq + Hkv].float(), s["k_w"], s["k_b"]), cos, sin)
    _plain_write(case, s, "k", k, live)
    _plain_write(case, s, "v", x[:, Hq + Hkv:].float(), live)
    return {**s["result"], "q": q.reshape(T, Hq * D).to(s["q"].dtype)}


def _plain_rows(case, s, name, page, place):
    """fp32 [...][heads][D] of the cache's tokens at (page, place)."""
    if case["cache"] == "e4m3":
        return s[name + "_cache"].view(torch.uint8)[page, place].view(DTYPES["e4m3"]).float() * s[name + "_scale"][page, place][..., None]
    return s[name + "_cache"][page, place].float()


def _plain_read(case, s):
    slot, page = s["slot"], case["page"]
    return {n: _plain_rows(case, s, n, slot // page, slot % page).to(s[n].dtype).view(case["T"], -1) for n in ("k", "v")}


def _plain_softmax(scores, seen):
    scores = torch.where(seen, scores, -math.inf)
    top = scores.amax(-1, keepdim=True)
    p = torch.where(seen, (scores - torch.where(top == -math.inf, 0.0, top)).exp(), 0.0)
    total = p.sum(-1, keepdim=True)
    return p / torch.where(total == 0, 1.0, total)


def _plain_prompt(case, s):
    """All sequences side by side, as long as the longest."""
    S, Hq, Hkv, D, Lq, Lk = case["S"], case["Hq"], case["Hkv"], case["D"], case["longest"], s["longest_key"]
    group = Hq // Hkv
    q0, k0 = s["q_begin"].long(), s["k_begin"].long()
    nq, nk = q0.diff(), k0.diff()
    i, j = torch.arange(Lq, device="cuda"), torch.arange(Lk, device="cuda")
    rows = lambda x, begin, at, most, H: x.float()[(begin[:-1, None] + at).clamp(max=most - 1)].view(S, len(at), H, D)  # noqa: E731
    q = rows(s["q"], q0, i, s["q_rows"], Hq).view(S, Lq, Hkv, group, D).permute(0, 2, 3, 1, 4).reshape(S * Hkv, group * Lq, D)
    k, v = (rows(s[n], k0, j, s["k_rows"], Hkv).permute(0, 2, 1, 3).reshape(S * Hkv, Lk, D) for n in ("k", "v"))
    seen = (j < nk[:, None])[:, None, :] & (i < nq[:, None])[:, :, None]
    if case["causal"]:
        seen = seen & (j <= i[None, :, None] + (nk - nq)[:, None, None])
    scores = (q @ k.transpose(1, 2)).mul_(s["scale"]).view(S, Hkv, group, Lq, Lk)
    p = _plain_softmax(scores, seen[:, None, None])
    o = (p.view(S * Hkv, group * Lq, Lk) @ v).view(S, Hkv, group, Lq, D).permute(0, 3, 1, 2, 4).reshape(S, Lq, Hq * D)
    of_row = torch.repeat_interleave(torch.arange(S, device="cuda"), nq, output_size=s["q_rows"])
    return o[of_row, torch.arange(s["q_rows"], device="cuda") - q0[of_row]].to(s["o"].dtype)


def _plain_token(case, s):
    S, Hq, Hkv, D, page = case["S"], case["Hq"], case["Hkv"], case["D"], case["page"]
    at = torch.arange(case["longest"], device="cuda")
    pages = s["table"].long()[:, at // page].clamp(min=0)
    k, v = (_plain_rows(case, s, n, pages, (at % page).expand_as(pages)).permute(0, 2, 1, 3) for n in ("k", "v"))
    q = s["q"].float().view(S, Hkv, Hq // Hkv, D)
    scores = (q @ k.transpose(2, 3)) * s["scale"]
    p = _plain_softmax(scores, (at < s["length"][:, None])[:, None, None])
    return (p @ v).view(S, Hq * D).to(s["o"].dtype)


# ---- the definition in 64 bits ---------------------------------------------------------------------------------

def _exact_norm(kind, v, w, b):
    if kind == "none":
        return v
    mean = v.sum(-1, keepdim=True) / v.shape[-1] if kind == "layer" else 0.0
    var = ((v - mean) ** 2).sum(-1, keepdim=True) / v.shape[-1]
    return (v - mean) / torch.sqrt(var + EPS) * w.double() + (b.double() if kind == "layer" else 0.0)


def _exact_codes(v):
    a = v.abs().max(-1).values
    scale = torch.where(a > 0, torch.maximum(a / 448, torch.full_like(a, 2.0 ** -126)), torch.ones_like(a))
    t = v / scale[..., None]
    # spacing of the values: 2^-9 below 2^-6, 2^(e - 3) from 2^e on
    step = torch.exp2(torch.floor(torch.log2(t.abs().clamp(min=2.0 ** -6))) - 3)
    return (t / step).round() * step, scale


def _exact_heads(case, s):
    T, Hq, Hkv, D, page = case["T"], case["Hq"], case["Hkv"], case["D"], case["page"]
    x = s["qkv"].double().view(T, -1, D)
    parts = {"q": x[:, :Hq], "k": x[:, Hq:Hq + Hkv], "v": x[:, Hq + Hkv:]}
    half = case["rotary"] // 2
    for n in ("q", "k"):
        y = _exact_norm(case["norm"], parts[n], s[n + "_w"], s[n + "_b"]).clone()
        if half:
            turn = torch.polar(torch.ones(T, half, dtype=torch.float64, device="cuda"), s["position"].double()[:, None] * s["freq"].double())
            first = slice(0, half) if case["pairs"] == "halves" else slice(0, 2 * half, 2)
            second = slice(half, 2 * half) if case["pairs"] == "halves" else slice(1, 2 * half, 2)
            z = torch.complex(y[..., first].contiguous(), y[..., second].contiguous()) * turn[:, None]
            y[..., first], y[..., second] = z.real, z.imag
        parts[n] = y
    out = {"q": parts["q"].reshape(T, Hq * D)}
    to = torch.nonzero(s["slot"] >= 0).flatten()
    flat = s["slot"][to]
    for n in ("k", "v"):
        pool = torch.zeros(s[n + "_cache"].shape, dtype=torch.float64, device="cuda").flatten(0, 1)
        scales = torch.ones(pool.shape[:2], dtype=torch.float64, device="cuda")
        if case["cache"] == "e4m3":
            pool[flat], scales[flat] = _exact_codes(parts[n][to])
        else:
            pool[flat] = parts[n][to]
        out[n] = pool.view(-1, page, Hkv, D)
        out[n + "_scale"] = scales.view(-1, page, Hkv) if case["cache"] == "e4m3" else None
    return out


def _exact_rows(case, s, name, slots):
    x = s[name + "_cache"][slots // case["page"], slots % case["page"]] if case["cache"] != "e4m3" else \
        s[name + "_cache"].view(torch.uint8)[slots // case["page"], slots % case["page"]].view(DTYPES["e4m3"])
    x = x.double()
    return x * s[name + "_scale"].double()[slots // case["page"], slots % case["page"]].unsqueeze(-1) if case["cache"] == "e4m3" else x


def exact(case, seed):
    s = prepare(case, seed)
    if case["kind"] == "heads":
        return _exact_heads(case, s)
    if case["kind"] == "read":
        return {n: _exact_rows(case, s, n, s["slot"]).view(case["T"], -1) for n in ("k", "v")}
    Hq, Hkv, D = case["Hq"], case["Hkv"], case["D"]
    group, lengths = Hq // Hkv, _lengths(case)
    out = torch.zeros(s["o"].shape, dtype=torch.float64, device="cuda")
    if case["kind"] == "prompt":
        q0, k0 = s["q_begin"].tolist(), s["k_begin"].tolist()
        for i, n in enumerate(lengths):
            m = k0[i + 1] - k0[i]
            hidden = None
            if case["causal"]:
                hidden = torch.ones(n, m, dtype=torch.bool, device="cuda").triu_(m - n + 1)
            for h in range(Hq):
                q, k, v = (s[x][b[i]:b[i + 1], c * D:c * D + D].double() for x, b, c in (("q", q0, h), ("k", k0, h // group), ("v", k0, h // group)))
                w = q @ k.t() * s["scale"]
                if hidden is not None:
                    w.masked_fill_(hidden, -math.inf)
                out[q0[i]:q0[i + 1], h * D:h * D + D] = torch.softmax(w, 1) @ v
        return out
    table = s["table"].tolist()
    for i, n in enumerate(lengths):
        slots = torch.cat([torch.arange(p * case["page"], (p + 1) * case["page"], device="cuda") for p in table[i][:-(-n // case["page"])]])[:n]
        k, v = (_exact_rows(case, s, x, slots) for x in ("k", "v"))
        for h in range(Hq):
            w = torch.softmax(k[:, h // group] @ s["q"][i, h * D:h * D + D].double() * s["scale"], 0)
            out[i, h * D:h * D + D] = w @ v[:, h // group]
    return out


def work(case):
    D, Hkv, t = case["D"], case["Hkv"], BYTES[case["dtype"]]
    kept = lambda rows: 2 * rows * Hkv * (D * BYTES[case["cache"]] + (4 if case["cache"] == "e4m3" else 0))  # noqa: E731
    if case["kind"] == "heads":
        T, Hq = case["T"], case["Hq"]
        return {"bytes": T * (2 * Hq + 2 * Hkv) * D * t + 12 * T + kept(T - T // 16), "flops": 10 * T * (Hq + Hkv) * D}
    if case["kind"] == "read":
        T = case["T"]
        return {"bytes": kept(T) + 8 * T + 2 * T * Hkv * D * t, "flops": 2 * T * Hkv * D}
    Hq, lengths = case["Hq"], _lengths(case)
    if case["kind"] == "token":
        return {"bytes": kept(sum(lengths)) + 2 * case["S"] * Hq * D * t, "flops": 4 * sum(lengths) * Hq * D}
    keys = [a + b for a, b in zip(lengths, _prefixes(case))]
    pairs = sum(n * m - (n * (n - 1) // 2 if case["causal"] else 0) for n, m in zip(lengths, keys))
    return {"bytes": (2 * sum(lengths) * Hq + 2 * sum(keys) * Hkv) * D * t, "flops": 4 * pairs * Hq * D}
