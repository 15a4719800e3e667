"""CPU checks of the attention entry points: what is refused, with which status, before anything touches a GPU, through the binding's
extension and through ctypes alike; and the tensors that descriptors are made of."""
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


def cache(nq, **kw):
    f = dict(d_k=A, d_v=A, d_k_scale=A, d_v_scale=A, pages=4, page_step=16 * 2 * 64, token_step=64, head_step=16 * 64, scale_page_step=32,
             scale_token_step=1, scale_head_step=16, type=nq.NQ_KV_E4M3, page_tokens=16, heads=2, head_dim=64)
    f.update(kw)
    return nq.nq_kv_cache(*[f[n] for n, _ in nq.nq_kv_cache._fields_])


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


BAD_CACHE = [(dict(pages=-1), "INVALID_ARG"), (dict(page_tokens=0), "INVALID_ARG"), (dict(type=0), "INVALID_ARG"), (dict(type=4), "INVALID_ARG"),
             (dict(heads=0), "INVALID_ARG"), (dict(head_dim=0), "INVALID_ARG"), (dict(head_dim=60), "SHAPE"), (dict(head_dim=264), "SHAPE"),
             (dict(heads=1025), "SHAPE"), (dict(page_step=-1), "INVALID_ARG"), (dict(token_step=-1), "INVALID_ARG"), (dict(head_step=-1), "INVALID_ARG"),
             (dict(pages=1 << 31), "SHAPE"), (dict(page_tokens=(1 << 20) + 1), "SHAPE"), (dict(page_step=(1 << 40) + 1), "SHAPE"),
             (dict(token_step=(1 << 26) + 1), "SHAPE"), (dict(head_step=(1 << 26) + 1), "SHAPE"), (dict(scale_page_step=-1), "INVALID_ARG"),
             (dict(scale_token_step=(1 << 26) + 1), "SHAPE"), (dict(scale_head_step=-1), "INVALID_ARG"), (dict(d_k=None), "INVALID_ARG"),
             (dict(d_v=None), "INVALID_ARG"), (dict(d_k_scale=None), "INVALID_ARG"), (dict(d_v_scale=None), "INVALID_ARG"),
             (dict(d_k_scale=A + 2), "ALIGN"), (dict(d_v_scale=A + 1), "ALIGN"), (dict(type=1, d_k=A + 1), "ALIGN"), (dict(type=2, d_v=A + 1), "ALIGN")]


@pytest.mark.parametrize("kw,want", BAD_CACHE)
def test_cache_descriptor(nq, kw, want):
    want, c = getattr(nq, "NQ_ERR_" + want), cache(nq, **kw)
    assert status(nq, "nq_cache_read", c, A, 0, A, 128, A, 128, 2) == want
    assert status(nq, "nq_head_norm", heads(nq, cache=c, kv_heads=c.heads, head_dim=c.head_dim), 0) == want or c.heads < 1 or c.head_dim < 1
    assert status(nq, "nq_attention_token", token(nq, cache=c)) == want


def test_no_cache_descriptor(nq):
    assert nq.binding._lib.nq_cache_read(None, A, 0, A, 128, A, 128, 2, 0) == nq.NQ_ERR_INVALID_ARG
    assert nq.binding._lib.nq_head_norm(None, 0, 0) == nq.NQ_ERR_INVALID_ARG
    assert nq.binding._lib.nq_attention_prompt(None, 0) == nq.NQ_ERR_INVALID_ARG
    assert nq.binding._lib.nq_attention_token(None, 0) == nq.NQ_ERR_INVALID_ARG


def test_cache_read(nq):
    call = lambda c=None, slot=A, T=4, k=A, ldk=128, v=A, ldv=128, dtype=2: status(nq, "nq_cache_read", c or cache(nq), slot, T, k, ldk, v, ldv, dtype)  # noqa: E731
    assert call(dtype=3) == call(dtype=-1) == call(T=-1) == call(slot=None) == nq.NQ_ERR_INVALID_ARG
    assert call(ldk=127) == call(ldv=127) == call(T=(1 << 30) + 1) == call(ldk=(1 << 32) + 1) == nq.NQ_ERR_SHAPE
    assert call(k=A + 1) == call(v=A + 2, dtype=0) == call(slot=A + 4) == nq.NQ_ERR_ALIGN
    assert call(T=0) == call(k=None, v=None) == call(T=0, k=None, v=None, slot=None) == nq.NQ_OK


def heads(nq, **kw):
    f = dict(q=A, ldq=256, k=A, ldk=128, v=A, ldv=128, dtype=2, q_heads=4, kv_heads=2, head_dim=64, q_norm=nq.make_norm(nq.NQ_NORM_RMS),
             k_norm=nq.make_norm(nq.NQ_NORM_RMS), freq=A, rotary=64, pairs=0, position=A, q_out=A, ldq_out=256, k_out=A, ldk_out=128, cache=None, slot=None)
    f.update(kw)
    return nq.make_head_norm(*f.values())


def test_head_norm(nq):
    call = lambda T=3, **kw: status(nq, "nq_head_norm", heads(nq, **kw), T)  # noqa: E731
    c = cache(nq)
    assert call(T=-1) == call(dtype=3) == call(dtype=-1) == call(pairs=2) == call(pairs=-1) == call(rotary=3) == call(rotary=-2) == nq.NQ_ERR_INVALID_ARG
    assert call(q_norm=nq.make_norm(3)) == call(k_norm=nq.make_norm(-1)) == call(q_heads=0) == call(kv_heads=-1) == nq.NQ_ERR_INVALID_ARG
    assert call(freq=None) == call(position=None) == call(q_out=None) == call(cache=c, slot=None) == nq.NQ_ERR_INVALID_ARG
    assert call(rotary=66) == call(head_dim=60, rotary=60) == call(head_dim=264) == call(T=(1 << 30) + 1) == nq.NQ_ERR_SHAPE
    assert call(ldq=255) == call(ldk=127) == call(ldv=127) == call(ldq_out=255) == call(ldk_out=127) == nq.NQ_ERR_SHAPE
    assert call(cache=cache(nq, heads=1), slot=A) == call(cache=cache(nq, head_dim=128), slot=A) == nq.NQ_ERR_SHAPE
    assert call(q=A + 1) == call(k=A + 1) == call(v=A + 1) == call(q_out=A + 1) == call(k_out=A + 1) == call(freq=A + 2) == call(position=A + 2) == nq.NQ_ERR_ALIGN
    assert call(cache=c, slot=A + 4) == call(q_norm=nq.make_norm(1, 1e-5, A + 2)) == nq.NQ_ERR_ALIGN
    assert call(T=0) == call(T=0, q=None, k=None, v=None, q_out=None, freq=None) == nq.NQ_OK
    assert call(q=None, k=None, v=None) == call(q=None, k_out=None) == call(q=None, cache=cache(nq, pages=0), slot=A, k_out=None) == nq.NQ_OK


def prompt(nq, **kw):
    f = dict(q=A, ldq=256, k=A, ldk=128, v=A, ldv=128, o=A, ldo=256, q_begin=A, k_begin=None, sequences=2, q_rows=5, k_rows=5, dtype=2, q_heads=4,
             kv_heads=2, head_dim=64, causal=1, scale=0.125)
    f.update(kw)
    return nq.make_attention_prompt(*f.values())


def test_attention_prompt(nq):
    call = lambda **kw: status(nq, "nq_attention_prompt", prompt(nq, **kw))  # noqa: E731
    assert call(sequences=-1) == call(q_rows=-1) == call(k_rows=-1) == call(dtype=3) == call(q_heads=0) == call(head_dim=-8) == nq.NQ_ERR_INVALID_ARG
    assert call(q=None) == call(k=None) == call(v=None) == call(o=None) == call(q_begin=None) == nq.NQ_ERR_INVALID_ARG
    assert call(q_heads=3) == call(kv_heads=4, q_heads=2) == call(head_dim=68) == call(head_dim=264) == call(q_heads=1026) == nq.NQ_ERR_SHAPE
    assert call(ldq=255) == call(ldk=127) == call(ldv=127) == call(ldo=255) == call(q_rows=(1 << 30) + 1) == nq.NQ_ERR_SHAPE
    assert call(k_rows=(1 << 30) + 1) == call(sequences=1 << 24) == call(q_rows=1 << 30) == nq.NQ_ERR_SHAPE
    assert call(dtype=0) == nq.NQ_ERR_UNSUPPORTED
    assert call(q=A + 1) == call(k=A + 1) == call(v=A + 1) == call(o=A + 1) == call(q_begin=A + 2) == call(k_begin=A + 1) == nq.NQ_ERR_ALIGN
    assert call(sequences=0) == call(q_rows=0, q=None, o=None) == nq.NQ_OK


def token(nq, **kw):
    f = dict(q=A, ldq=1 << 20, o=A, ldo=1 << 20, cache=None, table=A, length=A, sequences=3, max_length=100, dtype=2, q_heads=4, scale=0.125, workspace=A,
             ldtable=7, workspace_bytes=1 << 40)
    f.update(kw)
    size = f.pop("workspace_bytes")
    f["cache"] = f["cache"] or cache(nq)
    job = nq.make_attention_token(*f.values())
    job.workspace_bytes = size
    return job


def test_attention_token(nq):
    call = lambda **kw: status(nq, "nq_attention_token", token(nq, **kw))  # noqa: E731
    assert call(sequences=-1) == call(max_length=-1) == call(ldtable=-1) == call(dtype=3) == call(q_heads=0) == nq.NQ_ERR_INVALID_ARG
    assert call(q=None) == call(o=None) == call(table=None) == call(length=None) == nq.NQ_ERR_INVALID_ARG
    assert call(q_heads=3) == call(ldq=255) == call(ldo=255) == call(ldtable=6) == call(sequences=65536) == call(q_heads=1026) == nq.NQ_ERR_SHAPE
    assert call(max_length=(1 << 31) - 1, ldtable=1 << 30) == nq.NQ_ERR_SHAPE
    assert call(dtype=0) == call(dtype=1, cache=cache(nq, type=2)) == call(dtype=2, cache=cache(nq, type=1)) == nq.NQ_ERR_UNSUPPORTED
    assert call(q=A + 1) == call(o=A + 1) == call(table=A + 2) == call(length=A + 2) == nq.NQ_ERR_ALIGN
    long = dict(max_length=8192, ldtable=512)
    assert call(workspace=None, **long) == nq.NQ_ERR_INVALID_ARG
    assert call(workspace=A + 8, **long) == nq.NQ_ERR_ALIGN
    need = nq.nq_attention_token_workspace_bytes(3, 4, 2, 64, 8192)
    assert need > 0 and call(workspace_bytes=need - 1, **long) == nq.NQ_ERR_RANGE
    assert call(sequences=0) == call(sequences=0, q=None, o=None, table=None, length=None) == nq.NQ_OK


def test_workspace_bytes(nq):
    need = nq.nq_attention_token_workspace_bytes
    assert need(0, 4, 2, 64, 100) == need(1, 3, 2, 64, 100) == need(1, 4, 2, 60, 100) == need(-1, 4, 2, 64, 1000) == need(1, 4, 2, 64, 0) == 0
    assert need(1, 4, 2, 64, 100) == 0                       # one part: nothing to join
    assert need(100000, 32, 8, 128, 100000) == 0             # enough sequences to fill the card
    assert need(1, 32, 8, 128, 65536) > 0


def test_descriptor_of_a_cache(nq):
    k = torch.zeros(3, 2, 16, 64, dtype=torch.float8_e4m3fn).transpose(1, 2)
    s = torch.ones(3, 2, 16).transpose(1, 2)
    c = nq.make_kv_cache(k, k.clone(memory_format=torch.preserve_format), s, s)
    assert (c.pages, c.page_tokens, c.heads, c.head_dim, c.type) == (3, 16, 2, 64, nq.NQ_KV_E4M3)
    assert (c.page_step, c.token_step, c.head_step, c.scale_page_step, c.scale_token_step, c.scale_head_step) == (2048, 64, 1024, 32, 1, 16)
    f = torch.zeros(3, 16, 2, 64, dtype=torch.bfloat16)
    assert nq.make_kv_cache(f, f).type == nq.NQ_KV_BF16 and nq.make_kv_cache(f.half(), f.half()).type == nq.NQ_KV_F16
    for bad in (lambda: nq.make_kv_cache(f, f.half()), lambda: nq.make_kv_cache(f, f[:, :8]), lambda: nq.make_kv_cache(f.float(), f.float()),
                lambda: nq.make_kv_cache(f[0], f[0]), lambda: nq.make_kv_cache(f, f, s, s), lambda: nq.make_kv_cache(k, k), lambda: nq.make_kv_cache(k, k, s, None),
                lambda: nq.make_kv_cache(k, k, s.double(), s.double()), lambda: nq.make_kv_cache(k, k, s[:, :8], s), lambda: nq.make_kv_cache(k, k.contiguous(), s, s),
                lambda: nq.make_kv_cache(k, k, s, s.contiguous()), lambda: nq.make_kv_cache(f.transpose(2, 3), f.transpose(2, 3))):
        with pytest.raises(ValueError):
            bad()
    for dtype in (torch.float16, torch.bfloat16, torch.float8_e4m3fn):
        own = nq.KvCache(5, 32, 3, 80, dtype, device="cpu")
        assert (own.desc.pages, own.desc.page_tokens, own.desc.heads, own.desc.head_dim) == (5, 32, 3, 80) and own.k.shape == (5, 32, 3, 80)
        assert own.desc.token_step == 80 and (own.desc.d_k_scale is None) == (dtype != torch.float8_e4m3fn)


def test_tensors_of_the_jobs(nq):
    bf, i32, i64 = torch.bfloat16, torch.int32, torch.int64
    t = lambda *shape, dtype=bf: torch.zeros(*shape, dtype=dtype)  # noqa: E731
    for bad in (dict(q=t(3, 256, dtype=torch.half)), dict(k=t(3, 128, dtype=torch.float32)), dict(freq=t(31, dtype=torch.float32)),
                dict(freq=t(32, dtype=torch.float64)), dict(position=t(3, dtype=i64)), dict(slot=t(3, dtype=i32)),
                dict(q_norm=nq.make_norm(1, 1e-5, torch.ones(63)))):
        with pytest.raises(ValueError):
            heads(nq, **bad)
    for few in (dict(q=t(2, 256)), dict(q_out=t(2, 256)), dict(k=t(2, 128)), dict(v=t(2, 128)), dict(k_out=t(2, 128)), dict(position=t(2, dtype=i32)),
                dict(slot=t(2, dtype=i64), cache=cache(nq)), dict(q=t(3, 255))):
        with pytest.raises(ValueError, match="2 rows"):
            nq.nq_head_norm(heads(nq, **few), 3, stream=0)
    heads(nq, q=t(3, 512)[:, 256:], ldq=512, k=t(3, 128))
    for bad in (dict(q=t(4, 256)), dict(o=t(4, 256)), dict(k=t(4, 128)), dict(v=t(4, 128)), dict(q=t(5, 256, dtype=torch.half)), dict(q_begin=t(2, dtype=i32)),
                dict(q_begin=t(3, dtype=i64)), dict(k_begin=t(2, dtype=i32)), dict(q=t(9, 256)[4:, 8:])):
        with pytest.raises(ValueError):
            prompt(nq, **bad)
    for bad in (dict(q=t(2, 256), ldq=256), dict(o=t(2, 256), ldo=256), dict(length=t(2, dtype=i32)), dict(length=t(3, dtype=i64)), dict(table=t(2, 7, dtype=i32)),
                dict(table=t(3, 6, dtype=i32)), dict(table=t(3, 7, dtype=i64)), dict(table=t(7, 3, dtype=i32).t())):
        with pytest.raises(ValueError):
            token(nq, **bad)
    job = token(nq, table=t(3, 9, dtype=i32)[:, :7], ldtable=None, length=t(3, dtype=i32))
    assert job.ldtable == 9
    for bad in (dict(slot=t(3, dtype=i64)), dict(k=t(3, 128)), dict(v=t(4, 128, dtype=torch.half))):
        f = dict(slot=A, k=A, v=A)
        f.update(bad)
        with pytest.raises(ValueError):
            nq.nq_cache_read(cache(nq), f["slot"], 4, f["k"], 128, f["v"], 128, nq.NQ_DT_BF16, stream=0)
