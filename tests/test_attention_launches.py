"""CPU checks of what the attention calls launch, against the stub of the HIP runtime (hip_stub.c), each part in a process of its own."""
import os
import subprocess
import sys

import pytest

from test_fp8_launches import A, ROOT, Stub, stub  # noqa: F401


@pytest.mark.parametrize("part", ["sizes", "grants", "pieces", "dealt"])
def test_launches(stub, part):  # noqa: F811
    env = dict(os.environ, PYTHONPATH=os.pathsep.join((ROOT, os.path.join(ROOT, "tests"))))
    r = subprocess.run([sys.executable, os.path.abspath(__file__), stub, part], capture_output=True, text=True, env=env, timeout=300)
    assert r.returncode == 0, r.stdout[-2000:] + r.stderr[-4000:]


# ---- in the other process ------------------------------------------------------------------------------------------

def cache(nq, type=3, heads=8, dim=128, page=16, pages=1 << 20):
    return nq.nq_kv_cache(A, A, A, A, pages, page * heads * dim, dim, page * dim, page * heads, 1, page, type, page, heads, dim)


def heads(nq, c, dtype, Hq, T):
    none = nq.make_norm(nq.NQ_NORM_RMS)
    w = Hq * c.head_dim
    job = nq.make_head_norm(A, w, A, w, A, w, dtype, Hq, c.heads, c.head_dim, none, none, A, c.head_dim, 0, A, A, w, None, 0, c, A)
    nq.nq_head_norm(job, T, stream=0)


def prompt(nq, q_rows, k_rows, S, Hq, Hkv, D, dtype=2, q=A):
    nq.nq_attention_prompt(nq.make_attention_prompt(q, Hq * D, A, Hkv * D, A, Hkv * D, A, Hq * D, A, A, S, q_rows, k_rows, dtype, Hq, Hkv, D, True, 0.1), stream=0)


def token(nq, c, S, longest, Hq, dtype=2):
    nq.nq_attention_token(token_job(nq, c, S, longest, Hq, dtype), stream=0)


def token_job(nq, c, S, longest, Hq, dtype=2):
    job = nq.make_attention_token(A, Hq * c.head_dim, A, Hq * c.head_dim, c, A, A, S, longest, dtype, Hq, 0.1, A, ldtable=-(-longest // c.page_tokens))
    job.workspace_bytes = nq.nq_attention_token_workspace_bytes(S, Hq, c.heads, c.head_dim, longest)
    return job


def sizes(nq, stub):  # noqa: F811
    """From one row to the most that a call takes: no launch is too large for a dispatch, and every row has its threads."""
    most = (1 << 30) - 4096
    for dim in (8, 64, 72, 128, 256):
        c = cache(nq, dim=dim)
        for T in (1, 1000, 1 << 20, most):
            heads(nq, c, nq.NQ_DT_BF16, 32, T)
            lanes = 8 if dim <= 64 else 16 if dim <= 128 else 32
            assert sum(b * t for _, b, t, _ in stub.take()) >= min(T, 1 << 40) * 64 // (64 // lanes) // lanes
            nq.nq_cache_read(c, A, T, A, 8 * dim, A, 8 * dim, nq.NQ_DT_F16, stream=0)
            assert sum(b * t for _, b, t, _ in stub.take()) >= T * dim
    for q_rows, S, Hq in ((1, 1, 1), (8192, 1, 32), (1, 100000, 16), (1 << 20, 1000, 64), ((1 << 24) * 128 - 4096 * 128 >> 1, 1, 1), (most // 2, 7, 1)):
        for dim in (64, 128, 256):
            prompt(nq, q_rows, q_rows, S, Hq, 1, dim)
            (_, blocks, _, _), = stub.take()
            assert blocks >= -(-q_rows // 128) * Hq
    for S, longest, Hq, heads_ in ((1, 1, 1, 1), (1, 65536, 32, 8), (65535, 100, 1024, 1024), (1, (1 << 31) - 5000, 1, 1), (1024, 1 << 20, 16, 1), (65535, 1 << 20, 8, 8)):
        for type_ in (2, 3):
            token(nq, cache(nq, type_, heads_, 64), S, longest, Hq)
            assert len(stub.take()) in (1, 2)
    assert stub.v["refused"].value == 0


def grants(nq, stub):  # noqa: F811
    """LDS beyond 64 KB: asked for on every device, a refusal reported and asked for again."""
    for call in (lambda: prompt(nq, 8192, 8192, 1, 32, 8, 128), lambda: prompt(nq, 512, 512, 1, 8, 8, 64), lambda: prompt(nq, 4096, 4096, 1, 8, 8, 256, 1),
                 lambda: prompt(nq, 8192, 8192, 1, 32, 8, 128, 2, A + 2)):
        stub.v["device"].value, stub.v["fail_grants"].value = 0, 1
        try:
            call()
        except nq.NQError as e:
            assert e.status == nq.NQ_ERR_HIP
        else:
            raise AssertionError("a refused grant was not reported")
        assert not stub.take() and stub.v["refused"].value == 0, "launched without the grant"
        for device in (0, 3, 0, 3):
            stub.v["device"].value = device
            call()
            assert len(stub.take()) == 1 and stub.v["refused"].value == 0
    stub.v["device"].value = 0


def pieces(nq, stub):  # noqa: F811
    """The pieces that a call is launched with are those that its workspace was sized for, and a smaller one is refused."""
    for S, longest, Hq, Hkv, dim in ((1, 4096, 32, 8, 128), (1, 65536, 1, 1, 64), (96, 4096, 32, 8, 128), (1000, 300, 4, 1, 256), (256, 1 << 16, 32, 8, 128), (256, 1024, 32, 8, 128), (1024, 1 << 20, 8, 8, 64), (3, 129, 8, 8, 96)):
        c = cache(nq, 3, Hkv, dim)
        job = token_job(nq, c, S, longest, Hq)
        nq.nq_attention_token(job, stream=0)
        got = stub.take()
        blocks = Hkv * -(-(Hq // Hkv) // 16)
        if job.workspace_bytes:
            assert len(got) == 2 and got[0][1] // blocks * Hq * (dim + 2) * 4 + S * 8 == job.workspace_bytes
            job.workspace_bytes -= 1
            try:
                nq.nq_attention_token(job, stream=0)
            except nq.NQError as e:
                assert e.status == nq.NQ_ERR_RANGE
            else:
                raise AssertionError("a workspace that is too small was taken")
        else:
            assert len(got) == 1 and got[0][1] == blocks * S
        assert not stub.take()


def prompt_job(nq, S, q_rows, k_rows, Hq, Hkv, D, q=A):
    job = nq.make_attention_prompt(q, Hq * D, A, Hkv * D, A, Hkv * D, A, Hq * D, A, A, S, q_rows, k_rows, 2, Hq, Hkv, D, True, 0.1, A)
    job.workspace_bytes = nq.nq_attention_prompt_workspace_bytes(S, q_rows, k_rows, Hq, Hkv, D)
    return job


def dealt(nq, stub):  # noqa: F811
    """Prompts whose keys are dealt to workgroups: as many as the workspace was sized for, and a join; without a workspace, and where rows are not on
    16 bytes, one launch."""
    for S, q_rows, k_rows, Hq, Hkv, D in ((1, 16, 4016, 32, 8, 128), (1, 1, 1 << 20, 1, 1, 64), (4, 300, 20000, 8, 8, 96), (1, 512, 32768, 32, 8, 128), (1, 100, 5000, 4, 4, 256),
                                          (1, 8192, 8192, 32, 8, 128), (1000, 5000, 9000, 8, 8, 64), (1, 32768, 1 << 29, 1, 1, 8), (1, 1, 512, 1, 1, 8)):
        job = prompt_job(nq, S, q_rows, k_rows, Hq, Hkv, D)
        nq.nq_attention_prompt(job, stream=0)
        got = stub.take()
        if not job.workspace_bytes:
            assert len(got) == 1
            continue
        pieces = job.workspace_bytes // (q_rows * Hq * (D + 2) * 4)
        assert len(got) == 2 and 2 <= pieces <= 32 and got[0][1] % pieces == 0 and got[0][1] // pieces >= -(-q_rows // 128) * Hq
        assert got[1][1] * 256 >= q_rows * Hq * D // 4
        for q in (A + 2,):
            nq.nq_attention_prompt(prompt_job(nq, S, q_rows, k_rows, Hq, Hkv, D, q), stream=0)
            assert len(stub.take()) == 1
        for field, value, status in (("workspace_bytes", job.workspace_bytes - 1, nq.NQ_ERR_RANGE), ("d_workspace", A + 8, nq.NQ_ERR_ALIGN)):
            was = getattr(job, field)
            setattr(job, field, value)
            try:
                nq.nq_attention_prompt(job, stream=0)
            except nq.NQError as e:
                assert e.status == status
            else:
                raise AssertionError(f"{field} was taken")
            setattr(job, field, was)
        job.d_workspace, job.workspace_bytes = None, 0
        nq.nq_attention_prompt(job, stream=0)
        assert len(stub.take()) == 1
    assert stub.v["refused"].value == 0
    assert nq.nq_attention_prompt_workspace_bytes(0, 1, 1, 1, 1, 64) == 0 and nq.nq_attention_prompt_workspace_bytes(1, 16, 4000, 3, 2, 64) == 0


if __name__ == "__main__":
    the_stub = Stub(sys.argv[1])
    import paper_2506_17870_amd
    globals()[sys.argv[2]](paper_2506_17870_amd, the_stub)
