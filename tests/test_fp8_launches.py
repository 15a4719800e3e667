"""CPU checks of what the fp8 calls launch, against a stub of the HIP runtime (hip_stub.c): each part runs in a process of its own in which
the stub is loaded before the library."""
import ctypes
import os
import subprocess
import sys

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
A = 1 << 44                                      # an address nobody reads


@pytest.fixture(scope="module")
def stub(tmp_path_factory):
    so = str(tmp_path_factory.mktemp("stub") / "libstub.so")
    subprocess.run(["gcc", "-O1", "-shared", "-fPIC", "-o", so, os.path.join(ROOT, "tests", "hip_stub.c")], check=True)
    return so


def in_process(stub, part):
    env = dict(os.environ, PYTHONPATH=ROOT)
    r = subprocess.run([sys.executable, os.path.abspath(__file__), stub, part], capture_output=True, text=True, env=env, timeout=300)
    assert r.returncode == 0, r.stdout[-2000:] + r.stderr[-4000:]


@pytest.mark.parametrize("part", ["quantise_sizes", "product_sizes", "grants", "profile", "forms"])
def test_launches(stub, part):
    in_process(stub, part)


# ---- in the other process ------------------------------------------------------------------------------------------

class Launch(ctypes.Structure):
    _fields_ = [("kernel", ctypes.c_void_p), ("blocks", ctypes.c_uint64), ("threads", ctypes.c_uint64), ("lds", ctypes.c_uint64),
                ("start", ctypes.c_uint64), ("stop", ctypes.c_uint64)]


class Stub:
    def __init__(self, path):
        self.lib = ctypes.CDLL(path, mode=ctypes.RTLD_GLOBAL)
        self.launches = (Launch * (1 << 16)).in_dll(self.lib, "stub_launches")
        self.v = {n: ctypes.c_int.in_dll(self.lib, "stub_" + n) for n in ("count", "refused", "device", "fail_grants", "grant_calls")}

    def take(self):
        n, self.v["count"].value = self.v["count"].value, 0
        assert n <= 1 << 16
        return [(x.kernel, x.blocks, x.threads, x.lds) for x in self.launches[:n]]


def fp8(nq, rows, cols, block_rows=1, ld=None):
    ld = ld or -(-cols // 16) * 16
    return nq.nq_fp8(A, rows, cols, ld, A, 1, -(-rows // block_rows), block_rows, 0)


def quantise_sizes(nq, stub):
    """From one row to more than a dispatch can have threads for, every block of 128 columns once."""
    for block_rows in (1, 128):
        for dtype in (nq.NQ_DT_F32, nq.NQ_DT_BF16):
            for rows, cols in ((1, 1), (300, 1000), (1 << 20, 8192), (5 << 20, 8192), (1 << 20, 65536), ((1 << 28) + 1, 1), ((1 << 32) + 5, 100)):
                nq.nq_quantize_fp8(A, dtype, cols, None, cols, nq.NQ_ACT_NONE, fp8(nq, rows, cols, block_rows), stream=0)
                groups, got = -(-rows // block_rows) * -(-cols // 128), stub.take()
                if block_rows == 1:
                    assert groups <= sum(16 * b for _, b, _, _ in got) < groups + 16 * len(got)
                else:
                    assert sum(b for _, b, _, _ in got) == groups
    assert stub.v["refused"].value == 0


def product_sizes(nq, stub):
    """From one output to more tiles than a dispatch can have threads for, over rows and over columns, on 16 bytes and on any."""
    for dtype in (nq.NQ_DT_F32, nq.NQ_DT_F16):
        for aligned in (True, False):
            for M, N, K in ((1, 1, 1), (1, 4096, 4096), (24, 1 << 20, 130), (1, 1 << 30, 1), (300, (1 << 30) - 5, 16), (1 << 24, 4096, 128),
                            ((1 << 25) + 37, 70, 130), ((1 << 28) + 1, 1, 1), (1 << 22, 1 << 18, 256)):
                ld = None if aligned else K + 1 if (K + 1) % 16 else K
                nq.nq_gemm_fp8(fp8(nq, M, K, 1, ld), fp8(nq, N, K, 128, ld), None, A, dtype, N, stream=0)
                assert stub.take(), (M, N, K)
    assert stub.v["refused"].value == 0


def grants(nq, stub):
    """LDS beyond 64 KB: asked for on every device, not given twice, an error where it is refused, and asked for again after that."""
    def product(dtype=nq.NQ_DT_BF16, M=8192, N=8192):
        nq.nq_gemm_fp8(fp8(nq, M, 1024), fp8(nq, N, 1024, 128), None, A, dtype, N, stream=0)

    def norm(D=32768):
        none = nq.make_norm(nq.NQ_NORM_NONE)
        nq.nq_block_norm(nq.make_block_norm(A, 0, D, A, 0, D, None, 0, 0, 1.0, 1.0, none, none, A, D, None, 0), 8, D, stream=0)

    for call in (product, norm, lambda: product(nq.NQ_DT_F32), lambda: product(M=600, N=8192)):
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
        calls = stub.v["grant_calls"].value
        for device in (0, 3):
            stub.v["device"].value = device
            call()
        assert stub.v["grant_calls"].value == calls
        stub.take()
    stub.v["device"].value = 0
    calls = stub.v["grant_calls"].value
    norm(9000)                                   # (a smaller row changes nothing for a longer one)
    norm()
    assert stub.v["grant_calls"].value == calls and len(stub.take()) == 2


def profile(nq, stub):
    """The events of nq_profile_next_launch are taken by the next product, start by its first launch and stop by its last, once."""
    for M, N, ld in ((8, 300, None), (8, 300, 301), (1, 3 << 20, None)):
        nq.nq_profile_next_launch(0x111, 0x222)
        args = fp8(nq, M, 256, 1, ld), fp8(nq, N, 256, 128, ld), None, A, nq.NQ_DT_BF16, N
        nq.nq_gemm_fp8(*args, stream=0)
        n = stub.v["count"].value
        assert [x.start for x in stub.launches[:n]] == [0x111] + [0] * (n - 1) and [x.stop for x in stub.launches[:n]] == [0] * (n - 1) + [0x222]
        stub.take()
        nq.nq_gemm_fp8(*args, stream=0)
        n = stub.v["count"].value
        assert not any(x.start or x.stop for x in stub.launches[:n])
        stub.take()


def forms(nq, stub):
    """Which form the library runs: the sizes that the GPU tests have for each."""
    from fp8_forms import ANY_BYTE, FORMS
    call = lambda M, N, K, dt, ld=None: nq.nq_gemm_fp8(fp8(nq, M, K, 1, ld), fp8(nq, N, K, 128, ld), None, A, dt, N, stream=0)  # noqa: E731
    for dt, name, count in ((nq.NQ_DT_F32, "f32", 8), (nq.NQ_DT_F16, "16 bits", 12), (nq.NQ_DT_BF16, "16 bits", 12)):
        assert sorted(FORMS[name]) == list(range(count))
        for form, sizes in FORMS[name].items():
            for size in sizes:
                call(*size, dt)
                assert nq.nq_profile_last_kernel() == (12, form), (name, size)
        for variant, sizes in ANY_BYTE.items():
            for M, N, K in sizes:
                call(M, N, K, dt, K if K % 16 else K + 1)
                assert nq.nq_profile_last_kernel() == (12, variant), (name, M, N, K)
    for step, family in ((1 << 27, lambda v: v < 100), (1 << 28, lambda v: v >= 100)):      # scales too far apart for the tiles: another order
        x = nq.nq_fp8(A, 8, 256, 256, A, 1, step, 1, 0)
        nq.nq_gemm_fp8(x, fp8(nq, 300, 256, 128), None, A, nq.NQ_DT_F32, 300, stream=0)
        assert family(nq.nq_profile_last_kernel()[1])
    assert len({k for k, *_ in stub.take()}) == 8 + 12 + 12 + 3 * 2


if __name__ == "__main__":
    the_stub = Stub(sys.argv[1])
    import paper_2506_17870_amd
    globals()[sys.argv[2]](paper_2506_17870_amd, the_stub)
