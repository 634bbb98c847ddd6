"""MX4 entry points on the host: sizes, refusals. No call here reaches a kernel."""
import ctypes

import pytest

INVALID, TOO_SMALL = 1, 8
P = 1 << 20    # a pointer that a refused call does not follow (aligned)


@pytest.fixture(scope="module")
def b():
    from paper_2608_09291_b200 import binding
    return binding


@pytest.mark.parametrize("rows,K,tiles", [(1, 1, 1), (128, 256, 1), (129, 256, 2), (128, 257, 2), (300, 1000, 12), (0, 5, 0)])
def test_bytes_are_whole_tiles(b, rows, K, tiles):
    assert b.mx4_bytes(rows, K) == tiles * 17 * 1024


@pytest.mark.parametrize("rows,K", [(-1, 4), (4, 0), (4, -1), (1 << 31, 4), (4, (1 << 30) + 1)])
def test_shapes_out_of_range(b, rows, K):
    assert b._lib.us_mx4_bytes(rows, K) == -1
    with pytest.raises(b.UsError):
        b.mx4_bytes(rows, K)


def _quantize(b, X=P, t=0, ldx=64, rows=4, K=64, mx=P):
    return b._lib.us_mx4_quantize(X, t, ldx, rows, K, mx, None)


@pytest.mark.parametrize("kw", [dict(X=None), dict(mx=None), dict(t=3), dict(t=-1), dict(ldx=63), dict(ldx=-64), dict(K=0), dict(rows=-1), dict(X=P + 1),
                                dict(mx=P + 8), dict(t=2, X=P + 2)])
def test_quantize_refuses(b, kw):
    assert _quantize(b, **kw) == INVALID


@pytest.mark.parametrize("kw", [dict(out=None), dict(mx=None), dict(t=5), dict(ldo=63), dict(K=0), dict(out=P + 1), dict(mx=P + 4)])
def test_dequantize_refuses(b, kw):
    a = dict(mx=P, rows=4, K=64, out=P, t=1, ldo=64)
    a.update(kw)
    assert b._lib.us_mx4_dequantize(a["mx"], a["rows"], a["K"], a["out"], a["t"], a["ldo"], None) == INVALID


@pytest.mark.parametrize("kw", [dict(codes=None), dict(scales=None), dict(mx=None), dict(ldc=31), dict(lds=1), dict(mx=P + 1), dict(K=-1)])
def test_pack_and_unpack_refuse(b, kw):
    a = dict(codes=P, ldc=32, scales=P, lds=2, rows=4, K=64, mx=P)
    a.update(kw)
    assert b._lib.us_mx4_pack(a["codes"], a["ldc"], a["scales"], a["lds"], a["rows"], a["K"], a["mx"], None) == INVALID
    assert b._lib.us_mx4_unpack(a["mx"], a["rows"], a["K"], a["codes"], a["ldc"], a["scales"], a["lds"], None) == INVALID


@pytest.mark.parametrize("kw", [dict(X=None), dict(w=None), dict(Y=None), dict(t=3), dict(yt=-1), dict(ldx=511), dict(ldy=255), dict(M=0), dict(K=0), dict(N=-1),
                                dict(X=P + 1), dict(Y=P + 1), dict(w=P + 8), dict(M=1 << 31), dict(N=1 << 30, M=1 << 20)])
def test_linear_and_matmul_refuse(b, kw):
    a = dict(X=P, t=0, ldx=512, N=100, w=P, M=256, K=512, Y=P, yt=0, ldy=256)
    a.update(kw)
    args = (a["w"], a["M"], a["K"], a["Y"], a["yt"], a["ldy"])
    assert b._lib.us_mx4_linear(a["X"], a["t"], a["ldx"], a["N"], *args, P, 1 << 40, 0, None) == INVALID
    if not {"t", "ldx"} & set(kw):
        assert b._lib.us_mx4_matmul(a["X"], a["N"], *args, 0, None) == INVALID


def test_linear_wants_its_scratch(b):
    need = b._lib.us_mx4_linear_scratch(100, 256, 512)
    assert need == b.mx4_bytes(100, 512)
    for scratch, size in ((None, need), (P, need - 1), (P + 8, need)):
        assert b._lib.us_mx4_linear(P, 0, 512, 100, P, 256, 512, P, 0, 256, scratch, size, 0, None) == TOO_SMALL
    assert b._lib.us_mx4_linear_scratch(1, 256, 512) == 0          # a single token is quantised by the product
    assert b._lib.us_mx4_linear_scratch(0, 256, 512) == 0
    assert b._lib.us_mx4_linear_scratch(-1, 256, 512) == -1 and b._lib.us_mx4_linear_scratch(4, 0, 512) == -1


FAKE = r"""
#include <cuda_runtime_api.h>
#include <cstdlib>
#include <new>
/* A runtime whose launches do nothing, and a heap that is full when it is told so. */
extern "C" {
int full = 0, launches = 0;
cudaError_t cudaGetDevice(int* d) { *d = 0; return cudaSuccess; }
cudaError_t cudaGetSymbolAddress(void** p, const void*) { *p = &launches; return cudaSuccess; }
cudaError_t cudaFuncSetAttribute(const void*, cudaFuncAttribute, int) { return cudaSuccess; }
cudaError_t cudaLaunchKernelExC(const cudaLaunchConfig_t*, const void*, void**) { ++launches; return cudaSuccess; }
}
void* operator new(size_t n)
{
    void* p = full ? nullptr : malloc(n);
    if (!p) throw std::bad_alloc();
    return p;
}
"""
CALLS = """
import ctypes
from paper_2608_09291_b200 import binding as b
P, me = 1 << 20, ctypes.CDLL(None)
full, launches = (ctypes.c_int.in_dll(me, n) for n in ("full", "launches"))
for n in (1, 0):
    full.value = n
    status = b._lib.us_mx4_matmul(P, 5, P, 256, 512, P, 0, 256, 0, None)
    full.value = 0
    print(status, launches.value)
"""


def test_no_exception_leaves_a_call_that_launches(tmp_path):
    """Where there is no memory for a note of the host's, a product is launched all the same. On a fake of the runtime calls."""
    import os
    import subprocess
    import sys
    from pathlib import Path
    (tmp_path / "fake.cpp").write_text(FAKE)
    subprocess.run(["g++", "-shared", "-fPIC", "-I/usr/local/cuda/include", "fake.cpp", "-o", "fake.so"], cwd=tmp_path, check=True)
    env = dict(os.environ, LD_PRELOAD=str(tmp_path / "fake.so"))
    r = subprocess.run([sys.executable, "-c", CALLS], cwd=Path(__file__).resolve().parent.parent, env=env, capture_output=True, text=True, timeout=300)
    assert r.returncode == 0, (r.returncode, r.stderr[-500:])
    assert r.stdout.split() == ["0", "1", "0", "2"]


def test_nothing_to_do(b):
    assert b._lib.us_mx4_quantize(None, 0, 0, 0, 64, None, None) == 0
    assert b._lib.us_mx4_dequantize(None, 0, 64, None, 0, 0, None) == 0
    assert b._lib.us_mx4_pack(None, 0, None, 0, 0, 64, None, None) == 0
    assert b._lib.us_mx4_matmul(None, 0, None, 4, 64, None, 0, 0, 0, None) == 0
    assert b._lib.us_mx4_linear(None, 0, 0, 0, None, 4, 64, None, 0, 0, None, 0, 0, None) == 0


def test_tensors_have_to_be_on_the_device(b):
    torch = pytest.importorskip("torch")
    with pytest.raises((ValueError, RuntimeError)):
        b.mx4_quantize(torch.zeros(4, 64))
    with pytest.raises(ValueError):
        b.Mx4(4, 64, torch.zeros(17 * 1024, dtype=torch.uint8))
    with pytest.raises(TypeError):
        b.mx4_quantize([1.0, 2.0])
