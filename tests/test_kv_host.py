"""The 8-bit cache's entry points on the host: refusals and sizes. No call here reaches a kernel (device memory is not followed)."""
import ctypes

import pytest

INVALID, UNSUPPORTED, TOO_SMALL = 1, 4, 8
P = 1 << 20


@pytest.fixture(scope="module")
def b():
    from paper_2608_09291_b200 import binding
    return binding


@pytest.fixture()
def h(b):
    handle = b.us_kv_create(P, P, P, P, 100, 2, 64, 128)
    yield handle
    assert b._lib.us_kv_destroy(handle) == 0


def _create(b, kc=P, vc=P, ks=P, vs=P, n=100, heads=2, T=64, D=128):
    out = ctypes.c_void_p(5)
    st = b._lib.us_kv_create(kc, vc, ks, vs, n, heads, T, D, ctypes.byref(out))
    if st == 0:
        b._lib.us_kv_destroy(out.value)
    else:
        assert out.value is None
    return st


@pytest.mark.parametrize("kw,st", [(dict(kc=None), INVALID), (dict(vc=None), INVALID), (dict(ks=None), INVALID), (dict(vs=None), INVALID), (dict(n=0), INVALID),
                                   (dict(heads=0), INVALID), (dict(heads=70000), INVALID), (dict(kc=P + 8), INVALID), (dict(vs=P + 2), INVALID), (dict(T=0), INVALID),
                                   (dict(T=48), UNSUPPORTED), (dict(T=8), UNSUPPORTED), (dict(T=512), UNSUPPORTED), (dict(D=96), UNSUPPORTED), (dict(D=256), UNSUPPORTED),
                                   (dict(n=1 << 25), UNSUPPORTED), (dict(n=(1 << 24) - 1), 0), (dict(T=16), 0), (dict(T=256, D=64), 0)])
def test_create(b, kw, st):
    assert _create(b, **kw) == st


def test_create_wants_a_place_for_the_handle(b):
    assert b._lib.us_kv_create(P, P, P, P, 1, 1, 64, 128, None) == INVALID


def _seqs(b, **kw):
    a = dict(block_table=P, table_stride=10, lengths=P, cu_tokens=None, n_seqs=3, table_width=10)
    a.update(kw)
    return b.us_kv_seqs(**a)


def _append(b, h, q, N=3, K=P, V=P, t=0, kt=256, kh=128, vt=256, vh=128):
    return b._lib.us_kv_append(h, ctypes.byref(q) if q is not None else None, N, K, V, t, kt, kh, vt, vh, None)


def _attend(b, h, q, N=3, Q=P, t=0, heads=8, qt=1024, qh=128, scale=0.1, causal=1, window=0, out=P, ot=1024, oh=128, lse=None, scratch=P, size=1 << 40):
    return b._lib.us_kv_attention(h, ctypes.byref(q) if q is not None else None, N, Q, t, heads, qt, qh, scale, causal, window, out, ot, oh, lse, scratch, size, None)


BAD_SEQS = [dict(block_table=None), dict(lengths=None), dict(n_seqs=-1), dict(table_width=0), dict(table_width=1 << 25), dict(table_stride=9), dict(n_seqs=4),
            dict(block_table=P + 2), dict(lengths=P + 1), dict(cu_tokens=P + 3)]


@pytest.mark.parametrize("kw", BAD_SEQS)
def test_bad_sequences(b, h, kw):
    q = _seqs(b, **kw)
    assert _append(b, h, q) == INVALID
    assert _attend(b, h, q) == INVALID
    assert b._lib.us_kv_attention_scratch(h, ctypes.byref(q), 3, 8) == -1
    if "cu_tokens" not in kw and kw != dict(n_seqs=4):
        assert b._lib.us_kv_read(h, ctypes.byref(q), 5, P, P, 2, None) == INVALID


@pytest.mark.parametrize("kw", [dict(K=None), dict(V=None), dict(t=3), dict(t=-1), dict(N=-1), dict(kt=127), dict(vh=127), dict(kh=-128), dict(K=P + 1), dict(t=2, V=P + 2)])
def test_append_refuses(b, h, kw):
    assert _append(b, h, _seqs(b), **kw) == INVALID


@pytest.mark.parametrize("kw,st", [(dict(Q=None), INVALID), (dict(out=None), INVALID), (dict(t=2), UNSUPPORTED), (dict(t=4), INVALID), (dict(heads=7), INVALID), (dict(heads=0), INVALID),
                                   (dict(window=-1), INVALID), (dict(scale=float("nan")), INVALID), (dict(scale=float("inf")), INVALID), (dict(qt=127), INVALID), (dict(oh=64), INVALID),
                                   (dict(Q=P + 1), INVALID), (dict(lse=P + 2), INVALID), (dict(scratch=None), TOO_SMALL), (dict(scratch=P + 8), TOO_SMALL), (dict(size=100), TOO_SMALL)])
def test_attention_refuses(b, h, kw, st):
    assert _attend(b, h, _seqs(b), **kw) == st


FAKE = r"""
#include <cuda_runtime_api.h>
#include <stdlib.h>
#include <string.h>
/* Two devices: an address below 16 MB lies on device 0, one below 32 MB on device 1, others are managed; FAKE_DEVICE is the current one. */
cudaError_t cudaGetDevice(int* d) { *d = atoi(getenv("FAKE_DEVICE")); return cudaSuccess; }
cudaError_t cudaPointerGetAttributes(struct cudaPointerAttributes* a, const void* p)
{
    memset(a, 0, sizeof *a);
    a->type = (size_t)p >> 25 ? cudaMemoryTypeManaged : cudaMemoryTypeDevice;
    a->device = (int)((size_t)p >> 24);
    return cudaSuccess;
}
"""
CALLS = """
import ctypes, os, sys
from paper_2608_09291_b200 import binding as b
lib, P0, P1, P2 = b._lib, 1 << 20, (1 << 24) + (1 << 20), 1 << 26
out = ctypes.c_void_p()
print([lib.us_kv_create(k, v, s, t, 100, 2, 64, 128, ctypes.byref(out)) for k, v, s, t in
       ((P1, P0, P1, P1), (P1, P1, P0, P1), (P2, P1, P1, P0), (P2, P2, P2, P2), (P2, P2, P1, P1))])
q, h = b.us_kv_seqs(block_table=P1, table_stride=10, lengths=P1, cu_tokens=None, n_seqs=3, table_width=10), out.value
for n in (0, 1):
    os.environ["FAKE_DEVICE"] = str(n)
    ctypes.CDLL(None).setenv(b"FAKE_DEVICE", str(n).encode(), 1)
    print([lib.us_kv_append(h, ctypes.byref(q), 3, P1, P1, 0, 256, 128, 256, 128, None),
           lib.us_kv_read(h, ctypes.byref(q), 5, P1, P1, 2, None),
           lib.us_kv_attention(h, ctypes.byref(q), 3, P1, 0, 8, 1024, 128, 0.1, 1, 0, P1, 1024, 128, None, P1, 1 << 40, None)])
"""


def test_a_cache_belongs_to_a_device(tmp_path):
    """With another device current than the one that the pool lies on, the calls that launch refuse; a pool on two devices is none. On a
    fake of the two runtime calls that say what lies where: on the device the calls go on, and fail for want of a GPU here."""
    import os
    import subprocess
    import sys
    from pathlib import Path
    (tmp_path / "fake.c").write_text(FAKE)
    subprocess.run(["gcc", "-shared", "-fPIC", "-I/usr/local/cuda/include", "fake.c", "-o", "fake.so"], cwd=tmp_path, check=True)
    env = dict(os.environ, LD_PRELOAD=str(tmp_path / "fake.so"), FAKE_DEVICE="1", CUDA_VISIBLE_DEVICES="")
    r = subprocess.run([sys.executable, "-c", CALLS], cwd=Path(__file__).resolve().parent.parent, env=env, capture_output=True, text=True, timeout=300)
    assert r.returncode == 0, r.stderr
    made, elsewhere, there = [eval(line) for line in r.stdout.split("\n")[:3]]
    assert made == [INVALID, INVALID, INVALID, 0, 0]
    assert elsewhere == [INVALID, INVALID, INVALID]
    assert all(s not in (0, INVALID) for s in there)


def test_read_refuses(b, h):
    q = _seqs(b)
    for tokens, K, V, t in ((641, P, P, 2), (-1, P, P, 2), (5, None, P, 2), (5, P, P + 8, 2), (5, P, P, 3)):
        assert b._lib.us_kv_read(h, ctypes.byref(q), tokens, K, V, t, None) == INVALID


def test_no_handle(b):
    q = _seqs(b)
    assert _append(b, None, q) == INVALID and _attend(b, None, q) == INVALID and b._lib.us_kv_read(None, ctypes.byref(q), 5, P, P, 2, None) == INVALID
    assert b._lib.us_kv_attention_scratch(None, ctypes.byref(q), 3, 8) == -1 and b._lib.us_kv_destroy(None) == 0


def test_nothing_to_do(b, h):
    none = _seqs(b, n_seqs=0, block_table=None, lengths=None)
    assert _append(b, h, none, N=0, K=None, V=None) == 0 and _attend(b, h, none, N=0, Q=None, out=None, scratch=None, size=0) == 0
    assert b._lib.us_kv_attention_scratch(h, ctypes.byref(none), 0, 8) == 0
    assert b._lib.us_kv_read(h, ctypes.byref(_seqs(b)), 0, None, None, 2, None) == 0


def test_tensors_have_to_fit(b):
    torch = pytest.importorskip("torch")
    codes, steps = torch.zeros(4, 2, 64, 128, dtype=torch.int8), torch.zeros(4, 2)
    with pytest.raises(ValueError):
        b.KVCache(codes, codes, steps, steps)          # not on a device
    with pytest.raises(ValueError):
        b.KVCache(codes.float(), codes, steps, steps)


def test_status_text(b):
    assert "out of range" in b.us_status_string(9)
