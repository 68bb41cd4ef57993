"""CPU tests of the paged cache: sizes, refusals (judged before a context or a device is needed),
the kernels' index arithmetic in a host build, and the oracle against itself."""
import ctypes
import os
import shutil
import subprocess

import numpy as np
import pytest

import paper_2403_01164_amd as hg
from oracle import paged

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
INVALID, UNSUPPORTED = hg.ERR_INVALID_ARG, hg.ERR_UNSUPPORTED


def _kv(**over):
    return hg.PagedKV(**dict(dict(heads=4, head_dim=64, page_size=32, n_pages=10, dtype=hg.F16, format=hg.KV_SAME),
                             **over))


def _batch(**over):
    # addresses that are never read: a call without a context ends before any device is touched
    return hg.PagedBatch(**dict(dict(n_tokens=6, n_seq=3, max_new=4, max_pages=5, new_start=4096, kv_len=4096,
                                     page_table=4096), **over))


def _statuses(kv, batch, k=4096, v=8192, ld=256, heads=8, q=4096, ldq=512, out=8192, ldo=512, scale=0.125, ws=4096,
              n=None):
    lib = hg._lib
    n = lib.hetegen_paged_attention_ws_bytes(kv, batch, heads) if n is None else n
    return (lib.hetegen_paged_kv_write(None, kv, 4096, batch, k, v, ld, None),
            lib.hetegen_paged_kv_read(None, kv, 4096, batch, k, v, ld, None),
            lib.hetegen_paged_attention(None, kv, 4096, batch, heads, q, ldq, out, ldo, scale, ws, n, None))


def test_index_arithmetic(tmp_path):
    if shutil.which("g++") is None:
        pytest.skip("g++ not available")
    exe = str(tmp_path / "index_check")
    b = subprocess.run(["g++", "-std=c++17", "-O1", "-fsanitize=undefined", "-fno-sanitize-recover",
                        "-D__HIP_PLATFORM_AMD__", "-I" + os.path.join(os.environ.get("ROCM_PATH", "/opt/rocm"), "include"),
                        os.path.join(ROOT, "tests", "paged", "index_check.cpp"), "-o", exe],
                       capture_output=True, text=True, timeout=300)
    assert b.returncode == 0, b.stderr[-3000:]
    r = subprocess.run([exe], capture_output=True, text=True, timeout=300)
    assert r.returncode == 0 and "index check ok" in r.stdout, (r.stdout, r.stderr[-3000:])


@pytest.mark.parametrize("fmt", [paged.SAME, paged.I8, paged.E4M3])
def test_bytes_of_pages(fmt):
    for D in (64, 128):
        for page in (32, 64, 128, 256):
            kv = _kv(head_dim=D, page_size=page, format=fmt, heads=7, n_pages=13)
            assert hg.hetegen_paged_kv_bytes(kv) == 13 * 7 * paged.record_bytes(fmt, page, D)
    kv = _kv(head_dim=128, page_size=256, heads=1024, n_pages=2 ** 31 - 1, format=fmt)
    assert hg.hetegen_paged_kv_bytes(kv) == (2 ** 31 - 1) * 1024 * paged.record_bytes(fmt, 256, 128)


@pytest.mark.parametrize("fmt", [paged.SAME, paged.I8, paged.E4M3])
def test_every_byte_of_a_record_is_one_element(fmt):
    # the documented offsets are a permutation of the record
    for D, page in ((64, 32), (128, 64), (64, 256)):
        es = 2 if fmt == paged.SAME else 1
        o = np.concatenate([paged.offset(fmt, page, D, w, np.arange(page)[:, None], np.arange(D)[None]).ravel()
                            for w in (0, 1)])
        assert np.array_equal(np.sort(o), np.arange(2 * page * D) * es)
        if fmt != paged.SAME:
            s = np.concatenate([paged.scale_offset(page, D, w, np.arange(page)) for w in (0, 1)])
            assert np.array_equal(s, 2 * page * D + 4 * np.arange(2 * page))


@pytest.mark.parametrize("over,status", [
    (dict(heads=0), INVALID), (dict(heads=1025), INVALID), (dict(n_pages=0), INVALID),
    (dict(head_dim=80), UNSUPPORTED), (dict(head_dim=256), UNSUPPORTED), (dict(page_size=16), UNSUPPORTED),
    (dict(page_size=48), UNSUPPORTED), (dict(page_size=512), UNSUPPORTED), (dict(dtype=hg.F32), UNSUPPORTED),
    (dict(format=3), UNSUPPORTED), (dict(format=-1), UNSUPPORTED)])
def test_refused_caches(over, status):
    kv = _kv(**over)
    assert hg.hetegen_paged_kv_bytes(kv) == 0
    assert hg.hetegen_paged_attention_ws_bytes(kv, _batch(), 8) == 0
    assert _statuses(kv, _batch(), ld=1 << 20, ldq=1 << 20, ldo=1 << 20, n=1 << 40) == (status,) * 3


@pytest.mark.parametrize("over,status", [
    (dict(n_tokens=-1), INVALID), (dict(n_tokens=2 ** 22 + 1), INVALID), (dict(n_seq=-1), INVALID),
    (dict(n_seq=2 ** 20 + 1), INVALID), (dict(max_new=0), INVALID), (dict(max_pages=0), INVALID),
    (dict(max_pages=2 ** 25 + 1), INVALID), (dict(new_start=None), INVALID), (dict(kv_len=None), INVALID),
    (dict(page_table=None), INVALID), (dict(new_start=4098), UNSUPPORTED), (dict(kv_len=4097), UNSUPPORTED),
    (dict(page_table=4099), UNSUPPORTED)])
def test_refused_batches(over, status):
    assert _statuses(_kv(), _batch(**over), n=1 << 40) == (status,) * 3


def test_refused_products():
    kv = _kv(heads=1024)
    big = dict(ld=1 << 16, heads=1024, ldq=1 << 16, ldo=1 << 16, n=1 << 40)
    for over in (dict(n_tokens=2 ** 17 + 1), dict(n_seq=2 ** 11 + 1)):
        assert _statuses(kv, _batch(**over), **big) == (INVALID,) * 3
        assert hg.hetegen_paged_attention_ws_bytes(kv, _batch(**over), 1024) == 0
    assert hg.hetegen_paged_attention_ws_bytes(kv, _batch(n_tokens=2 ** 17, n_seq=2 ** 11), 1024) > 0


def test_refused_rows_and_workspaces():
    lib, kv, b = hg._lib, _kv(), _batch()
    for args, want in ((dict(k=0), INVALID), (dict(v=0), INVALID), (dict(k=4098), UNSUPPORTED),
                       (dict(v=8200), UNSUPPORTED), (dict(ld=248), INVALID), (dict(ld=260), UNSUPPORTED)):
        assert _statuses(kv, b, **args)[:2] == (want,) * 2, args
    assert lib.hetegen_paged_kv_read(None, kv, 4096, b, 4096, 4096, 256, None) == INVALID
    for args, want in ((dict(q=0), INVALID), (dict(out=0), INVALID), (dict(q=4104), UNSUPPORTED),
                       (dict(ldq=504), INVALID), (dict(ldo=516), UNSUPPORTED), (dict(heads=0), INVALID),
                       (dict(heads=6), INVALID), (dict(heads=1028), INVALID), (dict(scale=float("nan")), INVALID),
                       (dict(scale=float("inf")), INVALID), (dict(q=8192), INVALID), (dict(ws=0), INVALID),
                       (dict(n=262143), INVALID), (dict(ws=4104), UNSUPPORTED)):
        assert _statuses(kv, b, **dict(dict(n=1 << 40), **args))[2] == want, args
    assert _statuses(None, b, n=1 << 40) == (INVALID,) * 3 and _statuses(kv, None, n=1 << 40) == (INVALID,) * 3
    for f in (lib.hetegen_paged_kv_write, lib.hetegen_paged_kv_read):
        assert f(None, kv, None, b, 4096, 8192, 256, None) == INVALID
        assert f(None, kv, 4104, b, 4096, 8192, 256, None) == UNSUPPORTED
    # everything in order but the context
    assert _statuses(kv, b) == (INVALID,) * 3
    assert lib.hetegen_decode_step_paged(None, None, kv, 4096, b, 4096, 8192, 4096, 1 << 30, None) == INVALID
    assert lib.hetegen_decode_step_paged_ws_bytes(None, kv, b) == 0


@pytest.mark.parametrize("scale", [3.4e38, -3.4e38, 1e300, -1e300])
def test_scales_that_binary32_cannot_hold_are_refused(scale):
    # scale * log2(e) is what multiplies scores; the misplaced workspace would be refused after it
    assert _statuses(_kv(), _batch(), scale=scale, ws=4104)[2] == INVALID
    for held in (2.3e38, -2.3e38, 0.0, 1e-300):
        assert _statuses(_kv(), _batch(), scale=held, ws=4104)[2] == UNSUPPORTED


def test_workspace_does_not_shrink():
    kv = _kv(head_dim=128)
    for name, sizes in (("n_tokens", [0, 1, 2, 8, 100, 5000, 100000]), ("n_seq", [0, 1, 5, 300, 5000, 65536]),
                        ("max_new", [1, 2, 9, 100, 4000]), ("max_pages", [1, 2, 17, 1000, 100000])):
        got = [hg.hetegen_paged_attention_ws_bytes(kv, _batch(**{name: n}), 32) for n in sizes]
        assert got == sorted(got) and got[0] >= 262144, (name, got)
    assert max(hg.hetegen_paged_attention_ws_bytes(kv, _batch(n_tokens=t, n_seq=min(t, 65536), max_pages=2 ** 25), 32)
               for t in (1, 64, 4000, 10 ** 6)) < 200 << 20


def test_oracle_attention_is_the_dense_one():
    # one token, every page there: the decode attention of the dense cache
    from oracle import attention as oat
    rng = np.random.default_rng(3)
    q, K, V = rng.normal(size=(1, 4, 64)), rng.normal(size=(70, 4, 64)), rng.normal(size=(70, 4, 64))
    got, _, _ = paged.attend(q, K, V, [69], np.ones(70, bool), 64 ** -0.5)
    want = oat.attend(q.reshape(1, 256), K.reshape(1, 70, 256), V.reshape(1, 70, 256), 64)
    assert np.allclose(got.reshape(1, 256), want, rtol=1e-13)


def test_structures_match_the_header():
    assert ctypes.sizeof(hg.PagedKV) == 24 and ctypes.sizeof(hg.PagedBatch) == 40
