"""GPU tests of the paged cache's write and read-back: the pages' bytes and the rows read against
the oracle, bit for bit, with everything that a call may not touch checked as well."""
import numpy as np
import pytest

import oracle
from oracle import paged

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")
hg = pytest.importorskip("paper_2403_01164_amd")

from paged_model import GUARD, Batch, bits, device, stream  # noqa: E402


@pytest.fixture(scope="module")
def ctx():
    c = hg.hetegen_create(0)
    yield c
    hg.hetegen_destroy(c)


def _kv(dtype, fmt, D, page=64, heads=3):
    return dict(heads=heads, head_dim=D, page_size=page, dtype=dtype, format=fmt)


def _rows(b, seed, std=1.0):
    kv = b.kv
    w = kv["heads"] * kv["head_dim"]
    return bits(np.random.default_rng(seed).normal(0, std, (b.T, w)), kv["dtype"])


def _write(ctx, b, pages, k, v, ld=None, kd=None, vd=None):
    kd, vd = (device(k), device(v)) if kd is None else (kd, vd)
    hg.hetegen_paged_kv_write(ctx, b.desc, pages.data_ptr(), b.batch, kd.data_ptr(), vd.data_ptr(),
                              ld or k.shape[1], stream())
    torch.cuda.synchronize()
    return pages.cpu().numpy()


def _expected_write(b, fill, k, v):
    c = b.cache(fill)
    H, D = b.kv["heads"], b.kv["head_dim"]
    for s in range(len(b.lens)):
        for row, pos in b.positions(s):
            if 0 <= pos < b.held(s):
                c.write(b.table[s], pos, 0, k[row].reshape(H, D))
                c.write(b.table[s], pos, 1, v[row].reshape(H, D))
    return c


def _fill(b, seed=5):
    n = hg.hetegen_paged_kv_bytes(b.desc)
    return np.random.default_rng(seed).integers(0, 256, n, dtype=np.uint8)


RAGGED = dict(lens=[100, 1, 33, 70, 0, 200, 64, 65], new=[100, 1, 2, 17, 0, 129, 32, 1])


@pytest.mark.parametrize("page", [32, 128])
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("fmt", [paged.SAME, paged.I8, paged.E4M3])
@pytest.mark.parametrize("dtype", [0, 1])
def test_write_gives_the_documented_bytes(ctx, dtype, fmt, D, page):
    b = Batch(_kv(dtype, fmt, D, page), seed=1, lead=2, tail=3, **RAGGED)
    k, v, fill = _rows(b, 2), _rows(b, 3, 30.0), _fill(b)
    got = _write(ctx, b, device(fill), k, v)
    want = _expected_write(b, fill, k, v)
    assert np.array_equal(got.reshape(want.bytes.shape), want.bytes)


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("fmt", [paged.SAME, paged.I8, paged.E4M3])
@pytest.mark.parametrize("dtype", [0, 1])
def test_read_gives_the_stored_values(ctx, dtype, fmt, D):
    b = Batch(_kv(dtype, fmt, D), seed=4, lead=1, tail=2, **RAGGED)
    k, v, fill = _rows(b, 6), _rows(b, 7, 0.01), np.zeros(0, np.uint8)
    pages = torch.zeros(hg.hetegen_paged_kv_bytes(b.desc), dtype=torch.uint8, device="cuda")
    cache = b.cache(_write(ctx, b, pages, k, v))
    w = k.shape[1]
    out = [torch.full((b.T, w + 8), GUARD, dtype=torch.int16, device="cuda") for _ in range(2)]
    hg.hetegen_paged_kv_read(ctx, b.desc, pages.data_ptr(), b.batch, out[0].data_ptr(), out[1].data_ptr(), w + 8,
                             stream())
    torch.cuda.synchronize()
    for which, (o, src) in enumerate(zip(out, (k, v))):
        want = np.full((b.T, w + 8), GUARD, np.uint16)
        for s in range(len(b.lens)):
            rows = b.positions(s)
            if rows:
                vals, has = cache.read(b.table[s], rows[0][1], rows[-1][1] + 1, which)
                assert has.all()
                idx = [r for r, _ in rows]
                # a code times its scale in binary32 (one rounding), then one rounding to 16 bits
                want[idx, :w] = bits(vals.astype(np.float32).reshape(len(idx), w), dtype)
                if fmt == paged.SAME:
                    assert np.array_equal(want[idx, :w], src[idx])
                else:
                    # half a step of the code (int8: half a scale; e4m3: 2^-4 of the value, or half
                    # its smallest step 2^-9), then the rounding to 16 bits
                    x = oracle.decode(src[idx], dtype).astype(np.float64).reshape(len(idx), -1, D)
                    c = np.max(np.abs(x), axis=2, keepdims=True) / float(paged.QMAX[fmt])
                    step = c / 2 if fmt == paged.I8 else np.maximum(np.abs(x) * 2.0 ** -4, c * 2.0 ** -10)
                    u = 2.0 ** -11 if dtype == 0 else 2.0 ** -8
                    y = oracle.decode(want[idx, :w], dtype).astype(np.float64).reshape(x.shape)
                    assert (np.abs(y - x) <= 1.001 * step + u * (np.abs(x) + step) + 2.0 ** -25).all()
        assert np.array_equal(o.cpu().numpy().view(np.uint16), want), which


@pytest.mark.parametrize("fmt", [paged.I8, paged.E4M3])
@pytest.mark.parametrize("dtype", [0, 1])
def test_rows_of_zeros_extremes_and_no_numbers(ctx, dtype, fmt):
    b = Batch(_kv(dtype, fmt, 64, 32, heads=2), [40], [40], 8)
    x = oracle.decode(_rows(b, 9), dtype).astype(np.float32)
    top = 65504.0 if dtype == 0 else 3.3895313892515355e38
    x[0] = 0.0
    x[1] = top
    x[2] = 2.0 ** -24 if dtype == 0 else 2.0 ** -133  # the smallest subnormals
    x[3, 5], x[4, 64 + 7], x[5, 3] = np.inf, -np.inf, np.nan
    x[6] = -0.0
    x[7, ::2] = 1e-30 if dtype == 1 else 1e-7
    k, fill = bits(x, dtype), _fill(b)
    pages = device(fill)
    got = _write(ctx, b, pages, k, k[::-1].copy())
    want = _expected_write(b, fill, k, k[::-1].copy())
    assert np.array_equal(np.isnan(x[3:6]).any(1) | np.isinf(x[3:6]).any(1), [True] * 3)
    # a NaN's scale may be any NaN: compare those as numbers
    g, w = got.reshape(want.bytes.shape), want.bytes
    data = 2 * 32 * 64
    assert np.array_equal(g[..., :data], w[..., :data])
    gs, wsc = g[..., data:].copy().view(np.float32), w[..., data:].copy().view(np.float32)
    assert np.array_equal(gs, wsc, equal_nan=True)
    kd = torch.zeros((40, 128), dtype=torch.int16, device="cuda")
    vd = torch.zeros_like(kd)
    hg.hetegen_paged_kv_read(ctx, b.desc, pages.data_ptr(), b.batch, kd.data_ptr(), vd.data_ptr(), 128, stream())
    torch.cuda.synchronize()
    r = oracle.decode(kd.cpu().numpy().view(np.uint16), dtype).reshape(40, 2, 64)
    assert np.isnan(r[3, 0]).all() and np.isnan(r[4, 1]).all() and np.isnan(r[5, 0]).all()
    assert np.isfinite(r[3, 1]).all() and np.isfinite(r[4, 0]).all() and np.isfinite(r[5, 1]).all()
    assert (r[0] == 0).all() and (r[1] == top).all()
    assert np.array_equal(r[2], x[2].reshape(2, 64))


@pytest.mark.parametrize("fmt", [paged.I8, paged.E4M3])
@pytest.mark.parametrize("dtype", [0, 1])
def test_quotients_are_rounded_as_a_division_rounds(ctx, dtype, fmt):
    # rows of every magnitude of the type, many with values on or next to half a step
    b = Batch(_kv(dtype, fmt, 64, 64, heads=4), [1500], [1500], 18)
    rng = np.random.default_rng(19)
    lo, hi = (-24, 15) if dtype == 0 else (-133, 127)
    e = rng.integers(lo, hi + 1, (1500, 4, 1))
    x = rng.integers(-255, 256, (1500, 4, 64)) / 256.0 * 2.0 ** e
    x[..., 0] = np.where(rng.random((1500, 4)) < 0.5, 254 / 256 * 2.0 ** e[..., 0], x[..., 0])
    k = bits(x.reshape(1500, 256), dtype)
    v = bits(rng.normal(size=(1500, 256)) * 2.0 ** rng.uniform(lo / 2, hi / 2, (1500, 1)), dtype)
    fill = _fill(b)
    got = _write(ctx, b, device(fill), k, v)
    want = _expected_write(b, fill, k, v)
    assert np.array_equal(got.reshape(want.bytes.shape), want.bytes)


@pytest.mark.parametrize("fmt", [paged.SAME, paged.I8, paged.E4M3])
def test_missing_pages_positions_below_zero_and_behind_the_table(ctx, fmt):
    # sequence 0: pages that do not exist; 1: more new tokens than positions; 2: longer than the
    # table; 3: a length below zero; 4: more new tokens than max_new
    kv = _kv(0, fmt, 64, 32, heads=2)
    table = [[2, -1, 9, 12], [3, 4, -7, 5], [0, 1, 6, 7], [8, 8, 8, 8], [10, 11, 2147483647, -2147483648]]
    b = Batch(kv, [120, 20, 150, -5, 90], [100, 33, 60, 3, 80], 0, table=table, n_pages=12, max_new=60)
    k, v, fill = _rows(b, 10), _rows(b, 11), _fill(b)
    pages = device(fill)
    got = _write(ctx, b, pages, k, v)
    want = _expected_write(b, fill, k, v)
    assert np.array_equal(got.reshape(want.bytes.shape), want.bytes)
    out = [torch.full((b.T, k.shape[1]), GUARD, dtype=torch.int16, device="cuda") for _ in range(2)]
    hg.hetegen_paged_kv_read(ctx, b.desc, pages.data_ptr(), b.batch, out[0].data_ptr(), out[1].data_ptr(),
                             k.shape[1], stream())
    torch.cuda.synchronize()
    for which, o in enumerate(out):
        ref = np.full((b.T, k.shape[1]), GUARD, np.uint16)
        for s in range(5):
            for row, pos in b.positions(s):
                if pos < 0:
                    continue
                vals, has = want.read(b.table[s], pos, pos + 1, which)
                ref[row] = bits(vals.astype(np.float32).reshape(-1), 0) if has[0] and pos < b.held(s) else 0
        assert np.array_equal(o.cpu().numpy().view(np.uint16), ref), which


def test_unsound_offsets_stay_inside(ctx):
    # new_start that decreases or leaves the rows: what is written is undefined, but nothing
    # outside the pages and the rows is touched (guards on both sides of both)
    kv = _kv(0, paged.SAME, 64, 32, heads=2)
    b = Batch(kv, [90, 60, 45], [30, 30, 30], 12)
    n = hg.hetegen_paged_kv_bytes(b.desc)
    for start, lens in (([0, 200, -50, 90], [90, 60, 45]), ([70, 10, 30, 20], [2147483647, -2147483648, 45]),
                        ([-2147483648, 2147483647, 5, 2147483647], [90, 2147483647, 45])):
        b.start_d.copy_(torch.tensor(start, dtype=torch.int32))
        b.len_d.copy_(torch.tensor(lens, dtype=torch.int32))
        pages = torch.full((n + 512,), 7, dtype=torch.uint8, device="cuda")
        rows = torch.full((2, b.T + 4, 128), 3, dtype=torch.int16, device="cuda")
        hg.hetegen_paged_kv_write(ctx, b.desc, pages.data_ptr() + 256, b.batch, rows[0, 2:].data_ptr(),
                                  rows[1, 2:].data_ptr(), 128, stream())
        hg.hetegen_paged_kv_read(ctx, b.desc, pages.data_ptr() + 256, b.batch, rows[0, 2:].data_ptr(),
                                 rows[1, 2:].data_ptr(), 128, stream())
        torch.cuda.synchronize()
        assert (pages[:256] == 7).all() and (pages[-256:] == 7).all()
        assert (rows[:, :2] == 3).all() and (rows[:, -2:] == 3).all()


def test_strided_rows_of_a_qkv_output(ctx):
    b = Batch(_kv(1, paged.I8, 128, 64, heads=4), [75, 300], [7, 1], 13)
    w = 4 * 128
    qkv = bits(np.random.default_rng(14).normal(size=(b.T, 3 * w)), 1)
    d, fill = device(qkv), _fill(b)
    pages = device(fill)
    hg.hetegen_paged_kv_write(ctx, b.desc, pages.data_ptr(), b.batch, d.data_ptr() + 2 * w, d.data_ptr() + 4 * w,
                              3 * w, stream())
    torch.cuda.synchronize()
    want = _expected_write(b, fill, qkv[:, w:2 * w], qkv[:, 2 * w:])
    assert np.array_equal(pages.cpu().numpy().reshape(want.bytes.shape), want.bytes)


def test_many_sequences_of_one_token(ctx):
    # more sequences than a wavefront searches at once
    lens = [1 + (37 * i) % 150 for i in range(200)]
    b = Batch(_kv(0, paged.E4M3, 64, 32, heads=1), lens, [1] * 200, 15)
    k, v, fill = _rows(b, 16), _rows(b, 17), _fill(b)
    got = _write(ctx, b, device(fill), k, v)
    want = _expected_write(b, fill, k, v)
    assert np.array_equal(got.reshape(want.bytes.shape), want.bytes)


def test_empty_batches_do_nothing(ctx):
    kv = hg.PagedKV(2, 64, 32, 4, hg.F16, hg.KV_SAME)
    for t, n in ((0, 3), (5, 0), (0, 0)):
        batch = hg.PagedBatch(t, n, 1, 1, None, None, None)
        hg.hetegen_paged_kv_write(ctx, kv, 0, batch, 0, 0, 128, stream())
        hg.hetegen_paged_kv_read(ctx, kv, 0, batch, 0, 0, 128, stream())
        hg.hetegen_paged_attention(ctx, kv, 0, batch, 4, 0, 256, 0, 256, 0.125, 0, 0, stream())
    torch.cuda.synchronize()
