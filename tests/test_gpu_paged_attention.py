"""GPU tests of attention over a paged cache against float64 on the stored values, with bounds
from the arithmetic (paged_model.reference), and of the decode step that uses it."""
import numpy as np
import pytest

import oracle
import synth
from oracle import attention as oat
from oracle import paged
from common import TOL, U_ACT, rel_err

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")
hg = pytest.importorskip("paper_2403_01164_amd")

from gpu_model import Model  # noqa: E402
from paged_model import GUARD, TORCH, Batch, attention, bits, check, device, stream, workspace  # noqa: E402


@pytest.fixture(scope="module")
def ctx():
    c = hg.hetegen_create(0)
    yield c
    hg.hetegen_destroy(c)


def _kv(dtype, fmt, D, page=64, heads=2):
    return dict(heads=heads, head_dim=D, page_size=page, dtype=dtype, format=fmt)


def _stored(b, seed, garbage=True):
    """A cache whose positions are N(0, 1) rows, written by the oracle; everything else is NaN
    (or codes and scales that are)."""
    rng = np.random.default_rng(seed)
    kv = b.kv
    c = b.cache(np.full(hg.hetegen_paged_kv_bytes(b.desc), 0xFF if garbage else 0, np.uint8))
    H, D, P = kv["heads"], kv["head_dim"], kv["page_size"]
    for s in range(len(b.lens)):
        for j in range(-(-b.held(s) // P)):
            p = c.page(b.table[s], j * P)
            if p < 0:
                continue
            n = min(b.held(s) - j * P, P)
            for which in (0, 1):
                rows = bits(rng.normal(size=(n, H, D)), kv["dtype"])
                o = paged.offset(kv["format"], P, D, which, np.arange(n)[:, None], np.arange(D)[None])
                if kv["format"] == paged.SAME:
                    r = rows.transpose(1, 0, 2)
                    c.bytes[p][:, o], c.bytes[p][:, o + 1] = r & 255, r >> 8
                else:
                    codes, sc = paged.quantise(rows, kv["dtype"], kv["format"])
                    c.bytes[p][:, o] = codes.transpose(1, 0, 2)
                    at = int(paged.scale_offset(P, D, which, 0))
                    c.bytes[p][:, at:at + 4 * n] = np.ascontiguousarray(sc.T).view(np.uint8)
    return c


def _queries(b, heads, seed, std=1.0, extra=0):
    w = heads * b.kv["head_dim"] + extra
    return bits(np.random.default_rng(seed).normal(0, std, (b.T, w)), b.kv["dtype"])


def _run(ctx, b, heads, seed=0, std=1.0, scale=None, cache=None):
    cache = cache or _stored(b, seed)
    q = _queries(b, heads, seed + 1, std, extra=8)
    out = attention(ctx, b, device(cache.bytes), device(q), heads, scale)
    torch.cuda.synchronize()
    return check(b, cache, q, heads, out, scale)


ALL = [(dt, f, D) for dt in (0, 1) for f in (paged.SAME, paged.I8, paged.E4M3) for D in (64, 128)]


@pytest.mark.parametrize("dtype,fmt,D", ALL)
def test_single_tokens(ctx, dtype, fmt, D):
    lens = [1, 2, 15, 16, 17, 31, 32, 33, 63, 64, 65, 127, 128, 129, 255, 300, 511, 513, 700]
    _run(ctx, Batch(_kv(dtype, fmt, D, 32), lens, [1] * len(lens), 20, lead=1, tail=2), 2)


@pytest.mark.parametrize("dtype,fmt,D", ALL)
def test_grouped_heads_and_a_few_tokens(ctx, dtype, fmt, D):
    # 3 query heads to a key head: tiles of 16 rows begin and end inside a token
    _run(ctx, Batch(_kv(dtype, fmt, D, 64), [5, 90, 200, 7, 131], [5, 7, 2, 0, 11], 21), 6, seed=2)


@pytest.mark.parametrize("dtype,fmt,D", ALL)
def test_chunks_and_prompts(ctx, dtype, fmt, D):
    # a prompt from its first token, a chunk behind earlier positions, odd lengths, and a single token
    _run(ctx, Batch(_kv(dtype, fmt, D, 128), [150, 333, 64, 90], [150, 101, 64, 1], 22, lead=3, tail=4), 4, seed=4)


@pytest.mark.parametrize("group", [1, 2, 5, 8, 16, 17])
def test_group_sizes(ctx, group):
    _run(ctx, Batch(_kv(1, paged.SAME, 64, 32, heads=2), [130, 77, 40], [1, 9, 40], 23), 2 * group, seed=6)


@pytest.mark.parametrize("fmt", [paged.SAME, paged.I8])
@pytest.mark.parametrize("page", [32, 64, 128, 256])
def test_page_sizes(ctx, page, fmt):
    _run(ctx, Batch(_kv(0, fmt, 64, page, heads=1), [page - 1, page, page + 1, 3 * page + 7], [1, 2, 3, 70], 24), 2, seed=8)


@pytest.mark.parametrize("dtype,fmt", [(0, paged.SAME), (1, paged.SAME), (1, paged.I8), (0, paged.E4M3)])
@pytest.mark.parametrize("length", [1023, 1024, 1025, 2049, 8191, 8193, 20001])
def test_long_caches_split_over_workgroups(ctx, length, dtype, fmt):
    _run(ctx, Batch(_kv(dtype, fmt, 64, 256, heads=1), [length, 3], [1, 1], 25), 1, seed=10)
    _run(ctx, Batch(_kv(dtype, fmt, 128, 64, heads=1), [length], [3], 26), 4, seed=11)


def test_chunk_over_a_long_cache(ctx):
    _run(ctx, Batch(_kv(1, paged.SAME, 128, 128, heads=1), [9000], [70], 27), 2, seed=12)
    _run(ctx, Batch(_kv(0, paged.I8, 64, 64, heads=1), [9001, 40], [65, 1], 28), 2, seed=13)


@pytest.mark.parametrize("dtype,fmt", [(0, paged.SAME), (1, paged.SAME), (0, paged.I8), (1, paged.E4M3)])
def test_large_and_small_scores(ctx, dtype, fmt):
    # scores of hundreds: one position takes the whole weight; of thousandths: none does
    for std, scale in ((40.0, None), (1.0, 0.001), (1.0, -0.7), (1.0, 0.0)):
        _run(ctx, Batch(_kv(dtype, fmt, 64, 32), [40, 500, 90], [1, 1, 50], 29), 4, seed=14, std=std, scale=scale)


def test_bf16_queries_and_keys_near_the_largest(ctx):
    # sums of products that pass binary32 although the scores do not
    b = Batch(_kv(1, paged.SAME, 64, 32, heads=1), [40, 64], [1, 30], 30)
    c = _stored(b, 15)
    q = bits(np.full((b.T, 64), 2.0 ** 60), 1)
    for s in range(2):
        for j in range(b.held(s)):
            row = np.full((1, 64), 2.0 ** 62 * (1 + j % 5)) * np.where(np.arange(64) % 2, -1, 1)
            c.write(b.table[s], j, 0, bits(row, 1))
    out = attention(ctx, b, device(c.bytes), device(q), 1)
    check(b, c, q, 1, out)


def test_rows_that_see_nothing_are_zero(ctx):
    # more new tokens than positions, a length of 0 or less, and pages that do not exist
    kv = _kv(0, paged.SAME, 64, 32)
    table = [[0, 1, 2, 3], [-1, -1, -1, -1], [4, -1, 5, 99], [6, 7, 8, 9], [-1, 10, 11, 12]]
    for fmt in (paged.SAME, paged.I8, paged.E4M3):
        b = Batch(dict(kv, format=fmt), [3, 100, 120, -4, 97], [10, 20, 40, 2, 90], 0, table=table, n_pages=13)
        _run(ctx, b, 4, seed=16)
        b = Batch(dict(kv, format=fmt), [3, 100, 120, -4, 97], [4, 1, 1, 1, 1], 0, table=table, n_pages=13)
        _run(ctx, b, 2, seed=17)


def test_lengths_past_the_table_and_max_new(ctx):
    b = Batch(_kv(1, paged.SAME, 64, 32), [200, 50, 90], [3, 30, 80], 31, width=3, max_new=25)
    _run(ctx, b, 2, seed=18)
    b = Batch(_kv(1, paged.I8, 64, 32), [200, 50, 300], [150, 30, 280], 32, width=3, max_new=200)
    _run(ctx, b, 2, seed=19)


@pytest.mark.parametrize("dtype", [0, 1])
@pytest.mark.parametrize("new", [6, 40, 200])
def test_no_numbers_behind_a_token_stay_out_of_it(ctx, dtype, new):
    # keys and values of later tokens are infinities and NaNs: earlier tokens do not see them,
    # the others do
    b = Batch(_kv(dtype, paged.SAME, 64, 32, heads=1), [new + 21], [new], 33)
    for which, bad in ((0, np.nan), (0, -np.inf), (1, np.nan), (1, np.inf), (1, -np.inf)):
        c = _stored(b, 20)
        row = oracle.decode(bits(np.random.default_rng(1).normal(size=(1, 64)), dtype), dtype)
        row[0, 11] = bad
        for pos in (21 + new // 2, 21 + new - 1):
            c.write(b.table[0], pos, which, bits(row, dtype))
        q = np.abs(oracle.decode(_queries(b, 2, 21), dtype))
        q = bits(q, dtype)
        out = attention(ctx, b, device(c.bytes), device(q), 2)
        check(b, c, q, 2, out)
        got = oracle.decode(out.cpu().numpy().view(np.uint16)[:, :128], dtype)
        assert np.isfinite(got[:new // 2]).all()
        if not (which == 0 and bad < 0):
            assert not np.isfinite(got[new // 2:]).all(1).any()


@pytest.mark.parametrize("fmt", [paged.I8, paged.E4M3])
def test_no_numbers_in_8_bits(ctx, fmt):
    b = Batch(_kv(0, fmt, 64, 32, heads=1), [80], [50], 34)
    for which in (0, 1):
        c = _stored(b, 22)
        for pos, bad in ((60, np.inf), (70, np.nan)):
            row = np.ones((1, 64), np.float32)
            row[0, 3] = bad
            c.write(b.table[0], pos, which, bits(row, 0))
        q = _queries(b, 2, 23)
        out = attention(ctx, b, device(c.bytes), device(q), 2)
        check(b, c, q, 2, out)
        got = oracle.decode(out.cpu().numpy().view(np.uint16)[:, :128], 0)
        assert np.isfinite(got[:30]).all() and np.isnan(got[30:]).all()


def test_value_scales_far_apart(ctx):
    # the scales of values differ by 2^20 within a wavefront's keys; small ones come first
    for fmt in (paged.I8, paged.E4M3):
        b = Batch(_kv(1, fmt, 64, 32, heads=1), [300, 150], [1, 100], 35)
        c = _stored(b, 24)
        rng = np.random.default_rng(2)
        for s in range(2):
            for j in range(b.held(s)):
                c.write(b.table[s], j, 1, bits(rng.normal(size=(1, 64)) * 2.0 ** (-10 + 20 * j // b.held(s)), 1))
        q = _queries(b, 2, 25)
        check(b, c, q, 2, attention(ctx, b, device(c.bytes), device(q), 2))


def test_one_sequence_in_many_and_shared_pages(ctx):
    # 150 sequences, most without new tokens; two begin with the same pages
    n = 150
    b = Batch(_kv(0, paged.SAME, 64, 32, heads=1), [70 + i % 40 for i in range(n)], [int(i % 7 == 3) for i in range(n)], 36)
    b.table[10, 0] = b.table[3, 0]
    b.table[10, 1] = b.table[3, 1]
    b.table_d.copy_(torch.from_numpy(b.table))
    _run(ctx, b, 2, seed=26)


@pytest.mark.parametrize("dtype,fmt,D", [(0, paged.SAME, 128), (1, paged.I8, 64), (1, paged.SAME, 64), (0, paged.E4M3, 128)])
def test_more_sequences_than_a_wavefront_numbers(ctx, dtype, fmt, D):
    # over 64 sequences: long and short ones, one token, a few, chunks and none
    n = 70
    lens = [1 + (61 * i) % 400 + (5000 if i % 23 == 5 else 0) for i in range(n)]
    new = [min(l, (0, 1, 1, 2, 5)[i % 5]) for i, l in enumerate(lens)]
    _run(ctx, Batch(_kv(dtype, fmt, D, 64, heads=1), lens, new, 47, lead=1, tail=1), 2, seed=34)
    new[5], new[60] = 90, 70
    lens[60] += 100
    _run(ctx, Batch(_kv(dtype, fmt, D, 64, heads=1), lens, new, 48), 2, seed=35)


@pytest.mark.parametrize("seed", range(24))
def test_batches_drawn_at_random(ctx, seed):
    rng = np.random.default_rng(1000 + seed)
    fmt = int(rng.integers(0, 3))
    kv_heads, group = int(rng.integers(1, 5)), int(rng.choice([1, 2, 3, 4, 7]))
    n_seq = int(rng.choice([1, 2, 3, 7, 20]))
    budget = 500 // (n_seq * group)
    new = [int(rng.integers(0, 4)) if rng.random() < 0.6 else int(rng.integers(1, max(2, budget))) for _ in range(n_seq)]
    lens = [n + int(rng.choice([0, 1, 40, 500, 3000]) * rng.random()) for n in new]
    b = Batch(_kv(int(rng.integers(0, 2)), fmt, int(rng.choice([64, 128])), int(rng.choice([32, 64, 128, 256])), heads=kv_heads),
              lens, new, seed, lead=int(rng.integers(0, 3)), tail=int(rng.integers(0, 3)))
    if b.T == 0 or sum(new) == 0:
        b = Batch(b.kv, [9], [2], seed)
    _run(ctx, b, kv_heads * group, seed=2000 + seed)


def test_unsound_offsets_stay_inside(ctx):
    b = Batch(_kv(0, paged.SAME, 64, 32), [90, 60, 45], [30, 30, 30], 37)
    pages, ws = device(_stored(b, 27).bytes), workspace(b, 4)
    for start, lens in (([0, 200, -50, 90], [90, 60, 45]), ([70, 10, 30, 20], [2147483647, -2147483648, 45]),
                        ([-2147483648, 2147483647, 5, 2147483647], [90, 2147483647, 45])):
        b.start_d.copy_(torch.tensor(start, dtype=torch.int32))
        b.len_d.copy_(torch.tensor(lens, dtype=torch.int32))
        q = torch.ones((b.T, 256), dtype=torch.float16, device="cuda")
        out = torch.full((b.T + 4, 264), 3, dtype=torch.int16, device="cuda")
        attention(ctx, b, pages, q, 4, ws=ws, out=out[2:])
        torch.cuda.synchronize()
        assert (out[:2] == 3).all() and (out[-2:] == 3).all() and (out[:, 256:] == 3).all()


def test_same_bits_again_and_counters_back_to_zero(ctx):
    b = Batch(_kv(0, paged.I8, 128, 64), [3000, 900, 40], [1, 1, 1], 38)
    c = _stored(b, 28)
    pages, q, ws = device(c.bytes), device(_queries(b, 4, 29, extra=8)), workspace(b, 4)
    first = attention(ctx, b, pages, q, 4, ws=ws)
    for _ in range(20):
        assert torch.equal(attention(ctx, b, pages, q, 4, ws=ws), first)
    assert (ws[:262144] == 0).all()


def test_one_workspace_for_smaller_calls(ctx):
    big = Batch(_kv(0, paged.SAME, 64, 64), [5000, 4000, 70], [1, 2, 1], 39)
    ws = workspace(big, 8)
    for b in (Batch(_kv(0, paged.SAME, 64, 64), [900], [1], 40), big,
              Batch(_kv(0, paged.SAME, 64, 64), [700, 4100], [3, 1], 41)):
        c = _stored(b, 30)
        q = _queries(b, 8, 31)
        assert hg.hetegen_paged_attention_ws_bytes(b.desc, b.batch, 8) <= ws.numel()
        check(b, c, q, 8, attention(ctx, b, device(c.bytes), device(q), 8, ws=ws))


def test_pages_past_4_gib(ctx):
    # the pages of the sequence lie at both ends of a 9 GB cache
    kv = _kv(1, paged.SAME, 128, 256, heads=8)
    n_pages = 9 * 10 ** 9 // (8 * paged.record_bytes(paged.SAME, 256, 128))
    small = Batch(kv, [700], [3], 0, table=[[0, 1, 2]], n_pages=3)
    c = _stored(small, 32)
    b = Batch(kv, [700], [3], 0, table=[[0, n_pages - 1, n_pages // 2]], n_pages=n_pages)
    pages = torch.empty((n_pages,) + c.bytes.shape[1:], dtype=torch.uint8, device="cuda")
    for i, p in enumerate(b.table[0]):
        pages[int(p)] = device(c.bytes[i])
    q = _queries(b, 16, 33)
    check(small, c, q, 16, attention(ctx, b, pages, device(q), 16))
    k = device(_queries(b, 8, 34))
    hg.hetegen_paged_kv_write(ctx, b.desc, pages.data_ptr(), b.batch, k.data_ptr(), k.data_ptr(), 1024, stream())
    r = [torch.empty_like(k) for _ in range(2)]
    hg.hetegen_paged_kv_read(ctx, b.desc, pages.data_ptr(), b.batch, r[0].data_ptr(), r[1].data_ptr(), 1024, stream())
    torch.cuda.synchronize()
    assert torch.equal(r[0], k) and torch.equal(r[1], k)


@pytest.mark.parametrize("new", [1, 40])
def test_graph_replays_with_new_lengths(ctx, new):
    # write and attention captured once; lengths, table and rows change between replays
    kv = _kv(1, paged.I8, 64, 32, heads=2)
    steps = [Batch(kv, [new + 60 + 9 * i, new + 5 + 30 * i], [new, new], 42 + i, width=12, n_pages=20) for i in range(4)]
    b, w = steps[0], 3 * 128
    qkv = torch.empty((b.T, w), dtype=torch.int16, device="cuda")
    out = torch.full((b.T, 128 + 8), GUARD, dtype=torch.int16, device="cuda")
    pages = torch.empty(hg.hetegen_paged_kv_bytes(b.desc), dtype=torch.uint8, device="cuda")
    ws = workspace(b, 2)

    def step():
        p = qkv.data_ptr()
        hg.hetegen_paged_kv_write(ctx, b.desc, pages.data_ptr(), b.batch, p + 256, p + 512, w, stream())
        hg.hetegen_paged_attention(ctx, b.desc, pages.data_ptr(), b.batch, 2, p, w, out.data_ptr(), out.stride(0),
                                   0.125, ws.data_ptr(), ws.numel(), stream())

    def load(i):
        c = _stored(steps[i], 50 + i)
        pages.copy_(device(c.bytes).flatten())
        b.table_d.copy_(torch.from_numpy(steps[i].table))
        b.len_d.copy_(torch.tensor(steps[i].lens, dtype=torch.int32))
        rows = bits(np.random.default_rng(60 + i).normal(size=(b.T, w)), 1)
        qkv.copy_(device(rows))
        out.fill_(GUARD)
        for s in range(2):
            for r, pos in steps[i].positions(s):
                c.write(steps[i].table[s], pos, 0, rows[r, 128:256].reshape(2, 64))
                c.write(steps[i].table[s], pos, 1, rows[r, 256:].reshape(2, 64))
        return c, rows

    load(0)
    step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for i in (1, 2, 3, 0):
        c, rows = load(i)
        graph.replay()
        torch.cuda.synchronize()
        check(steps[i], c, rows, 2, out)
        captured = out.clone()
        out.fill_(GUARD)
        step()
        torch.cuda.synchronize()
        assert torch.equal(captured, out)


def test_two_streams_at_once(ctx):
    # calls that share the cache but nothing they write, on two streams
    b = Batch(_kv(0, paged.SAME, 128, 64), [4000, 3500, 90], [1, 1, 1], 43)
    c = _stored(b, 70)
    pages = device(c.bytes)
    qs = [device(_queries(b, 4, 71 + i)) for i in range(2)]
    wss = [workspace(b, 4) for _ in range(2)]
    want = [attention(ctx, b, pages, q, 4, ws=ws).clone() for q, ws in zip(qs, wss)]
    outs = [torch.full_like(want[0], GUARD) for _ in range(2)]
    streams = [torch.cuda.Stream() for _ in range(2)]
    torch.cuda.synchronize()
    for _ in range(20):
        for st, q, ws, o in zip(streams, qs, wss, outs):
            with torch.cuda.stream(st):
                attention(ctx, b, pages, q, 4, ws=ws, out=o)
    torch.cuda.synchronize()
    assert torch.equal(outs[0], want[0]) and torch.equal(outs[1], want[1])


# ---- the decode step over a paged cache ----

def _paged_state(m, b):
    n = hg.hetegen_paged_kv_bytes(b.desc)
    return torch.full((m.L, n), 0xFF, dtype=torch.uint8, device="cuda")


def _step(ctx, m, b, pages, x_bits, ws=None):
    x = device(x_bits)
    out = torch.full((b.T, m.H), GUARD, dtype=torch.int16, device="cuda")
    nb = hg.hetegen_model_trace_bytes(m.m, b.T)
    tr = torch.zeros((nb // 2,), dtype=torch.int16, device="cuda")
    if ws is None:
        ws = torch.zeros(hg.hetegen_decode_step_paged_ws_bytes(m.m, b.desc, b.batch), dtype=torch.uint8, device="cuda")
    hg.hetegen_model_set_trace(m.m, tr.data_ptr(), nb)
    hg.hetegen_decode_step_paged(ctx, m.m, b.desc, pages.data_ptr(), b.batch, x.data_ptr(), out.data_ptr(),
                                 ws.data_ptr(), ws.numel(), stream())
    torch.cuda.synchronize()
    hg.hetegen_model_set_trace(m.m, 0, 0)
    return out.cpu().numpy().view(np.uint16), tr.cpu().numpy().view(np.uint16)


@pytest.mark.parametrize("mode", ["resident", "streamed", "hetero"])
@pytest.mark.parametrize("dtype,fmt", [(0, paged.SAME), (1, paged.SAME), (0, paged.I8), (1, paged.E4M3)])
def test_decode_step_of_a_mixed_batch(ctx, dtype, fmt, mode):
    # three sequences of different lengths, 1, 4 and 2 new tokens: every linear teacher-forced, the
    # attention against float64 over the cache as the step left it
    L, H, F, D = 2, 256, 512, 64
    alpha = [0.4, 0.3, 0.5, 0.2] * L if mode == "hetero" else 0.0
    m = Model(ctx, L, H, F, dtype, alpha, int(mode == "resident"))
    try:
        b = Batch(dict(heads=H // D, head_dim=D, page_size=32, dtype=dtype, format=fmt), [70, 4, 150], [1, 4, 2], 44)
        start = [_stored(b, 80 + l) for l in range(L)]
        pages = torch.stack([device(c.bytes).flatten() for c in start])
        x = synth.normal((b.T, H), dtype, 0, synth.act_id(11))
        out, tr = _step(ctx, m, b, pages, x)

        def attn(l, qkv):
            c = b.cache(pages[l].cpu().numpy())
            want = b.cache(start[l].bytes)
            for s in range(3):
                for r, pos in b.positions(s):
                    want.write(b.table[s], pos, 0, qkv[r, H:2 * H].reshape(-1, D))
                    want.write(b.table[s], pos, 1, qkv[r, 2 * H:].reshape(-1, D))
            assert np.array_equal(c.bytes, want.bytes), l
            a = np.zeros((b.T, H))
            for s in range(3):
                K, has = c.read(b.table[s], 0, b.held(s), 0)
                V, _ = c.read(b.table[s], 0, b.held(s), 1)
                idx = [r for r, _ in b.positions(s)]
                q = oracle.decode(qkv[idx][:, :H], dtype).astype(np.float64).reshape(len(idx), -1, D)
                a[idx] = paged.attend(q, K, V, [p for _, p in b.positions(s)], has, D ** -0.5)[0].reshape(-1, H)
            return a

        last, _ = m.check_teacher_forced(x, tr, attn=attn)
        assert np.array_equal(out, last)
    finally:
        m.free()


def test_prompt_in_pieces_then_tokens_against_the_dense_cache(ctx):
    # a prompt of 19 tokens in pieces of 8, then two tokens: the last outputs are those of the
    # dense cache's steps, token by token, up to the rounding of both
    dtype, L, H, F, D = 0, 2, 256, 512, 64
    m = Model(ctx, L, H, F, dtype, 0.0, 1)
    try:
        kv = dict(heads=H // D, head_dim=D, page_size=32, dtype=dtype, format=paged.SAME)
        hg.hetegen_model_kv_create(ctx, m.m, 32, D)
        x = synth.normal((21, H), dtype, 0, synth.act_id(12))
        dense = np.concatenate([m.step_kv(x[t:t + 1], t) for t in range(21)])
        pages, at, got = None, 0, []
        for n in (8, 8, 3, 1, 1):
            b = Batch(kv, [at + n], [n], 0, table=[[3, 1]], n_pages=4)
            pages = _paged_state(m, b) if pages is None else pages
            got.append(_step(ctx, m, b, pages, x[at:at + n])[0])
            at += n
        a, c = oracle.decode(np.concatenate(got), dtype), oracle.decode(dense, dtype)
        # both round every intermediate: one rounding's difference per linear of the stack
        assert rel_err(a, c) <= 4 * L * (TOL + U_ACT[dtype])
    finally:
        m.free()


def test_decode_step_captured_into_a_graph(ctx):
    dtype, L, H, F, D = 0, 2, 256, 512, 64
    m = Model(ctx, L, H, F, dtype, 0.0, 1)
    try:
        kv = dict(heads=H // D, head_dim=D, page_size=32, dtype=dtype, format=paged.I8)
        b = Batch(kv, [40, 90], [1, 1], 45, width=4)
        c = _stored(b, 90)
        pages = torch.stack([device(c.bytes).flatten()] * L)
        ws = torch.zeros(hg.hetegen_decode_step_paged_ws_bytes(m.m, b.desc, b.batch), dtype=torch.uint8, device="cuda")
        x = torch.empty((2, H), dtype=torch.int16, device="cuda")
        out = torch.empty_like(x)

        def step():
            hg.hetegen_decode_step_paged(ctx, m.m, b.desc, pages.data_ptr(), b.batch, x.data_ptr(), out.data_ptr(),
                                         ws.data_ptr(), ws.numel(), stream())

        step()
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            step()
        for i in range(4):
            x.copy_(device(synth.normal((2, H), dtype, 0, synth.act_id(20 + i))))
            b.len_d.copy_(torch.tensor([40 - i, 90 + i], dtype=torch.int32))
            graph.replay()
            torch.cuda.synchronize()
            got = out.clone()
            out.fill_(-1)
            step()
            torch.cuda.synchronize()
            assert torch.equal(got, out)
    finally:
        m.free()


def test_decode_step_refusals(ctx):
    m = Model(ctx, 1, 256, 512, 0, 0.0, 1, max_batch=4)
    try:
        good = dict(heads=4, head_dim=64, page_size=32, dtype=0, format=paged.SAME)
        b = Batch(good, [40, 3], [1, 3], 46)
        pages, ws = _paged_state(m, b), torch.zeros(1 << 24, dtype=torch.uint8, device="cuda")
        x = torch.zeros((8, 256), dtype=torch.int16, device="cuda")
        o = torch.zeros_like(x)

        def call(b, x_ptr=None, out=None, n=None, model=m.m):
            hg.hetegen_decode_step_paged(ctx, model, b.desc, pages.data_ptr(), b.batch, x_ptr or x.data_ptr(),
                                         out or o.data_ptr(), ws.data_ptr(), ws.numel() if n is None else n, stream())

        call(b)
        for kv, status in ((dict(good, heads=2), hg.ERR_INVALID_ARG), (dict(good, dtype=1), hg.ERR_INVALID_ARG)):
            bad = Batch(kv, [40, 3], [1, 3], 46)
            assert hg.hetegen_decode_step_paged_ws_bytes(m.m, bad.desc, bad.batch) == 0
            with pytest.raises(hg.HetegenError) as e:
                call(bad)
            assert e.value.status == status
        many = Batch(good, [40, 3], [2, 3], 46)
        assert hg.hetegen_decode_step_paged_ws_bytes(m.m, many.desc, many.batch) == 0
        with pytest.raises(hg.HetegenError) as e:
            call(many)
        assert e.value.status == hg.ERR_UNSUPPORTED
        for args in (dict(x_ptr=o.data_ptr()), dict(n=1000), dict(model=None)):
            with pytest.raises(hg.HetegenError) as e:
                call(b, **args)
            assert e.value.status == hg.ERR_INVALID_ARG
        with pytest.raises(hg.HetegenError) as e:
            call(b, x_ptr=x.data_ptr() + 2)
        assert e.value.status == hg.ERR_UNSUPPORTED
        call(b)  # still usable
        torch.cuda.synchronize()
    finally:
        m.free()
