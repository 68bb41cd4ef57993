"""Batches over a paged cache for the GPU tests: device buffers, calls and the oracle's bounds."""
import numpy as np

import oracle
from oracle import paged
from common import U_ACT

import torch
import paper_2403_01164_amd as hg

TORCH = {0: torch.float16, 1: torch.bfloat16}
GUARD = 0x7C01  # a NaN in fp16; rows that no call may touch hold it


def bits(a, dtype):
    """float array -> 16-bit patterns, rounded half to even."""
    return torch.from_numpy(np.ascontiguousarray(a, np.float32)).to(TORCH[dtype]).view(torch.int16).numpy().view(np.uint16)


def device(a):
    a = np.ascontiguousarray(a)
    return torch.from_numpy((a.view(np.int16) if a.dtype == np.uint16 else a).copy()).cuda()


class Batch:
    """Sequences with lens[s] positions of which the last new[s] are the batch's rows.

    lead / tail: rows before the first and behind the last sequence.  The table's pages are
    drawn without repetition from n_pages; width: columns of the table."""

    def __init__(self, kv, lens, new, seed, lead=0, tail=0, width=None, max_new=None, table=None, n_pages=None):
        self.kv, self.lens, self.new = dict(kv), list(lens), list(new)
        rng = np.random.default_rng(seed)
        need = [-(-max(l, 0) // kv["page_size"]) for l in lens]
        self.n_pages = n_pages or sum(need) + 2
        width = width or max(max(need), 1)
        self.table = np.full((len(lens), width), -1, np.int32) if table is None else np.asarray(table, np.int32)
        order, at = rng.permutation(self.n_pages).astype(np.int32), 0
        for s, n in enumerate(need if table is None else []):
            n = min(n, width)
            self.table[s, :n] = order[at:at + n]
            at += n
        self.start = np.array([lead + sum(new[:s]) for s in range(len(new) + 1)], np.int32)
        self.T = int(self.start[-1]) + tail
        self.max_new = max_new or max([1] + self.new)
        self.desc = hg.PagedKV(n_pages=self.n_pages, **kv)
        self.start_d, self.table_d = device(self.start), device(self.table)
        self.len_d = device(np.array(lens, np.int32))
        self.batch = hg.PagedBatch(self.T, len(lens), self.max_new, self.table.shape[1], self.start_d.data_ptr(),
                                   self.len_d.data_ptr(), self.table_d.data_ptr())
        assert hg.hetegen_paged_kv_bytes(self.desc) == self.n_pages * kv["heads"] * paged.record_bytes(
            kv["format"], kv["page_size"], kv["head_dim"])

    def cache(self, fill=None):
        kv = self.kv
        return paged.Cache(kv["heads"], kv["head_dim"], kv["page_size"], self.n_pages, kv["dtype"], kv["format"], fill)

    def positions(self, s):
        """(row, position) of the tokens of sequence s that a call works on."""
        n = self.new[s]
        return [(int(self.start[s]) + i, self.lens[s] - n + i) for i in range(min(n, self.max_new))]

    def held(self, s):
        return min(max(self.lens[s], 0), self.table.shape[1] * self.kv["page_size"])


def stream():
    return torch.cuda.current_stream().cuda_stream


def attention(ctx, b, pages, q, heads, scale=None, ws=None, out=None, ldq=None):
    """q [T, ldq] on the device; returns out [T, heads * D + 8] (its last 8 columns guard the stride)."""
    D = b.kv["head_dim"]
    if out is None:
        out = torch.full((b.T, heads * D + 8), GUARD, dtype=torch.int16, device="cuda")
    if ws is None:
        ws = workspace(b, heads)
    hg.hetegen_paged_attention(ctx, b.desc, pages.data_ptr(), b.batch, heads, q.data_ptr(), ldq or q.stride(0),
                               out.data_ptr(), out.stride(0), D ** -0.5 if scale is None else scale, ws.data_ptr(),
                               ws.numel(), stream())
    return out


def workspace(b, heads):
    """Counters as zeros, the rest as NaN."""
    n = hg.hetegen_paged_attention_ws_bytes(b.desc, b.batch, heads)
    assert n >= 262144
    ws = torch.full((n,), 0xFF, dtype=torch.uint8, device="cuda")
    ws[:262144] = 0
    return ws


def reference(b, cache, q_bits, heads, scale=None):
    """Per sequence: rows, the oracle's output and the largest error that the arithmetic allows.

    The bound, relative to sum_j p_j |v_j| but for the first and last term:
      the output's rounding, half a step of |out|;
      a weight's rounding to 16 bits: half a step of fp16 (8-bit caches, too), or of bf16, and in
        binary32 the exponential (2^-21: its argument's rounding and its own) and the sums
        (n 2^-24 each);
      a score's error e moves a weight by e and the sum of weights by at most e: 2 e, with
        e = (D + 4) 2^-24 scale sum_d |q_d k_d| (products summed in binary32, the factors'
        roundings);
      fp16 weights below 2^-14 of the largest: steps of 2^-24, half a step each, at most n of
        them against a sum of at least 1."""
    D, dt, fmt = b.kv["head_dim"], b.kv["dtype"], b.kv["format"]
    scale = D ** -0.5 if scale is None else scale
    u = U_ACT[1] if dt == 1 and fmt == paged.SAME else U_ACT[0]
    for s in range(len(b.lens)):
        rows = b.positions(s)
        if not rows:
            continue
        n = b.held(s)
        K, has = cache.read(b.table[s], 0, n, 0)
        V, _ = cache.read(b.table[s], 0, n, 1)
        idx = [r for r, _ in rows]
        q = oracle.decode(q_bits[idx][:, :heads * D], dt).astype(np.float64).reshape(len(idx), heads, D)
        out, qk, mean = paged.attend(q, K, V, [p for _, p in rows], has, scale)
        e = (D + 4) * 2.0 ** -24 * abs(scale) * qk
        with np.errstate(all="ignore"):
            top = np.max(np.where(np.isfinite(V), np.abs(V), 0), axis=0) if n else np.zeros((b.kv["heads"], D))
            small = (n * 2.0 ** -25 if u == U_ACT[0] else 0.0) * np.repeat(top, heads // b.kv["heads"], axis=0)
            tol = U_ACT[dt] * np.abs(out) + (u + 2.0 ** -21 + 2 * n * 2.0 ** -24 + 2 * e[..., None]) * mean + small
        yield s, idx, out, tol * 1.01 + (2.0 ** -25 if dt == 0 else 1e-38)


def check(b, cache, q_bits, heads, out, scale=None):
    """out [T, heads * D + 8] (int16) against the oracle; every other element holds GUARD."""
    D = b.kv["head_dim"]
    got = out.cpu().numpy().view(np.uint16)
    touched = np.zeros(got.shape, bool)
    worst = 0.0
    for s, idx, want, tol in reference(b, cache, q_bits, heads, scale):
        o = oracle.decode(got[idx][:, :heads * D], b.kv["dtype"]).astype(np.float64).reshape(want.shape)
        touched[idx, :heads * D] = True
        same = (o == want) | (np.isnan(o) & np.isnan(want))
        with np.errstate(all="ignore"):
            ratio = np.where(same, 0.0, np.abs(o - want) / tol)
        ratio = np.where(np.isnan(ratio), np.inf, ratio)
        worst = max(worst, float(ratio.max()))
        assert worst <= 1.0, (s, np.argwhere(ratio > 1.0)[:4].tolist(), worst)
    assert (got[~touched] == GUARD).all()
    return worst
