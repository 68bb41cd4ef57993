"""The paged cache's operators as timed cases: writing it, reading it back, attention over it.

A paged cache keeps the keys and values of many sequences in pages of a fixed number of
positions; a table names each sequence's pages.  The cases write new tokens into it (as 16-bit
values, or as 8-bit codes with one scale for each token and head), read positions back, and let
new tokens (one of each sequence, or a chunk) attend to it.

`run` has two forms: the operators in elementary torch operations (own = False), and the calls
of paper_2403_01164_amd that do the same (own = True).

Layout of the pages.  A page holds, for every key/value head, `page` positions:
  keys    tiles of 16 positions: 8 dimensions of a position are contiguous (16-bit; the 8-bit
          formats hold two such groups, 32 dimensions apart, side by side)
  values  tiles of 32 positions: 8 positions of a dimension are contiguous; element e of lane
          group g is position 16 (e // 4) + 4 g + e % 4 of the tile
  8-bit formats: `page` binary32 scales of the keys, then `page` of the values
which `_pages_of` spells out as views.
"""
import math

import torch

own = False

DTYPE = {"f16": torch.float16, "bf16": torch.bfloat16}
QMAX = {"i8": 127.0, "e4m3": 448.0}


# ---- cases ------------------------------------------------------------------------------

def _case(op, dtype, fmt, heads, kv_heads, dim, page, lens, new):
    """lens[s]: positions of sequence s with its new tokens; new[s]: the new tokens."""
    return {"op": op, "dtype": dtype, "fmt": fmt, "heads": heads, "kv_heads": kv_heads, "dim": dim, "page": page,
            "lens": ",".join(map(str, lens)), "new": ",".join(map(str, new))}


def _ragged(base, n, spread):
    """n lengths around base, none alike, odd ones among them."""
    return [max(1, base + (i * 37) % (2 * spread + 1) - spread) for i in range(n)]


def listed():
    cases = [
        # a decode step's write: one token of each of 8 sequences, the layer of a 32-head model
        ("write_token_b8", _case("write", "f16", "same", 32, 32, 128, 64, _ragged(600, 8, 99), [1] * 8)),
        # prompts of several users quantised as they are written, ragged, bf16 to int8
        ("write_prompts_i8", _case("write", "bf16", "i8", 32, 32, 128, 64, [1931, 517, 1200, 63], [1931, 517, 1200, 63])),
        # chunks appended behind earlier positions, grouped heads, f16 to e4m3
        ("write_chunks_e4m3", _case("write", "f16", "e4m3", 32, 8, 64, 128, _ragged(5000, 8, 333), [1000, 512, 1, 700, 512, 333, 64, 900])),
        # an int8 cache read back, as for moving sequences to another machine
        ("read_i8", _case("read", "f16", "i8", 40, 40, 128, 64, [2049, 1000, 331, 2048], [2049, 1000, 331, 2048])),
        # the last positions of a few sequences
        ("read_tail_e4m3", _case("read", "bf16", "e4m3", 12, 12, 64, 32, [300, 77, 130], [17, 33, 5])),
        # one sequence's next token: latency
        ("attend_token_b1", _case("attend", "f16", "same", 32, 32, 128, 64, [513], [1])),
        # 8 sequences' next tokens over an int8 cache, one key head per query head
        ("attend_token_b8_i8", _case("attend", "f16", "i8", 40, 40, 128, 64, _ragged(4000, 8, 499), [1] * 8)),
        # long contexts, grouped heads, e4m3
        ("attend_token_long_e4m3", _case("attend", "bf16", "e4m3", 32, 8, 128, 128, [32001, 20000, 9999, 31337], [1] * 4)),
        # a few proposed tokens of each of 16 sequences, checked at once
        ("attend_few_b16", _case("attend", "bf16", "same", 32, 8, 128, 64, _ragged(2500, 16, 777), [5] * 16)),
        # a chunk of a long prompt over what is cached of it
        ("attend_chunk_f16", _case("attend", "f16", "same", 32, 8, 128, 128, [9217], [513])),
        # prompts from their first token on
        ("attend_prompts_bf16", _case("attend", "bf16", "same", 32, 32, 128, 64, [2048, 7000], [2048, 7000])),
        # one prompt's chunk among sequences that decode, int8
        ("attend_mixed_i8", _case("attend", "bf16", "i8", 32, 8, 64, 64, [3000] + _ragged(1500, 23, 400), [1024] + [1] * 23)),
    ]
    return [dict(c, name=n) for n, c in cases]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    """One case of the listed ones' range that costs no more than the largest of them."""
    limit = [max(work(c)[n] for c in listed()) for n in ("bytes", "flops")]
    while True:
        case = _draw(rng)
        if all(work(case)[n] <= top for n, top in zip(("bytes", "flops"), limit)):
            return case


def _draw(rng):
    op = rng.choice(["write", "read", "attend", "attend", "attend"])
    dim = rng.choice([64, 128])
    kv_heads = rng.choice([1, 2, 4, 5, 8, 12, 16, 32, 40])
    group = rng.choice([g for g in (1, 2, 3, 4, 8) if kv_heads * g <= 40])
    page = rng.choice([32, 64, 128, 256])
    n_seq = _log_int(rng, 1, 32)
    kind = rng.choice(["token", "few", "chunk"])
    new, lens = [], []
    for _ in range(n_seq):
        n = 1 if kind == "token" else rng.randint(1, 9) if kind == "few" else _log_int(rng, 10, max(20, 4000 // n_seq))
        new.append(n)
        lens.append(n + (0 if rng.random() < 0.2 else _log_int(rng, 1, 32000 // n_seq)))
    return _case(op, rng.choice(["f16", "bf16"]), rng.choice(["same", "i8", "e4m3"]), kv_heads * group, kv_heads, dim,
                 page, lens, new)


def _ints(text):
    return [int(v) for v in text.split(",")]


# ---- the cache's pages --------------------------------------------------------------------

def _elem(case):
    return 2 if case["fmt"] == "same" else 1


def _record_bytes(case):
    """Bytes of one head of one page."""
    data = 2 * case["page"] * case["dim"] * _elem(case)
    return data + (0 if case["fmt"] == "same" else 2 * case["page"] * 4)


def _stored_type(case):
    return {"same": DTYPE[case["dtype"]], "i8": torch.int8, "e4m3": torch.float8_e4m3fn}[case["fmt"]]


def _pages_of(case, pages):
    """Views of the pages [n, kv_heads, record] (uint8): keys, values, and their scales."""
    half = case["page"] * case["dim"] * _elem(case)
    t = _stored_type(case)
    out = {"k": pages[..., :half].view(t), "v": pages[..., half:2 * half].view(t)}
    if case["fmt"] != "same":
        out["k_scale"] = pages[..., 2 * half:2 * half + 4 * case["page"]].view(torch.float32)
        out["v_scale"] = pages[..., 2 * half + 4 * case["page"]:].view(torch.float32)
    return out


def _raw(t):
    """The same storage as an integer type that indexing takes."""
    return t.view(torch.int16 if t.element_size() == 2 else torch.uint8)


def _tile_views(case, stored):
    """Keys as [n, H, tile, D / c, 4, 16, c / 32, 8] and values as [n, H, tile, D / d, 4, 16, d / 16, 8]."""
    n, H = stored["k"].shape[:2]
    P, D = case["page"], case["dim"]
    c, d = (32, 16) if case["fmt"] == "same" else (64, 32)
    k, v = _raw(stored["k"]), _raw(stored["v"])
    return k.unflatten(2, (P // 16, D // c, 4, 16, c // 32, 8)), v.unflatten(2, (P // 32, D // d, 4, 16, d // 16, 8))


def _slots(case, table, lens, new, device):
    """Of every new token: its page and its position in the page."""
    seq = torch.repeat_interleave(torch.arange(len(new), device=device), torch.tensor(new, device=device))
    pos = torch.cat([torch.arange(l - n, l, device=device) for l, n in zip(lens, new)])
    return table[seq, pos // case["page"]].long(), pos % case["page"]


def _put(case, stored, page, off, k, v):
    """Stores rows k, v [T, H, D] (of the stored type) at their pages and positions."""
    T, H, D = k.shape
    kt, vt = _tile_views(case, stored)
    c, d = (32, 16) if case["fmt"] == "same" else (64, 32)
    h = torch.arange(H, device=k.device)[None]
    page, off = page[:, None], off[:, None]
    kt[page, h, off // 16, :, :, off % 16] = _raw(k).view(T, H, D // c, c // 32, 4, 8).transpose(3, 4)
    r = off % 32
    vt[page, h, off // 32, :, r % 16 // 4, :, :, r // 16 * 4 + r % 4] = _raw(v).view(T, H, D // d, d // 16, 16).transpose(3, 4)


def _take(case, stored, page, off):
    """Rows [T, H, D] of the stored type at pages and positions, keys and values."""
    T, H = page.shape[0], stored["k"].shape[1]
    kt, vt = _tile_views(case, stored)
    h = torch.arange(H, device=page.device)[None]
    page, off = page[:, None], off[:, None]
    r = off % 32
    k = kt[page, h, off // 16, :, :, off % 16].transpose(3, 4).reshape(T, H, case["dim"])
    v = vt[page, h, off // 32, :, r % 16 // 4, :, :, r // 16 * 4 + r % 4].transpose(3, 4).reshape(T, H, case["dim"])
    return k.view(_stored_type(case)), v.view(_stored_type(case))


# ---- inputs -------------------------------------------------------------------------------

def prepare(case, seed):
    """Pages with earlier positions in them, the table, and the new tokens' rows.

    Keys, values and queries are N(0, 1), keys and queries with a few dimensions eight times
    as large, as trained models have them.  The pages of a sequence lie in no order.
    """
    g = torch.Generator(device="cuda").manual_seed(seed)
    dt, D, Hk, Hq = DTYPE[case["dtype"]], case["dim"], case["kv_heads"], case["heads"]
    lens, new = _ints(case["lens"]), _ints(case["new"])
    need = [-(-l // case["page"]) for l in lens]
    n_pages, width, T = sum(need) + 3, max(need), sum(new)
    order = torch.randperm(n_pages, generator=g, device="cuda").int()
    table = torch.full((len(lens), width), -1, dtype=torch.int32, device="cuda")
    at = 0
    for s, n in enumerate(need):
        table[s, :n] = order[at:at + n]
        at += n
    start = torch.tensor([sum(new[:s]) for s in range(len(new) + 1)], dtype=torch.int32, device="cuda")
    state = {"case": case, "lens": lens, "new": new, "table": table, "start": start, "T": T,
             "kv_len": torch.tensor(lens, dtype=torch.int32, device="cuda")}
    loud = torch.ones(D, device="cuda")
    loud[torch.randperm(D, generator=g, device="cuda")[:max(1, D // 32)]] = 8.0

    def rows(heads, scale):
        return (torch.randn((T, heads, D), generator=g, device="cuda") * scale).to(dt).reshape(T, heads * D)

    if case["op"] != "read":
        # a token's query, keys and values are the parts of one row, as the qkv product leaves them
        state["qkv"] = torch.cat([rows(Hq, loud), rows(Hk, loud), rows(Hk, 1.0)], 1)
    pages = torch.empty((n_pages, Hk, _record_bytes(case)), dtype=torch.uint8, device="cuda")
    stored = _pages_of(case, pages)
    if case["fmt"] == "same":
        half = (n_pages, Hk, case["page"] * D)
        for name in ("k", "v"):
            stored[name].copy_(torch.randn(half, generator=g, device="cuda").to(dt))
        kt = stored["k"].unflatten(2, (-1, D // 32, 4, 16, 8))
        kt.mul_(loud.to(dt).view(D // 32, 4, 1, 8))
    else:
        for name in ("k", "v"):
            raw = torch.randn((n_pages, Hk, case["page"] * D), generator=g, device="cuda") * (QMAX[case["fmt"]] / 3.5)
            raw = raw.clamp_(-QMAX[case["fmt"]], QMAX[case["fmt"]])
            stored[name].view(torch.uint8).copy_((raw.round_() if case["fmt"] == "i8" else raw).to(_stored_type(case)).view(torch.uint8))
            stored[name + "_scale"].copy_((torch.rand((n_pages, Hk, case["page"]), generator=g, device="cuda") + 2.5) / QMAX[case["fmt"]])
    state["pages"] = pages
    if own:
        _prepare_own(state)
    return state


# ---- plain forms ----------------------------------------------------------------------------

def _quantise(case, x):
    """Codes (in the stored type) and scales of rows x [T, H, D] in 32 bits."""
    c = x.abs().amax(2) / QMAX[case["fmt"]]
    q = x / torch.where(c == 0, 1.0, c)[..., None]
    return (q.round().clamp(-127, 127) if case["fmt"] == "i8" else q).to(_stored_type(case)), c


def _kv_rows(state):
    case = state["case"]
    w = case["kv_heads"] * case["dim"]
    q = case["heads"] * case["dim"]
    qkv = state["qkv"]
    return qkv[:, :q], qkv[:, q:q + w], qkv[:, q + w:]


def _write(state):
    case = state["case"]
    _, k, v = _kv_rows(state)
    k, v = k.unflatten(1, (-1, case["dim"])), v.unflatten(1, (-1, case["dim"]))
    page, off = _slots(case, state["table"], state["lens"], state["new"], k.device)
    stored = _pages_of(case, state["pages"])
    if case["fmt"] == "same":
        _put(case, stored, page, off, k.contiguous(), v.contiguous())
        return stored
    (kq, kc), (vq, vc) = _quantise(case, k.float()), _quantise(case, v.float())
    _put(case, stored, page, off, kq, vq)
    h = torch.arange(kq.shape[1], device=kq.device)[None]
    stored["k_scale"][page[:, None], h, off[:, None]] = kc
    stored["v_scale"][page[:, None], h, off[:, None]] = vc
    return stored


def _values(case, stored, page, off):
    """Keys and values [T, H, D] in 32 bits at pages and positions."""
    k, v = _take(case, stored, page, off)
    k, v = k.float(), v.float()
    if case["fmt"] != "same":
        h = torch.arange(k.shape[1], device=k.device)[None]
        k = k * stored["k_scale"][page[:, None], h, off[:, None]][..., None]
        v = v * stored["v_scale"][page[:, None], h, off[:, None]][..., None]
    return k, v


def _read(state):
    case = state["case"]
    page, off = _slots(case, state["table"], state["lens"], state["new"], state["pages"].device)
    k, v = _values(case, _pages_of(case, state["pages"]), page, off)
    dt = DTYPE[case["dtype"]]
    return {"k": k.to(dt).flatten(1), "v": v.to(dt).flatten(1)}


def _attend(state):
    case = state["case"]
    D, Hk, Hq = case["dim"], case["kv_heads"], case["heads"]
    q, _, _ = _kv_rows(state)
    out = torch.empty((state["T"], Hq * D), dtype=q.dtype, device=q.device)
    stored = _pages_of(case, state["pages"])
    at = 0
    for s, (length, n) in enumerate(zip(state["lens"], state["new"])):
        pos = torch.arange(length, device=q.device)
        k, v = _values(case, stored, state["table"][s, pos // case["page"]].long(), pos % case["page"])
        qs = q[at:at + n].float().view(n, Hk, Hq // Hk, D).permute(1, 2, 0, 3)
        # a block of the chunk's tokens at a time: the scores of a long one would fill the card
        step = max(1, (1 << 28) // (length * Hq))
        for i in range(0, n, step):
            part = qs[:, :, i:i + step]
            m = part.shape[2]
            score = part.reshape(Hk, -1, D) @ k.permute(1, 2, 0).contiguous() * D ** -0.5
            score = score.view(Hk, Hq // Hk, m, length)
            sees = pos[None] <= (length - n + i + torch.arange(m, device=q.device))[:, None]
            score = score.masked_fill(~sees, -math.inf)
            weight = (score - score.amax(3, keepdim=True)).exp()
            weight = weight / weight.sum(3, keepdim=True)
            o = weight.view(Hk, -1, length) @ v.permute(1, 0, 2).contiguous()
            out[at + i:at + i + m] = o.view(Hk, Hq // Hk, m, D).permute(2, 0, 1, 3).reshape(m, -1).to(q.dtype)
        at += n
    return out


# ---- the framework's calls ------------------------------------------------------------------

_context = None


def _ctx(hg):
    """One context per process, as a serving program keeps it."""
    global _context
    if _context is None:
        _context = hg.hetegen_create(torch.cuda.current_device())
    return _context


def _prepare_own(state):
    import paper_2403_01164_amd as hg
    case = state["case"]
    fmt = {"same": hg.KV_SAME, "i8": hg.KV_I8, "e4m3": hg.KV_E4M3}[case["fmt"]]
    kv = hg.PagedKV(heads=case["kv_heads"], head_dim=case["dim"], page_size=case["page"],
                    n_pages=state["pages"].shape[0], dtype={"f16": hg.F16, "bf16": hg.BF16}[case["dtype"]], format=fmt)
    batch = hg.PagedBatch(n_tokens=state["T"], n_seq=len(state["new"]), max_new=max(state["new"]),
                          max_pages=state["table"].shape[1], new_start=state["start"].data_ptr(),
                          kv_len=state["kv_len"].data_ptr(), page_table=state["table"].data_ptr())
    assert hg.hetegen_paged_kv_bytes(kv) == state["pages"].numel()
    state.update(hg=hg, ctx=_ctx(hg), kv=kv, batch=batch)
    if case["op"] == "attend":
        n = hg.hetegen_paged_attention_ws_bytes(kv, batch, case["heads"])
        state["ws"] = torch.zeros(n, dtype=torch.uint8, device="cuda")


def _run_own(state):
    case, hg = state["case"], state["hg"]
    stream = torch.cuda.current_stream().cuda_stream
    call = (state["ctx"], state["kv"], state["pages"].data_ptr(), state["batch"])
    wq, wk = case["heads"] * case["dim"], case["kv_heads"] * case["dim"]
    if case["op"] == "read":
        dt = DTYPE[case["dtype"]]
        k = torch.empty((state["T"], wk), dtype=dt, device="cuda")
        v = torch.empty_like(k)
        hg.hetegen_paged_kv_read(*call, k.data_ptr(), v.data_ptr(), wk, stream)
        return {"k": k, "v": v}
    qkv = state["qkv"]
    ld, p = qkv.stride(0), qkv.data_ptr()
    if case["op"] == "write":
        hg.hetegen_paged_kv_write(*call, p + 2 * wq, p + 2 * (wq + wk), ld, stream)
        return _pages_of(case, state["pages"])
    out = torch.empty((state["T"], wq), dtype=qkv.dtype, device="cuda")
    hg.hetegen_paged_attention(*call, case["heads"], p, ld, out.data_ptr(), wq, case["dim"] ** -0.5,
                               state["ws"].data_ptr(), state["ws"].numel(), stream)
    return out


def run(state):
    if own:
        return _run_own(state)
    return {"write": _write, "read": _read, "attend": _attend}[state["case"]["op"]](state)


# ---- what a pass cannot do without -----------------------------------------------------------

def work(case):
    lens, new = _ints(case["lens"]), _ints(case["new"])
    D, Hk, Hq, T = case["dim"], case["kv_heads"], case["heads"], sum(new)
    stored = 2 * Hk * (D * _elem(case) + (0 if case["fmt"] == "same" else 4))  # one position, keys and values
    tables = 4 * (2 * len(lens) + 1 + sum(-(-l // case["page"]) for l in lens))
    if case["op"] != "attend":
        return {"bytes": T * (stored + 2 * Hk * D * 2) + tables, "flops": 4 * T * Hk * D}
    pairs = sum(n * (l - n) + n * (n + 1) // 2 for l, n in zip(lens, new))
    return {"bytes": sum(lens) * stored + 2 * T * Hq * D * 2 + tables, "flops": 4 * D * Hq * pairs}


# ---- the definition in 64 bits ----------------------------------------------------------------

def _unpack64(case, state, s, name, first, last):
    """Positions [first, last) of sequence s as [positions, H, D] in 64 bits, page by page."""
    P, D = case["page"], case["dim"]
    wide = case["fmt"] == "same"
    stored = _pages_of(case, state["pages"])
    out = []
    for j in range(first // P, -(-last // P)):
        page = int(state["table"][s, j])
        x = stored[name][page].double()
        H = x.shape[0]
        if name == "k":
            # [tile, block, group, position, part, 8] -> position, then dimension
            x = x.reshape(H, P // 16, D // (32 if wide else 64), 4, 16, 1 if wide else 2, 8)
            x = x.permute(1, 4, 0, 2, 5, 3, 6).reshape(P, H, D)
        else:
            # [tile, block, group, dimension, part, half, 4]: position 16 half + 4 group + last
            x = x.reshape(H, P // 32, D // (16 if wide else 32), 4, 16, 1 if wide else 2, 2, 4)
            x = x.permute(1, 6, 3, 7, 0, 2, 5, 4).reshape(P, H, D)
        if not wide:
            x = x * stored[name + "_scale"][page].double().T[:, :, None]
        out.append(x)
    return torch.cat(out)[first - first // P * P:][:last - first]


def exact(case, seed):
    state = prepare(case, seed)
    lens, new = state["lens"], state["new"]
    D, Hk, Hq, P = case["dim"], case["kv_heads"], case["heads"], case["page"]
    if case["op"] == "read":
        return {n: torch.cat([_unpack64(case, state, s, n, l - m, l) for s, (l, m) in enumerate(zip(lens, new))])
                .flatten(1) for n in ("k", "v")}
    if case["op"] == "write":
        # codes of 8 bits are whole steps of their scale, which 64 bits may take to the neighbour
        stored = {n: None for n in _pages_of(case, state["pages"])}
        w, first = Hk * D, Hq * D
        for n, at in (("k", first), ("v", first + w)):
            if case["fmt"] == "same":
                want = _pages_of(case, state["pages"])[n].double()
            else:
                want = _pages_of(case, state["pages"])[n + "_scale"].double()
            rows = state["qkv"][:, at:at + w].double().view(-1, Hk, D)
            t = 0
            for s, (l, m) in enumerate(zip(lens, new)):
                for j in range((l - m) // P, -(-l // P)):
                    page, lo, hi = int(state["table"][s, j]), max(l - m, j * P), min(l, (j + 1) * P)
                    part, o = rows[t + lo - (l - m):t + hi - (l - m)], lo - j * P
                    if case["fmt"] != "same":
                        want[page, :, o:o + hi - lo] = part.abs().amax(2).T / QMAX[case["fmt"]]
                        continue
                    if n == "k":
                        x = want[page].reshape(Hk, P // 16, D // 32, 4, 16, 8).permute(0, 1, 4, 2, 3, 5).reshape(Hk, P, D)
                        x[:, o:o + hi - lo] = part.transpose(0, 1)
                        x = x.view(Hk, P // 16, 16, D // 32, 4, 8).permute(0, 1, 3, 4, 2, 5)
                    else:
                        x = want[page].reshape(Hk, P // 32, D // 16, 4, 16, 2, 4).permute(0, 1, 5, 3, 6, 2, 4).reshape(Hk, P, D)
                        x[:, o:o + hi - lo] = part.transpose(0, 1)
                        x = x.view(Hk, P // 32, 2, 4, 4, D // 16, 16).permute(0, 1, 5, 3, 6, 2, 4)
                    want[page] = x.reshape(Hk, P * D)
                t += m
            stored[n if case["fmt"] == "same" else n + "_scale"] = want
        return stored
    out = torch.empty((state["T"], Hq, D), dtype=torch.float64, device="cuda")
    q = state["qkv"][:, :Hq * D].double().view(-1, Hq, D)
    at = 0
    for s, (l, n) in enumerate(zip(lens, new)):
        k, v = (_unpack64(case, state, s, name, 0, l) for name in ("k", "v"))
        hidden = torch.arange(l, device="cuda")[None] > torch.arange(l - n, l, device="cuda")[:, None]
        for h in range(Hq):
            score = (q[at:at + n, h] @ k[:, h // (Hq // Hk)].T) / math.sqrt(D)
            weight = score.masked_fill_(hidden, -math.inf).softmax(1)
            out[at:at + n, h] = weight @ v[:, h // (Hq // Hk)]
        at += n
    return out.flatten(1)
