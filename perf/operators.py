"""The operators of serving prompts of different lengths over a paged 8-bit KV cache, as measurable cases.

A server of block diffusion (or of single tokens) has prompts of every length in one batch, attends over them packed
(kind "prompt"), keeps the keys and values of the committed tokens in pages of 64 tokens as e4m3 with one scale per
page and head (kind "store": rows written into their pages and read back), attends from the active rows over those
pages (kind "attend"), forks sequences that share a prompt (kind "fork") and closes the gaps that finished sequences
leave in the pool (kind "compact").

``run`` computes each in elementary torch operations in 32 bits, or, where ``own`` is true, with the framework's
operators.  ``exact`` restates each from its definition in 64 bits.  Head counts and sizes are those of the presets in
``workloads``: tiny 4 heads of 64 (fp32), small 12 of 64, block 16 over 8 of 128, posttrain 32 over 16 of 128.
"""
from __future__ import annotations

import math
from types import SimpleNamespace

import torch

own = False

PAGE = 64                                   # tokens of a page
DIMS = {                                    # query heads, KV heads, head dim, layers, type of the activations
    "tiny": (4, 4, 64, 6, "f32"),
    "small": (12, 12, 64, 12, "bf16"),
    "block": (16, 8, 128, 22, "bf16"),
    "posttrain": (32, 16, 128, 62, "bf16"),
}
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16}


# ------------------------------------------------------------------ the cases
def listed():
    return [
        # Four short prompts of the fp32 model: the smallest packed call.
        {"name": "prompt_tiny_f32", "kind": "prompt", "dims": "tiny", "lens": "32,7,128,61", "window": 0},
        # Prefill of a serving batch of the block model: prompts of 1 to 512 tokens, packed.
        {"name": "prompt_block_ragged", "kind": "prompt", "dims": "block", "window": 0,
         "lens": "512,33,300,1,127,480,64,211,512,95,402,17,256,350,129,512,5,444,190,63,371,288,500,12"},
        # Prefill of the 27 B model with one long document among short prompts: the compute-bound case.
        {"name": "prompt_posttrain_long", "kind": "prompt", "dims": "posttrain", "lens": "8111,900,1,2500", "window": 0},
        # The same heads in a local layer: a sliding window of 1024 keys over prompts of a few thousand tokens.
        {"name": "prompt_posttrain_local", "kind": "prompt", "dims": "posttrain", "lens": "4096,1500,3333", "window": 1024},
        # One sequence, one token, a short context: the latency of a single decode call (heads of 64).
        {"name": "attend_small_token", "kind": "attend", "dims": "small", "rows": "1", "ctx": "700", "causal": True,
         "window": 0},
        # The serving batch of the block model: 32 sequences with 32 active rows each over contexts of 1 to 2000 tokens.
        {"name": "attend_block_step", "kind": "attend", "dims": "block", "causal": False, "window": 0,
         "rows": ",".join(["32"] * 32),
         "ctx": ",".join(str(v) for v in (512, 1999, 64, 1030, 1, 777, 1500, 320, 1984, 96, 1211, 640, 33, 1765, 900, 448,
                                          1337, 2000, 700, 128, 1601, 555, 1088, 250, 1900, 811, 416, 1440, 63, 975, 1152,
                                          1820))},
        # The 27 B model's block step over long documents: 8 sequences, contexts of 3000 to 30000 tokens.
        {"name": "attend_posttrain_step", "kind": "attend", "dims": "posttrain", "causal": False, "window": 0,
         "rows": ",".join(["32"] * 8), "ctx": "30000,4097,12345,3000,20011,8192,16000,6001"},
        # Single tokens over very long contexts, four sequences: the bytes of the cache are everything.
        {"name": "attend_block_long_tokens", "kind": "attend", "dims": "block", "causal": True, "window": 0,
         "rows": "1,1,1,1", "ctx": "131000,65537,100003,90000"},
        # One new token for each of 64 sequences, in the middle of their pages.
        {"name": "store_block_tokens", "kind": "store", "dims": "block", "rows": ",".join(["1"] * 64),
         "start": ",".join(str((37 * i * i + 11 * i) % 2000) for i in range(64))},
        # The keys and values of prompts of up to 2000 tokens, from the prefill into fresh pages; one continues a
        # sequence inside a page.
        {"name": "store_block_prompts", "kind": "store", "dims": "block", "rows": "2000,512,1,777,1500,64,333,1025",
         "start": "0,0,64,0,100,0,0,1"},
        # Sixteen prompts, each forked into three more branches (best of four): full pages are shared, the last page
        # of a prompt is copied in every layer.
        {"name": "fork_block_branches", "kind": "fork", "dims": "block", "seqs": 16, "branches": 3, "max_len": 1000,
         "spare": 8},
        # A pool of which finished sequences have left every other page empty: live pages move to the front.
        {"name": "compact_block_pool", "kind": "compact", "dims": "block", "pages": 384, "live": 0.5},
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _some(rng, n, lo, hi):
    return [_log(rng, lo, hi) for _ in range(n)]


def _text(values):
    return ",".join(str(v) for v in values)


def draw(rng):
    kind = rng.choice(["prompt", "prompt", "prompt", "attend", "attend", "attend", "attend", "store", "store", "fork",
                       "compact"])
    if kind == "prompt":
        dims = rng.choice(["tiny", "small", "block", "block", "posttrain"])
        if dims == "tiny":
            return {"kind": kind, "dims": dims, "lens": _text(_some(rng, rng.randint(1, 6), 1, 500)),
                    "window": rng.choice([0, 0, 50])}
        lens = _some(rng, _log(rng, 1, 24), 1, 4000)
        while sum(lens) > 9000:
            lens.pop()
        return {"kind": kind, "dims": dims, "lens": _text(lens), "window": rng.choice([0, 0, 0, 100, 1024])}
    if kind == "attend":
        dims = rng.choice(["tiny", "small", "block", "block", "posttrain"])
        batch = _log(rng, 1, 4 if dims == "tiny" else 40)
        most = rng.choice([1, 1, 8, 32, 32, 100])
        rows = [most if rng.random() < 0.7 else rng.randint(0, most) for _ in range(batch)]
        if not any(rows):
            rows[0] = most
        top = 600 if dims == "tiny" else max(200, min(100000, 200000 // batch))
        return {"kind": kind, "dims": dims, "rows": _text(rows), "ctx": _text(v - 1 for v in _some(rng, batch, 1, top)),
                "causal": rng.random() < 0.5, "window": rng.choice([0, 0, 0, 100, 1024])}
    if kind == "store":
        dims = rng.choice(["tiny", "small", "block", "block", "posttrain"])
        batch = _log(rng, 1, 64)
        most = rng.choice([1, 32, max(1, 8000 // batch)])
        rows = [most if most <= 32 else _log(rng, 1, most) for _ in range(batch)]
        return {"kind": kind, "dims": dims, "rows": _text(rows),
                "start": _text(rng.choice([0, v, v // PAGE * PAGE]) for v in _some(rng, batch, 1, 2000))}
    if kind == "fork":
        return {"kind": kind, "dims": rng.choice(["small", "block"]), "seqs": _log(rng, 1, 16),
                "branches": rng.randint(1, 4), "max_len": _log(rng, 50, 1500), "spare": rng.randint(0, 40)}
    return {"kind": kind, "dims": rng.choice(["small", "block"]), "pages": _log(rng, 20, 380),
            "live": round(rng.uniform(0.05, 0.95), 3)}


# ------------------------------------------------------------------ inputs
def _ints(text):
    return [int(v) for v in str(text).split(",")]


def _sum0(values):
    out = [0]
    for v in values:
        out.append(out[-1] + v)
    return out


def _i32(values):
    return torch.tensor(list(values), dtype=torch.int32, device="cuda")


def _pages(n):
    return (n + PAGE - 1) // PAGE


def _pow2(e):
    """2^e as fp32, for whole e between -126 and 127."""
    return ((e.to(torch.int32) + 127) << 23).view(torch.float32)


def _f8(x):
    """The values of e4m3 bytes in 32 bits."""
    return x.view(torch.float8_e4m3fn).float()


def _qkv(g, rows, heads, kv_heads, hd, dtype):
    """Q, K and V as a QKV projection leaves them: row-major slices of one buffer, a few channels of K larger than the
    others, as in trained heads."""
    x = torch.randn((rows, heads + 2 * kv_heads, hd), generator=g, device="cuda")
    x[:, heads:heads + kv_heads] *= torch.exp(0.5 * torch.randn((kv_heads, hd), generator=g, device="cuda"))
    x = x.to(dtype)
    return x[:, :heads], x[:, heads:heads + kv_heads], x[:, heads + kv_heads:]


def _pool(g, layers, pages, kv_heads, hd, key_gain=0.5):
    """A pool in use: e4m3 bytes of normal draws and their scales, powers of two that differ from page to page.
    K is [layers, pages, heads, 64, hd], V is transposed: [layers, pages, heads, hd, 64]."""
    def draws(shape):
        out = torch.empty(shape, dtype=torch.uint8, device="cuda")
        flat = out.view(-1)
        for at in range(0, flat.numel(), 1 << 28):        # in pieces: the 32-bit draws of a large pool would not fit
            n = min(1 << 28, flat.numel() - at)
            x = torch.randn(n, generator=g, device="cuda") * 80.0
            flat[at:at + n] = x.clamp_(-448.0, 448.0).to(torch.float8_e4m3fn).view(torch.uint8)
        return out

    def scales():
        return _pow2(torch.randint(-7, -5, (layers, pages, kv_heads), generator=g, device="cuda"))

    return SimpleNamespace(k=draws((layers, pages, kv_heads, PAGE, hd)), v=draws((layers, pages, kv_heads, hd, PAGE)),
                           k_scale=scales(), v_scale=scales())


def _scattered(g, counts, width, spare=0):
    """A page table [sequences, width] in which the pages of the sequences lie scattered over the pool; -1: none."""
    total = sum(counts)
    order = torch.randperm(total + spare, generator=g, device="cuda")[:total].to(torch.int32)
    table = torch.full((len(counts), width), -1, dtype=torch.int32, device="cuda")
    at = 0
    for b, n in enumerate(counts):
        table[b, :n] = order[at:at + n]
        at += n
    return table


def prepare(case, seed):
    heads, kv_heads, hd, layers, dtype = DIMS[case["dims"]]
    g = torch.Generator(device="cuda")
    g.manual_seed(int(seed))
    s = SimpleNamespace(case=case, heads=heads, kv_heads=kv_heads, hd=hd)
    kind = case["kind"]
    if kind == "prompt":
        lens = _ints(case["lens"])
        s.max_rows = max(lens)
        s.cu = _i32(_sum0(lens))
        s.q, s.k, s.v = _qkv(g, sum(lens), heads, kv_heads, hd, TYPES[dtype])
        s.o = torch.empty((sum(lens), heads, hd), dtype=s.q.dtype, device="cuda")
    elif kind == "attend":
        rows, ctx = _ints(case["rows"]), _ints(case["ctx"])
        lens = [r + c for r, c in zip(rows, ctx)]          # the active rows are the last ones of the cache
        s.max_rows, s.max_len = max(rows), max(lens)
        s.cu, s.lens = _i32(_sum0(rows)), _i32(lens)
        s.table = _scattered(g, [_pages(n) for n in lens], _pages(max(lens)) + 1, spare=3)
        s.pool = _pool(g, 1, sum(_pages(n) for n in lens) + 3, kv_heads, hd)
        s.q = _qkv(g, sum(rows), heads, kv_heads, hd, TYPES[dtype])[0]
        s.o = torch.empty((sum(rows), heads, hd), dtype=s.q.dtype, device="cuda")
    elif kind == "store":
        rows, start = _ints(case["rows"]), _ints(case["start"])
        ends = [r + c for r, c in zip(rows, start)]
        back = [r + c % PAGE for r, c in zip(rows, start)]  # read back from the start of the first page written
        s.max_rows, s.max_back = max(rows), max(back)
        s.cu, s.start = _i32(_sum0(rows)), _i32(start)
        s.cu_back, s.start_back = _i32(_sum0(back)), _i32(c - c % PAGE for c in start)
        s.table = _scattered(g, [_pages(n) for n in ends], _pages(max(ends)), spare=2)
        s.pool = _pool(g, 1, sum(_pages(n) for n in ends) + 2, kv_heads, hd)
        s.k, s.v = _qkv(g, sum(rows), heads, kv_heads, hd, TYPES[dtype])[1:]
        s.k_back = torch.empty((sum(back), kv_heads, hd), dtype=TYPES[dtype], device="cuda")
        s.v_back = torch.empty_like(s.k_back)
    elif kind == "fork":
        n, br = case["seqs"], case["branches"]
        lens = torch.randint(1, case["max_len"] + 1, (n,), generator=g, device="cuda").tolist()
        counts, width = [_pages(v) for v in lens], _pages(case["max_len"])
        pages = n * (width + br) + case["spare"]           # enough for the longest prompts
        s.table = torch.full((n * (br + 1), width), -1, dtype=torch.int32, device="cuda")
        s.table[:n] = _scattered(g, counts, width, spare=pages - sum(counts))
        s.lens = _i32(lens + [0] * (n * br))
        s.refs = torch.zeros(pages, dtype=torch.int32, device="cuda")
        s.refs[s.table[s.table >= 0].long()] = 1
        s.src = _i32(i % n for i in range(n * br))
        s.dst = _i32(n + i for i in range(n * br))
        s.pool = _pool(g, layers, s.refs.numel(), kv_heads, hd)
    else:
        pages = case["pages"]
        live = torch.rand(pages, generator=g, device="cuda") < case["live"]
        live[pages // 2] = True
        ids = torch.nonzero(live)[:, 0].to(torch.int32)
        ids = ids[torch.randperm(ids.numel(), generator=g, device="cuda")]
        width = 24
        s.table = torch.full((ids.numel() // width + 2, width), -1, dtype=torch.int32, device="cuda")
        s.table.view(-1)[:ids.numel()] = ids
        s.table[-1, :1] = s.table[0, :1]                    # a fork of the first sequence's first page
        s.refs = live.to(torch.int32)
        s.refs[s.table[0, 0].long()] += 1
        s.pool = _pool(g, layers, pages, kv_heads, hd)
    if kind in ("fork", "compact"):
        s.table_out, s.refs_out = torch.empty_like(s.table), torch.empty_like(s.refs)
        s.status = torch.zeros(1, dtype=torch.int32, device="cuda")
        if kind == "fork":
            s.lens_out = torch.empty_like(s.lens)
    if own:
        import paper_2609_37924_gb300.tadm as T
        s.T = T
        if kind == "prompt":
            return s
        s.handle = T.PagePool(s.pool.k, s.pool.v, s.pool.k_scale, s.pool.v_scale)
        if kind == "attend":
            need = T.tadm_page_attention_scratch_size(s.cu.numel() - 1, s.q.shape[0], s.max_rows, s.max_len, heads,
                                                      kv_heads, hd, 0 if dtype == "f32" else 1)
            s.scratch = torch.empty(max(need, 16), dtype=torch.uint8, device="cuda")
        elif kind in ("fork", "compact"):
            need = T.tadm_pages_scratch_size(s.refs.numel(), s.table.shape[0])
            s.scratch = torch.empty(max(need, 16), dtype=torch.uint8, device="cuda")
    return s


# ------------------------------------------------------------------ one pass
def run(s):
    kind, case = s.case["kind"], s.case
    if not own:
        return {"prompt": _plain_prompt, "attend": _plain_attend, "store": _plain_store, "fork": _plain_fork,
                "compact": _plain_compact}[kind](s)
    T = s.T
    if kind == "prompt":
        T.tadm_attention_packed(s.q, s.k, s.v, s.o, s.cu, s.max_rows, causal=True, window=case["window"])
        return s.o
    if kind == "attend":
        T.tadm_page_attention(s.q, s.handle, 0, s.o, s.cu, s.lens, s.table, s.max_rows, s.max_len, s.scratch,
                              causal=case["causal"], window=case["window"])
        return s.o
    if kind == "store":
        T.tadm_page_write(s.handle, 0, s.k, s.v, s.cu, s.start, s.table, s.max_rows)
        T.tadm_page_read(s.handle, 0, s.k_back, s.v_back, s.cu_back, s.start_back, s.table, s.max_back)
        return s.k_back, s.v_back
    if kind == "fork":
        T.tadm_pages_fork(s.handle, s.table, s.lens, s.refs, s.src, s.dst, s.table_out, s.lens_out, s.refs_out, s.status,
                          s.scratch)
        return _pages_out(s, s.lens_out)
    T.tadm_pages_compact(s.handle, s.table, s.refs, s.table_out, s.refs_out, s.status, s.scratch)
    return _pages_out(s, None)


def _pages_out(s, lens):
    p = s.pool
    out = {"table": s.table_out, "refs": s.refs_out, "status": s.status, "k": p.k.view(torch.float8_e4m3fn),
           "v": p.v.view(torch.float8_e4m3fn), "k_scale": p.k_scale, "v_scale": p.v_scale}
    if lens is not None:
        out["lens"] = lens
    return out


def _softmax_rows(x):
    """Softmax over the last axis; a row of -inf alone gives zeros."""
    m = x.amax(-1, keepdim=True)
    x = torch.exp(x.sub_(torch.where(torch.isfinite(m), m, torch.zeros_like(m))))
    return x.div_(x.sum(-1, keepdim=True).clamp_min(torch.finfo(x.dtype).tiny))


def _plain_prompt(s):
    """softmax(Q K^T / sqrt(hd)) V over the keys of a row's own sequence, up to itself, within the window."""
    rows, group, window = s.q.shape[0], s.heads // s.kv_heads, s.case["window"]
    q = s.q.float().transpose(0, 1).reshape(s.kv_heads, group * rows, s.hd)
    k, v = s.k.float().transpose(0, 1), s.v.float().transpose(0, 1)
    at = torch.arange(rows, device="cuda")
    seq = torch.searchsorted(s.cu[1:].contiguous().long(), at, right=True)
    see = (seq[:, None] == seq) & (at <= at[:, None])
    if window:
        see &= at[:, None] - at < window
    x = (torch.matmul(q, k.transpose(1, 2)) / math.sqrt(s.hd)).view(s.kv_heads, group, rows, rows)
    p = _softmax_rows(x.masked_fill_(~see, -math.inf))
    o = torch.matmul(p.view(s.kv_heads, group * rows, rows), v)
    s.o.copy_(o.view(s.heads, rows, s.hd).transpose(0, 1))
    return s.o


def _plain_values(p, table, pages):
    """K and V of the pages of every sequence: [sequences, heads, tokens, hd] in 32 bits."""
    at = table[:, :pages].clamp_min(0).long()
    k = _f8(p.k[0][at]) * p.k_scale[0][at][..., None, None]
    v = _f8(p.v[0][at]) * p.v_scale[0][at][..., None, None]
    n, h, hd = at.shape[0], k.shape[2], k.shape[4]
    return (k.permute(0, 2, 1, 3, 4).reshape(n, h, pages * PAGE, hd),
            v.permute(0, 2, 1, 4, 3).reshape(n, h, pages * PAGE, hd))


def _plain_attend(s):
    """softmax(Q K^T / sqrt(hd)) V over a sequence's pages; its rows are the last ones of its len tokens."""
    case, group = s.case, s.heads // s.kv_heads
    k, v = _plain_values(s.pool, s.table, _pages(s.max_len))
    n, keys = s.cu.numel() - 1, k.shape[2]
    r = torch.arange(s.max_rows, device="cuda")
    first, count = s.cu[:-1].long(), (s.cu[1:] - s.cu[:-1]).long()
    row = torch.where(r < count[:, None], first[:, None] + r, torch.zeros_like(r))
    q = s.q.float()[row].view(n, s.max_rows, s.kv_heads, group, s.hd).permute(0, 2, 3, 1, 4)
    x = torch.matmul(q.reshape(n, s.kv_heads, group * s.max_rows, s.hd), k.transpose(2, 3)) / math.sqrt(s.hd)
    x = x.view(n, s.kv_heads, group, s.max_rows, keys)
    j, pos = torch.arange(keys, device="cuda"), (s.lens.long() - count)[:, None] + r
    see = (j < s.lens[:, None, None]) & (r[:, None] < count[:, None, None])
    if case["causal"]:
        see = see & (j <= pos[..., None])
    if case["window"]:
        see = see & (pos[..., None] - j < case["window"])
    p = _softmax_rows(x.masked_fill_(~see[:, None, None], -math.inf))
    o = torch.matmul(p.view(n, s.kv_heads, group * s.max_rows, keys), v)
    o = o.view(n, s.heads, s.max_rows, s.hd).permute(0, 2, 1, 3)
    s.o.copy_(o[(r < count[:, None])])
    return s.o


def _needed_scale(amax):
    """The least power of two s, 2^-60 to 2^60, with amax <= 448 s."""
    frac, exp = torch.frexp(amax)                           # amax = frac 2^exp, 0.5 <= frac < 1
    e = exp - 9 + (frac > 0.875).to(exp.dtype)              # 448 = 0.875 * 2^9
    return _pow2(torch.where(amax > 0, e, torch.full_like(e, -60)).clamp_(-60, 60))


def _plain_store(s):
    """Rows into their pages as e4m3 x scale.  A page's scale is the larger of what its new rows need and, where it
    keeps earlier tokens, the one it has; kept tokens are re-encoded when the scale grows."""
    rows, n, width = s.k.shape[0], s.table.shape[0], s.table.shape[1]
    at = torch.arange(rows, device="cuda")
    seq = torch.searchsorted(s.cu[1:].contiguous().long(), at, right=True)
    pos = s.start.long()[seq] + at - s.cu.long()[seq]
    slot, place = pos % PAGE, seq * width + pos // PAGE
    page = s.table.view(-1)[place].long()
    first = (s.start.long() // PAGE).clamp_max(width - 1)
    old = s.table.gather(1, first[:, None])[:, 0].long().clamp_min(0)     # the first page that a sequence writes
    keeps = (s.start % PAGE != 0) & (s.cu[1:] > s.cu[:-1])
    kept = torch.arange(PAGE, device="cuda") < (s.start % PAGE)[:, None]  # [n, 64] its tokens that stay
    kept = kept & keeps[:, None]
    p, outs = s.pool, []
    for x, data, scale, token_last in ((s.k, p.k[0], p.k_scale[0], False), (s.v, p.v[0], p.v_scale[0], True)):
        x = x.float()
        amax = torch.zeros((n * width, s.kv_heads), device="cuda")
        amax.scatter_reduce_(0, place[:, None].expand(-1, s.kv_heads), x.abs().amax(-1), "amax")
        need = _needed_scale(amax)
        had = scale[old]                                                  # [n, heads]
        need = need.view(n, width, s.kv_heads)
        grown = torch.maximum(need.gather(1, first[:, None, None].expand(-1, 1, s.kv_heads))[:, 0], had)
        now = torch.where(keeps[:, None], grown, need.gather(1, first[:, None, None].expand(-1, 1, s.kv_heads))[:, 0])
        need.scatter_(1, first[:, None, None].expand(-1, 1, s.kv_heads), now[:, None])
        need = need.view(n * width, s.kv_heads)
        keep = _f8(data[old]) * (had / now)[..., None, None]             # [n, heads, 64, hd] or [n, heads, hd, 64]
        keep = (keep.transpose(2, 3) if token_last else keep).permute(0, 2, 1, 3)
        b, t = torch.nonzero(kept, as_tuple=True)
        new = (x / need[place][..., None]).to(torch.float8_e4m3fn).view(torch.uint8)
        keep = keep[b, t].to(torch.float8_e4m3fn).view(torch.uint8)
        if token_last:
            data[old[b], :, :, t] = keep
            data[page, :, :, slot] = new
        else:
            data[old[b], :, t] = keep
            data[page, :, slot] = new
        scale[page] = need[place]
    back = torch.arange(s.k_back.shape[0], device="cuda")
    seq = torch.searchsorted(s.cu_back[1:].contiguous().long(), back, right=True)
    pos = s.start_back.long()[seq] + back - s.cu_back.long()[seq]
    page, slot = s.table.view(-1)[seq * width + pos // PAGE].long(), pos % PAGE
    s.k_back.copy_(_f8(p.k[0][page, :, slot]) * p.k_scale[0][page][..., None])
    s.v_back.copy_(_f8(p.v[0][page, :, :, slot]) * p.v_scale[0][page][..., None])
    return s.k_back, s.v_back


def _plain_fork(s):
    """dst[i] becomes a copy of sequence src[i]: full pages are shared, a last page that is not full goes into the
    lowest free pages, in the order of the list."""
    src, dst = s.src.long(), s.dst.long()
    lens = s.lens[src]
    slot = torch.arange(s.table.shape[1], device="cuda")
    rows = torch.where(slot * PAGE < lens[:, None], s.table[src], torch.full_like(s.table[src], -1))
    part = lens % PAGE != 0
    free = torch.nonzero(s.refs == 0)[:, 0]
    rank = torch.cumsum(part.long(), 0) - 1
    who = torch.nonzero(part)[:, 0]
    last = (lens[who] // PAGE).long()
    old, new = rows[who, last].long(), free[rank[who]]
    s.refs_out.copy_(s.refs)
    rows[who, last] = new.to(torch.int32)
    whole = rows[(slot + 1) * PAGE <= lens[:, None]].long()
    s.refs_out.index_add_(0, whole, torch.ones_like(whole, dtype=torch.int32))
    s.refs_out[new] = 1
    s.table_out.copy_(s.table)
    s.table_out[dst] = rows
    s.lens_out.copy_(s.lens)
    s.lens_out[dst] = lens
    s.status.zero_()
    for x in (s.pool.k, s.pool.v, s.pool.k_scale, s.pool.v_scale):
        x[:, new] = x[:, old]
    return _pages_out(s, s.lens_out)


def _plain_compact(s):
    """The n pages in use move to the ids below n: the i-th of those above takes the i-th free one below."""
    live = s.refs > 0
    n = live.sum()
    ids = torch.arange(s.refs.numel(), device="cuda")
    holes, movers = torch.nonzero(~live & (ids < n))[:, 0], torch.nonzero(live & (ids >= n))[:, 0]
    to = ids.clone()
    to[movers] = holes
    s.table_out.copy_(torch.where(s.table >= 0, to[s.table.clamp_min(0).long()].to(torch.int32), s.table))
    s.refs_out.copy_(s.refs)
    s.refs_out[holes] = s.refs[movers]
    s.refs_out[movers] = 0
    s.status.copy_(n.to(torch.int32).view(1))
    for x in (s.pool.k, s.pool.v, s.pool.k_scale, s.pool.v_scale):
        x[:, holes] = x[:, movers]
    return _pages_out(s, None)


# ------------------------------------------------------------------ work
def _visible(rows, length, causal, window):
    """Keys that the last `rows` of `length` positions see, summed over the rows."""
    total = 0
    for r in range(rows):
        pos = length - rows + r
        hi = pos + 1 if causal else length
        total += max(0, hi - max(0, pos - window + 1 if window else 0))
    return total


def work(case):
    heads, kv_heads, hd, layers, dtype = DIMS[case["dims"]]
    es, kind = TYPES[dtype].itemsize, case["kind"]
    if kind == "prompt":
        lens = _ints(case["lens"])
        w = case["window"]
        pairs = sum(n * (n + 1) // 2 - (max(0, n - w) * (max(0, n - w) + 1) // 2 if w else 0) for n in lens)
        return {"bytes": 2 * sum(lens) * (heads + kv_heads) * hd * es, "flops": 4 * pairs * heads * hd}
    if kind == "attend":
        rows, ctx = _ints(case["rows"]), _ints(case["ctx"])
        pairs = sum(_visible(r, r + c, case["causal"], case["window"]) for r, c in zip(rows, ctx))
        keys = 0
        for r, c in zip(rows, ctx):
            keys += min(r + c, r + case["window"] - 1) if case["window"] and r else r + c if r else 0
        return {"bytes": keys * kv_heads * 2 * hd + 2 * sum(rows) * heads * hd * es, "flops": 4 * pairs * heads * hd}
    if kind == "store":
        rows, start = _ints(case["rows"]), _ints(case["start"])
        back = sum(r + c % PAGE for r, c in zip(rows, start))
        return {"bytes": 2 * kv_heads * hd * (sum(rows) * (es + 1) + back * (1 + es)), "flops": 0}
    page = layers * kv_heads * 2 * (PAGE * hd + 4)
    if kind == "fork":                                      # about one length in 64 ends with its page
        n = case["seqs"]
        return {"bytes": int(n * 63 / 64) * page * (1 + case["branches"]), "flops": 0}
    live = case["live"]
    return {"bytes": max(1, int(2 * case["pages"] * live * (1 - live))) * page, "flops": 0}


# ------------------------------------------------------------------ exact
def exact(case, seed):
    s = prepare(case, seed)
    kind = case["kind"]
    if kind == "prompt":
        return _exact_prompt(s)
    if kind == "attend":
        return _exact_attend(s)
    if kind == "store":
        return _exact_store(s)
    return _exact_pages(s)


def _exact_rows(q, k, v, pos, causal, window):
    """One head: rows q [r, hd] at positions pos over all keys of a sequence, in 64 bits."""
    out = torch.zeros_like(q)
    j = torch.arange(k.shape[0], device="cuda")
    for at in range(0, q.shape[0], 2048):
        x = q[at:at + 2048] @ k.T / math.sqrt(q.shape[1])
        p = pos[at:at + 2048, None]
        hide = torch.zeros_like(x, dtype=torch.bool)
        if causal:
            hide |= j > p
        if window:
            hide |= p - j >= window
        e = torch.exp(x.masked_fill(hide, -math.inf) - x.masked_fill(hide, -1e300).amax(1, keepdim=True))
        total = e.sum(1, keepdim=True)
        out[at:at + 2048] = torch.where(total > 0, e @ v / total.clamp_min(1e-300), torch.zeros_like(total))
    return out


def _exact_prompt(s):
    q, k, v = s.q.double(), s.k.double(), s.v.double()
    out, cu = torch.zeros_like(q), s.cu.tolist()
    for a, b in zip(cu[:-1], cu[1:]):
        pos = torch.arange(b - a, device="cuda")
        for h in range(s.heads):
            g = h * s.kv_heads // s.heads
            out[a:b, h] = _exact_rows(q[a:b, h], k[a:b, g], v[a:b, g], pos, True, s.case["window"])
    return out


def _exact_attend(s):
    out, cu, lens = s.q.double(), s.cu.tolist(), s.lens.tolist()
    out = torch.zeros_like(out)
    p = s.pool
    for b, n in enumerate(lens):
        at, to = cu[b], cu[b + 1]
        if at == to:
            continue
        ids = s.table[b, :_pages(n)].long()
        pos = torch.arange(n - (to - at), n, device="cuda")
        for g in range(s.kv_heads):
            k = _f8(p.k[0, ids, g]).double() * p.k_scale[0, ids, g].double()[:, None, None]
            v = _f8(p.v[0, ids, g]).double() * p.v_scale[0, ids, g].double()[:, None, None]
            k, v = k.reshape(-1, s.hd)[:n], v.transpose(1, 2).reshape(-1, s.hd)[:n]
            for h in range(g * s.heads // s.kv_heads, (g + 1) * s.heads // s.kv_heads):
                out[at:to, h] = _exact_rows(s.q[at:to, h].double(), k, v, pos, s.case["causal"], s.case["window"])
    return out


def _e4m3(x):
    """The nearest e4m3 value (ties to even) of x, |x| <= 448, in 64 bits: 3 bits after the leading one, and steps of
    2^-9 below 2^-6."""
    step = torch.exp2(torch.floor(torch.log2(x.abs().clamp_min(2.0 ** -6))) - 3)
    return torch.round(x / step) * step


def _exact_store(s):
    cu, start, width = s.cu.tolist(), s.start.tolist(), s.table.shape[1]
    outs = []
    for x, data, scale, token_last in ((s.k, s.pool.k[0], s.pool.k_scale[0], False),
                                       (s.v, s.pool.v[0], s.pool.v_scale[0], True)):
        x, parts = x.double(), []
        for b in range(len(start)):
            n, at = cu[b + 1] - cu[b], start[b]
            base = at - at % PAGE
            for first in range(base, at + n, PAGE):
                lo, hi = max(first, at), min(first + PAGE, at + n)
                new = x[cu[b] + lo - at:cu[b] + hi - at].transpose(0, 1)            # [heads, tokens, hd]
                amax = new.abs().amax((1, 2))
                e = torch.ceil(torch.log2((amax / 448.0).clamp_min(2.0 ** -60)))
                sc = torch.exp2(e.clamp(-60, 60))
                if lo > first:
                    page = int(s.table[b, first // PAGE])
                    had = scale[page].double()
                    sc = torch.maximum(sc, had)
                    f = _f8(data[page]).double()
                    f = f.transpose(1, 2) if token_last else f
                    kept = _e4m3(f[:, :lo - first] * (had / sc)[:, None, None]) * sc[:, None, None]
                    parts.append(kept.transpose(0, 1))
                parts.append((_e4m3(new / sc[:, None, None]) * sc[:, None, None]).transpose(0, 1))
        outs.append(torch.cat(parts))
    return tuple(outs)


def _exact_pages(s):
    table, refs = s.table.tolist(), s.refs.tolist()
    moves, out = {}, {}
    if s.case["kind"] == "fork":
        lens = s.lens.tolist()
        free = [i for i, r in enumerate(refs) if r == 0]
        for a, b in zip(s.src.tolist(), s.dst.tolist()):
            for j in range(_pages(lens[a])):
                table[b][j] = table[a][j]
                if (j + 1) * PAGE > lens[a]:
                    table[b][j] = free.pop(0)
                    moves[table[b][j]] = table[a][j]
                refs[table[b][j]] += 1
            lens[b] = lens[a]
        out["lens"] = _i32(lens)
        out["status"] = _i32([0])
    else:
        n = sum(r > 0 for r in refs)
        holes = [i for i in range(n) if refs[i] == 0]
        movers = [i for i in range(n, len(refs)) if refs[i] > 0]
        moves = dict(zip(holes, movers))
        to = {b: a for a, b in moves.items()}
        table = [[to.get(p, p) for p in row] for row in table]
        for a, b in moves.items():
            refs[a], refs[b] = refs[b], 0
        out["status"] = _i32([n])
    new, old = torch.tensor(list(moves), device="cuda").long(), torch.tensor(list(moves.values()), device="cuda").long()
    for name, x in (("k", s.pool.k), ("v", s.pool.v), ("k_scale", s.pool.k_scale), ("v_scale", s.pool.v_scale)):
        x[:, new] = x[:, old]
        out[name] = x if name.endswith("scale") else x.view(torch.float8_e4m3fn)
        out[name] = out[name].double()
    out["table"], out["refs"] = _i32(v for row in table for v in row).view(s.table.shape), _i32(refs)
    return out
