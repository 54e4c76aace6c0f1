"""Sequences of different lengths on the GPU: packed prompts, the paged 8-bit cache,
attention over it and its pages' bookkeeping, against plain definitions in 64 bits."""
import math

import numpy as np
import pytest

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")

PAGE = 64


@pytest.fixture(scope="module")
def T():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    import __graft_entry__ as g
    g.build()
    from paper_2609_37924_gb300 import tadm
    return tadm


def i32(v):
    return torch.tensor(list(v), dtype=torch.int32, device="cuda")


def cum(lens, first=0):
    out = [first]
    for n in lens:
        out.append(out[-1] + n)
    return out


def gen(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return g


def attend64(q, k, v, pos, causal, window):
    """q [r, Hq, hd] at positions pos, k, v [n, Hkv, hd], 64 bits: the output and sum_j p_j |v_j|; rows that see no
    key are zero."""
    group = q.shape[1] // k.shape[1]
    k, v = k.repeat_interleave(group, 1), v.repeat_interleave(group, 1)
    x = torch.einsum("rhd,nhd->hrn", q, k) / math.sqrt(q.shape[2])
    j, p = torch.arange(k.shape[0], device=q.device), pos[:, None]
    see = torch.ones((q.shape[0], k.shape[0]), dtype=torch.bool, device=q.device)
    if causal:
        see &= j <= p
    if window:
        see &= p - j < window
    e = torch.where(see, torch.exp(x - torch.where(see, x, -1e300).amax(-1, keepdim=True)), 0.0) if k.shape[0] else x
    w = e / e.sum(-1, keepdim=True).clamp_min(1e-300)
    return torch.einsum("hrn,nhd->rhd", w, v), torch.einsum("hrn,nhd->rhd", w, v.abs())


def close(got, ref, absum, dtype, v_max):
    """fp32: scores of up to a few tens carry an absolute error of some 1e-6, which scales the probabilities.  bf16:
    the probabilities' rounding (at most 2^-9 of each) and the output's (2^-9), and the fp32 path's error."""
    tol = 5e-5 * v_max + (2.0 ** -8 * absum if dtype == torch.bfloat16 else 0.0)
    err = (got.double() - ref).abs()
    assert torch.isfinite(got).all()
    assert (err <= tol).all(), (float(err.max()), float((err / (tol + 1e-30)).max()))


HEADS = [(4, 4, 64), (16, 8, 128), (6, 2, 64), (8, 1, 128), (5, 1, 64), (32, 16, 128), (14, 2, 128)]
LENS = [[1], [0, 5, 0, 130, 64, 1], [300, 1, 257, 63], [129, 128, 127, 2, 511], [700]]


# ------------------------------------------------------------------ packed prompts
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("heads", HEADS)
@pytest.mark.parametrize("lens", LENS)
@pytest.mark.parametrize("causal,window", [(True, 0), (False, 0), (True, 1), (True, 50), (False, 200)])
def test_packed_attention(T, dtype, heads, lens, causal, window):
    Hq, Hkv, hd = heads
    rows = sum(lens)
    x = torch.randn((rows, Hq + 2 * Hkv, hd), generator=gen(rows + Hq), device="cuda").to(dtype)
    q, k, v = x[:, :Hq], x[:, Hq:Hq + Hkv], x[:, Hq + Hkv:]
    o = torch.full((rows, Hq, hd), 7.0, dtype=dtype, device="cuda")
    T.tadm_attention_packed(q, k, v, o, i32(cum(lens)), max(lens), causal=causal, window=window)
    for a, n in zip(cum(lens), lens):
        s = slice(a, a + n)
        ref, absum = attend64(q[s].double(), k[s].double(), v[s].double(), torch.arange(n, device="cuda"), causal, window)
        if n:
            close(o[s], ref, absum, dtype, float(v[s].abs().max()))


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("causal", [True, False])
def test_packed_rows_outside_the_sequences(T, dtype, causal):
    """Rows before the first and after the last sequence, rows past max_rows, wider output rows: nothing of them is
    written, and nothing that they hold (NaN, infinities) reaches a row of a sequence; nor does another sequence."""
    Hq, Hkv, hd, lens = 4, 2, 64, [70, 33, 200]
    cu, total = cum(lens, first=3), 3 + sum(lens) + 5
    q, k, v = (torch.randn((total, h, hd), generator=gen(h + 1), device="cuda").to(dtype) for h in (Hq, Hkv, Hkv))
    for x in (q, k, v):
        x[:3] = math.nan
        x[-5:] = math.inf
    k[cu[1]:cu[2]], v[cu[1]:cu[2]] = math.nan, -math.inf       # the middle sequence is broken, its neighbours are not
    wide = torch.full((total, Hq * hd + 64), 7.0, dtype=dtype, device="cuda")
    o = wide[:, :Hq * hd].unflatten(1, (Hq, hd))
    T.tadm_attention_packed(q, k, v, o, i32(cu), 150, causal=causal)
    assert (wide[:, Hq * hd:] == 7.0).all() and (o[:3] == 7.0).all() and (o[-5:] == 7.0).all()
    assert (o[cu[2] + 150:cu[3]] == 7.0).all()
    for a, n in ((cu[0], 70), (cu[2], 150)):
        s = slice(a, a + n)
        ref, absum = attend64(q[s].double(), k[s].double(), v[s].double(), torch.arange(n, device="cuda"), causal, 0)
        close(o[s], ref, absum, dtype, float(v[s].abs().max()))


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_packed_large_scores(T, dtype):
    """Scores of several hundred, growing along the keys (every tile moves the running maximum) and falling."""
    n, H, hd = 900, 2, 128
    q, k, v = (torch.randn((n, H, hd), generator=gen(i), device="cuda") for i in range(3))
    ramp = torch.linspace(-1, 1, n, device="cuda")[:, None, None] * 3
    q[..., 0], k[:, 0, 0], k[:, 1, 0] = 400.0, ramp[:, 0, 0], -ramp[:, 0, 0]
    q, k, v = q.to(dtype), k.to(dtype), v.to(dtype)
    o = torch.empty_like(q)
    T.tadm_attention_packed(q, k, v, o, i32([0, n]), n, causal=False)
    ref, absum = attend64(q.double(), k.double(), v.double(), torch.arange(n, device="cuda"), False, 0)
    # scores up to 110: their fp32 error is a few 2^-24 of that, in a sum of 128 products
    tol = 4e-4 * float(v.abs().max()) + (2.0 ** -8 * absum if dtype == torch.bfloat16 else 0.0)
    assert ((o.double() - ref).abs() <= tol).all()


def test_packed_many_sequences(T):
    """More sequences than one warp scans at a time, most of them empty."""
    lens = [(7 * i) % 40 if i % 3 == 0 else 0 for i in range(200)]
    Hq, Hkv, hd, rows = 4, 2, 64, sum(lens)
    q, k, v = (torch.randn((rows, h, hd), generator=gen(h), device="cuda").bfloat16() for h in (Hq, Hkv, Hkv))
    o = torch.empty_like(q)
    T.tadm_attention_packed(q, k, v, o, i32(cum(lens)), max(lens))
    for a, n in zip(cum(lens), lens):
        s = slice(a, a + n)
        if n:
            ref, absum = attend64(q[s].double(), k[s].double(), v[s].double(), torch.arange(n, device="cuda"), True, 0)
            close(o[s], ref, absum, torch.bfloat16, float(v[s].abs().max()))


@pytest.mark.parametrize("heads", [(16, 8, 128), (12, 12, 64), (15, 3, 128), (10, 2, 64)])
@pytest.mark.parametrize("causal,window", [(True, 0), (True, 130), (False, 0)])
def test_packed_more_work_than_blocks_run(T, heads, causal, window):
    """More row tiles than the SMs take at a time, so that blocks go on with others' work, over more sequences than one warp
    scans at a time; every call gives the same bits, also on two streams at once."""
    Hq, Hkv, hd = heads
    lens = [(37 * i * i + 5 * i) % 600 if i % 5 else (i * 13) % 3 for i in range(75)] + [1500, 1]
    rows = sum(lens)
    x = torch.randn((rows, Hq + 2 * Hkv, hd), generator=gen(rows + Hq), device="cuda").bfloat16()
    q, k, v = x[:, :Hq], x[:, Hq:Hq + Hkv], x[:, Hq + Hkv:]
    outs = [torch.full((rows, Hq, hd), 7.0, dtype=torch.bfloat16, device="cuda") for _ in range(6)]
    streams, cu = [torch.cuda.Stream() for _ in range(2)], i32(cum(lens))
    torch.cuda.synchronize()
    for i, o in enumerate(outs):
        T.tadm_attention_packed(q, k, v, o, cu, max(lens), causal=causal, window=window, stream=streams[i % 2] if i > 1 else None)
    torch.cuda.synchronize()
    for o in outs[1:]:
        assert torch.equal(o, outs[0])
    for a, n in zip(cum(lens), lens):
        if n:
            s = slice(a, a + n)
            ref, absum = attend64(q[s].double(), k[s].double(), v[s].double(), torch.arange(n, device="cuda"), causal, window)
            close(outs[0][s], ref, absum, torch.bfloat16, float(v[s].abs().max()))


# ------------------------------------------------------------------ the cache
def e4m3_bytes(x):
    """Nearest e4m3 (ties to even) of float64 |x| <= 448, as bytes; NaN for what is not finite."""
    grid = torch.arange(127, dtype=torch.uint8).view(torch.float8_e4m3fn).double().numpy()   # 0 .. 448, ascending
    a = np.abs(x)
    at = np.clip(np.searchsorted(grid, a), 1, 126)
    lo, hi = grid[at - 1], grid[at]
    up = (a - lo > hi - a) | ((a - lo == hi - a) & (at % 2 == 0))
    code = np.where(up, at, at - 1).astype(np.uint8)
    out = code | np.where(np.signbit(x), 0x80, 0).astype(np.uint8)
    return np.where(np.isfinite(x), out, 0x7F).astype(np.uint8)


class Cache64:
    """What page_write has to leave in the pages: bytes of tokens and scales."""

    def __init__(self, pages, heads, hd):
        self.q = np.zeros((pages, heads, PAGE, hd), np.uint8)
        self.s = np.zeros((pages, heads), np.float64)

    def values(self, page):
        f = torch.from_numpy(self.q[page]).view(torch.float8_e4m3fn).double().numpy()
        return f * self.s[page][:, None, None]

    def write(self, x, start, row):
        n = x.shape[0]
        for first in range(start // PAGE * PAGE, start + n, PAGE):
            page, lo, hi = row[first // PAGE], max(first, start), min(first + PAGE, start + n)
            new = x[lo - start:hi - start].transpose(1, 0, 2)
            for h in range(x.shape[1]):
                a = np.abs(new[h][np.isfinite(new[h])])
                amax = a.max() if a.size else 0.0
                e = -60
                while e < 60 and amax > 448.0 * 2.0 ** e:
                    e += 1
                s = 2.0 ** e
                if lo > first:
                    s = max(s, self.s[page, h])
                    old = torch.from_numpy(self.q[page, h, :lo - first]).view(torch.float8_e4m3fn).double().numpy()
                    self.q[page, h, :lo - first] = e4m3_bytes(old * (self.s[page, h] / s))
                else:
                    self.q[page, h] = 0
                self.q[page, h, lo - first:hi - first] = e4m3_bytes(new[h] / s)
                self.s[page, h] = s


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("heads,hd", [(3, 64), (8, 128)])
def test_page_write_and_read(T, dtype, heads, hd):
    """Fresh pages, rows inside a page, a scale that grows, single tokens, a sequence without rows, all-zero rows,
    infinities and NaN: every byte and scale equal to the definition's; pages not named stay as they were."""
    pages, width = 40, 6
    pool = T.PagePool.empty(2, pages, heads, hd)
    pool.k.random_(generator=gen(5)), pool.v.random_(generator=gen(6))
    before = pool.k.clone(), pool.v.clone()
    order = torch.randperm(pages, generator=gen(7), device="cuda")[:24].cpu().numpy().reshape(4, width)
    table = torch.from_numpy(order.astype(np.int32)).cuda()
    ref = [Cache64(pages, heads, hd), Cache64(pages, heads, hd)]
    steps = [([0, 0, 0, 0], [130, 0, 64, 1], 1.0), ([130, 0, 64, 1], [1, 1, 1, 1], 30.0), ([131, 1, 65, 2], [40, 63, 200, 1], 0.1),
             ([171, 64, 265, 3], [100, 1, 0, 61], 3.0), ([64, 0, 128, 0], [7, 3, 1, 70], 1e-30)]
    for i, (start, rows, size) in enumerate(steps):
        x = torch.randn((sum(rows), 3 * heads, hd), generator=gen(i), device="cuda") * size
        if i == 2:
            x[5, :, 3], x[9, :, 1], x[11] = math.inf, math.nan, 0.0
        if i == 3:
            x[:100] = 0.0
        x = x.to(dtype)
        kv = x[:, heads:2 * heads], x[:, 2 * heads:]
        T.tadm_page_write(pool, 1, *kv, i32(cum(rows)), i32(start), table, max(rows))
        for b in range(4):
            for c in range(2):
                ref[c].write(kv[c][cum(rows)[b]:cum(rows)[b + 1]].cpu().to(torch.float64).numpy(), start[b], order[b])
        ends = [max(0, s + n) for s, n in zip(start, rows)]
        for c, (data, scale) in enumerate(((pool.k, pool.k_scale), (pool.v, pool.v_scale))):
            got = (data[1] if c == 0 else data[1].transpose(2, 3)).cpu().numpy()
            for b in range(4):
                for t in range(0, ends[b], PAGE):
                    n, p = min(PAGE, ends[b] - t), order[b, t // PAGE]
                    assert (got[p, :, :n] & 0x7F == ref[c].q[p, :, :n] & 0x7F).all(), (i, c, b, t)
                    same = got[p, :, :n] == ref[c].q[p, :, :n]
                    assert (same | (got[p, :, :n] & 0x7F == 0x7F)).all()             # the sign of a NaN is free
                    assert (scale[1, p].cpu().numpy() == ref[c].s[p]).all()
        back = [torch.empty((sum(ends), heads, hd), dtype=dtype, device="cuda") for _ in range(2)]
        T.tadm_page_read(pool, 1, *back, i32(cum(ends)), i32([0] * 4), table, max(ends))
        for c in range(2):
            got = back[c].double().cpu().numpy()
            for b in range(4):
                for t in range(0, ends[b], PAGE):
                    n = min(PAGE, ends[b] - t)
                    want = ref[c].values(order[b, t // PAGE])[:, :n].transpose(1, 0, 2)
                    a = cum(ends)[b] + t
                    # powers of two: exact, but for products below the type's normal range
                    assert np.array_equal(got[a:a + n], np.where(np.abs(want) < 2.0 ** -126, got[a:a + n], want), equal_nan=True)
    unused = np.setdiff1d(np.arange(pages), order)
    assert torch.equal(pool.k[0], before[0][0]) and torch.equal(pool.v[0], before[1][0])
    assert torch.equal(pool.k[1][unused], before[0][1][unused]) and torch.equal(pool.v[1][unused], before[1][1][unused])


def test_page_rows_skip_what_the_table_lacks(T):
    """A page id out of range is not followed: its tokens are not written and read as zeros; strided reads leave the
    columns between rows alone."""
    pool = T.PagePool.empty(1, 3, 2, 64)
    x = torch.ones((150, 2, 64), device="cuda")
    table = i32([2, -1, 1]).view(1, 3)
    T.tadm_page_write(pool, 0, x, x, i32([0, 150]), i32([0]), table, 150)
    table[0, 0] = 3
    wide = torch.full((150, 2, 2, 64), 7.0, device="cuda")
    T.tadm_page_read(pool, 0, wide[:, 0], wide[:, 1], i32([0, 150]), i32([0]), table, 150)
    assert (wide[:128] == 0).all() and (wide[128:] == 1).all()
    assert (pool.k[0, 0] == 0).all() and (pool.k[0, 2] != 0).all()


# ------------------------------------------------------------------ attention over the cache
def filled(T, lens, heads, hd, seed, spread=6, nan_tail=True):
    """A pool whose scattered pages hold draws, scales 2^-6 2^(0 .. spread) 1 .. 2, NaN in every slot past a sequence's length and in
    pages of nobody; the values of each sequence in 64 bits."""
    counts = [-(-n // PAGE) for n in lens]
    pages, width, g = sum(counts) + 3, max(counts + [1]) + 1, gen(seed)
    f8 = lambda shape: (torch.randn(shape, generator=g, device="cuda") * 60).clamp(-448, 448).to(torch.float8_e4m3fn)  # noqa: E731
    k, v = f8((2, pages, heads, PAGE, hd)).view(torch.uint8), f8((2, pages, heads, hd, PAGE)).view(torch.uint8)
    scale = lambda: torch.exp2(torch.rand((2, pages, heads), generator=g, device="cuda") - 6 +  # noqa: E731
                               torch.randint(0, spread + 1, (2, pages, heads), generator=g, device="cuda"))
    ks, vs = scale(), scale()
    ks = ks * 2.0 ** -spread                       # scores of a few units
    order = torch.randperm(pages, generator=g, device="cuda").tolist()
    table = torch.full((len(lens), width), -1, dtype=torch.int32, device="cuda")
    at, seqs = 0, []
    for b, n in enumerate(lens):
        mine = order[at:at + counts[b]]
        at += counts[b]
        if mine:
            table[b, :len(mine)] = i32(mine)
            kk = k[1, mine].view(torch.float8_e4m3fn).double() * ks[1, mine].double()[..., None, None]
            vv = v[1, mine].view(torch.float8_e4m3fn).double() * vs[1, mine].double()[..., None, None]
            seqs.append((kk.permute(0, 2, 1, 3).reshape(-1, heads, hd)[:n], vv.permute(0, 3, 1, 2).reshape(-1, heads, hd)[:n]))
            if nan_tail and n % PAGE:
                k[1, mine[-1], :, n % PAGE:] = 0x7F
                v[1, mine[-1], :, :, n % PAGE:] = 0xFF
        else:
            seqs.append((torch.zeros((0, heads, hd), dtype=torch.float64, device="cuda"),) * 2)
    for p in order[at:]:
        k[:, p], v[:, p], ks[:, p], vs[:, p] = 0x7F, 0x7F, math.nan, math.nan
    return T.PagePool(k, v, ks, vs), table, seqs


def run_paged(T, pool, table, q, cu, lens, max_rows, max_len, causal, window, fill=7.0):
    batch = len(cu) - 1
    wide = torch.full((q.shape[0], q.shape[1] * q.shape[2] + 64), fill, dtype=q.dtype, device="cuda")
    o = wide[:, :-64].unflatten(1, q.shape[1:])
    n = T.tadm_page_attention_scratch_size(batch, q.shape[0], max_rows, max_len, q.shape[1], pool.n_kv_heads, q.shape[2],
                                           1 if q.dtype == torch.bfloat16 else 0)
    scratch = torch.full((n + 64,), 0xFF, dtype=torch.uint8, device="cuda")
    T.tadm_page_attention(q, pool, 1, o, i32(cu), i32(lens), table, max_rows, max_len, scratch[:n], causal=causal,
                          window=window)
    assert (scratch[n:] == 0xFF).all() and (wide[:, -64:] == fill).all()
    return o


PAGED = [([1], [1]), ([1, 1, 1, 1, 1], [64, 1, 700, 129, 63]), ([32] * 4, [32, 33, 1000, 128]), ([0, 3, 0, 70, 1], [5, 3, 0, 70, 2000]),
         ([5, 4, 3], [0, 2, 64]), ([200, 1], [200, 3000]), ([100, 33, 7], [517, 40, 1025])]


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("heads", HEADS)
@pytest.mark.parametrize("rows,lens", PAGED)
@pytest.mark.parametrize("causal,window", [(True, 0), (False, 0), (True, 1), (True, 50), (False, 200)])
def test_page_attention(T, dtype, heads, rows, lens, causal, window):
    """Single tokens, blocks, chunks; empty sequences and sequences shorter than their rows (rows that see nothing are
    zero); pages that end inside a tile, with NaN behind the end."""
    Hq, Hkv, hd = heads
    pool, table, seqs = filled(T, lens, Hkv, hd, sum(lens) + Hq)
    q = torch.randn((sum(rows), 2 * Hq, hd), generator=gen(9), device="cuda").to(dtype)[:, Hq:]
    o = run_paged(T, pool, table, q, cum(rows), lens, max(rows), max(lens), causal, window)
    for b, n in enumerate(rows):
        if n == 0:
            continue
        s = slice(cum(rows)[b], cum(rows)[b] + n)
        k, v = seqs[b]
        pos = torch.arange(lens[b] - n, lens[b], device="cuda")
        if lens[b] == 0:
            assert (o[s] == 0).all()
            continue
        ref, absum = attend64(q[s].double(), k, v, pos, causal, window)
        close(o[s], ref, absum, dtype, float(v.abs().max()))


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_page_attention_limits(T, dtype):
    """max_len below a length leaves the later tokens out, max_rows the later rows; a page id out of range reads as
    zeros; scales 2^40 apart; values of one key only; a query of zeros."""
    Hq, Hkv, hd, lens, rows = 8, 4, 128, [600, 200, 64], [4, 9, 1]
    pool, table, seqs = filled(T, lens, Hkv, hd, 3, nan_tail=False)
    q = torch.randn((sum(rows), Hq, hd), generator=gen(4), device="cuda").to(dtype)
    q[-1] = 0.0
    o = run_paged(T, pool, table, q, cum(rows), lens, 8, 333, False, 0)
    assert (o[4 + 8:13] == 7.0).all()
    for b, (n, m) in enumerate(((4, 333), (8, 200), (1, 64))):
        s = slice(cum(rows)[b], cum(rows)[b] + n)
        k, v = (x[:m] for x in seqs[b])
        ref, absum = attend64(q[s].double(), k, v, torch.zeros(n, device="cuda"), False, 0)
        close(o[s], ref, absum, dtype, float(v.abs().max()))
    # a page that is not there: keys and values of zero
    bad = table.clone()
    bad[0, 2] = pool.pages + 7
    k, v = (x.clone() for x in seqs[0])
    k[128:192], v[128:192] = 0.0, 0.0
    o = run_paged(T, pool, bad, q[:4], [0, 4], [600], 4, 600, False, 0)
    ref, absum = attend64(q[:4].double(), k, v, torch.zeros(4, device="cuda"), False, 0)
    close(o, ref, absum, dtype, float(v.abs().max()))
    # V scales 2^40 apart: the small pages count where they hold all the weight
    page = table[0].tolist()
    pool.v_scale[1, page[3]] *= 2.0 ** 40
    v = seqs[0][1].clone()
    v[192:256] *= 2.0 ** 40
    o = run_paged(T, pool, table, q[:4], [0, 4], [600], 4, 600, False, 0)
    ref, absum = attend64(q[:4].double(), seqs[0][0], v, torch.zeros(4, device="cuda"), False, 0)
    close(o, ref, absum, dtype, float(v.abs().max()))
    o = run_paged(T, pool, table, q[:4], [0, 4], [192], 4, 600, False, 0)
    ref, absum = attend64(q[:4].double(), seqs[0][0][:192], v[:192], torch.zeros(4, device="cuda"), False, 0)
    close(o, ref, absum, dtype, float(v[:192].abs().max()))


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("heads", HEADS)
@pytest.mark.parametrize("causal,window", [(True, 1), (True, 70), (False, 150)])
def test_page_attention_behind_window(T, dtype, heads, causal, window):
    """Keys that the window hides from every row of a sequence reach none, whatever they, their page's scales or their table
    entry hold."""
    Hq, Hkv, hd = heads
    rows, lens = [1, 32, 5], [700, 1000, 389]
    pool, table, seqs = filled(T, lens, Hkv, hd, 21)
    q = torch.randn((sum(rows), Hq, hd), generator=gen(22), device="cuda").to(dtype)
    for b, n in enumerate(rows):
        lo = lens[b] - n - window + 1                # the first row's first key
        page = int(table[b, lo // PAGE])
        pool.k[1, page, :, :lo % PAGE] = 0x7F
        pool.v[1, page, :, :, :lo % PAGE] = 0xFF
        gone = table[b, :lo // PAGE].long()
        pool.k[1, gone], pool.v[1, gone], pool.k_scale[1, gone], pool.v_scale[1, gone] = 0x7F, 0x7F, math.nan, math.inf
        table[b, :lo // PAGE:2] = -1
    o = run_paged(T, pool, table, q, cum(rows), lens, max(rows), max(lens), causal, window)
    for b, n in enumerate(rows):
        s, (k, v) = slice(cum(rows)[b], cum(rows)[b] + n), seqs[b]
        ref, absum = attend64(q[s].double(), k, v, torch.arange(lens[b] - n, lens[b], device="cuda"), causal, window)
        close(o[s], ref, absum, dtype, float(v.abs().max()))


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("window", [2 ** 31 - 1, 300, 299, 40])
def test_windows_as_long_as_the_context(T, dtype, window):
    """Windows about the length of the longest context and the longest possible one, where some sequences are shorter than
    their rows (positions below zero)."""
    Hq, Hkv, hd, rows, lens = 8, 4, 64, [33, 5, 40, 2], [300, 2, 17, 0]
    pool, table, seqs = filled(T, lens, Hkv, hd, 31)
    q = torch.randn((sum(rows), Hq, hd), generator=gen(32), device="cuda").to(dtype)
    for causal in (True, False):
        o = run_paged(T, pool, table, q, cum(rows), lens, max(rows), max(lens), causal, window)
        for b, n in enumerate(rows):
            s, (k, v) = slice(cum(rows)[b], cum(rows)[b] + n), seqs[b]
            if lens[b] == 0:
                assert (o[s] == 0).all()
                continue
            ref, absum = attend64(q[s].double(), k, v, torch.arange(lens[b] - n, lens[b], device="cuda"), causal, window)
            close(o[s], ref, absum, dtype, float(v.abs().max()))
        k, v = (torch.randn((sum(rows), Hkv, hd), generator=gen(33 + i), device="cuda").to(dtype) for i in range(2))
        o = torch.empty_like(q)
        T.tadm_attention_packed(q, k, v, o, i32(cum(rows)), max(rows), causal=causal, window=window)
        for b, n in enumerate(rows):
            s = slice(cum(rows)[b], cum(rows)[b] + n)
            ref, absum = attend64(q[s].double(), k[s].double(), v[s].double(), torch.arange(n, device="cuda"), causal, window)
            close(o[s], ref, absum, dtype, float(v.abs().max()))


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("rows", [1, 32])
def test_page_attention_sink(T, dtype, rows):
    """One key holds nearly all the weight and a zero value; the rest of a long context, each key 2^-20 of it, makes
    the output: small probabilities are not lost."""
    n, Hq, Hkv, hd = 20000, 4, 2, 64
    pool, table, seqs = filled(T, [n], Hkv, hd, 8, spread=0)
    page = int(table[0, 0])
    q = torch.randn((rows, Hq, hd), generator=gen(2), device="cuda") * 0.05
    q[..., 0] = 8.0
    q = q.to(dtype)
    k, v = (x.clone() for x in seqs[0])
    kb = pool.k[1].view(torch.float8_e4m3fn)
    pool.k[1, table[0, :-1].long(), :, :, 0] = 0                     # dim 0: zero but for key 0
    pool.k_scale[1, page] = 2.0 ** -4
    pool.k[1, page, :, 0, 0] = torch.tensor(224.0).to(torch.float8_e4m3fn).view(torch.uint8).item()   # 14: score 8 * 14 / 8
    pool.v[1, page, :, :, 0] = 0
    kk = (kb[page].double() * pool.k_scale[1, page].double()[:, None, None]).transpose(0, 1)
    k[:, :, 0] = 0
    k[:PAGE] = kk[:min(PAGE, n)]
    v[0] = 0
    o = run_paged(T, pool, table, q, [0, rows], [n], rows, n, False, 0)
    ref, absum = attend64(q.double(), k, v, torch.zeros(rows, device="cuda"), False, 0)
    err = float((o.double() - ref).norm() / ref.norm())
    # rounding to bf16 once for the probabilities and once for the output; fp32 sums of 20000 terms
    assert err < (4e-3 if dtype == torch.bfloat16 else 2e-4), err


def test_page_attention_streams(T):
    """On a stream of its own, behind work of that stream, twice with one scratch; the same bits both times."""
    pool, table, seqs = filled(T, [3000, 100], 4, 128, 12)
    q = torch.randn((64, 8, 128), generator=gen(1), device="cuda").bfloat16()
    n = T.tadm_page_attention_scratch_size(2, 64, 32, 3000, 8, 4, 128, 1)
    scratch, s = torch.empty(max(n, 16), dtype=torch.uint8, device="cuda"), torch.cuda.Stream()
    outs = [torch.empty_like(q) for _ in range(3)]
    args = i32([0, 32, 64]), i32([3000, 100]), table, 32, 3000, scratch
    torch.cuda.synchronize()
    with torch.cuda.stream(s):
        late = torch.empty_like(q)
        late.copy_(q)
        for o in outs[:2]:
            T.tadm_page_attention(late, pool, 1, o, *args)
    T.tadm_page_attention(late, pool, 1, outs[2], *args, stream=s)
    s.synchronize()
    assert torch.equal(outs[0], outs[1]) and torch.equal(outs[0], outs[2])
    ref, absum = attend64(q[:32].double(), *seqs[0], torch.zeros(32, device="cuda"), False, 0)
    close(outs[0][:32], ref, absum, torch.bfloat16, float(seqs[0][1].abs().max()))


@pytest.mark.parametrize("heads,rows,lens", [((32, 16, 128), [200, 1], [200, 3000]), ((32, 16, 128), [100, 33, 7], [517, 40, 1025]),
                                             ((4, 2, 64), [1] * 5, [64, 1, 700, 129, 63])])
def test_page_attention_repeats(T, heads, rows, lens):
    """The same bits on every call: items of several tiles, split between CTAs, one behind the other."""
    Hq, Hkv, hd = heads
    pool, table, seqs = filled(T, lens, Hkv, hd, 5)
    q = torch.randn((sum(rows), Hq, hd), generator=gen(9), device="cuda").bfloat16()
    o, first = torch.empty_like(q), run_paged(T, pool, table, q, cum(rows), lens, max(rows), max(lens), False, 0)
    scratch = torch.empty(T.tadm_page_attention_scratch_size(len(rows), sum(rows), max(rows), max(lens), Hq, Hkv, hd, 1),
                          dtype=torch.uint8, device="cuda")
    args = i32(cum(rows)), i32(lens), table, max(rows), max(lens), scratch
    differ = torch.zeros((), dtype=torch.int64, device="cuda")
    for _ in range(300):
        T.tadm_page_attention(q, pool, 1, o, *args)
        differ += (o != first).sum()
    assert int(differ) == 0


# ------------------------------------------------------------------ bookkeeping
class Pages:
    """The bookkeeping in plain Python."""

    def __init__(self, table, lens, refs):
        self.table, self.lens, self.refs = [list(r) for r in table], list(lens), list(refs)

    def held(self, s):
        return [p for p in self.table[s] if p >= 0]

    def free(self):
        return [i for i, r in enumerate(self.refs) if r == 0]

    def reserve(self, seqs, new):
        free = self.free()
        for s, n in zip(seqs, new):
            for j in range(len(self.held(s)), -(-n // PAGE)):
                if not free:
                    return 1
                self.table[s][j] = free.pop(0)
                self.refs[self.table[s][j]] = 1
        return 0

    def fork(self, src, dst):
        free, moves = self.free(), []
        for a, b in zip(src, dst):
            n = self.lens[a]
            for j in range(-(-n // PAGE)):
                p = self.table[a][j]
                if (j + 1) * PAGE > n:
                    if not free:
                        return 1, []
                    moves.append((p, free.pop(0)))
                    p = moves[-1][1]
                self.table[b][j] = p
                self.refs[p] += 1
            self.lens[b] = n
        return 0, moves

    def release(self, seqs):
        for s in seqs:
            for p in self.held(s):
                self.refs[p] -= 1
            self.table[s], self.lens[s] = [-1] * len(self.table[s]), 0

    def compact(self):
        live = [i for i, r in enumerate(self.refs) if r > 0]
        n = len(live)
        holes, movers = [i for i in range(n) if self.refs[i] == 0], [i for i in live if i >= n]
        to = dict(zip(movers, holes))
        for a, b in to.items():
            self.refs[b], self.refs[a] = self.refs[a], 0
        self.table = [[to.get(p, p) for p in r] for r in self.table]
        return n, list(to.items())


class Device:
    """The same state on the device, with calls out of place or in place."""

    def __init__(self, T, pages, n_seqs, width, in_place, layers=2, heads=3, hd=64):
        self.T, self.in_place = T, in_place
        self.pool = T.PagePool.empty(layers, pages, heads, hd)
        for i, x in enumerate((self.pool.k, self.pool.v)):
            x.random_(generator=gen(20 + i))
        for i, x in enumerate((self.pool.k_scale, self.pool.v_scale)):
            x.uniform_(generator=gen(30 + i))
        self.table = torch.full((n_seqs, width), -1, dtype=torch.int32, device="cuda")
        self.lens, self.refs = i32([0] * n_seqs), i32([0] * pages)
        self.status = i32([77])
        self.scratch = torch.full((T.tadm_pages_scratch_size(pages, n_seqs) + 64,), 0xEE, dtype=torch.uint8, device="cuda")

    def call(self, name, *args, pool=False, lens=True):
        state = [self.table, self.lens, self.refs] if lens else [self.table, self.refs]
        out = state if self.in_place else [torch.full_like(x, -9) for x in state]
        kept = [x.clone() for x in state]
        head = (self.pool,) if pool else ()
        getattr(self.T, name)(*head, *state, *args, *out, self.status, self.scratch[:-64])
        assert (self.scratch[-64:] == 0xEE).all()
        if not self.in_place:
            assert all(torch.equal(a, b) for a, b in zip(state, kept))
        if lens:
            self.table, self.lens, self.refs = out
        else:
            self.table, self.refs = out
        return int(self.status)

    def same(self, m):
        assert self.table.tolist() == m.table and self.lens.tolist() == m.lens and self.refs.tolist() == m.refs

    def contents(self):
        return [x.clone() for x in (self.pool.k, self.pool.v, self.pool.k_scale, self.pool.v_scale)]

    def moved(self, before, moves):
        for x, b in zip((self.pool.k, self.pool.v, self.pool.k_scale, self.pool.v_scale), before):
            want = b.clone()
            for a, c in moves:
                want[:, c] = b[:, a]
            assert torch.equal(x, want)


@pytest.mark.parametrize("in_place", [False, True])
@pytest.mark.parametrize("pages,n_seqs,width", [(60, 12, 9), (5000, 70, 40), (1, 2, 1)])
def test_pages_bookkeeping(T, in_place, pages, n_seqs, width):
    """A random life of a pool: reserve, fork, free, compact, against the plain model; every table entry, reference,
    length and page of every layer."""
    rng = np.random.default_rng(pages)
    d = Device(T, pages, n_seqs, width, in_place)
    m = Pages(d.table.tolist(), d.lens.tolist(), d.refs.tolist())
    for step in range(40):
        empty = [s for s in range(n_seqs) if not m.held(s)]
        full = [s for s in range(n_seqs) if m.held(s)]
        kind = rng.choice(["reserve", "fork", "free", "compact"])
        before = d.contents()
        if kind == "reserve":
            seqs = rng.permutation(n_seqs)[:rng.integers(0, n_seqs + 1)].tolist()
            new = [int(rng.integers(0, width * PAGE + 1)) for _ in seqs]
            trial = Pages(m.table, m.lens, m.refs)
            want = trial.reserve(seqs, new)
            got = d.call("tadm_pages_reserve", i32(seqs), i32(new), lens=False)
            assert got == want
            if not want:
                m = trial
                # the sequences' tokens now fill some of what they hold
                m.lens = [int(rng.integers(0, len(m.held(s)) * PAGE + 1)) for s in range(n_seqs)]
                d.lens = i32(m.lens)
        elif kind == "fork" and full:
            dst = empty[:rng.integers(0, len(empty) + 1)]
            src = [int(rng.choice(full)) for _ in dst]
            trial = Pages(m.table, m.lens, m.refs)
            want, moves = trial.fork(src, dst)
            assert d.call("tadm_pages_fork", i32(src), i32(dst), pool=True) == want
            d.moved(before, moves)
            if not want:
                m = trial
        elif kind == "free":
            seqs = [s for s in range(n_seqs) if rng.random() < 0.3]
            assert d.call("tadm_pages_free", i32(seqs)) == 0
            m.release(seqs)
        elif kind == "compact":
            n, moves = m.compact()
            assert d.call("tadm_pages_compact", pool=True, lens=False) == n
            d.moved(before, moves)
        d.same(m)


@pytest.mark.parametrize("in_place", [False, True])
def test_pages_refusals_on_the_device(T, in_place):
    """Lists and states that the device finds wrong: the status says so and nothing changes."""
    d = Device(T, 20, 6, 4, in_place)
    assert d.call("tadm_pages_reserve", i32([0, 3]), i32([200, 65]), lens=False) == 0
    d.lens = i32([130, 0, 0, 64, 0, 0])
    m = Pages(d.table.tolist(), d.lens.tolist(), d.refs.tolist())
    before = d.contents()

    def refused(status, name, *args, **kw):
        assert d.call(name, *args, **kw) == status
        d.same(m)
        d.moved(before, [])

    bad, short = 2, 1
    for seqs, new in (([0, 0], [1, 1]), ([6], [1]), ([-1], [1]), ([1], [257]), ([1], [-1])):
        refused(bad, "tadm_pages_reserve", i32(seqs), i32(new), lens=False)
    refused(short, "tadm_pages_reserve", i32([1, 2, 4, 5]), i32([256] * 4), lens=False)
    for src, dst in (([0, 0], [1, 1]), ([0], [6]), ([7], [1]), ([-1], [1]), ([0, 1], [1, 2]), ([0], [3]), ([0], [0])):
        refused(bad, "tadm_pages_fork", i32(src), i32(dst), pool=True)
    for seqs in ([0, 0], [9], [-2]):
        refused(bad, "tadm_pages_free", i32(seqs))
    # a table that names a page nobody holds, and one that is not there
    page = int(d.table[0, 0])
    d.refs[page] = m.refs[page] = 0
    refused(bad, "tadm_pages_free", i32([0]))
    refused(bad, "tadm_pages_fork", i32([0]), i32([1]), pool=True)
    d.refs[page] = m.refs[page] = 1
    d.table[0, 0] = m.table[0][0] = 20
    refused(bad, "tadm_pages_free", i32([3, 0]))
    refused(bad, "tadm_pages_fork", i32([0]), i32([1]), pool=True)


def test_pages_copy(T):
    d = Device(T, 30, 1, 1, True, layers=3, heads=2, hd=128)
    before = d.contents()
    T.tadm_pages_copy(d.pool, i32([3, 3, 29, 40, 5]), i32([0, 7, 11, 12, -1]))
    d.moved(before, [(3, 0), (3, 7), (29, 11)])
    T.tadm_pages_copy(d.pool, i32([]), i32([]))
    d.moved(before, [(3, 0), (3, 7), (29, 11)])


# ------------------------------------------------------------------ together
def test_example_server(T):
    """The example runs the operators together: pages shared by branches, blocks and single tokens on top of them; every
    attention over the cache within bf16 rounding of 64 bits (the probabilities' 11 bits and the output's 8)."""
    import importlib.util
    import os
    at = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples", "ragged_server.py")
    spec = importlib.util.spec_from_file_location("ragged_server", at)
    m = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(m)
    for heads, kv_heads, hd, seed in ((16, 8, 128, 0), (6, 6, 64, 1)):
        x, peak, live, worst = m.serve(layers=2, prompts=4, branches=3, heads=heads, kv_heads=kv_heads, hd=hd, seed=seed, check=True)
        assert torch.isfinite(x).all() and 0 < live < peak and worst < 4e-3, (peak, live, worst)


def test_graph_replay(T):
    """Captured into a CUDA graph and replayed on new inputs in place: packed prompts, write, attention over the cache, read."""
    Hq, Hkv, hd, lens = 8, 4, 128, [70, 5, 200]
    cu, rows = i32(cum(lens)), sum(lens)
    pool, table = T.PagePool.empty(1, 12, Hkv, hd), torch.arange(12, dtype=torch.int32, device="cuda").view(3, 4)
    x = torch.randn((rows, Hq + 2 * Hkv, hd), generator=gen(1), device="cuda").bfloat16()
    q, k, v = x[:, :Hq], x[:, Hq:Hq + Hkv], x[:, Hq + Hkv:]
    o, p, kb, vb = (torch.empty((rows, h, hd), dtype=x.dtype, device="cuda") for h in (Hq, Hq, Hkv, Hkv))
    start, n = i32([0, 0, 0]), i32(lens)
    scratch = torch.empty(T.tadm_page_attention_scratch_size(3, rows, 200, 200, Hq, Hkv, hd, 1), dtype=torch.uint8, device="cuda")

    def once(stream=None):
        T.tadm_attention_packed(q, k, v, o, cu, 200, stream=stream)
        T.tadm_page_write(pool, 0, k, v, cu, start, table, 200, stream=stream)
        T.tadm_page_attention(q, pool, 0, p, cu, n, table, 200, 200, scratch, causal=True, stream=stream)
        T.tadm_page_read(pool, 0, kb, vb, cu, start, table, 200, stream=stream)

    once()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        once()
    x.copy_(torch.randn(x.shape, generator=gen(2), device="cuda"))
    graph.replay()
    torch.cuda.synchronize()
    got = [t.clone() for t in (o, p, kb, vb)]
    once()
    for a, b in zip(got, (o, p, kb, vb)):
        assert torch.equal(a, b)
    for a, m in zip(cum(lens), lens):
        s = slice(a, a + m)
        ref, absum = attend64(q[s].double(), k[s].double(), v[s].double(), torch.arange(m, device="cuda"), True, 0)
        close(o[s], ref, absum, torch.bfloat16, float(v[s].abs().max()))
        ref, absum = attend64(q[s].double(), kb[s].double(), vb[s].double(), torch.arange(m, device="cuda"), True, 0)
        close(p[s], ref, absum, torch.bfloat16, float(vb[s].abs().max()))


def test_offsets_past_32_bits(T):
    """The last pages of a pool whose K and V are over 4 GB each: rows written, read and attended over."""
    Hkv, hd, pages = 8, 128, 34000
    k = torch.empty((2, pages, Hkv, PAGE, hd), dtype=torch.uint8, device="cuda")
    v = torch.empty((2, pages, Hkv, hd, PAGE), dtype=torch.uint8, device="cuda")
    assert k.numel() > 1 << 32
    scales = [torch.ones((2, pages, Hkv), dtype=torch.float32, device="cuda") for _ in range(2)]
    pool, table = T.PagePool(k, v, *scales), i32([pages - 1, pages - 3, 5]).view(1, 3)
    x = torch.randn((150, 2, Hkv, hd), generator=gen(1), device="cuda").bfloat16()
    T.tadm_page_write(pool, 1, x[:, 0], x[:, 1], i32([0, 150]), i32([0]), table, 150)
    kb, vb = torch.empty_like(x[:, 0]).contiguous(), torch.empty_like(x[:, 1]).contiguous()
    T.tadm_page_read(pool, 1, kb, vb, i32([0, 150]), i32([0]), table, 150)
    assert (kb.float() - x[:, 0].float()).abs().max() <= 2.0 ** -4 * x.abs().max()     # e4m3: half of 2^-3 of a value
    q = torch.randn((1, 16, hd), generator=gen(2), device="cuda").bfloat16()
    o = run_paged(T, pool, table, q, [0, 1], [150], 1, 150, True, 0)
    ref, absum = attend64(q.double(), kb.double(), vb.double(), torch.tensor([149], device="cuda"), True, 0)
    close(o, ref, absum, torch.bfloat16, float(vb.abs().max()))
    status, refs = i32([0]), torch.zeros(pages, dtype=torch.int32, device="cuda")
    T.tadm_pages_copy(pool, i32([pages - 1]), i32([pages - 2]))
    assert torch.equal(k[:, pages - 1], k[:, pages - 2]) and torch.equal(v[1, pages - 1], v[1, pages - 2])
    assert int(status) == 0 and int(refs.sum()) == 0


def test_many_items_and_long_splits(T):
    """More sequences than a warp scans at once, most of them short; and one sequence that every SM has a part of."""
    Hq, Hkv, hd = 8, 4, 64
    lens = [(13 * i) % 150 for i in range(100)]
    pool, table, seqs = filled(T, lens, Hkv, hd, 21)
    rows = [1 if n else 0 for n in lens]
    q = torch.randn((sum(rows), Hq, hd), generator=gen(3), device="cuda").bfloat16()
    o = run_paged(T, pool, table, q, cum(rows), lens, 1, max(lens), True, 0)
    for b, n in enumerate(lens):
        if n:
            s = slice(cum(rows)[b], cum(rows)[b] + 1)
            ref, absum = attend64(q[s].double(), *seqs[b], torch.tensor([n - 1], device="cuda"), True, 0)
            close(o[s], ref, absum, torch.bfloat16, float(seqs[b][1].abs().max()))
    pool, table, seqs = filled(T, [70001], 1, hd, 22)
    for n in (1, 33):
        q = torch.randn((n, 2, hd), generator=gen(4), device="cuda").bfloat16()
        o = run_paged(T, pool, table, q, [0, n], [70001], n, 70001, False, 0)
        ref, absum = attend64(q.double(), *seqs[0], torch.zeros(n, device="cuda"), False, 0)
        close(o, ref, absum, torch.bfloat16, float(seqs[0][1].abs().max()))
