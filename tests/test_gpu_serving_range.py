"""Operators for sequences of different lengths over values of very different sizes, and in states at the edge of what
they accept, against plain definitions in 64 bits."""
import math

import pytest

torch = pytest.importorskip("torch")
from test_gpu_serving import Device, Pages, T, attend64, close, cum, filled, gen, i32, run_paged  # noqa: E402, F401

pytestmark = pytest.mark.gpu


# ------------------------------------------------------------------ queries of different sizes
def cached(pool, table, b, n, layer=1):
    """The first n tokens of sequence b as the pool's bytes and scales say, in 64 bits: k, v [n, heads, hd]."""
    at = table[b, :-(-n // 64)].long()
    f = lambda x, s: x[layer, at].view(torch.float8_e4m3fn).double() * s[layer, at].double()[..., None, None]  # noqa: E731
    k, v = f(pool.k, pool.k_scale), f(pool.v, pool.v_scale)
    return k.permute(0, 2, 1, 3).flatten(0, 1)[:n], v.permute(0, 3, 1, 2).flatten(0, 1)[:n]


def encode(x):
    return x.float().to(torch.float8_e4m3fn).view(torch.uint8)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("heads", [(16, 8, 128), (6, 2, 64), (8, 1, 128), (32, 16, 128)])
@pytest.mark.parametrize("n,length", [(1, 700), (8, 300), (33, 1025)])
@pytest.mark.parametrize("gain", [2.0 ** 11, 2.0 ** 12])
def test_page_attention_large_channel(T, dtype, heads, n, length, gain):
    """A channel of Q is `gain` times the others and K's as much smaller, so that all channels count alike: the others keep
    their bits.  The bf16 form holds Q to 2^-20 of a row's largest value; with q_top the largest of all rows and errors of
    q_top 2^-21 evenly spread over both signs, a score is off by |k| q_top 2^-21 / sqrt(3 hd), outputs by about twice that
    (relative), beside bf16's 2^-8."""
    Hq, Hkv, hd = heads
    pool, table, _ = filled(T, [length], Hkv, hd, length + Hq)
    pool.k[1, :, :, :, 5] = encode(pool.k[1, :, :, :, 5].contiguous().view(torch.float8_e4m3fn).float() / gain)
    k, v = cached(pool, table, 0, length)
    q = torch.randn((n, Hq, hd), generator=gen(6), device="cuda")
    q[..., 5] *= gain
    q = q.to(dtype)
    o = run_paged(T, pool, table, q, [0, n], [length], n, length, False, 0)
    ref, _ = attend64(q.double(), k, v, torch.zeros(n, device="cuda"), False, 0)
    err = (o.double() - ref).norm(dim=-1) / ref.norm(dim=-1)
    score = float(q.abs().max()) * 2.0 ** -21 / math.sqrt(3.0 * hd) * float(k.norm(dim=-1).mean())
    tol = math.sqrt(2.0 ** -16 + (2 * score) ** 2) if dtype == torch.bfloat16 else 1e-4
    assert err.square().mean().sqrt() <= tol and (err <= 4 * tol).all(), (float(err.square().mean().sqrt()), float(err.max()), tol)
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("heads", [(16, 8, 128), (6, 2, 64), (8, 1, 128), (32, 16, 128)])
@pytest.mark.parametrize("rows,lens", [([1, 1], [300, 64]), ([8, 3], [700, 40]), ([32, 33], [517, 1025])])
@pytest.mark.parametrize("large", [2.0 ** 6, 2.0 ** 12, 2.0 ** 20, 2.0 ** 60, math.inf, math.nan])
def test_page_attention_beside_large_rows(T, dtype, heads, rows, lens, large):
    """One query head of a sequence's first row and all heads of its last one (where it has more) are enlarged: every
    other row has its own accuracy, whatever shares its tile."""
    Hq, Hkv, hd = heads
    pool, table, seqs = filled(T, lens, Hkv, hd, sum(lens) + Hq)
    q = torch.randn((sum(rows), Hq, hd), generator=gen(5), device="cuda")
    grown = torch.zeros((sum(rows), Hq), dtype=torch.bool, device="cuda")
    for a, n in zip(cum(rows), rows):
        grown[a, Hq - 1] = True
        if n > 1:
            grown[a + n - 1] = True
    q = torch.where(grown[..., None], q * large, q).to(dtype)
    o = run_paged(T, pool, table, q, cum(rows), lens, max(rows), max(lens), False, 0)
    for b, n in enumerate(rows):
        s, (k, v) = slice(cum(rows)[b], cum(rows)[b] + n), seqs[b]
        ref, absum = attend64(torch.where(grown[s][..., None], 0.0, q[s].double()), k, v, torch.zeros(n, device="cuda"), False, 0)
        keep = ~grown[s]
        close(o[s][keep], ref[keep], absum[keep], dtype, float(v.abs().max()))


# ------------------------------------------------------------------ pages that nothing was written to
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("scale", [None, 0.0])
@pytest.mark.parametrize("n", [1, 20])
def test_unwritten_pages_are_zeros(T, dtype, scale, n):
    """Pages that a sequence holds but that no row was written to, between pages whose scores are far below zero, in a new
    pool and in one with scales of zero: their keys have score 0 and value 0."""
    Hq, Hkv, hd = 8, 4, 128
    pool, table = T.PagePool.empty(2, 6, Hkv, hd), i32([3, 0, 5, 1]).view(1, 4)
    if scale is not None:
        pool.k_scale.fill_(scale), pool.v_scale.fill_(scale)
    x = torch.randn((64, 2, Hkv, hd), generator=gen(1), device="cuda").to(dtype)
    x[:, 0] = -4.0                                             # scores of -4 * 4 * 128 / sqrt(128), 261 in log2 units below zero
    q = torch.full((n, Hq, hd), 4.0, dtype=dtype, device="cuda")
    for first in (0, 128):
        T.tadm_page_write(pool, 1, x[:, 0], x[:, 1], i32([0, 64]), i32([first]), table, 64)
    o = run_paged(T, pool, table, q, [0, n], [220], n, 220, False, 0)
    assert (o == 0).all()
    q = -q                                                     # and far above: the written pages have all the weight
    o = run_paged(T, pool, table, q, [0, n], [220], n, 220, False, 0)
    k, v = (torch.empty((64, Hkv, hd), dtype=dtype, device="cuda") for _ in range(2))
    T.tadm_page_read(pool, 1, k, v, i32([0, 64]), i32([0]), table, 64)
    ref = v.double().mean(0).repeat_interleave(Hq // Hkv, 0).expand(n, Hq, hd)
    close(o, ref, v.double().abs().mean(0).repeat_interleave(Hq // Hkv, 0).expand(n, Hq, hd), dtype, float(v.abs().max()))


def test_empty_pools_have_scales_that_attention_takes(T):
    pool = T.PagePool.empty(1, 3, 2, 64)
    for s in (pool.k_scale, pool.v_scale):
        assert (s == 2.0 ** -60).all()
    k, v = cached(pool, i32([0, 1, 2]).view(1, 3), 0, 192, layer=0)
    assert (k == 0).all() and (v == 0).all()


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_tokens_of_scale_zero_stay_zeros(T, dtype):
    """Rows written behind the tokens of a page whose scale is 0: those stay zeros, whatever their bytes are, when the page
    gets a scale."""
    pool = T.PagePool.empty(1, 2, 3, 64)
    for x in (pool.k, pool.v):
        x.copy_(encode(torch.randn(x.shape, generator=gen(1), device="cuda") * 60))
    pool.k_scale.zero_(), pool.v_scale.zero_()
    x = torch.randn((5, 2, 3, 64), generator=gen(2), device="cuda").to(dtype)
    table = i32([1]).view(1, 1)
    T.tadm_page_write(pool, 0, x[:, 0], x[:, 1], i32([0, 5]), i32([30]), table, 5)
    k, v = (torch.empty((35, 3, 64), dtype=dtype, device="cuda") for _ in range(2))
    T.tadm_page_read(pool, 0, k, v, i32([0, 35]), i32([0]), table, 35)
    for got, new in ((k, x[:, 0]), (v, x[:, 1])):
        assert (got[:30] == 0).all()
        assert ((got[30:] - new).abs() <= 2.0 ** -4 * new.abs().max()).all()


# ------------------------------------------------------------------ packed rows that weigh few keys
@pytest.mark.parametrize("heads", [(8, 8, 128), (4, 4, 64), (8, 4, 128)])
@pytest.mark.parametrize("n", [300, 1000])
@pytest.mark.parametrize("window", [0, 200])
def test_packed_rows_on_their_own_key(T, heads, n, window):
    """Rows of long prompts whose weight is nearly all on the key at their own position: what is left is the rounding of
    the output, 2^-8 of it, because the probabilities of the last keys are not rounded to 8 bits."""
    Hq, Hkv, hd = heads
    k, v = (torch.randn((n, Hkv, hd), generator=gen(i), device="cuda").bfloat16() for i in range(2))
    q = (k.float() * (1.0 if hd == 128 else 1.4)).bfloat16().repeat_interleave(Hq // Hkv, 1)
    o = torch.empty_like(q)
    T.tadm_attention_packed(q, k, v, o, i32([0, n]), n, window=window)
    ref, absum = attend64(q.double(), k.double(), v.double(), torch.arange(n, device="cuda"), True, window)
    close(o, ref, absum, torch.bfloat16, float(v.abs().max()))


# ------------------------------------------------------------------ scores of minus infinity
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("heads", [(4, 2, 64), (16, 8, 128)])
@pytest.mark.parametrize("n,hidden", [(300, 200), (300, 128), (300, 64), (700, 513), (40, 40)])
@pytest.mark.parametrize("causal,window", [(True, 0), (False, 0), (True, 150)])
def test_packed_scores_of_minus_infinity(T, dtype, heads, n, hidden, causal, window):
    """The first keys' scores are all minus infinity, over whole key tiles: they weigh nothing, and a row that sees no other
    key gets zeros as if it saw none."""
    Hq, Hkv, hd = heads
    q, k, v = (torch.randn((n, h, hd), generator=gen(h + 1), device="cuda") for h in (Hq, Hkv, Hkv))
    q[..., 3], k[:hidden, :, 3] = q[..., 3].abs() + 0.1, -math.inf
    q, k, v = q.to(dtype), k.to(dtype), v.to(dtype)
    o = torch.empty_like(q)
    T.tadm_attention_packed(q, k, v, o, i32([0, n]), n, causal=causal, window=window)
    pos, j = torch.arange(n, device="cuda")[:, None], torch.arange(n, device="cuda")
    see = (j >= hidden).expand(n, n)
    if causal:
        see = see & (j <= pos)
    if window:
        see = see & (pos - j < window)
    kk, vv = (x.double().repeat_interleave(Hq // Hkv, 1) for x in (k, v))
    kk[:hidden, :, 3] = 0.0
    x = (torch.einsum("rhd,nhd->hrn", q.double(), kk) / math.sqrt(hd)).masked_fill(~see, -math.inf)
    w = torch.exp(x - x.amax(-1, keepdim=True).clamp_min(-1e300))
    w = w / w.sum(-1, keepdim=True).clamp_min(1e-300)
    close(o, torch.einsum("hrn,nhd->rhd", w, vv), torch.einsum("hrn,nhd->rhd", w, vv.abs()), dtype, float(v.abs().max()))
    assert (o[~see.any(1)] == 0).all()


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("causal", [True, False])
def test_page_scores_of_minus_infinity(T, dtype, causal):
    """The same over the cache, with K of -448 2^60 (its largest) against a query that takes the scores past fp32."""
    Hq, Hkv, hd, n, length, hidden = 8, 4, 128, 5, 700, 384
    pool, table, _ = filled(T, [length], Hkv, hd, 2, nan_tail=False)
    at = table[0, :hidden // 64].long()
    pool.k[1, :, :, :, 7] = 0
    pool.k[1, at, :, :, :] = 0
    pool.k[1, at, :, :, 7] = 0xFE                               # -448
    pool.k_scale[1, at] = 2.0 ** 60
    k, v = cached(pool, table, 0, length)
    q = torch.randn((n, Hq, hd), generator=gen(3), device="cuda")
    q[..., 7] = 2.0 ** 70
    q = q.to(dtype)
    o = run_paged(T, pool, table, q, [0, n], [length], n, length, causal, 0)
    pos = torch.arange(length - n, length, device="cuda") - hidden
    qq = q.double()
    qq[..., 7] = 0.0
    ref, absum = attend64(qq, k[hidden:], v[hidden:], pos, causal, 0)
    if dtype == torch.float32:
        close(o, ref, absum, dtype, float(v.abs().max()))
    else:                                                      # q's other channels are below 2^-60 of its largest: no score of theirs is left
        flat = v[hidden:].repeat_interleave(Hq // Hkv, 1)
        mean = torch.stack([flat[:int(p) + 1 if causal else None].mean(0) for p in pos])
        close(o, mean, mean.abs().max().expand_as(mean), dtype, float(v.abs().max()))


# ------------------------------------------------------------------ bookkeeping
@pytest.mark.parametrize("in_place", [False, True])
@pytest.mark.parametrize("wrong", ["free", "past", "negative"])
def test_reserve_finds_contradictions(T, in_place, wrong):
    """A listed sequence that holds a page which the references call free (it would be handed out a second time), or an id
    that is no page: refused, nothing changes."""
    d = Device(T, 20, 6, 40, in_place)
    assert d.call("tadm_pages_reserve", i32([0, 3]), i32([200, 700]), lens=False) == 0
    d.lens = i32([130, 0, 0, 700, 0, 0])
    if wrong == "free":
        d.refs[int(d.table[3, 9])] = 0
    elif wrong == "past":
        d.table[3, 10] = 20
    else:
        d.refs[int(d.table[3, 2])] = -1
    m = Pages(d.table.tolist(), d.lens.tolist(), d.refs.tolist())
    for seqs, new in (([3], [900]), ([1, 3], [64, 10]), ([3, 0], [64, 64])):
        assert d.call("tadm_pages_reserve", i32(seqs), i32(new), lens=False) == 2
        d.same(m)
    assert d.call("tadm_pages_reserve", i32([0]), i32([300]), lens=False) == 0      # others go on


# ------------------------------------------------------------------ status
def test_no_call_gave_up(T):
    """What the tests of this file and the calls below left on the device's status word: nothing, on any stream, also
    where the calls were captured into a graph."""
    q = torch.randn((40, 4, 64), generator=gen(1), device="cuda").bfloat16()
    pool, table, _ = filled(T, [300], 2, 64, 1)
    o, scratch = torch.empty_like(q), torch.empty(T.tadm_page_attention_scratch_size(1, 40, 40, 300, 4, 2, 64, 1), dtype=torch.uint8, device="cuda")
    cu, lens, s = i32([0, 40]), i32([300]), torch.cuda.Stream()

    def once(stream=None):
        T.tadm_attention_packed(q, q[:, :2], q[:, 2:], o, cu, 40, stream=stream)
        T.tadm_page_attention(q, pool, 1, o, cu, lens, table, 40, 300, scratch, stream=stream)

    torch.cuda.synchronize()
    once(s)
    T.tadm_ragged_sync_status(s)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        once()
    graph.replay()
    T.tadm_ragged_sync_status()


# ------------------------------------------------------------------ pages of different scales
def by_dim(o, q, k8, v8, ks, vs, dtype):
    """Each output value against its own dim: what multiplies V in the bf16 form is p s, p the probability and s the page's
    scale, rounded to f16 (2^-11 of it) or, where it is below 2^-21 of the row's largest p s, to 2^-32 of that; the output to
    bf16 (2^-8); the rest is fp32."""
    group = q.shape[1] // k8.shape[1]
    k8, v8 = k8.repeat_interleave(group, 1), v8.repeat_interleave(group, 1)
    ks, vs = ks.repeat_interleave(group, 1), vs.repeat_interleave(group, 1)
    x = torch.einsum("rhd,nhd->hrn", q.double(), k8 * ks[..., None]) / math.sqrt(q.shape[2])
    w = torch.softmax(x, -1) * vs.T[:, None]
    ref, absum = torch.einsum("hrn,nhd->rhd", w, v8), torch.einsum("hrn,nhd->rhd", w, v8.abs())
    tol = 1e-4 * absum
    if dtype == torch.bfloat16:
        tol = tol + (2.0 ** -8 + 2.0 ** -11) * absum + 2.0 ** -32 * w.amax(-1).T[..., None] * v8.abs().sum(0)
    err = (o.double() - ref).abs()
    assert torch.isfinite(o).all() and (err <= tol).all(), (float((err / tol.clamp_min(1e-300)).max()))


def parts(pool, table, n):
    """Bytes and scales of the first n tokens of the one sequence: k8, v8 [n, heads, hd], ks, vs [n, heads]."""
    at = table[0, :-(-n // 64)].long()
    k, v = (x[1, at].view(torch.float8_e4m3fn).double() for x in (pool.k, pool.v))
    s = [x[1, at].double().repeat_interleave(64, 0)[:n] for x in (pool.k_scale, pool.v_scale)]
    return k.permute(0, 2, 1, 3).flatten(0, 1)[:n], v.permute(0, 3, 1, 2).flatten(0, 1)[:n], *s


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("n", [1, 4, 33])
@pytest.mark.parametrize("ratio", [2.0 ** 12, 2.0 ** 18, 2.0 ** 24])
def test_page_attention_one_large_dim(T, dtype, n, ratio):
    """The page in the middle has a V scale `ratio` times the others' and zeros in all dims but one: the other dims are the
    other pages' alone and keep their bits."""
    Hq, Hkv, hd, length = 8, 4, 128, 600
    pool, table, _ = filled(T, [length], Hkv, hd, 3, spread=0)
    page = int(table[0, 4])
    pool.v[1, page, :, 1:] = 0
    pool.v_scale[1, page] *= ratio
    q = (torch.randn((n, Hq, hd), generator=gen(4), device="cuda") * 0.2).to(dtype)
    o = run_paged(T, pool, table, q, [0, n], [length], n, length, False, 0)
    by_dim(o, q, *parts(pool, table, length), dtype)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("n", [1, 4, 33])
@pytest.mark.parametrize("page", [0, 3, 8])
def test_page_attention_scales_far_apart(T, dtype, n, page):
    """One page's V scale is 2^40 times the others' and its keys weigh 2^-40 of theirs: both count alike, all are seen at
    once, and every dim is judged by its own sum."""
    Hq, Hkv, hd, length = 8, 4, 128, 600
    pool, table, _ = filled(T, [length], Hkv, hd, 3, spread=0)
    q = torch.randn((n, Hq, hd), generator=gen(4), device="cuda") * 0.2
    q[..., 0] = 8.0
    q = q.to(dtype)
    at = int(table[0, page])
    pool.k[1, :, :, :, 0] = 0
    pool.k_scale[1, at] = 2.0 ** -3
    pool.k[1, at, :, :, 0] = encode(torch.tensor(-40.0 * math.log(2.0) * math.sqrt(hd) / 8.0 * 8.0)).item()   # score -40 ln 2
    pool.v_scale[1, at] *= 2.0 ** 40
    if at == int(table[0, length // 64]):                      # (the page that ends inside: its tail holds NaN)
        pool.k[1, at, :, length % 64:] = 0x7F
    o = run_paged(T, pool, table, q, [0, n], [length], n, length, False, 0)
    by_dim(o, q, *parts(pool, table, length), dtype)


def test_page_moves_past_32_bits(T):
    """fork and compact on a pool whose K and V are over 4 GB each: page contents and scales of both layers."""
    Hkv, hd, pages = 8, 128, 34000
    k = torch.empty((2, pages, Hkv, 64, hd), dtype=torch.uint8, device="cuda")
    v = torch.empty((2, pages, Hkv, hd, 64), dtype=torch.uint8, device="cuda")
    scales = [torch.ones((2, pages, Hkv), dtype=torch.float32, device="cuda") for _ in range(2)]
    assert k.numel() > 1 << 32
    pool = T.PagePool(k, v, *scales)
    own = [pages - 1, pages - 3, pages - 4]
    for i, x in enumerate((k, v)):
        x[:, own] = torch.randint(0, 256, (2, 3, Hkv) + tuple(x.shape[3:]), generator=gen(i), device="cuda").to(torch.uint8)
    for i, s in enumerate(scales):
        s[:, own] = torch.rand((2, 3, Hkv), generator=gen(9 + i), device="cuda")
    before = [x[:, own].clone() for x in (k, v, *scales)]
    refs = torch.ones(pages, dtype=torch.int32, device="cuda")
    refs[pages - 2] = 0                                        # the only free page
    tables = torch.full((2, 3), -1, dtype=torch.int32, device="cuda")
    tables[0] = i32(own)
    lens, status = i32([150, 0]), i32([7])
    scratch = torch.empty(T.tadm_pages_scratch_size(pages, 2), dtype=torch.uint8, device="cuda")
    T.tadm_pages_fork(pool, tables, lens, refs, i32([0]), i32([1]), tables, lens, refs, status, scratch)
    assert int(status) == 0 and tables.tolist() == [own, own[:2] + [pages - 2]] and lens.tolist() == [150, 150]
    assert refs[own].tolist() == [2, 2, 1] and int(refs[pages - 2]) == 1
    for x, b in zip((k, v, *scales), before):
        assert torch.equal(x[:, pages - 2], b[:, 2]) and torch.equal(x[:, own], b)
    refs.zero_()
    refs[own], refs[pages - 2] = i32([2, 2, 1]), 1
    refs[0] = refs[33000] = 1                                  # pages of nobody else's table: 0 stays, 33000 moves too
    T.tadm_pages_compact(pool, tables, refs, tables, refs, status, scratch)
    # in use: 0, 33000, then the four in ascending order; they take 1 .. 5
    to = {33000: 1, pages - 4: 2, pages - 3: 3, pages - 2: 4, pages - 1: 5}
    assert int(status) == 6 and tables.tolist() == [[to[p] for p in own], [to[p] for p in own[:2]] + [to[pages - 2]]]
    assert refs[:6].tolist() == [1, 1, 1, 2, 1, 2] and int(refs.sum()) == 8
    for x, b in zip((k, v, *scales), before):
        assert torch.equal(x[:, [to[p] for p in own]], b) and torch.equal(x[:, 4], b[:, 2])
