"""Sampling with settings per row, projections with an adapter per request, norms with gate and residual scale on the GPU,
against plain definitions in 64 bits."""
import math
import os
import subprocess
import sys

import numpy as np
import pytest

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")

F32, BF16 = torch.float32, torch.bfloat16


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


def f32(v):
    return torch.tensor(list(v), dtype=torch.float32, device="cuda")


def cum(lens, first=0):
    out = [first]
    for n in lens:
        out.append(out[-1] + n)
    return out


def gen(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return g


def randn(g, *shape):
    return torch.randn(shape, generator=g, device="cuda")


# ------------------------------------------------------------------ sampling
def draw64(logits, t, k, p, m, u, mask_id):
    """One row from the definition, in 64 bits: the token, its probability."""
    x = logits.astype(np.float64)
    x[np.isnan(x)] = -np.inf
    if mask_id >= 0:
        x[mask_id] = -np.inf
    ids = np.flatnonzero(x > -np.inf)
    if len(ids) == 0:
        return -1, 0.0
    x = x[ids]
    order = np.argsort(-x, kind="stable")
    if not t > 2.0 ** -100:
        return int(ids[order[0]]), 1.0
    with np.errstate(invalid="ignore", over="ignore", under="ignore"):
        w = np.where(x == x.max(), 1.0, np.exp((x - x.max()) / t))
    n = len(order) if k <= 0 else min(k, len(order))
    if m > 0:
        n = min(n, int(np.count_nonzero(w >= min(m, 1.0))))
    mass = np.cumsum(w[order[:n]])
    if p < 1:
        n = max(1, int(np.count_nonzero(np.concatenate([[0.0], mass[:-1]]) < p * mass[-1])))
    kept = np.sort(order[:n])
    mass = np.cumsum(w[kept])
    at = np.flatnonzero(mass > (u if u > 0 else 0.0) * mass[-1])
    at = int(at[0]) if len(at) else int(np.flatnonzero(w[kept] >= 2.0 ** -44)[-1])
    return int(ids[kept[at]]), float(w[kept[at]] / mass[-1])


def check_draws(T, logits, u, t=None, k=None, p=None, m=None, mask_id=-1):
    rows = logits.shape[0]
    before = logits.clone()
    tok = torch.full((rows,), -7, dtype=torch.int32, device="cuda")
    prob = torch.full((rows,), -7.0, device="cuda")
    T.tadm_sample(logits, u, tok, temperature=t, top_k=k, top_p=p, min_p=m, prob=prob, mask_id=mask_id)
    host = logits.float().cpu().numpy()
    get = lambda v, off: [off] * rows if v is None else [x.item() for x in v.cpu()]  # noqa: E731
    settings = list(zip(get(t, 1.0), get(k, 0), get(p, 1.0), get(m, 0.0), get(u, 0.0)))
    want = [draw64(host[r], *settings[r], mask_id) for r in range(rows)]
    got_t, got_p = tok.cpu().tolist(), prob.cpu().tolist()
    for r in range(rows):
        assert got_t[r] == want[r][0], (r, got_t[r], want[r], settings[r])
        # weights are right to 2^-34, their sums' remainders to 2^-44 a token; one rounding to fp32
        assert abs(got_p[r] - want[r][1]) <= 2.0 ** -23 * want[r][1] + 2.0 ** -24, (r, got_p[r], want[r], settings[r])
    bits = torch.int16 if logits.dtype == BF16 else torch.int32
    assert torch.equal(logits.contiguous().view(bits), before.contiguous().view(bits))
    alone = torch.empty_like(tok)
    T.tadm_sample(logits, u, alone, temperature=t, top_k=k, top_p=p, min_p=m, mask_id=mask_id)
    assert torch.equal(alone, tok)


def settings_of(g, rows, kind):
    pick = lambda *of: torch.tensor(of, device="cuda")[torch.randint(0, len(of), (rows,), generator=g, device="cuda")]  # noqa: E731
    t, k, p, m = pick(0.3, 0.7, 1.0, 1.5), None, None, None
    if "k" in kind:
        k = pick(1, 2, 40, 600, 0, 10 ** 9).to(torch.int32)
    if "p" in kind:
        p = pick(0.1, 0.5, 0.9, 0.99, 0.999999)
    if "m" in kind:
        m = pick(0.0, 1e-6, 0.05, 0.5)
    return t, k, p, m


VOCABS = [1, 2, 3, 31, 127, 128, 129, 1000, 4097, 30522, 32768]


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("kind", ["", "k", "p", "m", "kpm"])
@pytest.mark.parametrize("vocab", VOCABS)
def test_sample(T, dtype, kind, vocab):
    rows = 12
    g = gen(vocab + len(kind))
    x = 2.0 * randn(g, rows, vocab)
    x[::3] *= 0.25                                             # rows near a flat distribution
    if vocab > 100:
        x[1::3, ::50] += 7.0                                   # and rows with some tokens far above the others
    u = torch.rand(rows, generator=g, device="cuda")
    check_draws(T, x.to(dtype), u, *settings_of(g, rows, kind), mask_id=vocab - 1 if vocab % 2 else -1)


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("vocab,rows", [(128000, 3), (128001, 40), (262144, 2), (262144, 21), (1 << 19, 2)])
def test_sample_large_vocabularies(T, dtype, vocab, rows):
    g = gen(vocab + rows)
    x = randn(g, rows, vocab)
    x[::2] *= 3.0
    u = torch.rand(rows, generator=g, device="cuda")
    check_draws(T, x.to(dtype), u, *settings_of(g, rows, "kp"), mask_id=5)
    check_draws(T, x.to(dtype), u, *settings_of(g, rows, ""))


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("spread", [0.01, 1.0, 4.0])
@pytest.mark.parametrize("vocab", [9000, 70001])
def test_sample_cuts_of_thousands(T, dtype, spread, vocab):
    """Cuts far down the order, one setting alone and several at once: more ids than any list takes."""
    rows = 12
    g = gen(vocab)
    x = spread * randn(g, rows, vocab)
    u, n = torch.rand(rows, generator=g, device="cuda"), torch.arange(rows, device="cuda")
    k = (vocab * torch.tensor([0.05, 0.3, 0.7, 0.999], device="cuda")[n % 4]).to(torch.int32)
    p = torch.tensor([0.9, 0.5, 0.99], device="cuda")[n % 3]
    m = torch.tensor([1e-12, 0.01, 0.4], device="cuda")[n % 3]
    x = x.to(dtype)
    check_draws(T, x, u, k=k, mask_id=3)
    check_draws(T, x, u, p=p)
    check_draws(T, x, u, m=m, mask_id=vocab - 1)
    check_draws(T, x, u, k=k, p=p.flip(0))
    check_draws(T, x, u, p=p, m=m.roll(1))
    check_draws(T, x, u, k=k, m=m, p=p)


@pytest.mark.parametrize("vocab", [3000, 30000])
def test_sample_far_from_zero_and_nearly_cold(T, vocab):
    """Logits whose distance from zero, over the temperature, is past what the passes over a row count in."""
    rows = 12
    g = gen(vocab + 1)
    x = randn(g, rows, vocab)
    n = torch.arange(rows, device="cuda")
    x += torch.tensor([0.0, 3e4, -3e4, 1e6], device="cuda")[n % 4][:, None]
    t = torch.tensor([1.0, 1e-3, 3e-2], device="cuda")[n % 3]
    u = torch.rand(rows, generator=g, device="cuda")
    check_draws(T, x, u, t)
    check_draws(T, x, u, t, p=f32([0.9] * rows), mask_id=7)
    check_draws(T, x, u, t, k=i32([30] * rows), m=f32([0.01] * rows))
    check_draws(T, 1e5 * x, u, 1e5 * t, p=f32([0.7] * rows))


def half_way_tops(n):
    """Logits that lie, in steps of which 510 span a weight of 2^-44, half-way between two whole numbers once their product
    is rounded, and above that before."""
    per = np.float32(1.4426950408889634) * (np.float32(510) / np.float32(44))
    out = []
    for at in (0.5, 100.5, -20.5, 2000.5, 1e5 + 0.5, 1e6 + 0.5, 3e6 + 0.5):
        x = np.float32(at / np.float64(per))
        found = 0
        for _ in range(200000):
            x = np.nextafter(x, np.float32(np.inf))
            g = x * per
            if np.float64(g) - math.floor(g) == 0.5 and math.floor(g) % 2 == 0 and np.float64(x) * np.float64(per) > g:
                out.append(float(x))
                found += 1
                if found == n:
                    break
    return out


@pytest.mark.parametrize("vocab", [5000, 30000])
def test_sample_maxima_half_way_between_bins(T, vocab):
    """Every 8192 ids count their values from their own maximum; it must not round to a place in front of the first."""
    tops = half_way_tops(3)
    assert len(tops) >= 12
    rows = len(tops)
    g = gen(vocab + 2)
    x = torch.tensor(tops, device="cuda")[:, None] - 1.0 - 6.0 * torch.rand(rows, vocab, generator=g, device="cuda")
    for first in range(0, vocab, 8192):
        x[:, first + 77] = torch.tensor(tops, device="cuda")
    u = torch.rand(rows, generator=g, device="cuda")
    ones = torch.ones(rows, device="cuda")
    check_draws(T, x, u, ones, k=i32([30] * rows))
    check_draws(T, x, u, ones, k=i32([2] * rows))
    check_draws(T, x, u, ones, m=f32([0.1] * rows))
    check_draws(T, x, u, ones, m=f32([0.01] * rows), p=f32([0.9] * rows))


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("vocab", [7, 5000, 140000])
def test_sample_equal_logits(T, dtype, vocab):
    """Ties everywhere: every cut falls among equal logits and goes by the id."""
    rows = 24
    x = torch.full((rows, vocab), 1.25, device="cuda")
    x[8:16] = torch.where(torch.arange(vocab, device="cuda") % 3 == 1, 2.0, 0.5)
    x[16:] = torch.where(torch.arange(vocab, device="cuda") % 2 == 1, -0.0, 0.0)      # equal as numbers
    n = torch.arange(rows, device="cuda")
    u = ((n * 37 % 24).float() + 0.3) / 24
    k = (n % 5 * vocab // 6).to(torch.int32)
    p = torch.tensor([0.25, 0.5, 0.77, 1.0], device="cuda")[n % 4]
    check_draws(T, x.to(dtype), u, k=k, mask_id=2)
    check_draws(T, x.to(dtype), u, p=p)
    check_draws(T, x.to(dtype), u, k=k, p=p, mask_id=0)
    check_draws(T, x.to(dtype), u, t=torch.zeros(rows, device="cuda"), mask_id=1)


def test_sample_values_out_of_the_ordinary(T):
    g = gen(3)
    vocab, rows = 3000, 18
    x = randn(g, rows, vocab)
    low = torch.finfo(F32).min
    x[0] = -math.inf                                           # nothing to draw from
    x[1] = math.nan
    x[2, 100:] = -math.inf
    x[3, 7:] = math.nan
    x[4, 11] = math.inf                                        # all the weight
    x[5, [20, 30, 40]] = math.inf                              # in equal parts
    x[6, 10:] = low                                            # a mask of the type's lowest value
    x[7] = low
    x[8] = 1e30 * x[8]
    x[9, 5] = 3e38
    x[9, 6] = -3e38
    x[10] = 1e-30 * x[10]
    x[11] = x[11] + 1e6                                        # far from zero
    x[12, :] = -math.inf
    x[12, 17] = -1e4                                           # one token
    x[13, 9:] -= 200.0                                         # weights of nothing
    x[14, 0] = 1e5
    x[15, ::2] = -math.inf
    u = torch.rand(rows, generator=g, device="cuda")
    for t in (None, torch.full((rows,), 0.01, device="cuda"), torch.full((rows,), 50.0, device="cuda")):
        check_draws(T, x, u, t)
        check_draws(T, x, u, t, k=i32([7] * rows), mask_id=17)
        check_draws(T, x, u, t, p=f32([0.9] * rows), m=f32([0.01] * rows))
    check_draws(T, x[:, 1:], u)                                # rows that start off 16 bytes
    check_draws(T, x.bfloat16()[:, 1:], u, p=f32([0.9] * rows), mask_id=0)
    check_draws(T, x.bfloat16(), u, k=i32([50] * rows))


def test_sample_settings_out_of_the_ordinary(T):
    rows, vocab = 16, 2000
    g = gen(4)
    x = 2 * randn(g, rows, vocab)
    u = torch.rand(rows, generator=g, device="cuda")
    check_draws(T, x, u, t=f32([0.0, -1.0, math.nan, 1e-30, 1e-31, math.inf, 1e30, 2.0 ** -99] * 2))
    check_draws(T, x, u, k=i32([0, -5, 1, 2, vocab - 1, vocab, vocab + 1, 2 ** 31 - 1] * 2))
    check_draws(T, x, u, p=f32([0.0, -1.0, math.nan, 1e-30, 1.0, 2.0, 1 - 2.0 ** -24, 1e-7] * 2))
    check_draws(T, x, u, m=f32([0.0, -1.0, math.nan, 1e-30, 1.0, 2.0, 1 - 2.0 ** -24, 2.0 ** -40] * 2))
    last = 1 - 2.0 ** -24
    check_draws(T, x, f32([0.0, last, -1.0, 1.0, 5.0, math.inf, -0.0, 0.5] * 2), k=i32([3] * rows))
    check_draws(T, x, f32([0.0, last, 1.0, 2.0] * 4))
    nan = torch.empty(rows, dtype=torch.int32, device="cuda")
    T.tadm_sample(x, f32([math.nan] * rows), nan)
    zero = torch.empty_like(nan)
    T.tadm_sample(x, f32([0.0] * rows), zero)
    assert torch.equal(nan, zero)


def test_sample_draws_by_weight(T):
    """An even grid of random numbers meets each id as often as its probability says."""
    n = 4096
    x = torch.tensor([0.0, 1.0, -1.0, 0.5, 0.5, -20.0], device="cuda").repeat(n, 1)
    tok = torch.empty(n, dtype=torch.int32, device="cuda")
    T.tadm_sample(x, (torch.arange(n, device="cuda") + 0.5) / n, tok)
    share = torch.bincount(tok.long(), minlength=6).double() / n
    assert (share - torch.softmax(x[0].double(), 0)).abs().max() <= 1.0 / n
    assert bool((tok[1:] >= tok[:-1]).all())                   # in the order of ids


def test_sample_of_strided_rows_is_that_of_dense_ones(T):
    g = gen(5)
    big = randn(g, 9, 5003)
    u = torch.rand(9, generator=g, device="cuda")
    for cut in (slice(0, 5000), slice(3, 4001), slice(4, 12)):
        a, b = (torch.empty(9, dtype=torch.int32, device="cuda") for _ in range(2))
        T.tadm_sample(big[:, cut], u, a, top_p=f32([0.8] * 9))
        T.tadm_sample(big[:, cut].contiguous(), u, b, top_p=f32([0.8] * 9))
        assert torch.equal(a, b)


def test_sample_past_32_bits(T):
    """Rows further than 2^31 elements from the first."""
    stride, vocab = 1 << 30, 1000
    big = torch.empty(2 * stride + vocab + 8, dtype=BF16, device="cuda")
    x = torch.as_strided(big, (3, vocab), (stride, 1))
    x.copy_(randn(gen(6), 3, vocab))
    check_draws(T, x, f32([0.1, 0.6, 0.9]), p=f32([0.9] * 3))


# ------------------------------------------------------------------ adapters
def lora_case(g, lens, n_in, n_out, rank, n, dtype, spare=0, first=0, adapter=None):
    cu = cum(lens, first)
    total = cu[-1] + spare
    x = randn(g, total, n_in).to(dtype)
    w = (randn(g, n_out, n_in) / math.sqrt(n_in)).to(dtype)
    a = (randn(g, n, rank, n_in) / math.sqrt(n_in)).to(dtype)
    b = (randn(g, n, n_out, rank) / math.sqrt(rank)).to(dtype)
    scale = torch.exp(0.5 * randn(g, n))
    if adapter is None:
        adapter = [i % (n + 1) - 1 for i in range(len(lens))]
    return x, w, a, b, scale, cu, adapter


def project64(x, w, a, b, scale, cu, adapter):
    """The projection in 64 bits, the sums of its products' magnitudes, and those of the adapters' part; 0 outside."""
    y = torch.zeros((x.shape[0], w.shape[0]), dtype=torch.float64, device="cuda")
    mag, low = torch.zeros_like(y), torch.zeros_like(y)
    w = w.double()
    for i, ad in enumerate(adapter):
        at = slice(cu[i], cu[i + 1])
        v = x[at].double()
        y[at], mag[at] = v @ w.T, v.abs() @ w.abs().T
        if 0 <= ad < a.shape[0]:
            A, B, s = a[ad].double(), b[ad].double(), float(scale[ad])
            y[at] += s * (v @ A.T) @ B.T
            low[at] = s * (v @ A.T).abs() @ B.abs().T
            mag[at] += s * (v.abs() @ A.abs().T) @ B.abs().T
    return y, mag, low


def lora(T, x, w, y, cu, adapter, a, b, scale, stream=None, scratch=None):
    if scratch is None:
        need = T.tadm_lora_scratch_size(len(cu) - 1, x.shape[0], x.shape[1], w.shape[0], a.shape[0], a.shape[1],
                                        1 if x.dtype == BF16 else 0)
        scratch = torch.full((need,), 255, dtype=torch.uint8, device="cuda")           # NaN in every type
    T.tadm_lora_project(x, w, y, i32(cu), i32(adapter), a, b, scale, scratch, stream=stream)
    return y


def check_lora(T, x, w, a, b, scale, cu, adapter, y_dtype):
    y = torch.full((x.shape[0], w.shape[0]), 7.5, dtype=y_dtype, device="cuda")
    lora(T, x, w, y, cu, adapter, a, b, scale)
    T.tadm_ragged_sync_status()
    ref, mag, low = project64(x, w, a, b, scale, cu, adapter)
    # fp32 sums of n products: at most n half steps of the sum of magnitudes, twice that where a unit truncates; the low-rank
    # part's factor to 16 significant bits; the output's own rounding
    n = x.shape[1] + a.shape[1]
    tol = n * 2.0 ** -23 * mag + 1e-30
    if x.dtype == BF16:
        tol += 2.0 ** -16 * low
    if y_dtype == BF16:
        tol += 2.0 ** -8 * ref.abs()
    at = slice(cu[0], cu[-1])
    err = (y[at].double() - ref[at]).abs()
    assert torch.isfinite(y[at]).all()
    assert (err <= tol[at]).all(), float((err / tol[at]).max())
    assert (y[:cu[0]] == 7.5).all() and (y[cu[-1]:] == 7.5).all()                      # rows of no sequence
    return y


LENS = [[1], [0, 5, 0, 130, 64, 1], [1] * 70, [300, 1, 257, 63], [129, 127, 1, 255], [0, 0, 3]]


@pytest.mark.parametrize("dtype,y_dtype", [(F32, F32), (BF16, BF16), (BF16, F32)])
@pytest.mark.parametrize("lens", LENS)
@pytest.mark.parametrize("n_in,n_out,rank,n", [(64, 64, 8, 1), (256, 768, 16, 3), (200, 72, 24, 5), (768, 2304, 64, 9),
                                               (1000, 333, 40, 2), (8, 1, 8, 4), (512, 4096, 128, 70)])
def test_lora(T, dtype, y_dtype, lens, n_in, n_out, rank, n):
    g = gen(sum(lens) + n_in + rank)
    check_lora(T, *lora_case(g, lens, n_in, n_out, rank, n, dtype, spare=len(lens) % 3), y_dtype)


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("rank,n", [(256, 3), (8, 300), (16, 0)])
def test_lora_many_and_none(T, dtype, rank, n):
    """High ranks, an adapter for every row, no adapter at all; rows in front of the first sequence."""
    g = gen(rank)
    lens = [1] * 300 + [77]
    check_lora(T, *lora_case(g, lens, 256, 520, rank, n, dtype, spare=3, first=5), dtype)
    check_lora(T, *lora_case(g, lens, 256, 520, rank, n, dtype, adapter=[-1] * len(lens)), dtype)
    ids = [(7 * i) % (n + 3) - 1 if i % 2 else [-5, n, 2 ** 31 - 1, -2 ** 31][i // 2 % 4] for i in range(len(lens))]
    check_lora(T, *lora_case(g, lens, 256, 520, rank, n, dtype, adapter=ids), dtype)


@pytest.mark.parametrize("lens", [[2048, 1, 1000], [32] * 8])
def test_lora_larger(T, lens):
    g = gen(8)
    check_lora(T, *lora_case(g, lens, 2048, 4096, 16, 2, BF16, spare=7), BF16)
    check_lora(T, *lora_case(g, lens, 2056, 4104, 64, 3, BF16), BF16)


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("lens,first,spare", [([40, 0, 3], 700, 1500), ([300, 70], 0, 3000), ([0, 0], 30, 600), ([600], 511, 1)])
def test_lora_in_long_buffers(T, dtype, lens, first, spare):
    """Sequences that begin and end inside the buffer: rows in front of them and behind them are left alone."""
    for n_in, n_out, rank in ((256, 768, 16), (2048, 4096, 24)):
        check_lora(T, *lora_case(gen(first), lens, n_in, n_out, rank, 2, dtype, spare=spare, first=first), dtype)


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_lora_strides(T, dtype):
    """Operands that are parts of wider buffers: nothing around y is touched."""
    g = gen(9)
    x, w, a, b, scale, cu, adapter = lora_case(g, [40, 200, 3], 128, 144, 16, 2, dtype)
    want = torch.empty((x.shape[0], 144), dtype=dtype, device="cuda")
    lora(T, x, w, want, cu, adapter, a, b, scale)
    wide_x, wide_w = torch.full((243, 160), math.nan, device="cuda").to(dtype), torch.full((144, 136), math.nan, device="cuda").to(dtype)
    wide_x[:, 16:144], wide_w[:, :128] = x, w
    for left, width in ((8, 200), (3, 151), (0, 145)):          # rows on 16 bytes, and not
        wide_y = torch.full((243, width), 2.0, dtype=dtype, device="cuda")
        lora(T, wide_x[:, 16:144], wide_w[:, :128], wide_y[:, left:left + 144], cu, adapter, a, b, scale)
        assert torch.equal(wide_y[:, left:left + 144], want)
        assert (wide_y[:, :left] == 2).all() and (wide_y[:, left + 144:] == 2).all()


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_lora_rows_keep_to_themselves(T, dtype):
    """NaN and infinities in one row of x, in spare rows and in adapters that no row has reach nobody else."""
    g = gen(10)
    x, w, a, b, scale, cu, adapter = lora_case(g, [1] * 40 + [90], 256, 512, 16, 6, dtype, spare=20, adapter=[i % 5 - 1 for i in range(41)])
    clean = torch.zeros((150, 512), dtype=dtype, device="cuda")
    lora(T, x, w, clean, cu, adapter, a, b, scale)
    x[3], x[7, 5], x[100, 9], x[130:] = math.nan, math.inf, -math.inf, math.nan
    a[4:], b[4:], scale[4:] = math.nan, math.nan, math.nan
    y = torch.zeros_like(clean)
    lora(T, x, w, y, cu, adapter, a, b, scale)
    others = [r for r in range(150) if r not in (3, 7, 100)]
    assert torch.equal(y[others], clean[others])
    assert not torch.isfinite(y[[3, 7, 100]]).all(1).any()


def test_lora_low_rank_part_keeps_its_bits(T):
    """Where W gives nothing, the output is the adapters' part alone: no worse than one rounding of it."""
    g = gen(11)
    x, w, a, b, scale, cu, adapter = lora_case(g, [64, 33], 512, 256, 32, 2, BF16, adapter=[0, 1])
    check_lora(T, x, torch.zeros_like(w), a, b, scale, cu, adapter, F32)


# ------------------------------------------------------------------ norms
def norm64(x, y, post, gate, pre, scale, eps, seq):
    """In 64 bits, and the magnitudes of the two terms of x'."""
    u = y.double()
    if post is not None:
        u = u / torch.sqrt(u.square().mean(-1, keepdim=True) + eps) * post.double()
    if gate is not None:
        u = u * gate.double()[seq]
    xo = scale * x.double() + u
    r = 1 / torch.sqrt(xo.square().mean(-1, keepdim=True) + eps)
    g = pre.double() if pre is not None else 1.0
    return xo, xo * r * g, (scale * x.double()).abs() + u.abs(), r * (g.abs() if pre is not None else 1.0)


def step(dtype):
    return 2.0 ** -8 if dtype == BF16 else 2.0 ** -24


def check_norm(got, want, mag, rg):
    """Sums of squares of up to 6144 elements in fp32 (a thread's own 16, then trees: under 40 steps; 120 in the form for
    odd widths), their root, the products: 2^-16 of a term covers them with room; each output's own rounding."""
    xo, no = got
    assert ((xo.double() - want[0]).abs() <= step(xo.dtype) * want[0].abs() + 2.0 ** -16 * mag + 1e-30).all()
    if no is not None:
        err = (no.double() - want[1]).abs()
        tol = step(no.dtype) * want[1].abs() + 2.0 ** -15 * (want[1].abs() + mag * rg) + 1e-30
        assert (err <= tol).all(), float((err / tol).max())


@pytest.mark.parametrize("xt", [F32, BF16])
@pytest.mark.parametrize("yt", [F32, BF16])
@pytest.mark.parametrize("t", [F32, BF16])
@pytest.mark.parametrize("d", [1, 8, 13, 256, 768, 1000, 1032, 2048, 4100, 5376, 8200, 16392])
@pytest.mark.parametrize("form", ["all", "plain", "gate", "post", "no_norm"])
def test_residual_norm(T, xt, yt, t, d, form):
    g = gen(d)
    lens, spare, first = [5, 0, 1, 17], 3, 2
    cu = cum(lens, first)
    total = cu[-1] + spare
    x, y = randn(g, total, d).to(xt), (3 * randn(g, total, d)).to(yt)
    post = (1 + randn(g, d)).to(t) if form in ("all", "post") else None
    gate = randn(g, 4, d).to(t) if form in ("all", "gate") else None
    pre = (1 + randn(g, d)).to(t) if form not in ("plain", "no_norm") else None
    scale = 0.7 if form == "all" else 1.0
    xo = torch.full((total, d), 9.0, device="cuda").to(xt)
    no = None if form == "no_norm" else torch.full((total, d), 9.0, device="cuda").to(t)
    T.tadm_residual_norm(x, y, xo, no, cu_rows=i32(cu), post_gain=post, gate=gate, pre_gain=pre, residual_scale=scale)
    at = slice(cu[0], cu[-1])
    seq = torch.repeat_interleave(torch.arange(4, device="cuda"), torch.tensor(lens, device="cuda"))
    want = norm64(x[at], y[at], post, gate, pre, np.float32(scale), np.float32(1e-6), seq)
    check_norm((xo[at], None if no is None else no[at]), *[want[:2]], want[2], want[3])
    for o in (xo, no):
        if o is not None:
            assert (o[:cu[0]] == 9).all() and (o[cu[-1]:] == 9).all()


@pytest.mark.parametrize("xt,yt,t", [(F32, F32, BF16), (F32, BF16, BF16), (BF16, BF16, BF16), (BF16, F32, F32)])
@pytest.mark.parametrize("d", [1032, 2048, 5376, 8192, 16384])
def test_residual_norm_of_many_rows(T, xt, yt, t, d):
    """More rows than blocks at a time, strided and in place, rows in front of and behind the sequences."""
    g = gen(d)
    lens, spare, first = [700, 0, 1, 1500, 133], 9, 4
    cu = cum(lens, first)
    total = cu[-1] + spare
    wide = randn(g, total, d + 16).to(xt)
    x = wide[:, 8:8 + d]
    y, x0, around = (3 * randn(g, total, d)).to(yt), x.clone(), wide.clone()
    post, gate, pre = (1 + randn(g, d)).to(t), randn(g, 5, d).to(t), (1 + randn(g, d)).to(t)
    no = torch.full((total, d), 9.0, device="cuda").to(t)
    T.tadm_residual_norm(x, y, x, no, cu_rows=i32(cu), post_gain=post, gate=gate, pre_gain=pre, residual_scale=0.7)
    at = slice(cu[0], cu[-1])
    seq = torch.repeat_interleave(torch.arange(5, device="cuda"), torch.tensor(lens, device="cuda"))
    want = norm64(x0[at], y[at], post, gate, pre, np.float32(0.7), np.float32(1e-6), seq)
    check_norm((x[at], no[at]), want[:2], want[2], want[3])
    around[at, 8:8 + d] = x[at]
    assert torch.equal(wide, around) and (no[:cu[0]] == 9).all() and (no[cu[-1]:] == 9).all()
    plain = torch.empty_like(no)
    T.tadm_residual_norm(x0.clone(), y, torch.empty_like(x0), plain)
    want = norm64(x0, y, None, None, None, 1.0, np.float32(1e-6), None)
    check_norm((want[0], plain), want[:2], want[2], want[3])


def test_residual_norm_in_place_and_strided(T):
    g = gen(20)
    for d, left, width in ((512, 8, 1024), (512, 3, 1025), (1500, 0, 1501)):
        wide = randn(g, 33, width)
        y = randn(g, 33, d).bfloat16()
        x0, y0, pre = wide[:, left:left + d].clone(), y.clone(), randn(g, d).bfloat16()
        around = wide.clone()
        T.tadm_residual_norm(wide[:, left:left + d], y, wide[:, left:left + d], y, pre_gain=pre, eps=1e-5)
        want = norm64(x0, y0, None, None, pre, 1.0, np.float32(1e-5), None)
        check_norm((wide[:, left:left + d], y), want[:2], want[2], want[3])
        around[:, left:left + d] = wide[:, left:left + d]
        assert torch.equal(wide, around)


def test_residual_norm_of_many_sequences(T):
    """More sequences than a warp looks at in one step, empty ones among them, each with a gate of its own."""
    g = gen(21)
    lens = [(7 * i) % 4 for i in range(2500)]
    total, d = sum(lens), 64
    x, y, gate = randn(g, total, d), randn(g, total, d), randn(g, len(lens), d)
    xo, no = torch.empty_like(x), torch.empty_like(x)
    T.tadm_residual_norm(x, y, xo, no, cu_rows=i32(cum(lens)), gate=gate)
    seq = torch.repeat_interleave(torch.arange(len(lens), device="cuda"), torch.tensor(lens, device="cuda"))
    want = norm64(x, y, None, gate, None, 1.0, np.float32(1e-6), seq)
    check_norm((xo, no), want[:2], want[2], want[3])


def test_residual_norm_zeros_and_specials(T):
    d = 96
    z = torch.zeros((4, d), device="cuda")
    xo, no = torch.empty_like(z), torch.empty_like(z)
    T.tadm_residual_norm(z, z, xo, no, post_gain=z[0] + 1, pre_gain=z[0] + 1)
    assert (xo == 0).all() and (no == 0).all()
    x, y = torch.ones_like(z), torch.ones_like(z)
    y[1, 3], x[2, 4] = math.nan, math.inf
    T.tadm_residual_norm(x, y, xo, no, pre_gain=z[0] + 1)
    assert torch.isfinite(xo[[0, 3]]).all() and torch.isfinite(no[[0, 3]]).all()
    assert torch.isnan(xo[1, 3]) and torch.isnan(no[1]).all() and torch.isinf(xo[2, 4])


# ------------------------------------------------------------------ streams, graphs, a run of them together
def test_calls_in_a_graph_and_on_streams(T):
    """Captured once, replayed on new contents of the same buffers; eager calls on two streams at once give the same."""
    g = gen(30)
    lens, d, qkv, vocab = [1, 33, 0, 66], 256, 384, 5000
    x, w, a, b, scale, cu, adapter = lora_case(g, lens, d, qkv, 16, 2, BF16)
    total = x.shape[0]
    res, y_in, pre = randn(g, total, d), randn(g, total, d).bfloat16(), randn(g, d).bfloat16()
    logits, u = 3 * randn(g, total, vocab), torch.rand(total, generator=g, device="cuda")
    cu_t, ad_t = i32(cu), i32(adapter)
    need = T.tadm_lora_scratch_size(4, total, d, qkv, 2, 16, 1)

    def buffers():
        return (torch.empty_like(res), torch.empty_like(y_in), torch.empty((total, qkv), dtype=BF16, device="cuda"),
                torch.empty(total, dtype=torch.int32, device="cuda"), torch.empty(need, dtype=torch.uint8, device="cuda"))

    def calls(o, stream=None):
        T.tadm_residual_norm(res, y_in, o[0], o[1], cu_rows=cu_t, pre_gain=pre, stream=stream)
        T.tadm_lora_project(o[1], w, o[2], cu_t, ad_t, a, b, scale, o[4], stream=stream)
        T.tadm_sample(logits, u, o[3], top_p=torch.full((total,), 0.9, device="cuda") if stream is None else p9, stream=stream)

    p9 = torch.full((total,), 0.9, device="cuda")
    torch.cuda.synchronize()
    one, two, three = buffers(), buffers(), buffers()
    s1, s2 = torch.cuda.Stream(), torch.cuda.Stream()
    for _ in range(5):
        calls(one, s1)
        calls(two, s2)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        calls(three, torch.cuda.current_stream())
    for o in (res, y_in, logits):
        o.copy_(randn(g, *o.shape))
    graph.replay()
    calls(one, s1)
    calls(two, s2)
    torch.cuda.synchronize()
    T.tadm_ragged_sync_status()
    for p, q, r in zip(one[:4], two[:4], three[:4]):
        assert torch.equal(p, q) and torch.equal(p, r)


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("lens", [[3, 1, 0, 9], [200, 1, 333, 50]])
def test_a_chain_of_calls_is_that_of_calls_one_by_one(T, dtype, lens):
    """Each call reads what the one before wrote, in buffers and scratch memory that all share, with nothing between them."""
    g = gen(33)
    d, n = 256, 3
    cu, total = cum(lens), sum(lens)
    cu_t, ad_t = i32(cu), i32([i % (n + 1) - 1 for i in range(len(lens))])
    w, a, b = (randn(g, *sh).to(dtype) / 16 for sh in ((d, d), (n, 16, d), (n, d, 16)))
    scale, gain = torch.ones(n, device="cuda"), (1 + 0.1 * randn(g, d)).to(dtype)
    need = T.tadm_lora_scratch_size(len(lens), total, d, d, n, 16, 1 if dtype == BF16 else 0)
    scratch = torch.empty(need, dtype=torch.uint8, device="cuda")
    x0, u = randn(g, total, d).to(dtype), torch.rand(total, generator=g, device="cuda")
    x, y, z = (torch.zeros((total, d), dtype=dtype, device="cuda") for _ in range(3))
    wide, logits = (randn(g, 6000, d) / 4).to(dtype), torch.zeros((total, 6000), device="cuda")
    tok = torch.zeros(total, dtype=torch.int32, device="cuda")
    p = torch.full((total,), 0.9, device="cuda")
    room = torch.empty(T.tadm_sample_scratch_size(total, 6000), dtype=torch.uint8, device="cuda")

    def run(between):
        toks = []
        x.copy_(x0), z.zero_()
        for _ in range(4):
            T.tadm_residual_norm(x, z, x, y, cu_rows=cu_t, pre_gain=gain), between()
            T.tadm_lora_project(y, w, z, cu_t, ad_t, a, b, scale, scratch), between()
            T.tadm_residual_norm(x, z, x, y, cu_rows=cu_t, post_gain=gain, pre_gain=gain), between()
            T.tadm_lora_project(y, w, z, cu_t, ad_t, a, b, scale, scratch), between()
            T.tadm_gemm(z, wide, logits, dtype=1 if dtype == BF16 else 0), between()
            T.tadm_sample(logits, u, tok, top_p=p, scratch=room), between()
            toks.append(tok.clone())
        return [x.clone(), y.clone(), z.clone()] + toks

    want = run(torch.cuda.synchronize)
    for _ in range(10):
        for got, ref in zip(run(lambda: None), want):
            assert torch.equal(got, ref)
    T.tadm_ragged_sync_status()


def test_a_serving_step(T):
    """A layer and a draw of ragged prompts as a server runs them: norm, QKV with adapters, packed attention, output
    projection with adapters, residual and norm, logits, sampling; each stage against 64 bits from what the one before gave."""
    g = gen(31)
    lens, heads, kv, hd, vocab, n = [40, 1, 129, 7], 4, 2, 64, 3000, 3
    d, cu = heads * hd, cum(lens)
    total, width = cu[-1], (heads + 2 * kv) * hd
    h, zero = randn(g, total, d), torch.zeros((total, d), device="cuda")
    gain = [(1 + 0.1 * randn(g, d)).bfloat16() for _ in range(3)]
    _, wq, aq, bq, sq, _, adapter = lora_case(g, lens, d, width, 16, n, BF16)
    _, wo, ao, bo, so, _, _ = lora_case(g, lens, d, d, 16, n, BF16)
    head = (randn(g, vocab, d) / 4).bfloat16()
    cu_t = i32(cu)
    x, nx = torch.empty_like(h), torch.empty((total, d), dtype=BF16, device="cuda")
    T.tadm_residual_norm(h, zero, x, nx, cu_rows=cu_t, pre_gain=gain[0])
    seq = torch.repeat_interleave(torch.arange(4, device="cuda"), torch.tensor(lens, device="cuda"))
    want = norm64(h, zero, None, None, gain[0], 1.0, np.float32(1e-6), seq)
    check_norm((x, nx), want[:2], want[2], want[3])
    qkv = check_lora(T, nx, wq, aq, bq, sq, cu, adapter, BF16).view(total, heads + 2 * kv, hd)
    o = torch.empty((total, heads, hd), dtype=BF16, device="cuda")
    T.tadm_attention_packed(qkv[:, :heads], qkv[:, heads:heads + kv], qkv[:, heads + kv:], o, cu_t, max(lens))
    y = check_lora(T, o.view(total, d), wo, ao, bo, so, cu, adapter, BF16)
    x2, n2 = torch.empty_like(h), torch.empty_like(nx)
    T.tadm_residual_norm(x, y, x2, n2, cu_rows=cu_t, post_gain=gain[1], pre_gain=gain[2])
    want = norm64(x, y, gain[1], None, gain[2], 1.0, np.float32(1e-6), seq)
    check_norm((x2, n2), want[:2], want[2], want[3])
    last = n2[torch.tensor(cu[1:], device="cuda") - 1]
    logits = torch.empty((4, vocab), device="cuda")
    T.tadm_gemm(last, head, logits, dtype=1)
    check_draws(T, logits, torch.rand(4, generator=g, device="cuda"), t=f32([0.0, 0.7, 1.0, 1.3]), k=i32([0, 50, 0, 0]),
                p=f32([1.0, 0.9, 0.95, 1.0]), m=f32([0.0, 0.0, 0.0, 0.02]), mask_id=vocab - 1)


FIRST_CALLS = """
import torch
from paper_2609_37924_gb300 import tadm as T
s, dev = torch.cuda.Stream(), "cuda"
x, w = torch.ones(40, 64, device=dev).bfloat16(), torch.eye(64, device=dev).bfloat16()
a, b = torch.zeros(1, 16, 64, device=dev).bfloat16(), torch.zeros(1, 64, 16, device=dev).bfloat16()
cu, ad = torch.tensor([0, 40], dtype=torch.int32, device=dev), torch.zeros(1, dtype=torch.int32, device=dev)
y, scale = torch.zeros(40, 64, device=dev).bfloat16(), torch.ones(1, device=dev)
room = torch.empty(T.tadm_lora_scratch_size(1, 40, 64, 64, 1, 16, 1), dtype=torch.uint8, device=dev)
logits = torch.zeros(2, 9000, device=dev)
logits[0, 8999] = logits[1, 17] = 1.0
tok, u, k = torch.zeros(2, dtype=torch.int32, device=dev), torch.zeros(2, device=dev), torch.ones(2, dtype=torch.int32, device=dev)
xo, no = torch.zeros(40, 64, device=dev), torch.zeros(40, 64, device=dev)
torch.cuda.synchronize()
g = torch.cuda.CUDAGraph()
with torch.cuda.graph(g, stream=s):
    T.tadm_lora_project(x, w, y, cu, ad, a, b, scale, room)
    T.tadm_residual_norm(torch.ones_like(xo), y, xo, no, cu_rows=cu)
    T.tadm_sample(logits, u, tok, top_k=k)
g.replay()
torch.cuda.synchronize()
T.tadm_ragged_sync_status()
assert (y == 1).all() and (xo == 2).all() and ((no - 1).abs() < 1e-6).all() and tok.tolist() == [8999, 17]
print("captured")
"""


def test_the_first_calls_of_a_process_can_be_captured(T):
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    r = subprocess.run([sys.executable, "-c", FIRST_CALLS], cwd=root, capture_output=True, text=True, timeout=300)
    assert r.returncode == 0 and r.stdout.strip() == "captured", r.stderr[-2000:]


@pytest.mark.parametrize("rows", [24, 120])
def test_sample_rows_of_every_kind_in_one_call(T, rows):
    """Rows that are drawn from the whole, from a list, from a window, from nothing, and from one id, side by side: each as alone."""
    g = gen(40)
    vocab = 20000
    x = 2.0 * randn(g, rows, vocab)
    x[3], x[9, 5:] = -math.inf, -math.inf
    x[4] = 0.5
    x[11, 19999] = math.inf
    x[12] += 1e6
    n = torch.arange(rows, device="cuda")
    t = torch.tensor([1.0, 0.5, 0.0, 5.0], device="cuda")[n % 4]
    k = torch.tensor([0, 0, 50, 6000, 1], dtype=torch.int32, device="cuda")[n % 5]
    p = torch.tensor([1.0, 0.9, 1.0, 0.3, 0.99, 0.999, 1.0], device="cuda")[n % 7]
    m = torch.tensor([0.0, 0.0, 0.01], device="cuda")[n % 3]
    u = torch.rand(rows, generator=g, device="cuda")
    check_draws(T, x, u, t, k, p, m, mask_id=19998)
    together, alone = (torch.empty(rows, dtype=torch.int32, device="cuda") for _ in range(2))
    T.tadm_sample(x, u, together, t, k, p, m)
    for r in range(rows):
        T.tadm_sample(x[r:r + 1], u[r:r + 1], alone[r:r + 1], t[r:r + 1], k[r:r + 1], p[r:r + 1], m[r:r + 1])
    assert torch.equal(together, alone)
