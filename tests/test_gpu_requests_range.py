"""The operators for requests with settings of their own where their numbers are hard to keep: what an adapter's factor
holds, long sums, logits at the limits of the temperature's range, against plain definitions in 64 bits."""
import importlib.util
import math
import os

import numpy as np
import pytest

torch = pytest.importorskip("torch")
from test_gpu_requests import BF16, F32, T, check_draws, check_norm, f32, gen, i32, lora, lora_case, norm64, project64, randn  # noqa: E402, F401

pytestmark = pytest.mark.gpu


# ------------------------------------------------------------------ adapters
@pytest.mark.parametrize("lens", [[1], [1] * 64, [32] * 8, [300, 1, 257, 63], [2048, 1, 1000]])
@pytest.mark.parametrize("n_in,rank,n", [(64, 8, 1), (256, 24, 3), (512, 64, 7), (1000, 128, 40)])
def test_lora_factor_in_fp32(T, lens, n_in, rank, n):
    """W gives nothing, a row of x has one element, a row of B one column: an output is one product b h, h = s a x.  s a x
    rounds once to fp32 (2^-24; a x has 16 bits); b times each part of h is exact, and what remains are two sums of them in
    units that may truncate (2^-23 each) and that of the shares of K (2^-24; the others are zero): 3 x 2^-23 in all."""
    g = gen(n_in + rank)
    x, w, a, b, scale, cu, adapter = lora_case(g, lens, n_in, 200, rank, n, BF16, adapter=[i % n for i in range(len(lens))])
    one = torch.randint(0, n_in, (x.shape[0], 1), generator=g, device="cuda")
    x = torch.zeros_like(x).scatter_(1, one, x.gather(1, one))
    only = torch.arange(200, device="cuda")[:, None] % rank
    b = torch.zeros_like(b).scatter_(2, only.expand(n, 200, 1), b.gather(2, only.expand(n, 200, 1)))
    y = torch.full((x.shape[0], 200), 7.5, device="cuda")
    lora(T, x, torch.zeros_like(w), y, cu, adapter, a, b, scale)
    T.tadm_ragged_sync_status()
    ref = project64(x, torch.zeros_like(w), a, b, scale, cu, adapter)[0]
    assert ((y.double() - ref).abs() <= 3 * 2.0 ** -23 * ref.abs()).all(), float(((y.double() - ref).abs() / ref.abs()).nan_to_num().max() * 2.0 ** 23)


@pytest.mark.parametrize("lens", [[1] * 70, [300, 1, 257, 63]])
@pytest.mark.parametrize("n_in,rank", [(1000, 16), (2048, 16), (5376, 64)])
def test_lora_long_sums(T, lens, n_in, rank):
    """Every 16 products a sum is rounded, by 2^-23 of it at most where the unit truncates; sums of products of both signs
    stay within four times the root of their squares' sum.  The same for h, whose errors are as independent from rank to rank."""
    x, w, a, b, scale, cu, adapter = lora_case(gen(n_in), lens, n_in, 264, rank, 5, BF16, adapter=[i % 5 for i in range(len(lens))])
    y = torch.full((x.shape[0], 264), 7.5, device="cuda")
    lora(T, x, w, y, cu, adapter, a, b, scale)
    ref = project64(x, w, a, b, scale, cu, adapter)[0]
    sq = lambda t: t.double().square()  # noqa: E731
    of_y, of_h = sq(x) @ sq(w).T, torch.zeros_like(ref)
    for i, ad in enumerate(adapter):
        at, s2 = slice(cu[i], cu[i + 1]), float(scale[ad]) ** 2
        of_y[at] += s2 * sq(x[at].double() @ a[ad].double().T) @ sq(b[ad]).T
        of_h[at] = s2 * (sq(x[at]) @ sq(a[ad]).T) @ sq(b[ad]).T
    tol = (n_in + 3 * rank) / 16 * 2.0 ** -21 * (of_y.sqrt() + of_h.sqrt())
    err = (y.double() - ref).abs()
    assert (err <= tol).all(), float((err / tol).max())


# ------------------------------------------------------------------ sampling
@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("vocab,rows", [(3000, 9), (30000, 6), (30000, 120)])
def test_sample_maxima_of_minus_zero(T, dtype, vocab, rows):
    """Rows without a positive logit whose largest ones are -0, which counts as 0."""
    g = gen(vocab + rows)
    x = -0.01 - 2 * randn(g, rows, vocab).abs()
    for r in range(rows):
        x[r, [7 + r, vocab // 2 + r, vocab - 1 - r][:r % 3 + 1]] = -0.0
    x = x.to(dtype)
    u = torch.rand(rows, generator=g, device="cuda")
    ones = torch.ones(rows, device="cuda")
    check_draws(T, x, u)
    check_draws(T, x, u, 0 * ones)
    check_draws(T, x, u, k=i32([1] * rows))
    check_draws(T, x, u, k=i32([40, 2, 5000] * (rows // 3)), mask_id=7)
    check_draws(T, x, u, 0.5 * ones, p=0.9 * ones)
    check_draws(T, x, u, 0.5 * ones, m=0.3 * ones)
    check_draws(T, x, u, k=i32([600] * rows), p=0.9 * ones, m=0.01 * ones)


@pytest.mark.parametrize("sign", [-1.0, 1.0])
@pytest.mark.parametrize("t", [1.0, 1e-4])
@pytest.mark.parametrize("border,setting", [(2.0 ** 22 / 16 / math.log2(math.e), ""), (2.0 ** 22 / 16 / math.log2(math.e), "k"),
                                            (2.0 ** 22 / 16 / math.log2(math.e), "m"), (101600.0, "p")])
def test_sample_maxima_on_both_sides_of_a_limit(T, sign, t, border, setting):
    """The passes over 8192 ids count weights from 2^(j / 16) and values in bins of a width of their own, while the numbers
    of either stay below 2^22: rows whose maxima per 8192 ids lie on both sides of that, a little lower from one to the next."""
    vocab, rows, step = 16384, 96, 2.0 ** -6
    if setting == "p":                                         # 510 bins over the depth that top-p needs
        border = 2.0 ** 22 * (math.log2(vocab / 0.1) + 0.5) / 510 / math.log2(math.e)
    g = gen(int(border))
    top = sign * border + step * (torch.arange(rows, device="cuda", dtype=torch.float64)[:, None] - rows / 2)
    x = top - step * torch.randint(0, 64, (rows, vocab), generator=g, device="cuda")
    u = torch.rand(rows, generator=g, device="cuda")
    kw = {"k": dict(k=i32([40, 9000, 2] * 32)), "m": dict(m=f32([0.9, 0.3] * 48)), "p": dict(p=f32([0.9] * rows))}.get(setting, {})
    for first, down in ((slice(8192, vocab), 0.25), (slice(0, 8192), 0.25), (slice(8192, vocab), 3.0)):
        z = x.clone()
        z[:, first] -= down
        z = (z * t).float()
        ts = torch.full((rows,), t, device="cuda")
        check_draws(T, z, u, ts, **kw)                         # many rows
        for r in range(0, rows, 8):                            # few
            check_draws(T, z[r:r + 8], u[r:r + 8], ts[r:r + 8], **{n: v[r:r + 8] for n, v in kw.items()})


@pytest.mark.parametrize("vocab", [3000, 9000])
def test_sample_logits_a_whole_range_apart(T, vocab):
    """Temperatures at which logits count that lie further apart than the largest number."""
    rows, top = 14, float(np.finfo(np.float32).max)
    g = gen(vocab + 3)
    x = top * (2 * torch.rand(rows, vocab, generator=g, device="cuda") - 1)
    x[:, 5], x[:, 6] = top, -top
    t = f32([1e37, 1e38, 3e38, math.inf, 1e36, 5e37, top] * 2)
    x[7:] *= 0.25
    u = torch.rand(rows, generator=g, device="cuda")
    many = torch.arange(rows, device="cuda")
    for y in (x, (1e31 * randn(g, rows, vocab)), x.bfloat16().clamp(-3e38, 3e38)):
        s = t if y is x or y.dtype == BF16 else f32([1e31, 2e30, 1.4e30, 1.5e30, 1e32, 1e35, 1e29] * 2)
        check_draws(T, y, u, s)
        check_draws(T, y, u, s, k=(many * 100 + 3).int(), mask_id=5)
        check_draws(T, y, u, s, p=f32([0.9, 0.3] * 7))
        check_draws(T, y, u, s, m=f32([0.5, 0.01] * 7), p=f32([0.9, 0.3] * 7))


@pytest.mark.parametrize("vocab,rows", [(30000, 4), (30000, 80)])
def test_sample_cuts_beside_a_token_s_mass(T, vocab, rows):
    """A few tokens far apart above a tail: top-p ends within some 10^-6 of where one of them does, on either side."""
    g = gen(vocab + rows + 7)
    x = randn(g, rows, vocab)
    at = torch.randint(0, vocab - 1, (rows, 5), generator=g, device="cuda")
    x.scatter_(1, at, torch.tensor([16.0, 13.5, 12.0, 10.5, 9.0], device="cuda") + 0.2 * randn(g, rows, 5))
    w = torch.sort(x.double(), 1, descending=True).values
    w = torch.exp(w - w[:, :1])
    mass = torch.cumsum(w, 1) / w.sum(1, keepdim=True)
    u = torch.rand(rows, generator=g, device="cuda")
    for j in range(6):
        for off in (3e-6, -3e-6, 1e-4, -1e-4):
            check_draws(T, x, u, p=(mass[:, j] + off).float())
        check_draws(T, x, u, p=(mass[:, j] + 3e-6).float(), m=f32([1e-6] * rows), mask_id=vocab - 1)


@pytest.mark.parametrize("vocab", [300, 9000])
def test_sample_min_p_of_one(T, vocab):
    """The ids of the maximum; at an infinite temperature, where every one weighs as much, all of them."""
    rows = 12
    g = gen(vocab + 4)
    x = randn(g, rows, vocab)
    x[:4] = torch.round(2 * x[:4]) / 2
    x[11, [5, 8]] = math.inf
    t, u = f32([1.0, math.inf, 0.5] * 4), torch.rand(rows, generator=g, device="cuda")
    check_draws(T, x, u, t, m=f32([1.0, 1.0, 2.0, 2.0] * 3))
    check_draws(T, x, u, t, m=f32([1.0, 1.0, 2.0, 2.0] * 3), p=f32([0.9] * rows), mask_id=3)


# ------------------------------------------------------------------ norms
@pytest.mark.parametrize("xt,yt,t", [(F32, F32, BF16), (F32, BF16, BF16), (BF16, BF16, BF16), (BF16, F32, F32)])
@pytest.mark.parametrize("d", [1032, 2048, 4096, 5376, 8192])
def test_residual_norm_of_many_rows_without_gains(T, xt, yt, t, d):
    """Both outputs, and the residual add alone, where rows are many and no parameter is given."""
    g = gen(d + 1)
    total = 1500
    x, y = randn(g, total, d).to(xt), (3 * randn(g, total, d)).to(yt)
    xo, no = torch.full_like(x, 9.0), torch.full((total, d), 9.0, device="cuda").to(t)
    T.tadm_residual_norm(x, y, xo, no)
    want = norm64(x, y, None, None, None, 1.0, np.float32(1e-6), None)
    check_norm((xo, no), want[:2], want[2], want[3])
    alone = torch.full_like(x, 9.0)
    T.tadm_residual_norm(x, y, alone, cu_rows=i32([0, 700, 700, total]))
    assert torch.equal(alone, xo)
    T.tadm_ragged_sync_status()


# ------------------------------------------------------------------ the example
def test_the_example_adds_its_projection_in_fp32(T):
    """The output projection reaches the fp32 stream without a rounding to bf16: sums of 2048 products in fp32, each of
    whose 128 steps rounds by 2^-23 of four times the root of the squares' sum at most (bf16 would be 2^-9 of the value)."""
    at = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples", "ragged_server.py")
    spec = importlib.util.spec_from_file_location("ragged_server", at)
    mod = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(mod)
    s = mod.Server(1, 16, 8, 128, seqs=4, max_len=128, pages=8, seed=1)
    g = gen(50)
    d, rows = 2048, 40
    h, n = torch.zeros((rows, d), device="cuda"), torch.empty((rows, d), dtype=BF16, device="cuda")
    o = randn(g, rows, 16, 128).bfloat16()
    s.output(h, n, o, 0, i32([0, rows]), i32([-1]))
    v, w = o.view(rows, d).double(), s.wo[0].double()
    tol = 128 * 2.0 ** -21 * (v.square() @ w.square().T).sqrt()
    assert ((h.double() - v @ w.T).abs() <= tol).all()
