"""Window attention on the GPU against its formulas in float64.

Tolerances, before any run.  A score is a sum of D products, exact in float32 for bfloat16 and off by 2^-24 each for float32, of which at
most D follow one another: off by (D + 8) 2^-23 scale sum |q||k|.  The exponent s - lse (or s - max) is rounded once more, with what it is made of:
2^-22 (|s| + |lse|).  A weight is off by that, absolute in its exponent, twice in the forward (its sum of all weights too), by 2^-21 of the
exponential, and as bfloat16 operand by half a step, 2^-8.  Sums of n terms: (n + 16) 2^-23 of what is added up.  The products dout . v and
delta as the score.  At the end half a step of the storage type.

What falls below 2^-126 is 0 in float32 on this chip: a weight is off by up to that beside what it is off by relative to itself (exp(-88) is
where it ends; with scores of hundreds, most weights are there), and so is ds, by that times what the weight is multiplied with and once more
for the product itself."""
import math

import pytest
import torch

from paper_2210_10246_amd import binding as B

pytestmark = pytest.mark.gpu
DT = {"f32": torch.float32, "bf16": torch.bfloat16}
TINY = 2.0 ** -126


def seen(Sq, Sk, window, sinks, key_len, start, batch):
    """[batch, Sq, Sk]: which key a query sees."""
    i, j = torch.arange(Sq, device="cuda")[:, None], torch.arange(Sk, device="cuda")
    start = [Sk - Sq] * batch if start is None else start.tolist()
    key_len = [Sk] * batch if key_len is None else key_len.tolist()
    return torch.stack([(j <= s + i) & (j < n) & ((j > s + i - window) | (j < sinks)) for s, n in zip(start, key_len)])


def by_head(t, heads):
    """[B, S, n, D] -> [B, heads, S, D] in float64, shared heads repeated"""
    t = t.double().permute(0, 2, 1, 3)
    return t.repeat_interleave(heads // t.shape[1], 1) if t.shape[1] else t


def products(a, b, mask=None):
    """a b^T by head; where `mask` is false the pair is not made, whatever it holds."""
    out = torch.matmul(a, b.transpose(-1, -2))
    return out if mask is None else torch.where(mask, out, torch.zeros_like(out))


def weighted(p, v):
    """p v without the rows of v that have no weight: 0 times an element that is not finite is left out."""
    keep = (p != 0).any(-2)[..., None]
    return torch.matmul(p, torch.where(keep, v, torch.zeros_like(v)))


def reference(q, k, v, window, sinks, scale, key_len=None, start=None):
    heads, n = q.shape[2], k.shape[1]
    mask = seen(q.shape[1], n, window, sinks, key_len, start, q.shape[0])[:, None]
    qh, kh, vh = by_head(q, heads), by_head(k, heads), by_head(v, heads)
    s = torch.where(mask, products(qh, kh) * scale, -math.inf)
    lse = torch.logsumexp(s, -1) if n else torch.full(s.shape[:-1], -math.inf, device=s.device, dtype=s.dtype)
    some = torch.isfinite(lse)
    p = torch.exp(s - torch.where(some, lse, 0.0)[..., None])
    e = (q.shape[3] + 8) * 2.0 ** -23 * scale * products(qh.abs(), kh.abs(), mask)
    e = e + 2.0 ** -22 * (torch.where(mask, s.abs(), 0.0) + torch.where(some, lse, 0.0).abs()[..., None]) + 2.0 ** -21
    return mask, s, lse, p, e, vh, qh, kh


def near(got, want, off):
    assert got.shape == want.shape
    tol = off + want.abs() * torch.finfo(got.dtype).eps / 2
    over = (got.double() - want).abs() - tol
    assert bool((over <= 0).all()), f"{float(over.max())} beyond, at {int(over.argmax())} of {over.numel()}"


def half_step(dtype):
    return 2.0 ** -8 if dtype == torch.bfloat16 else 0.0


def check_forward(out, lse, q, k, v, window, sinks, scale, key_len=None, start=None):
    mask, s, want_lse, p, e, vh, _, _ = reference(q, k, v, window, sinks, scale, key_len, start)
    n = k.shape[1]
    worst = e.amax(-1, keepdim=True) if n else e.sum(-1, keepdim=True)
    rel = 2 * worst + half_step(q.dtype) + (n + 16) * 2.0 ** -22
    near(out.permute(0, 2, 1, 3), weighted(p, vh), rel * weighted(p, vh.abs()))
    if lse is not None:
        some = torch.isfinite(want_lse)
        assert torch.equal(torch.isneginf(lse), ~some)
        near(torch.where(some, lse, 0.0), torch.where(some, want_lse, 0.0), worst[..., 0] + (n + 16) * 2.0 ** -23)


def grouped(t, kv):
    """The sum over the heads that share one: [B, heads, S, D] -> [B, S, kv, D]"""
    return t.unflatten(1, (kv, -1)).sum(2).permute(0, 2, 1, 3)


def check_backward(dq, dk, dv, dout, q, k, v, out, lse, window, sinks, scale, key_len=None, start=None):
    heads, kv, n, D = q.shape[2], k.shape[2], k.shape[1], q.shape[3]
    mask, s, _, _, e, vh, qh, kh = reference(q, k, v, window, sinks, scale, key_len, start)
    p = torch.where(mask, torch.exp(torch.where(mask, s, 0.0) - torch.where(torch.isfinite(lse), lse, 0.0).double()[..., None]), 0.0)
    do, o = by_head(dout, heads), by_head(out, heads)
    dp, delta = products(do, vh, mask), (do * o).sum(-1, keepdim=True)
    ds = torch.where(mask, p * (dp - delta), 0.0)
    off = (D + 8) * 2.0 ** -23 * (products(do.abs(), vh.abs(), mask) + (do * o).abs().sum(-1, keepdim=True))
    h, rows = half_step(q.dtype), q.shape[1] * (heads // kv)
    ods = torch.where(mask, ds.abs() * (e + h) + p * off * (1 + e) + TINY * ((dp - delta).abs() + 1), 0.0)
    near(dq.permute(0, 2, 1, 3), scale * weighted(ds, kh), scale * weighted(ods + (n + 16) * 2.0 ** -23 * ds.abs(), kh.abs()))
    t = lambda x: x.transpose(-1, -2)  # noqa: E731
    sums = (rows + 16) * 2.0 ** -22
    near(dk, scale * grouped(weighted(t(ds), qh), kv), scale * grouped(weighted(t(ods + sums * ds.abs()), qh.abs()), kv))
    near(dv, grouped(weighted(t(p), do), kv), grouped(weighted(t(p * (e + h + sums) + mask * TINY), do.abs()), kv))


def normal(*shape, dtype, seed, scale=1.0):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return (scale * torch.randn(*shape, generator=g, device="cuda")).to(DT[dtype])


def guarded(*shape, dtype):
    """A tensor, and what lies behind it."""
    n = math.prod(shape)
    room = torch.full((n + 64,), 777.0, device="cuda", dtype=dtype)
    return room[:n].view(*shape), room[n:]


def inputs(batch, Sq, Sk, heads, kv, D, dtype):
    return normal(batch, Sq, heads, D, dtype=dtype, seed=1), normal(batch, Sk, kv, D, dtype=dtype, seed=2), \
        normal(batch, Sk, kv, D, dtype=dtype, seed=3)


def ints(values):
    return None if values is None else torch.tensor(values, dtype=torch.int32, device="cuda")


def kept(q, k, v, window, sinks, scale, key_len, start):
    """What a forward keeps, of the definition in 64 bits."""
    _, _, lse, p, _, vh, _, _ = reference(q, k, v, window, sinks, scale, key_len, start)
    return weighted(p, vh).permute(0, 2, 1, 3).to(q.dtype).contiguous(), lse.float()


def both_ways(batch, Sq, Sk, heads, kv, D, window, sinks, dtype, key_len=None, start=None, scale=None):
    q, k, v = inputs(batch, Sq, Sk, heads, kv, D, dtype)
    key_len, start = ints(key_len), ints(start)
    factor = D ** -0.5 if scale is None else scale
    (out, e1), (lse, e2) = guarded(batch, Sq, heads, D, dtype=q.dtype), guarded(batch, heads, Sq, dtype=torch.float32)
    B.tempo_window_attn_fwd(q, k, v, out, lse, window, sinks, scale, key_len, start)
    check_forward(out, lse, q, k, v, window, sinks, factor, key_len, start)
    alone = torch.empty_like(out)
    B.tempo_window_attn_fwd(q, k, v, alone, None, window, sinks, scale, key_len, start)
    assert torch.equal(alone, out)
    dout = normal(batch, Sq, heads, D, dtype=dtype, seed=4)
    o, l = kept(q, k, v, window, sinks, factor, key_len, start)
    (dq, e3), (dk, e4), (dv, e5) = (guarded(*t.shape, dtype=q.dtype) for t in (q, k, v))
    B.tempo_window_attn_bwd(dout, q, k, v, o, l, dq, dk, dv, window, sinks, scale, key_len, start)
    check_backward(dq, dk, dv, dout, q, k, v, o, l, window, sinks, factor, key_len, start)
    for end in (e1, e2, e3, e4, e5):
        assert bool((end == 777).all())


SIZES = [  # batch, Sq, Sk, heads, kv, D, window, sinks
    (1, 1, 1, 1, 1, 1, 1, 0), (1, 1, 1, 2, 1, 64, 5, 3), (2, 5, 5, 4, 2, 64, 3, 0), (1, 33, 33, 3, 1, 80, 7, 2), (2, 130, 130, 2, 2, 64, 40, 1),
    (1, 257, 257, 6, 2, 128, 100, 4), (1, 300, 300, 2, 1, 256, 64, 70), (2, 64, 200, 4, 4, 32, 50, 3), (1, 200, 64, 3, 3, 83, 20, 2),
    (3, 77, 77, 5, 5, 7, 1, 0), (1, 500, 500, 1, 1, 128, 1000, 0), (1, 129, 129, 12, 1, 33, 16, 200), (2, 31, 1000, 8, 1, 96, 128, 129),
    (1, 1, 2000, 8, 2, 128, 700, 4), (5, 2, 513, 7, 7, 200, 65, 33), (1, 1, 9, 1, 1, 255, 1 << 40, 1 << 40), (1, 640, 640, 2, 2, 64, 31, 0),
    (2, 0, 7, 2, 1, 16, 3, 1), (2, 7, 0, 2, 1, 16, 3, 1)]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("size", SIZES, ids=lambda s: "-".join(map(str, s)))
def test_sizes_both_ways(size, dtype):
    both_ways(*size, dtype)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("D", [*range(1, 18), *range(57, 64), *range(121, 128), 129, 160, 187, 192])
def test_rows_that_end_in_a_piece(D, dtype):
    """Every number of elements in a row's last piece of 16 bytes, with few rows and with many."""
    both_ways(2, 3, 70, 4, 2, D, 40, 1, dtype)
    both_ways(1, 70, 70, 2, 1, D, 40, 1, dtype)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("size,key_len,start", [
    ((4, 90, 90, 4, 2, 64, 20, 0), [90, 1, 0, 47], None),                     # padded; rows behind a sequence see nothing
    ((4, 90, 90, 4, 2, 64, 20, 3), [90, 1, 0, 47], None),
    ((3, 1, 400, 8, 2, 128, 50, 4), [400, 1, 77], [399, 0, 76]),              # a token each from a cache
    ((3, 4, 400, 6, 2, 64, 50, 0), [400, 4, 77], [396, 0, 73]),
    ((2, 40, 60, 2, 2, 48, 9, 2), None, [-25, 100]),                          # before the first key, behind the last
    ((2, 40, 60, 2, 2, 48, 9, 2), [1000, -3], [2 ** 31 - 1, -2 ** 31]),       # lengths beyond the keys and below none
    ((1, 200, 300, 2, 1, 128, 2 ** 31, 0), [211], [5]),
    ((2, 40, 60, 2, 2, 48, 100, 5), None, [200, 10]),                         # beyond a window that holds all keys: the first ones alone
    ((1, 600, 600, 4, 2, 64, 50, 300), [577], None),                          # first keys in several tiles
    ((2, 300, 300, 2, 1, 96, 33, 40), None, [0, 45]),
], ids=str)
def test_lengths_and_places(size, key_len, start, dtype):
    both_ways(*size, dtype, key_len, start)


MANY = [  # tiles enough for the whole chip, so that neither keys nor queries of a tile are in parts; key_len, start
    ((8, 400, 400, 16, 16, 64, 150, 1), None, None),
    ((8, 400, 400, 16, 16, 64, 150, 40), None, None),
    ((8, 400, 400, 16, 16, 64, 1000, 0), None, None),
    ((16, 300, 300, 16, 8, 128, 90, 3), [300, 299, 128, 129, 1, 0, 257, 256, 31, 32, 33, 200, 300, 90, 64, 5], None),
    ((16, 300, 300, 8, 8, 83, 90, 35), [300, 299, 128, 129, 1, 0, 257, 256, 31, 32, 33, 200, 300, 90, 64, 5], None),
    ((4, 1500, 1500, 8, 8, 96, 700, 130), None, None),                    # first keys in two tiles, then a window of many
    ((4, 1500, 1500, 8, 8, 64, 31, 7), None, [0, 3000, -700, 40]),
    ((16, 280, 280, 8, 8, 192, 60, 20), None, None),
    ((8, 400, 400, 12, 12, 256, 110, 2), None, None),
    ((2, 3300, 3300, 8, 8, 128, 2000, 4), [3300, 2999], None)]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("size,key_len,start", MANY, ids=str)
def test_many_tiles(size, key_len, start, dtype):
    both_ways(*size, dtype, key_len, start)
    torch.cuda.empty_cache()


@pytest.mark.parametrize("size", [(0, 3, 3, 2, 1), (1, 3, 3, 0, 0), (1, 0, 0, 2, 2)], ids=str)
def test_nothing_to_do(size):
    batch, Sq, Sk, heads, kv = size
    q, k, v = inputs(batch, Sq, Sk, heads, kv, 16, "f32")
    out, lse = torch.empty_like(q), torch.empty(batch, heads, Sq, device="cuda")
    grads = [torch.full_like(t, 7.0) for t in (q, k, v)]
    B.tempo_window_attn_fwd(q, k, v, out, lse, 3, 1)
    B.tempo_window_attn_bwd(q, q, k, v, out, lse, *grads, 3, 1)
    assert all(t.numel() == 0 for t in grads)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("Sq", [3, 200])
@pytest.mark.parametrize("window", [2 ** 31 - 1, 2 ** 31, 2 ** 31 + 30, 2 ** 40, 2 ** 63 - 1])
def test_windows_and_positions_next_to_2_to_31(window, Sq, dtype):
    """A window of more than 2^31 keys holds what it says at the furthest positions too."""
    both_ways(3, Sq, 60, 2, 2, 48, window, 0, dtype, None, [2 ** 31 - 1, 2 ** 31 - 25, -2 ** 31])
    both_ways(2, Sq, 60, 2, 1, 48, window, 2, dtype, [60, 41], [2 ** 31 - 1, 2 ** 31 - 200])


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("batch,Sq,Sk,kv,D", [(1, 3, 3, 2, 16), (2, 0, 300, 3, 83), (2, 70, 300, 1, 256)])
def test_key_heads_that_no_head_reads(batch, Sq, Sk, kv, D, dtype):
    """No heads of queries beside heads of keys: gradients of zeros, through both halves of the binding."""
    q, k, v = inputs(batch, Sq, Sk, 0, kv, D, dtype)
    out, lse = torch.empty_like(q), torch.empty(batch, 0, Sq, device="cuda")
    for stream in (None, torch.cuda.current_stream()):
        B.tempo_window_attn_fwd(q, k, v, out, lse, 3, 1, stream=stream)
        (dk, e1), (dv, e2) = (guarded(*t.shape, dtype=t.dtype) for t in (k, v))
        B.tempo_window_attn_bwd(out, q, k, v, out, lse, out, dk, dv, 3, 1, stream=stream)
        assert bool((dk == 0).all() and (dv == 0).all() and (e1 == 777).all() and (e2 == 777).all())


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_scales(dtype):
    both_ways(1, 70, 70, 2, 1, 64, 33, 1, dtype, scale=1.5)
    both_ways(1, 70, 70, 2, 1, 64, 33, 1, dtype, scale=1e-3)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("D", [64, 83, 128])
def test_strides(D, dtype):
    """Heads out of a projection, keys by head, one key head for all by a stride of 0 in v, gradients into a projection's."""
    batch, S, heads, kv, window, sinks, scale = 2, 150, 4, 2, 60, 3, D ** -0.5
    qkv = normal(batch, S, heads + 2 * kv, D, dtype=dtype, seed=5)
    q, k = qkv[:, :, :heads], normal(batch, kv, S, D + 3, dtype=dtype, seed=6)[..., 1:D + 1].transpose(1, 2)
    v = normal(batch, S, 1, D, dtype=dtype, seed=7).expand(batch, S, kv, D)
    out = torch.full((batch, heads, S, D + 1), 777.0, device="cuda", dtype=DT[dtype])
    lse = torch.empty(batch, heads, S, device="cuda")
    B.tempo_window_attn_fwd(q, k, v, out[..., :D].transpose(1, 2), lse, window, sinks)
    assert bool((out[..., D] == 777).all())
    check_forward(out[..., :D].transpose(1, 2), lse, q, k, v, window, sinks, scale)
    o, l = kept(q, k, v, window, sinks, scale, None, None)
    dout = normal(batch, heads, S, D, dtype=dtype, seed=8).transpose(1, 2)
    room = torch.full((batch, S, heads + 2 * kv + 1, D), 777.0, device="cuda", dtype=DT[dtype])
    dq, dk, dv = room[:, :, :heads], room[:, :, heads:heads + kv], room[:, :, heads + kv:heads + 2 * kv]
    B.tempo_window_attn_bwd(dout, q, k, v, o, l, dq, dk, dv, window, sinks)
    check_backward(dq, dk, dv, dout, q, k, v, o, l, window, sinks, scale)
    assert bool((room[:, :, -1] == 777).all())


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("what", [math.nan, math.inf, -math.inf])
def test_what_is_not_seen_is_not_looked_at(what, dtype):
    """A cache whose slots behind a sequence and before its window hold anything; padded queries and gradients."""
    lens = [300, 90, 7]
    batch, Sk, heads, kv, D, window, sinks = 3, 400, 4, 2, 64, 40, 2
    q, k, v = inputs(batch, 1, Sk, heads, kv, D, dtype)
    key_len, start = ints(lens), ints([n - 1 for n in lens])
    clean = torch.empty_like(q), torch.empty(batch, heads, 1, device="cuda")
    B.tempo_window_attn_fwd(q, k, v, *clean, window, sinks, None, key_len, start)
    for b, n in enumerate(lens):
        for t in (k, v):
            t[b, n:] = what
            t[b, sinks:max(n - window, sinks)] = what
    out = torch.empty_like(q), torch.empty(batch, heads, 1, device="cuda")
    B.tempo_window_attn_fwd(q, k, v, *out, window, sinks, None, key_len, start)
    assert torch.equal(out[0], clean[0]) and torch.equal(out[1], clean[1])
    # a padded batch in training, without first keys: rows far behind a sequence see nothing
    S, window, sinks = 300, 20, 0
    q, k, v = inputs(batch, S, S, heads, kv, D, dtype)
    dout = normal(batch, S, heads, D, dtype=dtype, seed=4)
    for b, n in enumerate(lens):
        k[b, n:], v[b, n:] = what, what
        q[b, n + window - 1:], dout[b, n + window - 1:] = what, what
    out, lse = torch.empty_like(q), torch.empty(batch, heads, S, device="cuda")
    B.tempo_window_attn_fwd(q, k, v, out, lse, window, sinks, None, key_len)
    grads = [torch.empty_like(t) for t in (q, k, v)]
    B.tempo_window_attn_bwd(dout, q, k, v, out, lse, *grads, window, sinks, None, key_len)
    for t in (out, *grads):
        assert bool(torch.isfinite(t).all())
    for b, n in enumerate(lens):
        assert bool((out[b, n + window - 1:] == 0).all() and (grads[0][b, n + window - 1:] == 0).all())
        assert bool(torch.isneginf(lse[b, :, n + window - 1:]).all())
        assert bool((grads[1][b, n:] == 0).all() and (grads[2][b, n:] == 0).all())


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_what_is_seen_and_not_finite_shows(dtype):
    q, k, v = inputs(1, 40, 40, 2, 1, 64, dtype)
    v[0, 30, 0, 5] = math.nan
    out, lse = torch.empty_like(q), torch.empty(1, 2, 40, device="cuda")
    B.tempo_window_attn_fwd(q, k, v, out, lse, 5, 0)
    assert bool(torch.isnan(out[0, 30:35, :, 5]).all()) and bool(torch.isfinite(out[..., 6:]).all())
    q[0, 3, 1, 0] = math.nan
    B.tempo_window_attn_fwd(q, k, v, out, lse, 5, 0)
    assert bool(torch.isnan(out[0, 3, 1]).all()) and bool(torch.isnan(lse[0, 1, 3]))


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_large_scores(dtype):
    """Scores of hundreds, maxima that grow by far along the keys: nothing overflows, what is far below counts for nothing."""
    both_ways(1, 300, 300, 2, 2, 64, 150, 2, dtype, scale=8.0)
    q, k, v = inputs(1, 1, 500, 2, 2, 64, dtype)
    k = k * torch.linspace(0.1, 12.0, 500, device="cuda", dtype=k.dtype)[:, None, None]
    out, lse = torch.empty_like(q), torch.empty(1, 2, 1, device="cuda")
    B.tempo_window_attn_fwd(q, k, v, out, lse, 500, 0, 1.0)
    check_forward(out, lse, q, k, v, 500, 0, 1.0)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_gradients_against_differences(dtype):
    """sum(out w) along a direction, in 64 bits on both sides of the inputs; the kernels' gradients of it by theirs.  The second
    difference's error is h^2 / 6 times a third derivative of about the sum's own size: 1e-5 of it at h = 2^-8; bfloat16 gradients are
    off by 2^-8 each of what they are, at random: 1e-2 of the norms is 2^-8 times 2.5."""
    size = 2, 70, 70, 4, 2, 64
    window, sinks, scale = 30, 3, 0.2
    x = [t.double() for t in inputs(*size, dtype)]
    w = normal(2, 70, 4, 64, dtype=dtype, seed=9)
    q, k, v = (t.to(DT[dtype]) for t in x)
    out, lse = torch.empty_like(q), torch.empty(2, 4, 70, device="cuda")
    B.tempo_window_attn_fwd(q, k, v, out, lse, window, sinks, scale)
    grads = [torch.empty_like(t) for t in (q, k, v)]
    B.tempo_window_attn_bwd(w, q, k, v, out, lse, *grads, window, sinks, scale)

    def value(q, k, v):
        _, _, _, p, _, vh, _, _ = reference(q, k, v, window, sinks, scale)
        return (weighted(p, vh).permute(0, 2, 1, 3) * w.double()).sum()
    h = 2.0 ** -8
    for n in range(3):
        d = torch.randn(x[n].shape, generator=torch.Generator(device="cuda").manual_seed(n), device="cuda", dtype=torch.float64)
        moved = [[t + way * h * d if i == n else t for i, t in enumerate(x)] for way in (1, -1)]
        slope = (value(*moved[0]) - value(*moved[1])) / (2 * h)
        got = (grads[n].double() * d).sum()
        assert abs(got - slope) <= (1e-4 if dtype == "f32" else 1e-2) * grads[n].double().norm() * d.norm() / d.numel() ** 0.5 * 3


def test_same_bits_each_time_and_both_halves_of_the_binding():
    q, k, v = inputs(2, 700, 700, 4, 2, 64, "bf16")
    dout = normal(2, 700, 4, 64, dtype="bf16", seed=4)
    results = []
    for stream in (None, None, torch.cuda.current_stream()):      # an explicit stream goes through ctypes
        out, lse = torch.empty_like(q), torch.empty(2, 4, 700, device="cuda")
        B.tempo_window_attn_fwd(q, k, v, out, lse, 300, 130, stream=stream)
        grads = [torch.empty_like(t) for t in (q, k, v)]
        B.tempo_window_attn_bwd(dout, q, k, v, out, lse, *grads, 300, 130, stream=stream)
        results.append((out, lse, *grads))
    for other in results[1:]:
        assert all(torch.equal(a, b) for a, b in zip(results[0], other))


def test_given_workspaces_side_by_side_on_two_streams_and_replays():
    """Two graphs, a workspace each, replayed at the same time and again after other work; the inputs change between replays."""
    size, window, sinks = (2, 260, 260, 4, 2, 64), 100, 5
    args = (2, 260, 260, 4, 2, 64, window, sinks)
    sides = []
    for seed in (0, 1):
        q, k, v = (t + seed for t in inputs(*size, "f32"))
        state = dict(q=q, k=k, v=v, out=torch.empty_like(q), lse=torch.empty(2, 4, 260, device="cuda"), dout=torch.ones_like(q),
                     grads=[torch.empty_like(t) for t in (q, k, v)])
        state["ws"] = [torch.empty(n(*args, torch.float32), dtype=torch.uint8, device="cuda")
                       for n in (B.tempo_window_attn_fwd_workspace_bytes, B.tempo_window_attn_bwd_workspace_bytes)]
        sides.append(state)

    def step(s, ws):
        B.tempo_window_attn_fwd(s["q"], s["k"], s["v"], s["out"], s["lse"], window, sinks, workspace=ws[0])
        B.tempo_window_attn_bwd(s["dout"], s["q"], s["k"], s["v"], s["out"], s["lse"], *s["grads"], window, sinks, workspace=ws[1])
    graphs, streams = [], [torch.cuda.Stream() for _ in sides]
    for s in sides:
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            step(s, s["ws"])
        graphs.append(graph)
    for turn in range(4):
        for s in sides:
            s["q"].mul_(1.0 + 0.1 * turn)
        torch.cuda.synchronize()
        for graph, stream in zip(graphs, streams):
            with torch.cuda.stream(stream):
                graph.replay()
        torch.cuda.synchronize()
        for s in sides:
            got = [t.clone() for t in (s["out"], s["lse"], *s["grads"])]
            step(s, (None, None))
            assert all(torch.equal(a, b) for a, b in zip(got, (s["out"], s["lse"], *s["grads"])))


def test_a_cache_beyond_2_to_32_elements():
    """Offsets of a batch, a token and a head that pass 32 bits."""
    Sk, kv, D, window, sinks = 1 << 18, 65, 256, 100, 3
    cache = torch.zeros(1, Sk, kv, D, device="cuda", dtype=torch.bfloat16)
    assert cache.numel() > 2 ** 32
    near_keys = normal(1, 128, kv, D, dtype="bf16", seed=1)
    cache[:, -128:] = near_keys
    cache[:, :sinks] = near_keys[:, :sinks] * 0.5
    q = normal(1, 1, kv, D, dtype="bf16", seed=2)
    out, lse = torch.empty_like(q), torch.empty(1, kv, 1, device="cuda")
    B.tempo_window_attn_fwd(q, cache, cache, out, lse, window, sinks)
    short = torch.cat((cache[:, :sinks], cache[:, -window:]), 1)
    check_forward(out, lse, q, short, short, window + sinks, 0, D ** -0.5)
    del cache
    torch.cuda.empty_cache()


def test_on_another_stream_than_its_own():
    q, k, v = inputs(1, 300, 300, 4, 4, 64, "bf16")
    want, out = torch.empty_like(q), torch.empty_like(q)
    B.tempo_window_attn_fwd(q, k, v, want, None, 64, 1)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        B.tempo_window_attn_fwd(q, k, v, out, None, 64, 1)
    side.synchronize()
    assert torch.equal(out, want)
