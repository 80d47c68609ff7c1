"""Residual norms on the GPU against their formulas in float64.

Tolerances, before any run; u = 2^-23, of one float32 step or two.  A row's sum: a lane adds at most 16 elements (or every 1024th of a long row), then 6
steps across the wave and at most 16 waves: k = 40 + M / 1024 additions follow one another, each off by u of what is added up.  What is made of
one or two roundings is off by 2 u of itself.  A variance is off by (k + 4) u of itself, 1 / sqrt of it by half of that and its own rounding.
A column's sum over N rows: at most N + 40 additions.  At the end half a step of the storage type."""
import itertools

import pytest
import torch

from paper_2210_10246_amd import binding as B

pytestmark = pytest.mark.gpu
DT = {"f32": torch.float32, "bf16": torch.bfloat16}
U = 2.0 ** -23
EPS = 1e-5


def near(got, want, off):
    assert got.shape == want.shape
    tol = off + want.abs() * torch.finfo(got.dtype).eps / 2
    over = (got.double() - want).abs() - tol
    assert bool((over <= 0).all()), f"{float(over.max())} beyond, at {int(over.argmax())} of {over.numel()}"


def normal(*shape, dtype="f32", seed, scale=1.0, shift=0.0):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return (shift + scale * torch.randn(*shape, generator=g, device="cuda")).to(DT[dtype])


def additions(M):
    return 40 + M / 1024


def statistics(t, kind):
    """Mean and rstd, and how far they may be off."""
    k = additions(t.shape[1])
    mean = t.mean(1, keepdim=True) if kind == "layer" else torch.zeros_like(t[:, :1])
    off = k * U * t.abs().mean(1, keepdim=True) if kind == "layer" else torch.zeros_like(mean)
    rstd = (((t - mean) ** 2).mean(1, keepdim=True) + EPS) ** -0.5
    # a mean that is off adds its square to the variance
    return mean, rstd, off, rstd * ((k + 8) * U + (off * rstd) ** 2)


def hat(t, kind):
    mean, rstd, om, orstd = statistics(t, kind)
    h = (t - mean) * rstd
    return h, h.abs() * (orstd / rstd + 4 * U) + om * rstd, mean, rstd, om, orstd


def wide(t, M, value):
    return torch.full((M,), value, device="cuda", dtype=torch.float64) if t is None else t.double()


def rows_of(gate, N, M):
    return torch.ones(1, M, device="cuda", dtype=torch.float64) if gate is None else \
        gate.double().reshape(-1, M).repeat_interleave(N // gate.reshape(-1, M).shape[0], 0)


def check_stats(stats, mean, rstd, om, orstd):
    near(stats[:, :1], mean, om)
    near(stats[:, 1:], rstd, orstd)


def check_forward(x, f, gate, y, h, post, pre, alpha, beta):
    """post, pre: (kind, weight, bias, stats)"""
    N, M = x.shape
    fd, fo = f.double(), torch.zeros_like(f, dtype=torch.float64)
    by, b = rows_of(gate, N, M) * beta, 0.0
    if post[0] is not None:
        fd, fo, *st = hat(fd, post[0])
        if post[3] is not None:
            check_stats(post[3], *st)
        by, b = by * wide(post[1], M, 1.0), by * wide(post[2], M, 0.0)
    n = fd * by + b
    near(y, alpha * x.double() + n, by.abs() * (fo + 4 * U * fd.abs()) + 4 * U * ((alpha * x.double()).abs() + n.abs() + abs(b)))
    if pre[0] is None:
        return
    yh, yo, *st = hat(y.double(), pre[0])
    if pre[3] is not None:
        check_stats(pre[3], *st)
    w, b = wide(pre[1], M, 1.0), wide(pre[2], M, 0.0)
    near(h, yh * w + b, w.abs() * (yo + 4 * U * yh.abs()) + 4 * U * b.abs())


def through(g, og, t_hat, rstd, kind):
    """The gradient of what a norm is of, from that of t_hat, and how far it may be off."""
    k = additions(g.shape[1]) + 8
    mean = lambda v: v.mean(1, keepdim=True)  # noqa: E731
    s1, o1 = mean(g * t_hat), mean(og * t_hat.abs()) + k * U * mean((g * t_hat).abs())
    s2, o2 = (mean(g), mean(og) + k * U * mean(g.abs())) if kind == "layer" else (torch.zeros_like(s1), torch.zeros_like(s1))
    return rstd * (g - t_hat * s1 - s2), rstd * (og + 8 * U * (g.abs() + (t_hat * s1).abs() + s2.abs()) + t_hat.abs() * o1 + o2)


def check_backward(dy, dh, f, y, gate, post, pre, got, alpha, beta):
    """got: dx, df, dgate, dpost_weight, dpost_bias, dpre_weight, dpre_bias"""
    N, M = f.shape
    dx, df, dgate, dpw, dpb, dqw, dqb = got
    d = dy.double() if dy is not None else torch.zeros_like(f, dtype=torch.float64)
    od = 2 * U * d.abs()
    columns = lambda v, o: (v.sum(0), o.sum(0) + (N + 40) * U * v.abs().sum(0))  # noqa: E731
    if pre[0] is not None:
        mean, rstd = pre[3][:, :1].double(), pre[3][:, 1:].double()
        yh = (y.double() - mean) * rstd
        g = dh.double() * wide(pre[1], M, 1.0)
        more, om = through(g, 2 * U * g.abs(), yh, rstd, pre[0])
        d, od = d + more, od + om + 2 * U * (d.abs() + more.abs())
        if dqw is not None:
            near(dqw, *columns(dh.double() * yh, 4 * U * (dh.double() * yh).abs()))
        if dqb is not None:
            near(dqb, *columns(dh.double(), 0 * yh))
    near(dx, alpha * d, abs(alpha) * (od + 2 * U * d.abs()))
    gates = rows_of(gate, N, M) * beta
    fh, w, b = f.double(), wide(None, M, 1.0), wide(None, M, 0.0)
    if post[0] is not None:
        mean, rstd = post[3][:, :1].double(), post[3][:, 1:].double()
        fh, w, b = (fh - mean) * rstd, wide(post[1], M, 1.0), wide(post[2], M, 0.0)
    e, oe = gates * w * d, (gates * w).abs() * (od + 4 * U * d.abs())
    if post[0] is not None:
        near(df, *through(e, oe, fh, rstd, post[0]))
    else:
        near(df, e, oe)
    if dgate is not None:
        G = gate.reshape(-1, M).shape[0]
        of = lambda v: v.reshape(G, N // G, M).sum(1)  # noqa: E731
        n, on = fh * w + b, (fh * w).abs() * 6 * U + b.abs() * 2 * U
        parts = ((fh * w).abs() + b.abs()) * d.abs()      # the two sums are made apart
        near(dgate.reshape(G, M), beta * of(n * d), abs(beta) * (of(on * d.abs() + ((fh * w).abs() + b.abs()) * od) + (N + 48) * U * of(parts)))
    o = gates.abs() * (od + 6 * U * d.abs())
    if dpw is not None:
        near(dpw, *columns(gates * d * fh, o * fh.abs()))
    if dpb is not None:
        near(dpb, *columns(gates * d, o))


def guarded(*shape, dtype):
    n = 1
    for s in shape:
        n *= s
    room = torch.full((n + 64,), 777.0, device="cuda", dtype=dtype)
    return room[:n].view(*shape), room[n:]


def both_ways(N, M, dtype, post, pre, groups=1, gated=True, weights=True, biases=False, alpha=1.0, beta=1.0, dy=True):
    x, f = normal(N, M, dtype=dtype, seed=1), normal(N, M, dtype=dtype, seed=2, scale=2.0, shift=0.3)
    gate = normal(groups, M, seed=3) if gated else None
    ends = []

    def room(*shape, dt=torch.float32):
        t, end = guarded(*shape, dtype=dt)
        ends.append(end)
        return t
    norms = []
    for n, kind in enumerate((post, pre)):
        norms.append((kind, normal(M, seed=4 + n, scale=0.3, shift=1.0) if kind and weights else None,
                      normal(M, seed=6 + n) if kind and biases else None, room(N, 2) if kind else None))
    y, h = room(N, M, dt=x.dtype), room(N, M, dt=x.dtype) if pre else None
    args = [a for n in norms for a in n]
    B.tempo_residual_norm_fwd(x, f, gate, y, h, *args, alpha, beta, EPS, EPS)
    check_forward(x, f, gate, y, h, *norms, alpha, beta)
    again, h2 = x.clone(), torch.empty_like(x) if pre else None      # in place, without statistics
    B.tempo_residual_norm_fwd(again, f, gate, again, h2, *args[:3], None, *args[4:7], None, alpha, beta, EPS, EPS)
    assert torch.equal(again, y) and (not pre or torch.equal(h2, h))
    dy = normal(N, M, dtype=dtype, seed=8) if dy else None
    dh = normal(N, M, dtype=dtype, seed=9) if pre else None
    like = lambda t: None if t is None else room(*t.shape)  # noqa: E731
    got = [room(N, M, dt=x.dtype), room(N, M, dt=x.dtype), like(gate), like(norms[0][1]), like(norms[0][2]), like(norms[1][1]), like(norms[1][2])]

    def backward(dy, got, **more):
        B.tempo_residual_norm_bwd(dy, dh, f, y if pre else None, gate, *got[:3], *norms[0], *got[3:5], norms[1][0], norms[1][1], norms[1][3],
                                  *got[5:], alpha, beta, **more)
    backward(dy, got)
    check_backward(dy, dh, f, y, gate, *norms, got, alpha, beta)
    if dy is not None:      # in place, without the parameters' gradients; then again, through ctypes
        into = dy.clone()
        backward(into, [into, torch.empty_like(f)] + [None] * 5)
        assert torch.equal(into, got[0])
    other = [None if t is None else torch.empty_like(t) for t in got]
    backward(dy, other, stream=torch.cuda.current_stream())
    assert all(a is None or torch.equal(a, b) for a, b in zip(got, other))
    for end in ends:
        assert bool((end == 777).all())


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("N,M", [(1, 1), (1, 8), (3, 5), (2, 64), (5, 513), (7, 1001), (64, 1024), (37, 2056), (3, 4096), (2, 8192), (3, 8200),
                                 (1, 16384), (2, 16390), (2, 40001), (700, 96), (5000, 40)])
@pytest.mark.parametrize("post,pre,biases", [("rms", "rms", False), ("layer", "layer", True), (None, "rms", False), ("rms", None, False),
                                             ("layer", "rms", True)])
def test_sizes_both_ways(N, M, post, pre, biases, dtype):
    both_ways(N, M, dtype, post, pre, biases=biases, alpha=0.75, beta=0.5)


# Rows whose last piece begins earlier, within what the wave before it has: a wave of pieces, several, and one more element each.
ONE_BEHIND_A_WAVE = {"f32": (257, 259, 513, 1025, 4097), "bf16": (513, 519, 1025, 4097, 8193)}


@pytest.mark.parametrize("post,pre", [(None, None), (None, "rms"), ("layer", None), ("rms", "layer")])
@pytest.mark.parametrize("dtype,M", [(dtype, M) for dtype, widths in ONE_BEHIND_A_WAVE.items() for M in widths])
def test_in_place_where_two_waves_share_elements(dtype, M, post, pre):
    """y = x and dx = dy, over thousands of rows: the same bits as into tensors of their own, which are right."""
    both_ways(9, M, dtype, post, pre, alpha=0.75, beta=0.5)
    N, alpha, beta = 20011, 0.75, 0.5
    x, f, dy = (normal(N, M, dtype=dtype, seed=s) for s in (1, 2, 3))
    dh = normal(N, M, dtype=dtype, seed=4) if pre else None
    w = [normal(M, seed=5 + n, shift=1.0) if kind else None for n, kind in enumerate((post, pre))]
    st = [torch.empty(N, 2, device="cuda") if kind else None for kind in (post, pre)]
    y, h, h2 = torch.empty_like(x), *(torch.empty_like(x) if pre else None for _ in range(2))

    def forward(x, y, h):
        B.tempo_residual_norm_fwd(x, f, None, y, h, post, w[0], None, st[0], pre, w[1], None, st[1], alpha, beta, EPS, EPS)

    def backward(dy, dx, df):
        grads = [torch.empty_like(t) if t is not None else None for t in w]
        B.tempo_residual_norm_bwd(dy, dh, f, y if pre else None, None, dx, df, None, post, w[0], None, st[0], grads[0], None, pre, w[1], st[1],
                                  grads[1], None, alpha, beta)
        return [g for g in grads if g is not None]
    forward(x, y, h)
    dx, df, df2 = (torch.empty_like(x) for _ in range(3))
    grads = backward(dy, dx, df)
    for _ in range(3):
        into, into_dy = x.clone(), dy.clone()
        forward(into, into, h2)
        assert torch.equal(into, y) and (not pre or torch.equal(h2, h))
        again = backward(into_dy, into_dy, df2)
        assert torch.equal(into_dy, dx) and torch.equal(df2, df) and all(torch.equal(a, b) for a, b in zip(again, grads))


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("N,groups", [(12, 12), (96, 4), (1000, 8), (4096, 2), (3000, 1)])
@pytest.mark.parametrize("post,biases", [(None, False), ("rms", True), ("layer", False)])
def test_gates_of_groups(N, groups, post, biases, dtype):
    both_ways(N, 264, dtype, post, "rms", groups, biases=biases, beta=-2.0)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("post,pre,gated,weights,dy", itertools.product((None, "rms", "layer"), ("rms", "layer"), (True, False), (True, False),
                                                                       (True, False)))
def test_what_may_be_left_out(post, pre, gated, weights, dy, dtype):
    both_ways(33, 200, dtype, post, pre, gated=gated, weights=weights, dy=dy)


def test_no_rows():
    x, gate, w = torch.empty(0, 16, device="cuda"), torch.ones(1, 16, device="cuda"), torch.ones(16, device="cuda")
    stats = torch.empty(0, 2, device="cuda")
    B.tempo_residual_norm_fwd(x, x, gate, x, x, "rms", w, None, stats, "rms", w, None, stats)
    grads = [torch.full((16,), 7.0, device="cuda") for _ in range(5)]
    B.tempo_residual_norm_bwd(x, x, x, x, gate, x, x, grads[0], "rms", w, None, stats, grads[1], grads[2], "rms", w, stats, grads[3], grads[4])
    assert all(bool((g == 0).all()) for g in grads)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_large_offsets_and_not_finite(dtype):
    """A LayerNorm of values far from zero, whose variance is taken around their mean; a row that is not finite stays alone."""
    N, M = 6, 1000
    x, f = normal(N, M, dtype=dtype, seed=1), normal(N, M, dtype=dtype, seed=2, scale=1.0, shift=300.0)
    y, h, stats = torch.empty_like(x), torch.empty_like(x), [torch.empty(N, 2, device="cuda") for _ in range(2)]
    B.tempo_residual_norm_fwd(x, f, None, y, h, "layer", None, None, stats[0], "layer", None, None, stats[1])
    check_forward(x, f, None, y, h, ("layer", None, None, stats[0]), ("layer", None, None, stats[1]), 1.0, 1.0)
    f[2, 7] = float("nan")
    f[4, 0] = float("inf")
    y2, h2 = torch.empty_like(x), torch.empty_like(x)
    B.tempo_residual_norm_fwd(x, f, None, y2, h2, "layer", None, None, None, "layer", None, None, None)
    for n in range(N):
        if n in (2, 4):
            assert bool(torch.isnan(h2[n]).all())
        else:
            assert torch.equal(y2[n], y[n]) and torch.equal(h2[n], h[n])


def test_gradients_against_differences():
    """sum(y v + h w) along a direction in 64 bits; second differences at h = 2^-8 are good to about 1e-5 of the sum's size."""
    N, M, alpha, beta = 9, 50, 0.8, 0.5
    x, f, v, w = (normal(N, M, seed=s) for s in range(4))
    gate, pw, pb, qw, qb = normal(3, M, seed=4), *(normal(M, seed=s, shift=1.0) for s in range(5, 9))
    y, h = torch.empty_like(x), torch.empty_like(x)
    st = [torch.empty(N, 2, device="cuda") for _ in range(2)]
    B.tempo_residual_norm_fwd(x, f, gate, y, h, "layer", pw, pb, st[0], "rms", qw, qb, st[1], alpha, beta, EPS, EPS)
    inputs = [x, f, gate, pw, pb, qw, qb]
    grads = [torch.empty_like(t) for t in inputs]
    B.tempo_residual_norm_bwd(v, w, f, y, gate, grads[0], grads[1], grads[2], "layer", pw, pb, st[0], grads[3], grads[4], "rms", qw, st[1],
                              grads[5], grads[6], alpha, beta)

    def value(x, f, gate, pw, pb, qw, qb):
        n = hat(f, "layer")[0] * pw + pb
        y = alpha * x + beta * gate.repeat_interleave(3, 0) * n
        return (y * v.double()).sum() + ((hat(y, "rms")[0] * qw + qb) * w.double()).sum()
    wide_inputs, step = [t.double() for t in inputs], 2.0 ** -8
    for n, g in enumerate(grads):
        d = normal(*g.shape, seed=20 + n).double()
        moved = [[t + way * step * d if i == n else t for i, t in enumerate(wide_inputs)] for way in (1, -1)]
        slope = (value(*moved[0]) - value(*moved[1])) / (2 * step)
        assert abs((g.double() * d).sum() - slope) <= 1e-3 * g.double().norm()


def test_replays_and_another_stream():
    N, M = 300, 768
    x, f, gate = normal(N, M, dtype="bf16", seed=1), normal(N, M, dtype="bf16", seed=2), normal(2, M, seed=3)
    w = torch.ones(M, device="cuda")
    y, h, st = torch.empty_like(x), torch.empty_like(x), [torch.empty(N, 2, device="cuda") for _ in range(2)]
    grads = [torch.empty_like(x), torch.empty_like(x), torch.empty_like(gate), torch.empty_like(w), torch.empty_like(w)]
    ws = torch.empty(B.tempo_residual_norm_bwd_workspace_bytes(N, M, 2, x.dtype), dtype=torch.uint8, device="cuda")

    def step(ws):
        B.tempo_residual_norm_fwd(x, f, gate, y, h, "rms", w, None, st[0], "rms", w, None, st[1])
        B.tempo_residual_norm_bwd(y, h, f, y, gate, grads[0], grads[1], grads[2], "rms", w, None, st[0], grads[3], None, "rms", w, st[1], grads[4],
                                  None, workspace=ws)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step(ws)
    side = torch.cuda.Stream()
    for turn in range(4):
        f.mul_(1.5)
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):
            graph.replay()
        side.synchronize()
        got = [t.clone() for t in (y, h, *st, *grads)]
        step(None)
        assert all(torch.equal(a, b) for a, b in zip(got, (y, h, *st, *grads)))


def test_beyond_2_to_32_elements():
    N, M = 70000, 61440 + 8
    x = torch.zeros(N, M, device="cuda", dtype=torch.bfloat16)
    assert x.numel() > 2 ** 32
    x[-2:] = normal(2, M, dtype="bf16", seed=1)
    y, w = torch.empty_like(x), normal(M, seed=2)
    B.tempo_residual_norm_fwd(x, x, None, y, y, "rms", w, None, None, None, None, None, None)
    check_forward(x[-2:], x[-2:], None, y[-2:], None, ("rms", w, None, None), (None,) * 4, 1.0, 1.0)
    assert bool((y[:-2] == 0).all())
    del x, y
    torch.cuda.empty_cache()


def test_rows_of_2_to_26_columns():
    """More columns than one launch of the sums' kernel has lanes for."""
    both_ways(2, 2 ** 26 + 5, "bf16", None, "rms", biases=True, gated=False, dy=False)
    torch.cuda.empty_cache()


def test_the_longest_row():
    """Columns up to 2^31 - 2: the turn of the last ones does not begin anew below 0, and nothing behind them is touched."""
    M, alpha, beta = 2 ** 31 - 1, 0.75, 0.5
    x, f = (torch.empty(1, M, device="cuda", dtype=torch.bfloat16) for _ in range(2))
    y, end = guarded(1, M, dtype=torch.bfloat16)
    for n, t in enumerate((x, f)):
        t.view(-1)[:].copy_(normal(2 ** 20 + 1, dtype="bf16", seed=n).repeat(2 ** 11)[:M])
    B.tempo_residual_norm_fwd(x, f, None, y, None, None, None, None, None, None, None, None, None, alpha, beta)
    for a, b, got in zip(*(t[0].split(2 ** 28) for t in (x, f, y))):
        want = alpha * a.double() + beta * b.double()
        near(got, want, 4 * U * ((alpha * a.double()).abs() + (beta * b.double()).abs()))
    assert bool((end == 777).all())
    del x, f, y
    torch.cuda.empty_cache()
