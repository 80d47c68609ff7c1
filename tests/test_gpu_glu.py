"""The gated feed-forward unit on the GPU against its formulas in float64.

Tolerances, before any run.  A sum of K products of bfloat16 values, which are exact in float32, is made of sums of a few of
them: at most K / 4 + 16 additions follow one another, each off by at most 2^-23 of what has been added up, in all
(K / 4 + 16) 2^-23 sum |a| |b|.  Three-way products of float32 leave out less than 2^-21 of sum |a| |b|.  act and act' are off
by at most 2^-20 (1 + |g|) (a sigmoid or Phi off by 2^-22, times at most 3 |g|), and have slopes of at most 1.2.  Then half
a step of the storage type."""
import math

import pytest
import torch

from paper_2210_10246_amd import binding as B

pytestmark = pytest.mark.gpu
DT = {"f32": torch.float32, "bf16": torch.bfloat16}
KINDS = ["silu", "gelu_erf", "gelu_tanh"]


def act(g, kind):
    if kind == "silu":
        s = torch.sigmoid(g)
        return g * s, s * (1 + g * (1 - s))
    if kind == "gelu_erf":
        phi = 0.5 * torch.erfc(-g / math.sqrt(2))
        return g * phi, phi + g * torch.exp(-0.5 * g * g) / math.sqrt(2 * math.pi)
    a = math.sqrt(2 / math.pi)
    t = torch.tanh(a * (g + 0.044715 * g ** 3))
    return 0.5 * g * (1 + t), 0.5 * (1 + t) + 0.5 * g * (1 - t * t) * a * (1 + 3 * 0.044715 * g * g)


def near(got, want, off):
    assert got.shape == want.shape
    tol = off + want.abs() * torch.finfo(got.dtype).eps / 2
    over = (got.double() - want).abs() - tol
    assert bool((over <= 0).all()), f"{float(over.max())} beyond, at {int(over.argmax())} of {over.numel()}"


def sums(a, b, dtype):
    """a b^T in float64, and how far the kernel's may be off."""
    total = a.abs() @ b.abs().t()
    return a @ b.t(), ((a.shape[1] / 4 + 16) * 2.0 ** -23 + (2.0 ** -21 if dtype == "f32" else 0)) * total


def normal(*shape, dtype, seed, scale=1.0):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return (scale * torch.randn(*shape, generator=g, device="cuda")).to(DT[dtype])


def inputs(T, H, F, dtype, bias=True):
    x, w = normal(T, H, dtype=dtype, seed=1), normal(2 * F, H, dtype=dtype, seed=2, scale=1 / math.sqrt(max(H, 1)))
    return x, w, normal(2 * F, dtype=dtype, seed=3, scale=0.5) if bias else None


def guarded(*shape, dtype):
    """A tensor, and what lies behind it."""
    n = math.prod(shape)
    room = torch.full((n + 64,), 777.0, device="cuda", dtype=DT[dtype])
    return room[:n].view(*shape), room[n:]


def check_forward(x, w, bias, gu, h, kind, dtype):
    F = w.shape[0] // 2
    want, off = sums(x.double(), w.double(), dtype)
    if bias is not None:
        want = want + bias.double()
        off = off + want.abs() * 2.0 ** -24
    if gu is not None:
        near(gu, want, off)
    g, u, og, ou = want[:, :F], want[:, F:], off[:, :F], off[:, F:]
    a, _ = act(g, kind)
    oa = 1.2 * og + 2.0 ** -20 * (1 + g.abs())
    near(h, a * u, oa * (u.abs() + ou) + a.abs() * ou + (a * u).abs() * 2.0 ** -23)


def check_backward(dh, gu, x, w, dgu, h, dx, dw, dbias, kind, dtype):
    F = w.shape[0] // 2
    d, g, u = dh.double(), gu[:, :F].double(), gu[:, F:].double()
    a, slope = act(g, kind)
    oa = 2.0 ** -20 * (1 + g.abs())
    if h is not None:
        near(h, a * u, oa * u.abs() + (a * u).abs() * 2.0 ** -23)
    want = torch.cat((d * u * slope, d * a), 1)
    off = torch.cat(((d * u).abs() * oa, d.abs() * oa), 1) + want.abs() * 2.0 ** -22
    near(dgu, want, off)
    stored = dgu.double()
    if dx is not None:
        near(dx, *sums(stored, w.double().t(), dtype))
    if dw is not None:
        near(dw, *sums(stored.t(), x.double().t(), dtype))
    if dbias is not None:
        near(dbias, want.sum(0), off.sum(0) + want.shape[0] * 2.0 ** -24 * want.abs().sum(0))


def both_ways(T, H, F, dtype, kind, bias):
    x, w, b = inputs(T, H, F, dtype, bias)
    (gu, e1), (h, e2) = guarded(T, 2 * F, dtype=dtype), guarded(T, F, dtype=dtype)
    B.tempo_glu_fwd(x, w, b, gu, h, kind)
    check_forward(x, w, b, gu, h, kind, dtype)
    alone = torch.empty_like(h)
    B.tempo_glu_fwd(x, w, b, None, alone, kind)
    assert torch.equal(alone, h)
    dh = normal(T, F, dtype=dtype, seed=4)
    (dgu, e3), (h2, e4), (dx, e5), (dw, e6) = (guarded(*s, dtype=dtype) for s in ((T, 2 * F), (T, F), (T, H), (2 * F, H)))
    db, e7 = guarded(2 * F, dtype=dtype) if bias else (None, h[:0])
    B.tempo_glu_bwd(dh, gu, x, w, dgu, h2, dx, dw, db, kind)
    check_backward(dh, gu, x, w, dgu, h2, dx, dw, db, kind, dtype)
    for end in (e1, e2, e3, e4, e5, e6, e7):
        assert bool((end == 777).all())


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("T,H,F", [
    (1, 1, 1), (1, 64, 64), (1, 1024, 515), (2, 7, 3), (3, 8, 8), (5, 65, 33), (16, 96, 40), (17, 257, 100), (31, 33, 129),
    (32, 130, 64), (33, 64, 32), (64, 64, 64), (65, 40, 31), (127, 129, 257), (128, 512, 128), (300, 264, 200), (257, 1, 96),
    (1000, 24, 1)])
@pytest.mark.parametrize("kind,bias", [("silu", False), ("gelu_erf", True), ("gelu_tanh", True)])
def test_sizes_both_ways(T, H, F, dtype, kind, bias):
    both_ways(T, H, F, dtype, kind, bias)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("T,H,F,bias", [(4096, 128, 2048, False), (4099, 72, 2050, True), (2048, 2048, 1024, False),
                                        (2050, 1031, 1029, True), (512, 4096, 1024, True), (40, 512, 8192, True),
                                        (8200, 1031, 4099, True), (8200, 1024, 4099, False), (8200, 1031, 4100, False)])
def test_sizes_of_every_tile(T, H, F, bias, dtype):
    both_ways(T, H, F, dtype, "silu", bias)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("T", [1, 15, 16, 17, 48, 63, 64, 65])
@pytest.mark.parametrize("H,F", [(64, 40), (72, 516), (520, 2048), (1000, 2052), (96, 10300), (1024, 31), (1001, 2050)])
def test_few_rows(T, H, F, dtype):
    x, w, b = inputs(T, H, F, dtype)
    (gu, e1), (h, e2) = guarded(T, 2 * F, dtype=dtype), guarded(T, F, dtype=dtype)
    B.tempo_glu_fwd(x, w, b, gu, h, "gelu_tanh")
    check_forward(x, w, b, gu, h, "gelu_tanh", dtype)
    assert bool((e1 == 777).all() and (e2 == 777).all())


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("T,H,F", [(0, 16, 8), (5, 0, 8), (5, 16, 0), (0, 0, 0)])
def test_sums_of_nothing(T, H, F, dtype):
    x, w, b = inputs(T, H, F, dtype)
    gu, h = (torch.full(s, 7.0, device="cuda", dtype=DT[dtype]) for s in ((T, 2 * F), (T, F)))
    B.tempo_glu_fwd(x, w, b, gu, h)
    check_forward(x, w, b, gu, h, "silu", dtype)
    dgu, h2, dx, dw, db = (torch.full(s, 7.0, device="cuda", dtype=DT[dtype]) for s in ((T, 2 * F), (T, F), (T, H), (2 * F, H), (2 * F,)))
    B.tempo_glu_bwd(normal(T, F, dtype=dtype, seed=4), gu, x, w, dgu, h2, dx, dw, db)
    assert T > 0 or (bool((dw == 0).all()) and bool((db == 0).all()))
    assert F > 0 or bool((dx == 0).all())


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_backward_in_place_and_in_part(dtype):
    """dgu in gu's place, and every output left out in turn: the same bits."""
    T, H, F = 70, 96, 130
    x, w, b = inputs(T, H, F, dtype)
    gu, dh = normal(T, 2 * F, dtype=dtype, seed=5), normal(T, F, dtype=dtype, seed=6)
    like = (torch.empty_like(gu), torch.empty_like(dh), torch.empty_like(x), torch.empty_like(w), torch.empty_like(b))
    B.tempo_glu_bwd(dh, gu, x, w, *like)
    place = gu.clone()
    outs = [torch.empty_like(t) for t in like[1:]]
    B.tempo_glu_bwd(dh, place, x, w, place, *outs)
    assert torch.equal(place, like[0]) and all(torch.equal(a, c) for a, c in zip(outs, like[1:]))
    for left in range(1, 5):
        outs = [None if i == left else torch.empty_like(t) for i, t in enumerate(like)]
        B.tempo_glu_bwd(dh, gu, x, w, *outs)
        assert all(a is None or torch.equal(a, c) for a, c in zip(outs, like))


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("kind", KINDS)
def test_gates_of_any_size(kind, dtype):
    """Gates from the deep tails to where squares overflow, and special values: the limits of the formulas."""
    g = torch.cat([torch.linspace(-30, 30, 997), torch.tensor([0.0, -0.0, 1e-30, -1e-30, 60.0, -60.0, 1e20, -1e20, 3e38, -3e38])])
    T, F = 1, g.numel()
    gu = torch.cat([g, torch.ones(F)])[None].to("cuda", DT[dtype])
    dh = torch.ones(1, F, device="cuda", dtype=DT[dtype])
    x, w = torch.zeros(1, 8, device="cuda", dtype=DT[dtype]), torch.zeros(2 * F, 8, device="cuda", dtype=DT[dtype])
    dgu, h = torch.empty_like(gu), torch.empty_like(dh)
    B.tempo_glu_bwd(dh, gu, x, w, dgu, h, None, None, None, kind)
    assert bool(torch.isfinite(dgu).all()) and bool(torch.isfinite(h).all())
    gate = gu[:, :F].double()
    inner = gate.abs() <= 30
    a, slope = act(gate, kind)
    near(h[inner], a[inner], (2.0 ** -20 * (1 + gate.abs()))[inner])
    near(dgu[:, :F][inner], slope[inner], (2.0 ** -20 * (1 + gate.abs()))[inner])
    # beyond: g or 1 on the right, 0 on the left, but for at most 60 exp(-60) = 5.3e-25 (SiLU at 60)
    far = ~inner
    assert bool(((h[far].double() - gate[far].clamp(min=0.0)).abs() <= 6e-25).all())
    assert bool(((dgu[:, :F][far].double() - (gate[far] > 0).double()).abs() <= 6e-25).all())


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_what_is_not_finite_stays_in_its_row(dtype):
    T, H, F = 130, 72, 96
    x, w, b = inputs(T, H, F, dtype)
    clean_gu, clean_h = torch.empty(T, 2 * F, device="cuda", dtype=DT[dtype]), torch.empty(T, F, device="cuda", dtype=DT[dtype])
    B.tempo_glu_fwd(x, w, b, clean_gu, clean_h)
    x[7, 3], x[T - 1, H - 1] = float("nan"), float("inf")
    gu, h = torch.empty_like(clean_gu), torch.empty_like(clean_h)
    B.tempo_glu_fwd(x, w, b, gu, h)
    rows = torch.ones(T, dtype=torch.bool, device="cuda")
    rows[7] = rows[T - 1] = False
    assert torch.equal(gu[rows], clean_gu[rows]) and torch.equal(h[rows], clean_h[rows])
    assert bool(torch.isnan(gu[7]).all()) and not bool(torch.isfinite(gu[T - 1]).any())


def test_gradients_agree_with_differences():
    """dx, dw and dbias of sum(h dh) against central differences of the kernel's own forward, float32."""
    T, H, F = 6, 20, 12
    x, w, b = inputs(T, H, F, "f32")
    dh = normal(T, F, dtype="f32", seed=8)

    def loss(x, w, b, kind):
        h = torch.empty_like(dh)
        B.tempo_glu_fwd(x, w, b, None, h, kind)
        return float((h.double() * dh.double()).sum())
    for kind in KINDS:
        gu, h = torch.empty(T, 2 * F, device="cuda"), torch.empty_like(dh)
        B.tempo_glu_fwd(x, w, b, gu, h, kind)
        dgu, dx, dw, db = torch.empty_like(gu), torch.empty_like(x), torch.empty_like(w), torch.empty_like(b)
        B.tempo_glu_bwd(dh, gu, x, w, dgu, None, dx, dw, db, kind)
        for at, (t, grad) in enumerate(((x, dx), (w, dw), (b, db))):
            way = normal(*t.shape, dtype="f32", seed=20 + at)
            step = 2.0 ** -7
            args = [x, w, b]
            args[at] = t + step * way
            up = loss(*args, kind)
            args[at] = t - step * way
            down = loss(*args, kind)
            slope = float((grad.double() * way.double()).sum())
            # third derivatives along `way` are at most some |way|^3 |dh|; the step's square is 6e-5
            assert abs((up - down) / (2 * step) - slope) <= 2e-3 * float((grad.double() * way.double()).abs().sum())


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_replays_streams_and_workspaces(dtype):
    """Two captured calls of split sums, each with its own workspace or one of the caller's; replays after eager calls."""
    T, H, F = 24, 2048, 96
    x, w, b = inputs(T, H, F, dtype)
    dh = normal(T, F, dtype=dtype, seed=6)
    bufs = lambda: [torch.empty(s, device="cuda", dtype=DT[dtype]) for s in ((T, 2 * F), (T, F), (T, 2 * F), (T, H), (2 * F, H), (2 * F,))]  # noqa: E731

    def step(gu, h, dgu, dx, dw, db, ws=None, stream=None):
        B.tempo_glu_fwd(x, w, b, gu, h, "silu", ws, stream=stream)
        B.tempo_glu_bwd(dh, gu, x, w, dgu, None, dx, dw, db, "silu", ws, stream=stream)
    eager, one, two = bufs(), bufs(), bufs()
    step(*eager)
    need = max(B.tempo_glu_fwd_workspace_bytes(T, H, F, DT[dtype]), B.tempo_glu_bwd_workspace_bytes(T, H, F, DT[dtype]))
    mine = torch.empty(max(need, 16), dtype=torch.uint8, device="cuda")
    graphs = [torch.cuda.CUDAGraph(), torch.cuda.CUDAGraph()]
    with torch.cuda.graph(graphs[0]):
        step(*one)
    with torch.cuda.graph(graphs[1]):
        step(*two, ws=mine)
    for turn in range(3):
        x.copy_(normal(T, H, dtype=dtype, seed=30 + turn))
        step(*eager)
        for g in graphs:
            g.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, c) and torch.equal(a, d) for a, c, d in zip(eager, one, two))
    side, other = torch.cuda.Stream(), bufs()
    side.wait_stream(torch.cuda.current_stream())
    step(*other, stream=side)
    side.synchronize()
    assert all(torch.equal(a, c) for a, c in zip(eager, other))
    if need > 16:
        with pytest.raises(B.TempoError, match="workspace"):
            step(*other, ws=mine[:16])


def test_more_than_2_32_elements():
    """[g | u] and h beyond 2^32 elements; the last rows, and every row's sum over the tiles, against float64."""
    T, H, F = 70001, 32, 32768
    x, w, _ = inputs(T, H, F, "bf16", False)
    gu, h = torch.empty(T, 2 * F, device="cuda", dtype=torch.bfloat16), torch.empty(T, F, device="cuda", dtype=torch.bfloat16)
    B.tempo_glu_fwd(x, w, None, gu, h)
    rows = torch.tensor([0, 32767, 32768, 65535, 65536, T - 2, T - 1], device="cuda")
    check_forward(x[rows], w, None, gu[rows], h[rows], "silu", "bf16")
    dx, dw = torch.empty_like(x), torch.empty_like(w)
    B.tempo_glu_bwd(h, gu, x, w, gu, None, dx, dw, None)      # dgu in gu's place, h as its gradient
    near(dx[rows], *sums(gu[rows].double(), w.double().t(), "bf16"))
    columns = torch.tensor([0, F - 1, F, 2 * F - 1], device="cuda")
    near(dw[columns], *sums(gu[:, columns].double().t(), x.double().t(), "bf16"))
