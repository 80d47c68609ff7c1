"""Rotary positions with several axes on the GPU against their formula in float64.

Tolerance, before any run: c and n are good to 2^-22 of the scale; y = x1 c -+ x2 n is two products and a sum, each rounded once,
2^-24 each of |x1 c| + |x2 n| twice; then half a step of the storage type: 1.5 * 2^-22 scale (|x1| + |x2|) and that half step."""
import pytest
import torch

from paper_2210_10246_amd import binding as B

pytestmark = pytest.mark.gpu
DT = {"f32": torch.float32, "bf16": torch.bfloat16}


def normal(*shape, dtype, seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return torch.randn(*shape, generator=g, device="cuda").to(DT[dtype])


def expected(x, freqs, axes, positions, layout, scale, start, way):
    """The turned x and how far each element may be off."""
    B_, S = x.shape[:2]
    n = freqs.numel()
    p = positions if positions.dim() == 3 else positions[:, None]
    at = (p.expand(-1, B_, -1).double() + start)[axes.long().clamp(max=p.shape[0] - 1)]      # [pairs, B, S]
    turn = (at * freqs[:, None, None]).permute(1, 2, 0)[:, :, None]
    c, s = scale * torch.cos(turn), way * scale * torch.sin(turn)
    first = slice(0, n) if layout == "half" else slice(0, 2 * n, 2)
    second = slice(n, 2 * n) if layout == "half" else slice(1, 2 * n, 2)
    y, off = x.double().clone(), torch.zeros_like(x, dtype=torch.float64)
    x1, x2 = x[..., first].double(), x[..., second].double()
    y[..., first], y[..., second] = x1 * c - x2 * s, x2 * c + x1 * s
    off[..., first] = off[..., second] = 1.5 * 2.0 ** -22 * scale * (x1.abs() + x2.abs())
    return y, off


def near(got, want, off):
    tol = off + want.abs() * torch.finfo(got.dtype).eps / 2
    over = (got.double() - want).abs() - tol
    assert bool((over <= 0).all()), float(over.max())


def frequencies(n):
    return 100.0 ** (-torch.arange(n, dtype=torch.float64, device="cuda") / n)


@pytest.mark.parametrize("way", ["fwd", "bwd"])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("layout", ["half", "interleaved"])
@pytest.mark.parametrize("batch,S,heads,kv,D,pairs,axes,bits", [
    (1, 1, 1, 1, 2, 1, 1, 64), (2, 17, 3, 1, 64, 32, 2, 64), (1, 33, 5, 2, 83, 19, 3, 32), (3, 50, 4, 4, 128, 64, 4, 64), (2, 7, 2, 2, 30, 15, 3, 32),
    (1, 3000, 24, 8, 128, 64, 3, 64), (1, 2, 1, 1, 600, 300, 3, 64)])
def test_sizes(batch, S, heads, kv, D, pairs, axes, bits, layout, dtype, way):
    g = torch.Generator(device="cuda").manual_seed(0)
    dt = torch.int64 if bits == 64 else torch.int32
    positions = torch.randint(-50, 500, (axes, batch, S), generator=g, device="cuda", dtype=dt)
    of_pair = torch.randint(0, axes, (pairs,), generator=g, device="cuda").to(torch.uint8)
    freqs, q, k = frequencies(pairs), normal(batch, S, heads, D, dtype=dtype, seed=1), normal(batch, S, kv, D, dtype=dtype, seed=2)
    call = B.tempo_rotary_axes_fwd if way == "fwd" else B.tempo_rotary_axes_bwd
    q_out, k_out = (torch.full((t.shape[0], t.shape[2], S, D), 7.0, device="cuda", dtype=t.dtype).transpose(1, 2) for t in (q, k))
    call(q, k, freqs, of_pair, positions, q_out, k_out, layout, 1.25, 3)
    for t, out in ((q, q_out), (k, k_out)):
        near(out, *expected(t, freqs, of_pair, positions, layout, 1.25, 3, 1 if way == "fwd" else -1))
    shared = positions[:, 0]      # for the whole batch, and through ctypes; in place
    for p in (shared, shared[:, None], shared.t().contiguous().t()):
        a, b = q.clone(), k.clone()
        call(a, b, freqs, of_pair, p, a, b, layout, stream=torch.cuda.current_stream())
        c, d = q.clone(), k.clone()
        call(c, d, freqs, of_pair, p, c, d, layout)
        assert torch.equal(a, c) and torch.equal(b, d)
        near(a, *expected(q, freqs, of_pair, p, layout, 1.0, 0, 1 if way == "fwd" else -1))


@pytest.mark.parametrize("layout", ["half", "interleaved"])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_the_same_place_on_every_axis_is_one_axis(layout, dtype):
    q, freqs = normal(2, 40, 3, 64, dtype=dtype, seed=1), frequencies(30)
    p = torch.arange(40, device="cuda") * (1 << 40) - 12345
    one, several = torch.empty_like(q), torch.empty_like(q)
    B.tempo_rotary_fwd(q, None, freqs, p, one, None, layout, 1.1, 2)
    of_pair = (torch.arange(30, device="cuda") % 3).to(torch.uint8)
    B.tempo_rotary_axes_fwd(q, None, freqs, of_pair, p.expand(3, -1), several, None, layout, 1.1, 2)
    assert torch.equal(one, several)
    back = torch.empty_like(q)
    B.tempo_rotary_axes_bwd(several, None, freqs, of_pair, p.expand(3, -1), back, None, layout, 1 / 1.1, 2)
    # the turn back: twice what one is off by, of values that a turn leaves as they are together
    off = 2 * 1.5 * 2.0 ** -22 * 8 + 2 * torch.finfo(q.dtype).eps / 2 * 8
    assert bool(((back.double() - q.double()).abs() <= off).all())


def test_an_axis_beyond_the_last_is_the_last():
    q, freqs = normal(1, 5, 2, 16, dtype="f32", seed=1), frequencies(8)
    p = torch.arange(10, device="cuda").view(2, 5)
    out, same = torch.empty_like(q), torch.empty_like(q)
    B.tempo_rotary_axes_fwd(q, None, freqs, torch.tensor([0, 1, 2, 3, 255, 0, 1, 9], dtype=torch.uint8, device="cuda"), p, out, None)
    B.tempo_rotary_axes_fwd(q, None, freqs, torch.tensor([0, 1, 1, 1, 1, 0, 1, 1], dtype=torch.uint8, device="cuda"), p, same, None)
    assert torch.equal(out, same)


def test_replays():
    q, freqs = normal(2, 64, 4, 32, dtype="bf16", seed=1), frequencies(16)
    p, of_pair = torch.arange(192, device="cuda").view(3, 64).contiguous(), (torch.arange(16, device="cuda") // 6).to(torch.uint8)
    out, want = torch.empty_like(q), torch.empty_like(q)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        B.tempo_rotary_axes_fwd(q, None, freqs, of_pair, p, out, None)
    for _ in range(3):
        p += 17
        graph.replay()
        B.tempo_rotary_axes_fwd(q, None, freqs, of_pair, p, want, None)
        assert torch.equal(out, want)
