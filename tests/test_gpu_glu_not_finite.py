"""The gated unit's forward at gates whose squares overflow and at gates that are infinite, in a plan that makes each sum in one piece
and in one that makes it in parts: h is what act(g) u is in float64, and what the backward makes of the stored gates.

Tolerances: test_gpu_glu's.  Infinities and NaN have to be where the formula has them: act(+inf) = +inf for all three, and -inf
times a sigmoid or Phi of 0 is NaN."""
import pytest
import torch

from paper_2210_10246_amd import binding as B
from test_gpu_glu import DT, KINDS, act, check_forward, normal

pytestmark = pytest.mark.gpu
# few rows on tiles of their own, tiles of 64 and 128, odd row lengths, sums in parts
SIZES = [(3, 64, 2048), (40, 128, 2048), (130, 72, 96), (130, 73, 95), (1030, 264, 1000), (8, 4096, 64)]


def forward(x, w, dtype, kind):
    T, F = x.shape[0], w.shape[0] // 2
    gu, h = torch.empty(T, 2 * F, device="cuda", dtype=DT[dtype]), torch.empty(T, F, device="cuda", dtype=DT[dtype])
    B.tempo_glu_fwd(x, w, None, gu, h, kind)
    again = torch.empty_like(h)
    dgu, dh = torch.empty_like(gu), torch.ones_like(h)
    B.tempo_glu_bwd(dh, gu, x, w, dgu, again, None, None, None, kind)
    return gu, h, again


def rows_of(gates, T, H, F, dtype):
    """x and w whose gates are those, one after the other (column 0 alone counts in them), and whose u are ordinary."""
    x, w = normal(T, H, dtype=dtype, seed=1), normal(2 * F, H, dtype=dtype, seed=2, scale=H ** -0.5)
    x[:, 0] = 1
    w[:F] = 0
    w[:F, 0] = torch.tensor(gates, device="cuda").to(DT[dtype]).repeat(F // len(gates) + 1)[:F]
    w[F:, 0] = 0
    return x, w


def test_a_size_whose_sums_are_made_in_parts():
    for dtype in DT:
        assert B.tempo_glu_fwd_workspace_bytes(8, 4096, 64, DT[dtype]) >= 2 * 8 * 128 * 4


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("T,H,F", SIZES)
def test_gates_whose_squares_overflow(T, H, F, kind, dtype):
    x, w = rows_of([60.0, -60.0, 200.0, -200.0, 1e4, -1e4, 3e19, -3e19, 1e30, -1e30, 1e37, -1e37], T, H, F, dtype)
    gu, h, again = forward(x, w, dtype, kind)
    assert bool(torch.isfinite(h).all()) and bool(torch.isfinite(again).all())
    check_forward(x, w, None, gu, h, kind, dtype)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("T,H,F", SIZES)
def test_gates_that_are_infinite(T, H, F, kind, dtype):
    """Sums of two finite products that are beyond the type."""
    x, w = rows_of([1.0, -1.0, 0.5], T, H, F, dtype)
    big = 3e38
    x[T // 2, 0] = x[T // 2, 1] = big
    w[:F, 1] = w[:F, 0]
    w[F:, 1] = 0
    x[:T // 2, 1] = x[T // 2 + 1:, 1] = 0
    w[2:F:3, :2] = 0                        # gates that stay finite in that row
    gu, h, again = forward(x, w, dtype, kind)
    g, u = gu[:, :F].double(), gu[:, F:].double()
    assert bool((g[T // 2, 0::3] == float("inf")).all()) and bool((g[T // 2, 1::3] == -float("inf")).all())
    assert bool((g[T // 2, 2::3] == 0).all()) and bool(torch.isfinite(u).all())
    want = act(g, kind)[0] * u
    for got in (h, again):
        assert torch.equal(torch.isnan(got), torch.isnan(want))
        far = torch.isinf(want)
        assert bool(far[T // 2, 0::3].all()) and torch.equal(got[far].double(), want[far])
    rows = torch.arange(T, device="cuda") != T // 2
    check_forward(x[rows], w, None, gu[rows], h[rows], kind, dtype)


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("T,H,F", SIZES)
def test_an_infinite_input(T, H, F, kind):
    """bfloat16: a sum is what its products make, +-inf here."""
    x, w = rows_of([1.0, -1.0, 0.5], T, H, F, "bf16")
    x[T - 1, 0] = float("inf")
    w[F:, 0] = 0.25
    gu, h, again = forward(x, w, "bf16", kind)
    want = torch.full((F,), float("nan"), device="cuda", dtype=torch.bfloat16)
    want[0::3] = want[2::3] = float("inf")
    for got in (h, again):
        assert torch.equal(got[T - 1].isnan(), want.isnan()) and torch.equal(got[T - 1][~want.isnan()], want[~want.isnan()])
    check_forward(x[:-1], w, None, gu[:-1], h[:-1], kind, "bf16")
