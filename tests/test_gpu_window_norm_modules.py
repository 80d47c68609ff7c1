"""Window attention, residual norms and rotary positions of several axes as modules, alone and together in a pre-norm model: outputs and
gradients against float64 autograd, what is kept, captured training steps.

Tolerances, before any run, relative to max(|reference|, its rms).  float32: products over up to 96 values are off by at most
(K / 4 + 16) 2^-23 sum |a| |b|, and that sum is about 0.8 sqrt(K) of the rms: 4e-5; the attention is two of them forward and five backward, around exponentials
that add 2^-21 of themselves: 2e-4, a whole block of some ten such steps 1e-3.  bfloat16: each of the roundings is off by up to 2^-8 of an element; the
attention makes three of them (weights, output, inputs of the next product) forward and as many backward, which add up at random, and an element may be
four times as far off as they are on average: 6 2^-8 and four times that, 1e-1."""
import math

import pytest
import torch
import torch.nn.functional as F

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def M():
    from paper_2210_10246_amd import binding, modules
    binding.load()
    return modules


def near(got, want, tol):
    assert got.shape == want.shape
    rms = want.square().mean().sqrt()
    off = float(((got.double() - want).abs() / torch.maximum(want.abs(), rms)).max())
    assert off <= tol, off


def normal(*shape, seed=0, dtype=torch.float32, scale=1.0):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return (scale * torch.randn(*shape, generator=g, device="cuda")).to(dtype)


def attention(q, k, v, window, sinks, scale=None, key_len=None):
    """q [B, heads, S, D] float64"""
    S, D, heads = q.shape[2], q.shape[3], q.shape[1]
    k, v = (t.repeat_interleave(heads // t.shape[1], 1) for t in (k, v))
    i, j = torch.arange(S, device="cuda")[:, None], torch.arange(S, device="cuda")
    seen = (j <= i) & ((j > i - window) | (j < sinks))
    if key_len is not None:
        seen = seen & (j < key_len[:, None, None, None])
    s = (q @ k.transpose(-1, -2)) * (D ** -0.5 if scale is None else scale)
    return torch.softmax(s.masked_fill(~seen, -math.inf), -1) @ v


def norm(t, kind, w=None, b=None, eps=1e-5):
    t = t - t.mean(-1, keepdim=True) if kind == "layer" else t
    t = t * (t.square().mean(-1, keepdim=True) + eps) ** -0.5
    t = t if w is None else t * w
    return t if b is None else t + b


@pytest.mark.parametrize("dtype,tol", [(torch.float32, 2e-4), (torch.bfloat16, 1e-1)])
def test_window_attention_gradients(M, dtype, tol):
    """Views of one projection, shared key heads, gradients that are broadcast, each gradient alone."""
    core = M.TempoWindowAttention(9, 2)
    qkv = normal(2, 41, 8, 16, dtype=dtype).requires_grad_()
    parts = lambda t: (t[:, :, :4].transpose(1, 2), t[:, :, 4:6].transpose(1, 2), t[:, :, 6:].transpose(1, 2))  # noqa: E731
    key_len = torch.tensor([41, 30], dtype=torch.int32, device="cuda")
    out = core(*parts(qkv), key_len)
    ref = qkv.detach().double().requires_grad_()
    want = attention(*parts(ref), 9, 2, None, key_len)
    near(out.detach(), want.detach(), tol)
    for weight in (normal(2, 4, 41, 16, seed=1, dtype=dtype), normal(2, 1, 41, 1, seed=2, dtype=dtype), torch.ones((), device="cuda", dtype=dtype)):
        got, = torch.autograd.grad((out * weight).sum(), qkv, retain_graph=True)
        near(got, torch.autograd.grad((want * weight.double()).sum(), ref, retain_graph=True)[0], tol)
    q, k, v = (t.detach().contiguous() for t in parts(qkv))
    all_of = None
    for which in ((0, 1, 2), (0,), (1,), (2,)):
        leaves = [t.clone().requires_grad_(n in which) for n, t in enumerate((q, k, v))]
        grads = torch.autograd.grad(core(*leaves, key_len).square().sum(), [leaves[n] for n in which])
        all_of = all_of or grads
        assert all(torch.equal(g, all_of[n]) for g, n in zip(grads, which))
    with torch.no_grad():
        assert torch.equal(core(*parts(qkv), key_len), out)
    with torch.autocast("cuda", dtype=torch.bfloat16):
        assert core(q.float(), k, v).dtype == torch.bfloat16


def test_no_second_derivatives(M):
    q = normal(1, 2, 5, 16).requires_grad_()
    with pytest.raises(RuntimeError, match="no second derivative"):
        torch.autograd.grad(M.TempoWindowAttention(3)(q, q, q).sum(), q, create_graph=True)
    x = normal(3, 16).requires_grad_()
    with pytest.raises(RuntimeError, match="no second derivative"):
        torch.autograd.grad(M.TempoResidualNorm(16).cuda()(x, x)[1].sum(), x, create_graph=True)


@pytest.mark.parametrize("dtype,tol", [(torch.float32, 2e-4), (torch.bfloat16, 1e-1)])
@pytest.mark.parametrize("post,pre,gate,affine", [(None, "rms", None, True), ("rms", "rms", 0.3, True), ("layer", "layer", "rows", True), ("rms", None, "all", False),
                                                  (None, "layer", "2d", True), (None, None, 0.1, False)])
def test_residual_norm_gradients(M, post, pre, gate, affine, dtype, tol):
    torch.manual_seed(3)
    place = M.TempoResidualNorm(48, post, pre, gate if isinstance(gate, float) else None, alpha=0.9, beta=0.5, affine=affine).cuda()
    with torch.no_grad():
        for p in place.parameters():
            p.add_(0.2 * torch.randn_like(p))
    x, f = normal(3, 7, 48, dtype=dtype).requires_grad_(), normal(3, 7, 48, seed=1, dtype=dtype).requires_grad_()
    given = {"rows": (3, 1, 48), "all": (48,), "2d": (3, 48)}.get(gate)
    given = None if given is None else normal(*given, seed=2, dtype=dtype).requires_grad_()
    y, h = place(x, f, given)
    leaves = [x, f] + ([given] if given is not None else []) + list(place.parameters())
    ref = [t.detach().double().requires_grad_() for t in leaves]
    names = dict(zip([n for n, _ in place.named_parameters()], ref[len(ref) - len(list(place.parameters())):]))
    g = ref[2] if given is not None else names.get("gate")
    if gate == "2d":
        g = g[:, None]
    wide = ref[1] if post is None else norm(ref[1], post, names.get("post_weight"), names.get("post_bias"))
    wy = 0.9 * ref[0] + 0.5 * (wide if g is None else g * wide)
    near(y.detach(), wy.detach(), tol)
    v, w = normal(3, 7, 48, seed=4, dtype=dtype), normal(3, 7, 48, seed=5, dtype=dtype)
    outs, wants = [(y * v).sum()], [(wy * v.double()).sum()]
    if pre is None:
        assert h is None
    else:
        wh = norm(wy, pre, names.get("pre_weight"), names.get("pre_bias"))
        near(h.detach(), wh.detach(), tol)
        outs += [(h * w).sum(), (y * v).sum() + (h * w).sum()]      # the gradient of one of the two alone, and of both
        wants += [(wh * w.double()).sum(), (wy * v.double()).sum() + (wh * w.double()).sum()]
    for out, want in zip(outs, wants):
        got = torch.autograd.grad(out, leaves, retain_graph=True, allow_unused=True)
        for a, b in zip(got, torch.autograd.grad(want, ref, retain_graph=True, allow_unused=True)):
            assert a is not None or b is None or float(b.abs().max()) == 0
            if b is not None:
                near(a, b, tol) if float(b.abs().max()) > 0 else None
            elif a is not None:
                assert float(a.abs().max()) == 0


@pytest.mark.parametrize("order,own", [("blocks", False), ("cyclic", True)])
def test_rotary_axes_gradients(M, order, own):
    r = M.RotaryPositions(16, sections=(2, 3, 3), order=order, own=own).cuda()
    q, k = normal(2, 4, 6, 16).requires_grad_(), normal(2, 2, 6, 16, seed=1).requires_grad_()
    positions = torch.randint(0, 99, (3, 2, 6), device="cuda")
    turn = (positions[r.axes.long()].double() * r.freqs[:, None, None]).permute(1, 2, 0)[:, None]

    def turned(x):
        c, s, x1, x2 = turn.cos(), turn.sin(), x[..., :8], x[..., 8:]
        return torch.cat((x1 * c - x2 * s, x2 * c + x1 * s), -1)
    out = r(q, k, positions)
    ref = [t.detach().double().requires_grad_() for t in (q, k)]
    want = [turned(t) for t in ref]
    for a, b in zip(out, want):
        near(a.detach(), b.detach(), 1e-6)
    got = torch.autograd.grad(sum((t ** 3).sum() for t in out), (q, k), create_graph=True)
    exact = torch.autograd.grad(sum((t ** 3).sum() for t in want), ref, create_graph=True)
    for a, b in zip(got, exact):
        near(a.detach(), b.detach(), 1e-5)
    for a, b in zip(torch.autograd.grad(sum(t.square().sum() for t in got), (q, k)), torch.autograd.grad(sum(t.square().sum() for t in exact), ref)):
        near(a, b, 1e-4)


class Model(torch.nn.Module):
    """Two pre-norm layers over patches and text: attention through rotary positions of three axes and a window, a gated block, the places
    between them with their gates, a norm behind each block in the second half."""

    def __init__(self, M, hidden=64, heads=4, kv=2, ffn=96, window=11, sinks=3, dtype=torch.float32):
        super().__init__()
        self.hidden, self.heads, self.kv, self.dim, self.window, self.sinks = hidden, heads, kv, hidden // heads, window, sinks
        self.rotary = M.RotaryPositions(self.dim, sections=(2, 3, 3))
        self.core = M.TempoWindowAttention(window, sinks)
        linear = lambda *a: torch.nn.Linear(*a, bias=False, dtype=dtype)  # noqa: E731
        self.qkv = torch.nn.ModuleList(linear(hidden, (heads + 2 * kv) * self.dim) for _ in range(2))
        self.out = torch.nn.ModuleList(linear(hidden, hidden) for _ in range(2))
        self.ffn = torch.nn.ModuleList(M.TempoGatedFFN(hidden, ffn, dtype=dtype) for _ in range(2))
        self.first = M.TempoResidualNorm(hidden, None, "rms")
        self.places = torch.nn.ModuleList(M.TempoResidualNorm(hidden, "rms" if n > 1 else None, "rms" if n < 3 else "layer", gate=0.7, beta=0.8)
                                          for n in range(4))

    def forward(self, x, positions, key_len=None):
        B, S, _ = x.shape
        x, h = self.first(x, torch.zeros_like(x))
        for n in range(2):
            qkv = self.qkv[n](h).view(B, S, -1, self.dim)
            q, k, v = (t.transpose(1, 2) for t in qkv.split((self.heads, self.kv, self.kv), 2))
            q, k = self.rotary(q, k, positions)
            a = self.core(q, k, v, key_len).transpose(1, 2).reshape(B, S, self.hidden)
            x, h = self.places[2 * n](x, self.out[n](a))
            x, h = self.places[2 * n + 1](x, self.ffn[n](h))
        return h

    def exact(self, x, positions, p, key_len=None):
        """The same in the type of x and p, elementary steps."""
        B, S, _ = x.shape
        turn = (positions[self.rotary.axes.long()].double() * self.rotary.freqs[:, None, None]).permute(1, 2, 0)[:, None]

        def turned(t):
            half = t.shape[-1] // 2
            c, s, a, b = turn.cos(), turn.sin(), t[..., :half], t[..., half:]
            return torch.cat((a * c - b * s, b * c + a * s), -1)

        def place(name, x, f):
            m = self.get_submodule(name)
            if m.post:
                f = norm(f, m.post, p[name + ".post_weight"])
            x = x + 0.8 * p[name + ".gate"] * f
            return x, norm(x, m.pre, p[name + ".pre_weight"], p.get(name + ".pre_bias"))
        h = norm(x, "rms", p["first.pre_weight"])
        for n in range(2):
            qkv = F.linear(h, p[f"qkv.{n}.weight"]).view(B, S, -1, self.dim)
            q, k, v = (t.transpose(1, 2) for t in qkv.split((self.heads, self.kv, self.kv), 2))
            a = attention(turned(q), turned(k), v, self.window, self.sinks, None, key_len).transpose(1, 2).reshape(B, S, self.hidden)
            x, h = place(f"places.{2 * n}", x, F.linear(a, p[f"out.{n}.weight"]))
            g, u = F.linear(h, p[f"ffn.{n}.gate_up_weight"]).chunk(2, -1)
            x, h = place(f"places.{2 * n + 1}", x, F.linear(F.silu(g) * u, p[f"ffn.{n}.down_weight"]))
        return h


def positions_of(B, S):
    p = torch.stack((torch.arange(S) // 20, torch.arange(S) // 5 % 4, torch.arange(S) % 5)).cuda()
    return p[:, None].expand(3, B, S)


@pytest.mark.parametrize("dtype,tol", [(torch.float32, 1e-3), (torch.bfloat16, 2.5e-1)])
def test_all_of_them_in_a_model(M, dtype, tol):
    """bfloat16: some twenty roundings of 2^-8 one after the other, at random 5 2^-8 on average, an element ten times as far off: 2e-1 and its own."""
    torch.manual_seed(1)
    model = Model(M, dtype=dtype).cuda()
    x = normal(2, 45, 64, dtype=dtype).requires_grad_()
    key_len = torch.tensor([45, 38], dtype=torch.int32, device="cuda")
    positions = positions_of(2, 45)
    h = model(x, positions, key_len)
    p = {n: t.detach().double().requires_grad_() for n, t in model.named_parameters()}
    ref = x.detach().double().requires_grad_()
    want = model.exact(ref, positions, p, key_len)
    near(h.detach(), want.detach(), tol)
    w = normal(2, 45, 64, seed=7, dtype=dtype)
    got = torch.autograd.grad((h * w).sum(), [x, *model.parameters()])
    exact = torch.autograd.grad((want * w.double()).sum(), [ref, *p.values()])
    for (name, _), a, b in zip([("x", None), *model.named_parameters()], got, exact):
        off = float((a.double() - b).norm() / b.norm())
        assert off <= tol / (4 if dtype == torch.bfloat16 else 1), (name, off)


def test_token_by_token_from_a_cache_is_the_whole_sequence(M):
    """The attention of a prompt and then of one token after the other over a cache that is longer than the sequences, which have different
    lengths, is that of the whole sequences."""
    B, heads, kv, D, room, window, sinks = 3, 4, 2, 32, 64, 10, 2
    core, r = M.TempoWindowAttention(window, sinks), M.RotaryPositions(D, sections=(4, 6, 6)).cuda()
    lens = [50, 33, 41]
    q, k, v = (normal(B, n, room, D, seed=s) for s, n in enumerate((heads, kv, kv)))
    place = torch.arange(room, device="cuda").expand(3, -1)
    tq, tk = r(q, k, place)
    key_len = torch.tensor(lens, dtype=torch.int32, device="cuda")
    whole = core(tq, tk, v, key_len)
    cache_k, cache_v = torch.full_like(k, float("nan")), torch.full_like(v, float("nan"))
    done = torch.tensor([20, 3, 11], dtype=torch.int32, device="cuda")
    for b, n in enumerate(done.tolist()):
        cache_k[b, :, :n], cache_v[b, :, :n] = tk[b, :, :n], v[b, :, :n]
    for _ in range(25):
        at = done.long()
        for b, n in enumerate(at.tolist()):
            cache_k[b, :, n], cache_v[b, :, n] = tk[b, :, n], v[b, :, n]
        new = torch.stack([tq[b, :, n] for b, n in enumerate(at.tolist())])[:, :, None]
        out = core(new, cache_k, cache_v, done + 1, done)
        for b, n in enumerate(at.tolist()):
            if n < lens[b]:
                near(out[b, :, 0], whole[b, :, n].double(), 1e-5)
        done += (done + 1 < key_len).int()


def test_replays_of_a_captured_training_step(M):
    """A step captured on a side stream, no eager graph of the leaves alive; each replay against the eager step on the same values."""
    torch.manual_seed(1)
    model = Model(M).cuda()
    x, positions, w = normal(2, 45, 64), positions_of(2, 45).contiguous(), normal(2, 45, 64, seed=7)
    params = list(model.parameters())

    def step():
        for p in params:
            p.grad = None
        loss = (model(x, positions) * w).sum()
        loss.backward()
        return loss.detach(), [p.grad for p in params]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step()
        for p in params:
            p.grad = None
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        loss, grads = step()
    captured = list(grads)
    for turn in range(3):
        x.copy_(normal(2, 45, 64, seed=20 + turn))
        graph.replay()
        torch.cuda.synchronize()
        got = [loss.clone(), *[g.clone() for g in captured]]
        with torch.cuda.stream(side):
            want, eager = step()
        torch.cuda.synchronize()
        for a, b in zip(got, [want, *eager]):
            near(a, b.double(), 1e-5) if b.dim() else None
