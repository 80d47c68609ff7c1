"""Rotary positions and the gated feed-forward block as modules, alone and together in an encoder layer: outputs and gradients
against float64, what is kept for the backward, captured training steps.

Tolerances, before any run, relative to max(|reference|, its rms).  A float32 product over K <= 96 values is off by at most
(K / 4 + 16) 2^-23 sum |a| |b|, and sum |a| |b| is about 0.8 sqrt(K) of the rms: 4e-5.  A block is three of them one after the
other each way, with activations that stretch by at most 1.2: 3e-4.  An encoder layer has two more products and the attention's
two, and normalizes twice: 1e-3.  In bfloat16 the block rounds x, [g | u], h, dh, dgu and the output, half a step of 2^-8
each, the sums of rounded values less than that: 6 2^-8 = 2.4e-2, and an element can be four times as far off as they are on
average: 1e-1."""
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
    rms = want.square().mean().sqrt()
    off = float(((got.double() - want).abs() / torch.maximum(want.abs(), rms)).max())
    assert off <= tol, off


def turned(x, positions, freqs, scale, layout):
    """x [B, A, S, D] float64; positions [B, S]"""
    half = freqs.numel()
    a = (positions.double()[:, :, None] * freqs)[:, None]
    c, n = scale * a.cos(), scale * a.sin()
    if layout == "half":
        x1, x2 = x[..., :half], x[..., half:2 * half]
        y = torch.cat((x1 * c - x2 * n, x2 * c + x1 * n), -1)
    else:
        x1, x2 = x[..., :2 * half:2], x[..., 1:2 * half:2]
        y = torch.stack((x1 * c - x2 * n, x2 * c + x1 * n), -1).flatten(-2)
    return torch.cat((y, x[..., 2 * half:]), -1)


def act(g, kind):
    return {"silu": F.silu, "gelu_erf": F.gelu, "gelu_tanh": lambda t: F.gelu(t, approximate="tanh")}[kind](g)


def gated(x, wi, bi, wo, bo, kind):
    g, u = F.linear(x, wi, bi).chunk(2, -1)
    return F.linear(act(g, kind) * u, wo, bo)


def normal(*shape, seed=0, dtype=torch.float32):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return torch.randn(*shape, generator=g, device="cuda").to(dtype)


@pytest.mark.parametrize("layout,dim,kv", [("half", 16, 4), ("interleaved", 10, 1), ("half", 8, 0)])
def test_rotary_gradients(M, layout, dim, kv):
    """Against float64 autograd: views of a projection as inputs, gradients that are broadcast, one of the two alone, twice."""
    r = M.RotaryPositions(dim, layout=layout, scaling="parts", factor=4.0, trained=64).cuda()
    qkv = normal(2, 7, 4 + kv, 16).requires_grad_()
    q, k = qkv[:, :, :4].transpose(1, 2), qkv[:, :, 4:].transpose(1, 2)
    positions = torch.randint(0, 500, (2, 7), device="cuda")
    yq, yk = r(q, k if kv else None, positions)
    ref = qkv.detach().double().requires_grad_()
    wq = turned(ref[:, :, :4].transpose(1, 2), positions, r.freqs, r.scale, layout)
    near(yq.detach(), wq.detach(), 1e-6)     # 2^-21 (|x1| + |x2|) and half a step, tests/test_gpu_rotary.py
    near(torch.autograd.grad(yq.sum(), qkv, retain_graph=True)[0], torch.autograd.grad(wq.sum(), ref, retain_graph=True)[0], 1e-5)
    if not kv:
        return
    wk = turned(ref[:, :, 4:].transpose(1, 2), positions, r.freqs, r.scale, layout)
    near(yk.detach(), wk.detach(), 1e-6)
    near(torch.autograd.grad(yk.sum(), qkv, retain_graph=True)[0], torch.autograd.grad(wk.sum(), ref, retain_graph=True)[0], 1e-5)
    got = torch.autograd.grad((yq.square().sum() + (yk ** 3).sum()), qkv, create_graph=True)[0]
    want = torch.autograd.grad((wq.square().sum() + (wk ** 3).sum()), ref, create_graph=True)[0]
    near(got.detach(), want.detach(), 1e-5)
    near(torch.autograd.grad(got.square().sum(), qkv)[0], torch.autograd.grad(want.square().sum(), ref)[0], 1e-4)


@pytest.mark.parametrize("dtype,tol", [(torch.float32, 3e-4), (torch.bfloat16, 1e-1)])
@pytest.mark.parametrize("kind,bias", [("silu", False), ("gelu_erf", True), ("gelu_tanh", True)])
def test_gated_block_gradients(M, kind, bias, dtype, tol):
    torch.manual_seed(5)
    block = M.TempoGatedFFN(48, 96, kind, bias, dtype).cuda()
    x = normal(3, 11, 48, dtype=dtype).requires_grad_()
    dy = normal(3, 11, 48, seed=1, dtype=dtype)
    params = [p for p in (block.gate_up_weight, block.gate_up_bias, block.down_weight, block.down_bias) if p is not None]
    y = block(x)
    ref = [t.detach().double().requires_grad_() for t in (x, *params)]
    wi, bi, wo, bo = (ref[1], ref[2], ref[3], ref[4]) if bias else (ref[1], None, ref[2], None)
    want = gated(ref[0], wi, bi, wo, bo, kind)
    near(y.detach(), want.detach(), tol)
    grads = torch.autograd.grad(want, ref, dy.double())
    all_of = torch.autograd.grad(y, [x, *params], dy, retain_graph=True)
    for got, g in zip(all_of, grads):
        near(got, g, tol)
    for i, t in enumerate([x, *params]):     # each alone, the same bits
        assert torch.equal(torch.autograd.grad(y, t, dy, retain_graph=True)[0], all_of[i])
    with torch.no_grad():
        assert torch.equal(block(x), y)


def test_gated_block_refuses_second_derivatives(M):
    block = M.TempoGatedFFN(16, 16).cuda()
    x = normal(2, 16).requires_grad_()
    with pytest.raises(RuntimeError, match="no second derivative"):
        torch.autograd.grad(block(x).sum(), x, create_graph=True)


def test_gated_block_keeps_its_input_and_the_projections(M):
    T, H, Fn = 64, 32, 128
    block = M.TempoGatedFFN(H, Fn, dtype=torch.bfloat16).cuda()
    x = normal(T, H, dtype=torch.bfloat16).requires_grad_()
    kept = []
    with torch.autograd.graph.saved_tensors_hooks(lambda t: kept.append(t) or t, lambda t: t):
        block(x)
    names = {block.gate_up_weight.data_ptr(), block.down_weight.data_ptr()}
    assert sorted(t.numel() for t in kept if t.data_ptr() not in names) == [T * H, T * 2 * Fn]


def test_gated_block_under_autocast_and_at_any_address(M):
    block = M.TempoGatedFFN(24, 40, "silu", True).cuda()
    x = normal(9, 24).requires_grad_()
    with torch.autocast("cuda", dtype=torch.bfloat16):
        y = block(x)
    assert y.dtype == torch.bfloat16
    y.sum().backward()
    assert x.grad.dtype == torch.float32 and block.down_weight.grad.dtype == torch.float32
    room = normal(9 * 24 + 1)
    assert torch.equal(block(room[1:].view(9, 24)), block(room[1:].view(9, 24).clone()))
    assert torch.equal(block(x.detach().t().contiguous().t()), block(x.detach()))


def layer_reference(layer, x, key_len, positions):
    """The layer's formulas in float64, without dropout."""
    p = {n: t.detach().double().requires_grad_() for n, t in layer.named_parameters()}
    Bn, S, H = x.shape
    heads = layer.heads
    q, k, v = F.linear(x, p["qkv.weight"], p["qkv.bias"]).view(Bn, S, 3, heads, H // heads).permute(2, 0, 3, 1, 4)
    r = layer.rotary
    q, k = (turned(t, positions, r.freqs, r.scale, r.layout) for t in (q, k))
    scores = q @ k.transpose(-1, -2) / math.sqrt(H // heads)
    if key_len is not None:
        scores = scores.masked_fill(torch.arange(S, device="cuda") >= key_len[:, None, None, None], -math.inf)
    a = (torch.softmax(scores, -1) @ v).permute(0, 2, 1, 3).reshape(Bn, S, H)
    norm = lambda t, n, eps: F.layer_norm(t, (H,), p[n + ".weight"], p[n + ".bias"], eps)  # noqa: E731
    x = norm(x + F.linear(a, p["proj.weight"], p["proj.bias"]), "ln1", layer.ln1.eps)
    y = gated(x, p["ffn.gate_up_weight"], p["ffn.gate_up_bias"], p["ffn.down_weight"], p["ffn.down_bias"], layer.ffn.kind)
    return norm(x + y, "ln2", layer.ln2.eps), p


@pytest.mark.parametrize("S,padded", [(1, False), (13, True), (40, False)])
def test_encoder_layer_with_both(M, S, padded):
    torch.manual_seed(2)
    layer = M.TempoEncoderLayer(64, 4, 96, p_attn=0.0, eps=1e-5, rotary=M.RotaryPositions(12), gated="silu").cuda()
    x = normal(3, S, 64).requires_grad_()
    dy = normal(3, S, 64, seed=1)
    key_len = torch.tensor([S, max(1, S // 2), 1], dtype=torch.int32, device="cuda") if padded else None
    positions = torch.arange(S, device="cuda") + torch.tensor([[0], [7], [900]], device="cuda")
    out = layer(x, key_len, positions)
    ref = x.detach().double().requires_grad_()
    want, p = layer_reference(layer, ref, key_len, positions)
    near(out.detach(), want.detach(), 1e-3)
    names = [n for n, _ in layer.named_parameters()]
    got = torch.autograd.grad(out, [x, *layer.parameters()], dy)
    for name, a, b in zip(["x", *names], got, torch.autograd.grad(want, [ref, *(p[n] for n in names)], dy.double())):
        if S == 1 and name in ("qkv.weight", "qkv.bias"):     # of one key: no gradient to q and k, zeros but for rounding
            a, b = a[128:], b[128:]
        near(a, b, 1e-3)


def test_captured_training_step_of_a_layer_with_both(M):
    """Forward and backward captured, replayed with new inputs between eager steps of a copy of the layer."""
    make = lambda: M.TempoEncoderLayer(64, 4, 96, p_attn=0.0, eps=1e-5, rotary=M.RotaryPositions(16), gated="gelu_tanh").cuda()  # noqa: E731
    torch.manual_seed(4)
    layer, copy = make(), make()
    copy.load_state_dict(layer.state_dict())
    x = normal(2, 24, 64)

    def step(of):
        for p in of.parameters():
            p.grad = None
        out = of(x)
        out.square().sum().backward()
        return [out.detach(), *(p.grad for p in of.parameters())]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step(layer)
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        captured = step(layer)
    for turn in range(3):
        x.copy_(normal(2, 24, 64, seed=20 + turn))
        graph.replay()
        torch.cuda.synchronize()
        for a, b in zip(captured, step(copy)):
            near(a, b.double(), 1e-4)
