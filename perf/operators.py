"""Rotary positions and the gated feed-forward unit, as a training or decoding program calls them.

`own` false: their plain forms, elementary torch in 32 bits (angles in 64).  `own` true: the binding's
calls on buffers that the program owns, as in `perf/cases.py`.  A case is one direction of one
operator; what the backward of the gated unit works from (the kept projections) is its input.
"""
import math

import torch

own = False

_DT = {"f32": torch.float32, "bf16": torch.bfloat16}
_SIZE = {"f32": 4, "bf16": 2}


# ---- the cases ------------------------------------------------------------------------------
def _rotary(batch, seq, heads, kv_heads, dim, rotated, dtype, layout="half", way="fwd", far=False):
    """far: positions of a long context beyond the trained one, frequencies and scale to match."""
    return {"op": "rotary", "batch": batch, "seq": seq, "heads": heads, "kv_heads": kv_heads, "dim": dim,
            "rotated": rotated, "dtype": dtype, "layout": layout, "way": way, "far": far}


def _glu(rows, hidden, ffn, dtype, kind="silu", way="fwd", bias=False, keep=True):
    """keep: the projections are kept for a backward (a forward in training)."""
    return {"op": "glu", "rows": rows, "hidden": hidden, "ffn": ffn, "dtype": dtype, "kind": kind, "way": way,
            "bias": bias, "keep": keep}


def listed():
    named = [
        # one new token of a gpt2-small-sized model: what a call costs
        ("rotary-token", _rotary(1, 1, 12, 12, 64, 64, "bf16")),
        # bert-large at 512 tokens, q and k out of one projection
        ("rotary-bert-large", _rotary(16, 512, 16, 16, 64, 64, "bf16")),
        # the backward at sizes that fit no vector and no tile: neighbours in pairs, part of the head
        ("rotary-odd-bwd", _rotary(3, 1021, 9, 3, 83, 38, "f32", "interleaved", "bwd")),
        # a long context in training: shared key heads, positions beyond the trained range
        ("rotary-long", _rotary(1, 65536, 32, 8, 128, 128, "bf16", "half", "fwd", True)),
        # the feed-forward of one new token: the weights are read for a single row
        ("glu-token", _glu(1, 1024, 4096, "bf16", keep=False)),
        # one new token of 48 sequences in a wide model
        ("glu-tokens-wide", _glu(48, 4096, 11008, "bf16", keep=False)),
        # two sequences of 128 tokens at bert-base width, float32
        ("glu-base-f32", _glu(256, 768, 2048, "f32", "gelu_erf")),
        # bert-large width, 64 sequences of 128 tokens: training, both ways
        ("glu-large-fwd", _glu(8192, 1024, 4096, "bf16")),
        ("glu-large-bwd", _glu(8192, 1024, 4096, "bf16", way="bwd")),
        # odd sizes everywhere, with a bias
        ("glu-odd-bwd", _glu(1021, 1001, 2729, "bf16", "gelu_tanh", "bwd", True)),
        # float32 training of a middle-sized model
        ("glu-wide-f32-bwd", _glu(4096, 2048, 5504, "f32", "silu", "bwd")),
        # a wide model's training forward, the largest call
        ("glu-wide-fwd", _glu(16384, 4096, 11008, "bf16")),
    ]
    return [{"name": name, **case} for name, case in named]


_MOST_ROTATED = 1 * 65536 * 40 * 128           # elements of q and k
_MOST_PRODUCTS = 2 * 16384 * 4096 * 11008      # multiplications


def _spread(rng, low, high, odd=0.5):
    n = int(round(math.exp(rng.uniform(math.log(low), math.log(high)))))
    if rng.random() < odd:
        return min(max(n, low), high)
    return max(low, n // 16 * 16)


def draw(rng):
    dtype = rng.choice(["bf16", "bf16", "f32"])
    way = rng.choice(["fwd", "bwd"])
    if rng.random() < 0.4:
        dim = rng.choice([32, 64, 64, 80, 96, 128, 128, 256, rng.randrange(20, 200)])
        rotated = dim // 2 * 2 if rng.random() < 0.6 else 2 * rng.randrange(1, dim // 2 + 1)
        kv = rng.choice([1, 2, 3, 4, 8, 12])
        heads = kv * rng.choice([1, 1, 2, 4, 5])
        tokens = _spread(rng, 1, _MOST_ROTATED // ((heads + kv) * dim) // 2)
        batch = min(tokens, rng.choice([1, 1, 2, 3, 8, 16, 64]))
        return _rotary(batch, tokens // batch, heads, kv, dim, rotated, dtype, rng.choice(["half", "interleaved"]),
                       way, rng.random() < 0.3)
    hidden = _spread(rng, 64, 4096, 0.25)
    ffn = _spread(rng, 128, 11008, 0.25)
    cost = (1 if way == "fwd" else 2) * (1 if dtype == "bf16" else 4)
    rows = _spread(rng, 1, max(2, min(16384, _MOST_PRODUCTS // (2 * hidden * ffn * cost))))
    return _glu(rows, hidden, ffn, dtype, rng.choice(["silu", "gelu_erf", "gelu_tanh"]), way, rng.random() < 0.3,
                way == "bwd" or rng.random() < 0.6)


# ---- inputs ---------------------------------------------------------------------------------
def _frequencies(half, far, device):
    """base^(-i / half) radians per position; far: those that turn less than once in the 4096
    trained positions are slowed down 8 times, those that turn 32 times and more are left."""
    f = 10000.0 ** (-torch.arange(half, dtype=torch.float64, device=device) / half)
    if not far:
        return f, 1.0
    left = ((4096.0 * f / (2 * math.pi) - 1.0) / 31.0).clamp(0.0, 1.0)
    return f * (left + (1.0 - left) / 8.0), 0.1 * math.log(8.0) + 1.0


def _prepare_rotary(case, g):
    B, S, A, K, D = (case[n] for n in ("batch", "seq", "heads", "kv_heads", "dim"))
    dt = _DT[case["dtype"]]
    normal = lambda *shape: torch.randn(*shape, generator=g, device="cuda", dtype=torch.float32).to(dt)  # noqa: E731
    freqs, scale = _frequencies(case["rotated"] // 2, case["far"], "cuda")
    # a sequence starts at its own place, as after a prompt or a document before it
    start = torch.randint(0, 32768 if case["far"] else 2048, (B, 1), generator=g, device="cuda")
    state = {"positions": start + torch.arange(S, device="cuda"), "freqs": freqs, "scale": scale}
    if case["way"] == "fwd":      # q and k lie in one projection; attention wants them by head
        qkv = normal(B, S, A + 2 * K, D)
        state["q"], state["k"] = qkv[:, :, :A], qkv[:, :, A:A + K]
        state["q_out"] = torch.empty(B, A, S, D, device="cuda", dtype=dt).transpose(1, 2)
        state["k_out"] = torch.empty(B, K, S, D, device="cuda", dtype=dt).transpose(1, 2)
    else:                         # the other way round
        state["q"] = normal(B, A, S, D).transpose(1, 2)
        state["k"] = normal(B, K, S, D).transpose(1, 2)
        dqkv = torch.empty(B, S, A + 2 * K, D, device="cuda", dtype=dt)
        state["q_out"], state["k_out"] = dqkv[:, :, :A], dqkv[:, :, A:A + K]
    return state


def _prepare_glu(case, g):
    T, H, F = case["rows"], case["hidden"], case["ffn"]
    dt = _DT[case["dtype"]]
    normal = lambda *shape: torch.randn(*shape, generator=g, device="cuda", dtype=torch.float32)  # noqa: E731
    empty = lambda *shape: torch.empty(*shape, device="cuda", dtype=dt)  # noqa: E731
    state = {"x": normal(T, H).to(dt), "w": (normal(2 * F, H) / math.sqrt(H)).to(dt), "h": empty(T, F), "bias": None}
    if case["way"] == "fwd":
        state["bias"] = (0.1 * normal(2 * F)).to(dt) if case["bias"] else None
        state["gu"] = empty(T, 2 * F) if case["keep"] else None
    else:
        state["dh"], state["gu"] = normal(T, F).to(dt), normal(T, 2 * F).to(dt)
        state["dgu"], state["dx"], state["dw"] = empty(T, 2 * F), empty(T, H), empty(2 * F, H)
        state["dbias"] = empty(2 * F) if case["bias"] else None
    return state


def prepare(case, seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    state = _prepare_rotary(case, g) if case["op"] == "rotary" else _prepare_glu(case, g)
    state["case"] = case
    return state


# ---- one pass -------------------------------------------------------------------------------
def run(state):
    if own:
        return _own_rotary(state) if state["case"]["op"] == "rotary" else _own_glu(state)
    return _plain_rotary(state) if state["case"]["op"] == "rotary" else _plain_glu(state)


def _own_rotary(state):
    from paper_2210_10246_amd import binding as B
    call = B.tempo_rotary_fwd if state["case"]["way"] == "fwd" else B.tempo_rotary_bwd
    call(state["q"], state["k"], state["freqs"], state["positions"], state["q_out"], state["k_out"],
         state["case"]["layout"], state["scale"])
    return {"q": state["q_out"], "k": state["k_out"]}


def _own_glu(state):
    from paper_2210_10246_amd import binding as B
    kind = state["case"]["kind"]
    if state["case"]["way"] == "fwd":
        B.tempo_glu_fwd(state["x"], state["w"], state["bias"], state["gu"], state["h"], kind)
        return {"gu": state["gu"], "h": state["h"]}
    B.tempo_glu_bwd(state["dh"], state["gu"], state["x"], state["w"], state["dgu"], state["h"], state["dx"],
                    state["dw"], state["dbias"], kind)
    return {"h": state["h"], "dx": state["dx"], "dw": state["dw"], "dbias": state["dbias"]}


def _plain_rotary(state):
    case = state["case"]
    angle = state["positions"].double()[:, :, None, None] * state["freqs"]
    c = (angle.cos() * state["scale"]).float()
    s = (angle.sin() * state["scale"]).float()
    if case["way"] == "bwd":
        s = -s
    half = case["rotated"] // 2

    def turned(x):
        f = x[..., :2 * half].float()
        if case["layout"] == "half":
            x1, x2 = f[..., :half], f[..., half:]
            y = torch.cat((x1 * c - x2 * s, x2 * c + x1 * s), -1)
        else:
            x1, x2 = f[..., ::2], f[..., 1::2]
            y = torch.stack((x1 * c - x2 * s, x2 * c + x1 * s), -1).flatten(-2)
        return torch.cat((y.to(x.dtype), x[..., 2 * half:]), -1)
    return {"q": turned(state["q"]), "k": turned(state["k"])}


def _act(g, kind):
    """act(g) and act'(g)"""
    if kind == "silu":
        s = torch.sigmoid(g)
        return g * s, s * (1 + g * (1 - s))
    if kind == "gelu_erf":
        phi = 0.5 * torch.erfc(g * -math.sqrt(0.5))
        return g * phi, phi + g * torch.exp(-0.5 * g * g) * (1 / math.sqrt(2 * math.pi))
    a = math.sqrt(2 / math.pi)
    s = torch.sigmoid(2 * a * (g + 0.044715 * g * g * g))      # (1 + tanh) / 2
    return g * s, s + g * (s * (1 - s)) * (2 * a) * (1 + 3 * 0.044715 * g * g)


def _plain_glu(state):
    case = state["case"]
    dt, F = _DT[case["dtype"]], case["ffn"]
    x, w = state["x"].float(), state["w"].float()
    if case["way"] == "fwd":
        gu = x @ w.t()
        if state["bias"] is not None:
            gu = gu + state["bias"].float()
        h = _act(gu[:, :F], case["kind"])[0] * gu[:, F:]
        return {"gu": gu.to(dt) if case["keep"] else None, "h": h.to(dt)}
    dh, g, u = state["dh"].float(), state["gu"][:, :F].float(), state["gu"][:, F:].float()
    a, d = _act(g, case["kind"])
    dgu = torch.cat((dh * u * d, dh * a), 1)
    return {"h": (a * u).to(dt), "dx": (dgu @ w).to(dt), "dw": (dgu.t() @ x).to(dt),
            "dbias": dgu.sum(0).to(dt) if case["bias"] else None}


# ---- what one pass cannot do without --------------------------------------------------------
def work(case):
    size = _SIZE[case["dtype"]]
    if case["op"] == "rotary":
        tokens, heads = case["batch"] * case["seq"], case["heads"] + case["kv_heads"]
        return {"bytes": 2 * size * tokens * heads * case["dim"] + 8 * tokens + 4 * case["rotated"],
                "flops": 3 * tokens * heads * case["rotated"]}
    T, H, F = case["rows"], case["hidden"], case["ffn"]
    if case["way"] == "fwd":
        return {"bytes": size * (T * H + 2 * F * H + (2 * F if case["bias"] else 0) + T * F + (2 * T * F if case["keep"] else 0)),
                "flops": 4 * T * H * F}
    return {"bytes": size * (4 * T * F + 2 * T * H + 4 * F * H + (2 * F if case["bias"] else 0)), "flops": 8 * T * H * F}


# ---- the definition in 64 bits --------------------------------------------------------------
def exact(case, seed):
    state = prepare(case, seed)
    if case["op"] == "rotary":
        way = 1.0 if case["way"] == "fwd" else -1.0
        turn = torch.outer(state["positions"].reshape(-1).double(), state["freqs"])
        # multiplication by scale * e^(i angle)
        by = torch.polar(torch.full_like(turn, state["scale"]), turn * way).reshape(case["batch"], case["seq"], 1, -1)
        half = case["rotated"] // 2
        out = {}
        for name in ("q", "k"):
            x = state[name].double()
            first = slice(0, half) if case["layout"] == "half" else slice(0, 2 * half, 2)
            second = slice(half, 2 * half) if case["layout"] == "half" else slice(1, 2 * half, 2)
            z = torch.complex(x[..., first], x[..., second]) * by
            y = x.clone()
            y[..., first], y[..., second] = z.real, z.imag
            out[name] = y
        return out
    F, kind = case["ffn"], case["kind"]
    x, w = state["x"].double(), state["w"].double()
    with torch.enable_grad():
        if case["way"] == "fwd":
            g, u = x.mm(w[:F].t()), x.mm(w[F:].t())
            if state["bias"] is not None:
                g, u = g + state["bias"][:F].double(), u + state["bias"][F:].double()
        else:
            g, u = (state["gu"][:, at:at + F].double().requires_grad_() for at in (0, F))
        if kind == "silu":
            a = g / (1.0 + torch.exp(-g))
        elif kind == "gelu_erf":
            a = g * (0.5 + 0.5 * torch.erf(g / math.sqrt(2.0)))
        else:
            a = 0.5 * g * (1.0 + torch.tanh(math.sqrt(2.0 / math.pi) * (g + 0.044715 * g ** 3)))
        h = a * u
        if case["way"] == "fwd":
            return {"gu": torch.cat((g, u), 1) if case["keep"] else None, "h": h}
        dg, du = torch.autograd.grad(h, (g, u), state["dh"].double())
    return {"h": h.detach(), "dx": dg.mm(w[:F]) + du.mm(w[F:]), "dw": torch.cat((dg.t().mm(x), du.t().mm(x))),
            "dbias": torch.cat((dg.sum(0), du.sum(0))) if case["bias"] else None}
