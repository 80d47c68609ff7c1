"""Window attention, residual norms and rotary positions of several axes, as a training or decoding
program calls them.

`own` false: their plain forms, elementary torch in 32 bits (angles in 64).  `own` true: the binding's
calls on buffers that the program owns.  A case is one direction of one operator; what a backward works
from (the forward's output and its statistics) is its input.
"""
import math

import torch

own = False

_DT = {"f32": torch.float32, "bf16": torch.bfloat16}
_SIZE = {"f32": 4, "bf16": 2}


# ---- the cases ------------------------------------------------------------------------------
def _attn(batch, queries, keys, heads, kv_heads, dim, window, sinks, dtype, way="fwd", padded=False, keep=False):
    """queries == keys: whole sequences, `padded` to the longest of them; else the last queries of sequences in a
    cache that holds `keys` tokens each.  keep: the forward of a training step, which keeps its statistics."""
    return {"op": "attn", "batch": batch, "queries": queries, "keys": keys, "heads": heads, "kv_heads": kv_heads, "dim": dim,
            "window": window, "sinks": sinks, "dtype": dtype, "way": way, "padded": padded, "keep": keep}


def _norm(rows, hidden, dtype, kind="rms", way="fwd", post=True, groups=1, gated=True, alpha=1.0, beta=1.0):
    """groups: sequences with a gate each, or one gate for all; post: a norm after the block too."""
    return {"op": "norm", "rows": rows, "hidden": hidden, "dtype": dtype, "kind": kind, "way": way, "post": post,
            "groups": groups, "gated": gated, "alpha": alpha, "beta": beta}


def _axes(batch, frames, height, width, heads, kv_heads, dim, sections, dtype, layout="half", way="fwd"):
    """A text of 64 tokens, at one place on every axis, then frames of height x width patches."""
    return {"op": "axes", "batch": batch, "frames": frames, "height": height, "width": width, "heads": heads,
            "kv_heads": kv_heads, "dim": dim, "sections": "-".join(map(str, sections)), "dtype": dtype, "layout": layout,
            "way": way}


def listed():
    named = [
        # one new token of a gpt2-small-sized model with a short window: what a call costs
        ("attn-token", _attn(1, 1, 1024, 12, 12, 64, 256, 4, "bf16")),
        # one new token of each of 48 sequences, shared key heads, a long window in a longer cache
        ("attn-tokens-batch", _attn(48, 1, 8192, 32, 8, 128, 4096, 4, "bf16")),
        # a prompt of 8192 tokens, or a forward in training
        ("attn-prompt", _attn(1, 8192, 8192, 32, 8, 128, 1024, 4, "bf16", keep=True)),
        # bert-large-sized training
        ("attn-large-bwd", _attn(8, 2048, 2048, 16, 16, 64, 512, 1, "bf16", "bwd")),
        # float32 at sizes that fit no tile, padded sequences, shared key heads
        ("attn-odd-f32-bwd", _attn(3, 1021, 1021, 9, 3, 83, 200, 5, "f32", "bwd", True)),
        # a long context in training, the largest call
        ("attn-long-bwd", _attn(1, 32768, 32768, 32, 8, 128, 4096, 16, "bf16", "bwd")),
        # the residual of one new token
        ("norm-token", _norm(1, 1024, "bf16", groups=1)),
        # 16 sequences of 512 tokens, a gate for each, depth-scaled branches
        ("norm-gated-fwd", _norm(8192, 4096, "bf16", groups=16, beta=0.25)),
        # odd sizes, float32, LayerNorm before the next block alone, the residual scaled down
        ("norm-odd-bwd", _norm(3063, 1001, "f32", "layer", "bwd", False, 3, alpha=0.75)),
        # a wide model's training backward
        ("norm-wide-bwd", _norm(65536, 4096, "bf16", "rms", "bwd")),
        # images at sizes that fit no vector, neighbours in pairs, part of the head
        ("axes-odd-fwd", _axes(3, 1, 45, 37, 9, 3, 83, (7, 6, 6), "f32", "interleaved")),
        # a video of 30 frames of 32 x 32 patches, time, height and width, the backward
        ("axes-video-bwd", _axes(1, 30, 32, 32, 40, 8, 128, (16, 24, 24), "bf16", "half", "bwd")),
    ]
    return [{"name": name, **case} for name, case in named]


_MOST_PAIRS = 32768 * 4096 * 32 * 128 * 5 // 2       # of an attention: visible pairs x elements x products / 2
_MOST_NORM = 65536 * 4096
_MOST_TURNED = 32768 * 48 * 128


def _spread(rng, low, high, odd=0.5):
    n = int(round(math.exp(rng.uniform(math.log(low), math.log(high)))))
    if rng.random() < odd:
        return min(max(n, low), high)
    return max(low, n // 16 * 16)


def draw(rng):
    op = rng.choice(["attn", "attn", "attn", "norm", "norm", "axes"])
    dtype = rng.choice(["bf16", "bf16", "f32"])
    way = rng.choice(["fwd", "bwd"])
    if op == "norm":
        hidden = _spread(rng, 64, 8192)
        rows = _spread(rng, 1, min(65536, _MOST_NORM // hidden // (2 if dtype == "f32" else 1)))
        gated = rng.random() < 0.7
        groups = max(g for g in range(1, rng.choice([1, 1, 16, 64]) + 1) if rows % g == 0) if gated else 1
        return _norm(rows, hidden, dtype, rng.choice(["rms", "rms", "layer"]), way, rng.random() < 0.6, groups, gated,
                     rng.choice([1.0, 1.0, 0.75]), rng.choice([1.0, 1.0, 0.25]))
    kv = rng.choice([1, 2, 3, 4, 8])
    heads = kv * rng.choice([1, 1, 2, 3, 4, 8])
    dim = rng.choice([32, 64, 64, 80, 96, 128, 128, 128, rng.randrange(16, 200), 256])
    if op == "axes":
        dim = dim // 2 * 2
        pairs = rng.choice([dim // 2, dim // 2, rng.randrange(3, dim // 2 + 1)])
        first = rng.randrange(1, pairs - 1)
        second = rng.randrange(1, pairs - first)
        frames, height, width = _spread(rng, 1, 32), _spread(rng, 4, 40), _spread(rng, 4, 40)
        most = _MOST_TURNED // ((heads + kv) * dim * (frames * height * width + 64)) // (2 if dtype == "f32" else 1)
        return _axes(max(1, min(most, rng.choice([1, 1, 2, 3, 8]))), frames, height, width, heads, kv, dim,
                     (first, second, pairs - first - second), dtype, rng.choice(["half", "interleaved"]), way)
    sinks = rng.choice([1, 1, 4, 4, 16, rng.randrange(1, 100)])
    if way == "fwd" and rng.random() < 0.5:          # decoding: one token, or a few that are looked at together
        window = _spread(rng, 16, 4096)
        keys = window + sinks + 16 + rng.randrange(0, 4096)
        batch = max(1, min(_spread(rng, 1, 64), (1 << 30) // (keys * kv * dim * _SIZE[dtype])))
        return _attn(batch, rng.choice([1, 1, 1, 2, 5, 16]), keys, heads, kv, dim, window, sinks, dtype)
    window = _spread(rng, 16, 4096)
    cost = heads * dim * (5 if way == "bwd" else 2) * (4 if dtype == "f32" else 1)
    tokens = _spread(rng, 8, max(16, min(32768, 2 * _MOST_PAIRS // (cost * window))))
    batch = min(tokens, rng.choice([1, 1, 2, 3, 8]))
    length = tokens // batch
    return _attn(batch, length, length, heads, kv, dim, window, sinks, dtype, way, rng.random() < 0.3, way == "fwd" and rng.random() < 0.5)


# ---- inputs ---------------------------------------------------------------------------------
def _lengths(case):
    """Tokens of each sequence of a padded batch."""
    S, B = case["keys"], case["batch"]
    return [S - b * S // (4 * B) for b in range(B)]


def _prepare_attn(case, g):
    B, Sq, Sk, A, K, D = (case[n] for n in ("batch", "queries", "keys", "heads", "kv_heads", "dim"))
    dt = _DT[case["dtype"]]
    normal = lambda *shape: torch.randn(*shape, generator=g, device="cuda", dtype=torch.float32).to(dt)  # noqa: E731
    state = {"key_len": None, "query_start": None, "scale": 1.0 / math.sqrt(D), "lse": None}
    if Sq == Sk:      # q and k by head, as rotary positions leave them; v in the projection
        state["q"], state["k"] = normal(B, A, Sq, D).transpose(1, 2), normal(B, K, Sk, D).transpose(1, 2)
        state["v"] = normal(B, Sk, A + 2 * K, D)[:, :, A + K:]
        if case["padded"]:
            state["key_len"] = torch.tensor(_lengths(case), dtype=torch.int32, device="cuda")
    else:             # a cache by head, each sequence with its own length
        state["q"] = normal(B, Sq, A, D)
        state["k"], state["v"] = (normal(B, K, Sk, D).transpose(1, 2) for _ in range(2))
        low = min(Sk, case["window"] + case["sinks"] + Sq)
        state["key_len"] = torch.randint(low, Sk + 1, (B,), generator=g, device="cuda", dtype=torch.int32)
        state["query_start"] = state["key_len"] - Sq
    state["out"] = torch.empty(B, Sq, A, D, device="cuda", dtype=dt)
    if case["keep"]:
        state["lse"] = torch.empty(B, A, Sq, device="cuda", dtype=torch.float32)
    if case["way"] == "bwd":
        kept = _plain_attn_fwd({**state, "case": case}, True)
        state["out"], state["lse"] = kept["out"], kept["lse"]
        state["dout"] = normal(B, Sq, A, D)
        state["dq"], state["dk"] = (torch.empty(B, n, Sq, D, device="cuda", dtype=dt).transpose(1, 2) for n in (A, K))
        state["dv"] = torch.empty(B, Sk, A + 2 * K, D, device="cuda", dtype=dt)[:, :, A + K:]
    return state


def _prepare_norm(case, g):
    N, M = case["rows"], case["hidden"]
    dt = _DT[case["dtype"]]
    normal = lambda *shape: torch.randn(*shape, generator=g, device="cuda", dtype=torch.float32)  # noqa: E731
    empty = lambda *shape, dtype=dt: torch.empty(*shape, device="cuda", dtype=dtype)  # noqa: E731
    layer = case["kind"] == "layer"
    state = {"f": normal(N, M).mul_(2.0).to(dt), "eps": 1e-5}
    state["gate"] = 0.5 * normal(case["groups"], M) if case["gated"] else None
    for name, there in (("post", case["post"]), ("pre", True)):
        state[name + "_weight"] = 1.0 + 0.1 * normal(M) if there else None
        state[name + "_bias"] = 0.1 * normal(M) if there and layer else None
        state[name + "_stats"] = empty(N, 2, dtype=torch.float32) if there else None
    if case["way"] == "fwd":
        state["x"], state["y"], state["h"] = normal(N, M).to(dt), empty(N, M), empty(N, M)
        return state
    state["y"], state["dy"], state["dh"] = normal(N, M).mul_(1.5).to(dt), normal(N, M).to(dt), normal(N, M).to(dt)
    for name, t in (("post", state["f"]), ("pre", state["y"])):
        if state[name + "_stats"] is not None:
            state[name + "_stats"] = _plain_stats(t, case["kind"], state["eps"])
    state["dx"], state["df"] = empty(N, M), empty(N, M)
    for name in ("gate", "post_weight", "post_bias", "pre_weight", "pre_bias"):
        state["d" + name] = None if state[name] is None else torch.empty_like(state[name])
    return state


def _prepare_axes(case, g):
    B, A, K, D = (case[n] for n in ("batch", "heads", "kv_heads", "dim"))
    dt = _DT[case["dtype"]]
    normal = lambda *shape: torch.randn(*shape, generator=g, device="cuda", dtype=torch.float32).to(dt)  # noqa: E731
    sections = [int(n) for n in case["sections"].split("-")]
    pairs = sum(sections)
    text = torch.arange(64, device="cuda").expand(3, 64)
    sizes = (case["frames"], case["height"], case["width"])
    patches = torch.stack(torch.meshgrid(*(torch.arange(n, device="cuda") for n in sizes), indexing="ij")).reshape(3, -1) + 64
    start = torch.randint(0, 1024, (1, B, 1), generator=g, device="cuda")      # what came before in each sequence
    positions = torch.cat((text, patches), 1)[:, None] + start
    S = positions.shape[-1]
    state = {"positions": positions, "axes": torch.repeat_interleave(
        torch.arange(3, device="cuda"), torch.tensor(sections, device="cuda")).to(torch.uint8),
        "freqs": 10000.0 ** (-torch.arange(pairs, dtype=torch.float64, device="cuda") / pairs)}
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


def prepare(case, seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    state = {"attn": _prepare_attn, "norm": _prepare_norm, "axes": _prepare_axes}[case["op"]](case, g)
    state["case"] = case
    return state


# ---- one pass -------------------------------------------------------------------------------
def run(state):
    op, way = state["case"]["op"], state["case"]["way"]
    if own:
        return {"attn": _own_attn, "norm": _own_norm, "axes": _own_axes}[op](state)
    if op == "axes":
        return _plain_axes(state)
    if op == "norm":
        return _plain_norm_fwd(state) if way == "fwd" else _plain_norm_bwd(state)
    return _plain_attn_fwd(state, state["case"]["keep"]) if way == "fwd" else _plain_attn_bwd(state)


def _own_attn(state):
    from paper_2210_10246_amd import binding as B
    case = state["case"]
    if case["way"] == "fwd":
        B.tempo_window_attn_fwd(state["q"], state["k"], state["v"], state["out"], state["lse"], case["window"], case["sinks"],
                                state["scale"], state["key_len"], state["query_start"])
        return {"out": state["out"], "lse": state["lse"]}
    B.tempo_window_attn_bwd(state["dout"], state["q"], state["k"], state["v"], state["out"], state["lse"], state["dq"],
                            state["dk"], state["dv"], case["window"], case["sinks"], state["scale"], state["key_len"],
                            state["query_start"])
    return {"dq": state["dq"], "dk": state["dk"], "dv": state["dv"]}


def _own_norm(state):
    from paper_2210_10246_amd import binding as B
    case, s = state["case"], state
    post, pre = case["kind"] if case["post"] else None, case["kind"]
    if case["way"] == "fwd":
        B.tempo_residual_norm_fwd(s["x"], s["f"], s["gate"], s["y"], s["h"], post, s["post_weight"], s["post_bias"],
                                  s["post_stats"], pre, s["pre_weight"], s["pre_bias"], s["pre_stats"], case["alpha"],
                                  case["beta"], s["eps"], s["eps"])
        return {"y": s["y"], "h": s["h"], "post_stats": s["post_stats"], "pre_stats": s["pre_stats"]}
    B.tempo_residual_norm_bwd(s["dy"], s["dh"], s["f"], s["y"], s["gate"], s["dx"], s["df"], s["dgate"], post, s["post_weight"],
                              s["post_bias"], s["post_stats"], s["dpost_weight"], s["dpost_bias"], pre, s["pre_weight"],
                              s["pre_stats"], s["dpre_weight"], s["dpre_bias"], case["alpha"], case["beta"])
    return {n: s[n] for n in ("dx", "df", "dgate", "dpost_weight", "dpost_bias", "dpre_weight", "dpre_bias")}


def _own_axes(state):
    from paper_2210_10246_amd import binding as B
    call = B.tempo_rotary_axes_fwd if state["case"]["way"] == "fwd" else B.tempo_rotary_axes_bwd
    call(state["q"], state["k"], state["freqs"], state["axes"], state["positions"], state["q_out"], state["k_out"],
         state["case"]["layout"])
    return {"q": state["q_out"], "k": state["k_out"]}


def _windows(state):
    """Queries a stretch at a time, with the keys that any of them sees: (queries, keys, k and v [B, kv, keys, D] in 32 bits,
    which pair is visible [B or 1, 1, queries, keys])."""
    case = state["case"]
    B, Sq, Sk, A, W, sinks = (case[n] for n in ("batch", "queries", "keys", "heads", "window", "sinks"))
    where = torch.arange(Sk, device="cuda")
    by_head = lambda t: t.permute(0, 2, 1, 3).float()  # noqa: E731
    if Sq != Sk:      # a few queries at the end of each sequence: the keys are collected for each
        span = torch.arange(min(sinks, Sk), device="cuda"), torch.arange(1 - W, Sq, device="cuda")
        start = state["query_start"].long()[:, None]
        keys = torch.cat((span[0].expand(B, -1), start + span[1]), 1)
        first = torch.arange(keys.shape[1], device="cuda") < len(span[0])
        at = (start + torch.arange(Sq, device="cuda"))[:, :, None]
        seen = (keys[:, None] >= 0) & (keys[:, None] <= at) & (first | ((keys[:, None] > at - W) & (keys[:, None] >= sinks)))
        rows, keys = torch.arange(B, device="cuda")[:, None], keys.clamp(0, Sk - 1)
        yield slice(0, Sq), None, by_head(state["k"][rows, keys]), by_head(state["v"][rows, keys]), seen[:, None]
        return
    stretch = max(16, min(Sq, 1024, (1 << 28) // (B * A * (W + sinks + 1024)), max(W, 256)))
    for i in range(0, Sq, stretch):
        queries = slice(i, min(i + stretch, Sq))
        low = max(0, i - W + 1)
        keys = where[low:queries.stop]
        if low > 0:
            keys = torch.cat((where[:min(sinks, low)], keys))
        at = where[queries, None]
        seen = ((keys <= at) & ((keys > at - W) | (keys < sinks)))[None]
        if state["key_len"] is not None:
            seen = seen & (keys < state["key_len"][:, None, None])
        yield queries, keys, by_head(state["k"][:, keys]), by_head(state["v"][:, keys]), seen[:, None]


def _rows(t, queries, kv):
    """[B, S, heads, D] -> [B, kv, heads / kv * queries, D] in 32 bits"""
    t = t[:, queries].permute(0, 2, 1, 3).float()
    return t.reshape(t.shape[0], kv, -1, t.shape[-1])


def _plain_attn_fwd(state, keep):
    case = state["case"]
    B, Sq, A, K, D = (case[n] for n in ("batch", "queries", "heads", "kv_heads", "dim"))
    out, lse = [], []
    for queries, _, k, v, seen in _windows(state):
        s = torch.matmul(_rows(state["q"], queries, K), k.transpose(-1, -2).contiguous()) * state["scale"]
        s = s.view(B, A, -1, k.shape[2]).masked_fill(~seen, -math.inf)
        top = s.amax(-1, keepdim=True)
        p = torch.exp(s - top)
        total = p.sum(-1, keepdim=True)
        o = torch.matmul(p.view(B, K, -1, k.shape[2]), v).view(B, A, -1, D) / total
        out.append(o.permute(0, 2, 1, 3).to(_DT[case["dtype"]]))
        lse.append((top + torch.log(total))[..., 0])
    return {"out": torch.cat(out, 1), "lse": torch.cat(lse, 2) if keep else None}


def _plain_attn_bwd(state):
    case = state["case"]
    B, Sq, A, K, D, sinks = (case[n] for n in ("batch", "queries", "heads", "kv_heads", "dim", "sinks"))
    dt = _DT[case["dtype"]]
    dq = []
    dk, dv = (torch.zeros(B, K, case["keys"], D, device="cuda") for _ in range(2))
    for queries, keys, k, v, seen in _windows(state):
        q, dout, out = (_rows(state[n], queries, K) for n in ("q", "dout", "out"))
        s = torch.matmul(q, k.transpose(-1, -2).contiguous()) * state["scale"]
        s = s.view(B, A, -1, k.shape[2]) - state["lse"][:, :, queries, None]
        p = torch.exp(s).masked_fill(~seen, 0.0).view(B, K, -1, k.shape[2])
        ds = p * (torch.matmul(dout, v.transpose(-1, -2).contiguous()) - (dout * out).sum(-1, keepdim=True)) * state["scale"]
        dq.append(torch.matmul(ds, k).view(B, A, -1, D).permute(0, 2, 1, 3).to(dt))
        dk.index_add_(2, keys, torch.matmul(ds.transpose(-1, -2).contiguous(), q))
        dv.index_add_(2, keys, torch.matmul(p.transpose(-1, -2).contiguous(), dout))
    return {"dq": torch.cat(dq, 1), "dk": dk.permute(0, 2, 1, 3).to(dt), "dv": dv.permute(0, 2, 1, 3).to(dt)}


def _plain_stats(t, kind, eps):
    t = t.float()
    mean = t.mean(-1, keepdim=True) if kind == "layer" else torch.zeros_like(t[:, :1])
    return torch.cat((mean, torch.rsqrt(((t - mean) ** 2).mean(-1, keepdim=True) + eps)), 1)


def _affine(t, stats, weight, bias):
    n = (t.float() - stats[:, :1]) * stats[:, 1:] * weight
    return n if bias is None else n + bias


def _gates(state):
    """beta * gate of every row [groups, rows of a group or 1, M], or beta"""
    return state["case"]["beta"] if state["gate"] is None else state["case"]["beta"] * state["gate"][:, None]


def _plain_norm_fwd(state):
    case, dt = state["case"], _DT[state["case"]["dtype"]]
    N, M, groups = case["rows"], case["hidden"], case["groups"]
    stats = _plain_stats(state["f"], case["kind"], state["eps"]) if case["post"] else None
    n = _affine(state["f"], stats, state["post_weight"], state["post_bias"]) if case["post"] else state["f"].float()
    y = case["alpha"] * state["x"].float() + (n.view(groups, -1, M) * _gates(state)).view(N, M)
    y = y.to(dt)      # the next block's residual, which its norm is of
    pre = _plain_stats(y, case["kind"], state["eps"])
    return {"y": y, "h": _affine(y, pre, state["pre_weight"], state["pre_bias"]).to(dt), "post_stats": stats, "pre_stats": pre}


def _plain_norm_grad(d, t, stats, weight, kind):
    """The gradients of t, the weight and the bias from that of norm(t)."""
    hat = (t.float() - stats[:, :1]) * stats[:, 1:]
    dw = d * weight
    dt = dw - hat * (dw * hat).mean(-1, keepdim=True)
    if kind == "layer":
        dt = dt - dw.mean(-1, keepdim=True)
    return dt * stats[:, 1:], (d * hat).sum(0), d.sum(0)


def _plain_norm_bwd(state):
    case, dt = state["case"], _DT[state["case"]["dtype"]]
    N, M, groups, layer = case["rows"], case["hidden"], case["groups"], case["kind"] == "layer"
    through, dpw, dpb = _plain_norm_grad(state["dh"].float(), state["y"], state["pre_stats"], state["pre_weight"], case["kind"])
    d = state["dy"].float() + through
    out = {"dx": (case["alpha"] * d).to(dt), "dpre_weight": dpw, "dpre_bias": dpb if layer else None, "dgate": None,
           "dpost_weight": None, "dpost_bias": None}
    if case["gated"]:
        n = _affine(state["f"], state["post_stats"], state["post_weight"], state["post_bias"]) if case["post"] else state["f"].float()
        out["dgate"] = case["beta"] * (n * d).view(groups, -1, M).sum(1)
    d = (d.view(groups, -1, M) * _gates(state)).view(N, M)
    if case["post"]:
        d, out["dpost_weight"], db = _plain_norm_grad(d, state["f"], state["post_stats"], state["post_weight"], case["kind"])
        out["dpost_bias"] = db if layer else None
    return {**out, "df": d.to(dt)}


def _plain_axes(state):
    case = state["case"]
    at = state["positions"].double()[state["axes"].long()].permute(1, 2, 0)      # [B, S, pairs]
    angle = (at * state["freqs"])[:, :, None]
    c, s = angle.cos().float(), angle.sin().float()
    if case["way"] == "bwd":
        s = -s
    half = state["freqs"].numel()

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


# ---- what one pass cannot do without --------------------------------------------------------
def work(case):
    size = _SIZE[case["dtype"]]
    if case["op"] == "axes":
        tokens, heads = case["batch"] * (64 + case["frames"] * case["height"] * case["width"]), case["heads"] + case["kv_heads"]
        pairs = sum(int(n) for n in case["sections"].split("-"))
        return {"bytes": 2 * size * tokens * heads * case["dim"] + 24 * tokens + 9 * pairs, "flops": 6 * tokens * heads * pairs}
    if case["op"] == "norm":
        N, M, norms = case["rows"], case["hidden"], 2 if case["post"] else 1
        columns = norms * (2 if case["kind"] == "layer" else 1) + (case["groups"] if case["gated"] else 0)
        if case["way"] == "fwd":
            return {"bytes": 4 * size * N * M + 8 * norms * N + 4 * columns * M, "flops": 10 * N * M}
        return {"bytes": 6 * size * N * M + 8 * norms * N + 8 * columns * M, "flops": 25 * N * M}
    B, Sq, Sk, A, K, D, W, sinks = (case[n] for n in ("batch", "queries", "keys", "heads", "kv_heads", "dim", "window", "sinks"))
    if Sq == Sk:
        pairs, seen = 0, 0
        for n in _lengths(case) if case["padded"] else [Sk] * B:
            for_row = lambda i: min(i + 1, n) - max(0, min(i + 1 - W, n) - min(sinks, n, max(i + 1 - W, 0)))  # noqa: E731
            pairs += sum(for_row(i) for i in range(Sk))
            seen += n
    else:
        low = min(Sk, W + sinks + Sq)      # the shortest sequence
        pairs = B * sum(min(low - Sq + 1 + i, W + sinks) for i in range(Sq))
        seen = B * min(low, W + sinks + Sq - 1)
    rows = B * Sq * A
    if case["way"] == "fwd":
        return {"bytes": size * D * (2 * rows + 2 * seen * K) + (4 * rows if case["keep"] else 0), "flops": 4 * D * pairs * A}
    return {"bytes": size * D * (4 * rows + 4 * seen * K) + 4 * rows, "flops": 10 * D * pairs * A}


# ---- the definition in 64 bits --------------------------------------------------------------
def _exact_attn(case, state):
    B, Sq, Sk, A, K, D, W, sinks = (case[n] for n in ("batch", "queries", "keys", "heads", "kv_heads", "dim", "window", "sinks"))
    if B * A * Sq * Sk > 1 << 37:
        return None
    key = torch.arange(Sk, device="cuda")
    out = torch.empty(B, Sq, A, D, device="cuda", dtype=torch.float64)
    lse = torch.empty(B, A, Sq, device="cuda", dtype=torch.float64)
    dq = torch.empty_like(out)
    dk, dv = (torch.zeros(B, Sk, K, D, device="cuda", dtype=torch.float64) for _ in range(2))
    for b in range(B):
        start = 0 if state["query_start"] is None else int(state["query_start"][b])
        there = Sk if state["key_len"] is None else int(state["key_len"][b])
        for a in range(A):
            k, v = state["k"][b, :, a * K // A].double(), state["v"][b, :, a * K // A].double()
            for i in range(0, Sq, 4096):
                rows = slice(i, i + 4096)
                q = state["q"][b, rows, a].double()
                back = (start + torch.arange(i, i + len(q), device="cuda"))[:, None] - key      # how far back a key lies
                hidden = (back < 0) | ((back >= W) & (key >= sinks)) | (key >= there)
                s = (q.mm(k.t()) * state["scale"]).masked_fill_(hidden, -math.inf)
                if case["way"] == "fwd":
                    lse[b, a, rows] = torch.logsumexp(s, 1)
                    out[b, rows, a] = torch.softmax(s, 1).mm(v)
                    continue
                dout = state["dout"][b, rows, a].double()
                p = s.sub_(state["lse"][b, a, rows].double()[:, None]).exp_()
                dv[b, :, a * K // A] += p.t().mm(dout)
                ds = dout.mm(v.t()).sub_((dout * state["out"][b, rows, a].double()).sum(1)[:, None]).mul_(p).mul_(state["scale"])
                dq[b, rows, a] = ds.mm(k)
                dk[b, :, a * K // A] += ds.t().mm(q)
    if case["way"] == "fwd":
        return {"out": out, "lse": lse if case["keep"] else None}
    return {"dq": dq, "dk": dk, "dv": dv}


def _exact_norm(case, state):
    N, M, groups, eps = case["rows"], case["hidden"], case["groups"], state["eps"]
    wide = {n: None if state[n] is None else state[n].double()
            for n in ("gate", "post_weight", "post_bias", "pre_weight", "pre_bias")}

    def hat(t, name):      # with the statistics of the forward, where this is a backward, and what a forward keeps
        if case["way"] == "bwd":
            kept = state[name + "_stats"].double()
            return (t - kept[:, 0, None]) * kept[:, 1, None], None
        centre = t.mean(1) if case["kind"] == "layer" else t.new_zeros(N)
        spread = torch.sqrt((t - centre[:, None]).square().sum(1) / M + eps)
        return (t - centre[:, None]) / spread[:, None], torch.stack((centre, 1.0 / spread), 1)

    def scaled(n, name):
        n = n * wide[name + "_weight"]
        return n if wide[name + "_bias"] is None else n + wide[name + "_bias"]
    rows = torch.full((N, 1), case["beta"], device="cuda", dtype=torch.float64)
    if case["gated"]:
        rows = rows * wide["gate"].repeat_interleave(N // groups, 0)
    f = state["f"].double()
    fh, post_stats = hat(f, "post") if case["post"] else (f, None)
    n = scaled(fh, "post") if case["post"] else f
    if case["way"] == "fwd":
        y = case["alpha"] * state["x"].double() + rows * n
        yh, pre_stats = hat(y.to(_DT[case["dtype"]]).double(), "pre")      # the norm is of what the next block's residual holds
        return {"y": y, "h": scaled(yh, "pre"), "post_stats": post_stats, "pre_stats": pre_stats}

    def grad(d, t_hat, name):      # through a norm
        g = d * wide[name + "_weight"]
        left = t_hat * (g * t_hat).sum(1, keepdim=True) / M
        if case["kind"] == "layer":
            left = left + g.sum(1, keepdim=True) / M
        return (g - left) * state[name + "_stats"][:, 1:].double()
    yh = hat(state["y"].double(), "pre")[0]
    dh, layer = state["dh"].double(), case["kind"] == "layer"
    d = state["dy"].double() + grad(dh, yh, "pre")
    dn = rows * d
    return {"dx": case["alpha"] * d, "df": grad(dn, fh, "post") if case["post"] else dn,
            "dgate": case["beta"] * (n * d).reshape(groups, N // groups, M).sum(1) if case["gated"] else None,
            "dpost_weight": (dn * fh).sum(0) if case["post"] else None,
            "dpost_bias": dn.sum(0) if case["post"] and layer else None,
            "dpre_weight": (dh * yh).sum(0), "dpre_bias": dh.sum(0) if layer else None}


def _exact_axes(case, state):
    way = 1.0 if case["way"] == "fwd" else -1.0
    half = state["freqs"].numel()
    place = torch.stack([state["positions"][a].double() * f for a, f in zip(state["axes"].tolist(), state["freqs"].tolist())], -1)
    by = torch.polar(torch.ones_like(place), place * way)[:, :, None]      # multiplication by e^(i angle)
    first = slice(0, half) if case["layout"] == "half" else slice(0, 2 * half, 2)
    second = slice(half, 2 * half) if case["layout"] == "half" else slice(1, 2 * half, 2)
    out = {}
    for name in ("q", "k"):
        y = state[name].double()
        z = torch.complex(y[..., first], y[..., second]) * by
        y = y.clone()
        y[..., first], y[..., second] = z.real, z.imag
        out[name] = y
    return out


def exact(case, seed):
    state = prepare(case, seed)
    return {"attn": _exact_attn, "norm": _exact_norm, "axes": _exact_axes}[case["op"]](case, state)
