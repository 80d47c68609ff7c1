"""Refusals of window attention, residual norms and rotary positions of several axes, which need no GPU: the C ABI's, the binding's, the
modules'."""
import ctypes
import math

import pytest
import torch

from paper_2210_10246_amd import binding as B
from paper_2210_10246_amd.modules import RotaryPositions, TempoResidualNorm, TempoWindowAttention, rotary_axes, rotary_frequencies

OK, INVALID, UNSUPPORTED, WORKSPACE = 0, 1, 2, 3


def heads(p=32, strides=(64, 16, 8)):
    return B._AttnHeads(p, (ctypes.c_int64 * 3)(*strides))


def window_fwd(q=heads(), k=heads(), v=heads(), out=heads(), lse=32, key_len=None, start=None, ws=None, size=0, B_=2, S=4, Sk=4, A=2, K=2, D=8,
               window=3, sinks=1, scale=1.0, dt=0):
    return B.load().tempo_window_attn_fwd(q, k, v, out, lse, key_len, start, ws, size, B_, S, Sk, A, K, D, window, sinks, scale, dt, None)


def window_bwd(dout=heads(), q=heads(), k=heads(), v=heads(), out=heads(), lse=32, dq=heads(), dk=heads(), dv=heads(), key_len=None, start=None,
               ws=16, size=0, B_=2, S=4, Sk=4, A=2, K=2, D=8, window=3, sinks=1, scale=1.0, dt=0):
    return B.load().tempo_window_attn_bwd(dout, q, k, v, out, lse, dq, dk, dv, key_len, start, ws, size, B_, S, Sk, A, K, D, window, sinks,
                                          scale, dt, None)


def test_window_attention_arguments_are_checked_before_any_launch():
    big = 1 << 62
    for call in (window_fwd, window_bwd):
        for args in (dict(q=None), dict(k=None), dict(v=None), dict(out=None), dict(B_=-1), dict(S=-1), dict(Sk=-1), dict(A=-1), dict(K=-1), dict(K=0),
                     dict(A=3), dict(D=0), dict(D=-1), dict(window=0), dict(window=-1), dict(sinks=-1), dict(scale=0.0), dict(scale=-1.0),
                     dict(scale=math.nan), dict(scale=math.inf), dict(scale=1e-39), dict(scale=3e38), dict(dt=2), dict(dt=-1), dict(S=1 << 31), dict(Sk=1 << 31), dict(B_=big), dict(D=big),
                     dict(A=big, K=big), dict(q=heads(strides=(-1, 1, 1))), dict(k=heads(strides=(64, -1, 1))), dict(v=heads(strides=(1 << 50, 1, 1))),
                     dict(q=heads(None)), dict(k=heads(None)), dict(v=heads(None)), dict(out=heads(None))):
            assert call(**args) == INVALID, args
        for args in (dict(D=257), dict(q=heads(34)), dict(k=heads(33), dt=1), dict(v=heads(34)), dict(out=heads(34)), dict(lse=34), dict(key_len=34),
                     dict(start=33), dict(ws=8, size=1 << 30), dict(A=1 << 29, K=1, S=4, B_=1, q=heads(strides=(0, 0, 0)), out=heads(strides=(1 << 31, 8, 8)))):
            assert call(**args) in (UNSUPPORTED, INVALID), args
        for args in (dict(D=257), dict(q=heads(34)), dict(lse=34), dict(ws=8, size=1 << 30)):
            assert call(**args) == UNSUPPORTED, args
        for args in (dict(B_=0), dict(A=0, K=0), dict(S=0, Sk=0)):
            nothing = {n: heads(None) for n in ("q", "k", "v", "out")}
            assert call(**args, **nothing) == OK, args
    for strides in ((0, 16, 8), (64, 0, 8), (64, 16, 0)):
        assert window_fwd(out=heads(strides=strides)) == INVALID
        for name in ("dq", "dk", "dv"):
            assert window_bwd(**{name: heads(strides=strides)}) == INVALID
    for name in ("dout", "dq", "dk", "dv"):
        assert window_bwd(**{name: None}) == INVALID and window_bwd(**{name: heads(None)}) == INVALID
        assert window_bwd(**{name: heads(34)}) == UNSUPPORTED
    assert window_bwd(lse=None) == INVALID
    # a workspace that is too small, or none where one is needed
    sizes = dict(B_=1, S=1, Sk=4000, A=1, K=1, D=64, window=4000)
    assert B.tempo_window_attn_fwd_workspace_bytes(1, 1, 4000, 1, 1, 64, 4000, 1, torch.float32) > 16
    assert window_fwd(**sizes) == WORKSPACE and window_fwd(ws=16, size=16, **sizes) == WORKSPACE
    assert window_bwd(**sizes) == WORKSPACE and window_bwd(ws=None, size=1 << 30, **sizes) == WORKSPACE


def test_key_heads_that_no_head_reads_have_gradients():
    """Where there are no heads of queries, a backward needs k, v and what it writes zeros to, and no workspace, as for no queries."""
    none = heads(None)
    sizes = dict(A=0, K=2, Sk=4)
    assert window_fwd(q=none, k=none, v=none, out=none, **sizes) == OK
    nothing = dict(q=none, out=none, dout=none, dq=none, lse=None)
    for name in ("k", "v", "dk", "dv"):
        assert window_bwd(**{**nothing, name: none}, **sizes) == INVALID
    for sizes_of in ((2, 4, 4, 0, 2), (2, 0, 4, 2, 2)):
        assert B.tempo_window_attn_bwd_workspace_bytes(*sizes_of, 8, 3, 1, torch.float32) == 0
    assert window_bwd(**nothing, **{**sizes, "Sk": 0}) == OK


def test_window_attention_workspaces_of_any_sizes():
    """Every size is looked at before it divides anything, and none overflows."""
    for way in (B.tempo_window_attn_fwd_workspace_bytes, B.tempo_window_attn_bwd_workspace_bytes):
        for n in range(8):
            for value in (-1, 0, 1, (1 << 31) - 1, 1 << 31, 1 << 40, (1 << 63) - 1):
                sizes = [2, 100, 300, 4, 2, 64, 50, 3]
                sizes[n] = value
                assert way(*sizes, torch.bfloat16) >= 0 and way(*sizes, torch.float32) >= 0
        assert way(2, 100, 300, 4, 0, 64, 50, 3, torch.float32) == 0 and way(2, 100, 300, 4, 3, 64, 50, 3, torch.float32) == 0


def norm(kind=0, weight=32, bias=None, eps=1e-5, stats=32):
    return B._Norm(kind, weight, bias, eps, stats)


def norm_fwd(x=16, f=16, gate=None, groups=1, post=norm(), pre=norm(), y=16, h=16, N=4, M=8, dt=0):
    return B.load().tempo_residual_norm_fwd(x, f, gate, groups, post, pre, y, h, 1.0, 1.0, N, M, dt, None)


def norm_bwd(dy=16, dh=16, f=16, y=16, gate=None, groups=1, post=norm(), pre=norm(), dx=16, df=16, dgate=None, dpw=None, dpb=None, dqw=None,
             dqb=None, ws=None, size=0, N=4, M=8, dt=0):
    return B.load().tempo_residual_norm_bwd(dy, dh, f, y, gate, groups, post, pre, dx, df, dgate, dpw, dpb, dqw, dqb, 1.0, 1.0, ws, size, N, M,
                                            dt, None)


def test_residual_norm_arguments_are_checked_before_any_launch():
    big = 1 << 62
    for call in (norm_fwd, norm_bwd):
        for args in (dict(N=-1), dict(M=-1), dict(N=big), dict(M=big), dict(M=1 << 31), dict(groups=0), dict(groups=-1), dict(groups=3), dict(dt=2),
                     dict(post=norm(kind=2)), dict(pre=norm(kind=-1)), dict(post=norm(eps=-1.0)), dict(pre=norm(eps=math.nan)), dict(f=None)):
            assert call(**args) == INVALID, args
        for args in (dict(f=8), dict(y=24), dict(gate=34), dict(post=norm(weight=33)), dict(pre=norm(stats=36)),
                     dict(gate=16, N=1 << 24, groups=1 << 24)):
            assert call(**args) == UNSUPPORTED, args
        assert call(M=0) == OK
    for args in (dict(x=None), dict(y=None), dict(h=None)):
        assert norm_fwd(**args) == INVALID, args
    assert norm_fwd(N=0, x=None, f=None, y=None, h=None) == OK
    for args in (dict(dx=None), dict(df=None), dict(dh=None), dict(y=None), dict(dy=None, pre=None), dict(post=norm(stats=None)),
                 dict(pre=norm(stats=None)), dict(dgate=16), dict(post=None, dpw=16), dict(post=None, dpb=16), dict(pre=None, dqw=16), dict(pre=None, dqb=16)):
        assert norm_bwd(**args) == INVALID, args
    for args in (dict(dx=8), dict(dqw=33, ws=16, size=1 << 30), dict(ws=8)):
        assert norm_bwd(**args) == UNSUPPORTED, args
    assert norm_bwd(dqw=16) == WORKSPACE and norm_bwd(dqw=16, ws=16, size=16) == WORKSPACE
    need = B.tempo_residual_norm_bwd_workspace_bytes
    assert need(4, 8, 1, torch.float32) >= 4 * 8 * 2 * 4
    assert all(need(*a, torch.bfloat16) == 0 for a in ((-1, 8, 1), (4, -1, 1), (4, 0, 1), (4, 8, 3), (4, 8, 0), (big, 8, 1), (4, big, 1)))


def rotary_heads(x=32, y=32, n=2, strides=(64, 16, 8)):
    return B._RotaryHeads(x, y, n, (ctypes.c_int64 * 3)(*strides), (ctypes.c_int64 * 3)(*strides))


def test_rotary_axes_arguments_are_checked_before_any_launch():
    def call(way, axes=32, n=3, positions=32, stride=8, bits=64, q=rotary_heads(), freqs=32, R=8):
        at = B._RotaryPositions(positions, bits, (ctypes.c_int64 * 2)(0, 1), 0)
        return getattr(B.load(), "tempo_rotary_axes_" + way)(q, None, freqs, axes, n, at, stride, 2, 4, 8, R, 0, 1.0, 0, None)
    for way in ("fwd", "bwd"):
        for args in (dict(axes=None), dict(n=0), dict(n=-1), dict(n=5), dict(positions=None), dict(stride=-1), dict(stride=1 << 50), dict(bits=16),
                     dict(freqs=None), dict(R=3), dict(R=10), dict(q=rotary_heads(x=None))):
            assert call(way, **args) == INVALID, args
        for args in (dict(positions=36), dict(freqs=36), dict(q=rotary_heads(x=34))):
            assert call(way, **args) == UNSUPPORTED, args


def test_binding_refuses_other_forms():
    t = lambda *s, dtype=torch.float32: torch.zeros(*s, dtype=dtype)  # noqa: E731
    q, k, lse = t(2, 4, 4, 8), t(2, 6, 2, 8), t(2, 4, 4)
    good = dict(q=q, k=k, v=k, out=q, lse=lse, window=3)
    for message, args in (
            ("float32 or bfloat16", dict(q=q.half(), k=k.half(), v=k.half(), out=q.half())), ("v must be", dict(v=k.bfloat16())),
            ("adjacent", dict(q=t(2, 4, 4, 16)[..., ::2])), ("adjacent", dict(k=t(2, 6, 16))), ("shape", dict(out=t(2, 4, 4, 9))),
            ("shape", dict(v=t(2, 5, 2, 8))), ("batch and elements", dict(k=t(1, 6, 2, 8), v=t(1, 6, 2, 8))), ("multiple", dict(k=t(2, 6, 3, 8), v=t(2, 6, 3, 8))),
            ("window", dict(window=0)), ("sinks", dict(sinks=-1)), ("window", dict(window=1 << 63)), ("scale", dict(scale=0.0)), ("scale", dict(scale=math.nan)),
            ("elements", dict(q=t(2, 4, 4, 0), k=t(2, 6, 2, 0), v=t(2, 6, 2, 0), out=t(2, 4, 4, 0))), ("lse", dict(lse=lse.double())), ("lse", dict(lse=t(2, 4, 3))), ("key_len", dict(key_len=t(2, dtype=torch.int64))),
            ("query_start", dict(query_start=t(3, dtype=torch.int32))), ("CUDA", {})):
        with pytest.raises(ValueError, match=message):
            B.tempo_window_attn_fwd(**{**good, **args})
    back = dict(dout=q, q=q, k=k, v=k, out=q, lse=lse, dq=q, dk=k, dv=k, window=3)
    for message, args in (("lse", dict(lse=None)), ("dk must have shape", dict(dk=q)), ("dout must be", dict(dout=q.bfloat16())), ("CUDA", {})):
        with pytest.raises(ValueError, match=message):
            B.tempo_window_attn_bwd(**{**back, **args})
    x, g, st = t(6, 8), t(8), t(6, 2)
    good = dict(x=x, f=x, gate=None, y=x, h=x, post="rms", post_weight=g, post_bias=None, post_stats=st, pre="layer", pre_weight=g, pre_bias=g,
                pre_stats=None)
    for message, args in (
            ("x must be", dict(x=x.half())), ("f must be", dict(f=x.bfloat16())), ("f must have", dict(f=t(5, 8))), ("h is needed", dict(h=None)),
            ("post must be", dict(post="batch")), ("there is no post_weight", dict(post=None)), ("pre_bias must have", dict(pre_bias=t(7))),
            ("post_stats must have", dict(post_stats=t(6))), ("gate must be torch", dict(gate=g.bfloat16())), ("gate must be \\[", dict(gate=t(9))),
            ("do not divide", dict(gate=t(4, 8))), ("CUDA", {})):
        with pytest.raises(ValueError, match=message):
            B.tempo_residual_norm_fwd(**{**good, **args})
    back = dict(dy=x, dh=x, f=x, y=x, gate=None, dx=x, df=x, dgate=None, post="rms", post_weight=g, post_bias=None, post_stats=st, dpost_weight=g,
                dpost_bias=None, pre="rms", pre_weight=g, pre_stats=st, dpre_weight=g, dpre_bias=None)
    for message, args in (("needed", dict(dx=None)), ("needed", dict(dh=None)), ("stats", dict(post_stats=None)), ("dgate", dict(dgate=g)),
                          ("None", dict(pre=None, pre_weight=None, pre_stats=None)), ("dh must be", dict(dh=x.bfloat16())), ("CUDA", {})):
        with pytest.raises(ValueError, match=message):
            B.tempo_residual_norm_bwd(**{**back, **args})
    f, axes, p = t(4, dtype=torch.float64), t(4, dtype=torch.uint8), t(3, 4, dtype=torch.int64)
    good = dict(q=q, k=None, freqs=f, axes=axes, positions=p, q_out=q, k_out=None)
    for message, args in (("needed", dict(axes=None)), ("needed", dict(positions=None)), ("axes must be", dict(axes=axes.int())),
                          ("axes must be", dict(axes=t(3, dtype=torch.uint8))), ("positions must be \\[", dict(positions=t(4, dtype=torch.int64))),
                          ("positions must be \\[", dict(positions=t(5, 4, dtype=torch.int64))), ("positions must be \\[", dict(positions=t(3, 3, 4, dtype=torch.int64))),
                          ("int32 or int64", dict(positions=p.float())), ("CUDA", {})):
        for call in (B.tempo_rotary_axes_fwd, B.tempo_rotary_axes_bwd):
            names = good if call is B.tempo_rotary_axes_fwd else None
            with pytest.raises(ValueError, match=message):
                call(*{**good, **args}.values()) if names is None else call(**{**good, **args})


def test_which_axis_a_pair_turns_by():
    assert rotary_axes((2, 3, 1)).tolist() == [0, 0, 1, 1, 1, 2]
    assert rotary_axes((2, 3, 1), "cyclic").tolist() == [0, 1, 2, 0, 1, 1]
    assert rotary_axes((0, 2)).tolist() == [1, 1]
    for args in (((),), ((1, 1, 1, 1, 1),), ((-1, 2),), ((0, 0),), ((1, 2), "mixed")):
        with pytest.raises(ValueError):
            rotary_axes(*args)
    r = RotaryPositions(12, sections=(2, 3, 1), own=True)
    assert r.axes.dtype == torch.uint8 and torch.equal(r.freqs[2:5], rotary_frequencies(6)[0]) and torch.equal(r.freqs[:2], rotary_frequencies(4)[0])
    assert torch.equal(RotaryPositions(12, sections=(2, 3, 1)).freqs, rotary_frequencies(12)[0])
    r.bfloat16().type(torch.float32)
    assert r.axes.dtype == torch.uint8 and r.freqs.dtype == torch.float64 and r.axes.tolist() == [0, 0, 1, 1, 1, 2]
    assert RotaryPositions(12).axes is None and not r.state_dict()
    for args in (dict(sections=(2, 3)), dict(own=True)):
        with pytest.raises(ValueError):
            RotaryPositions(12, **args)
    with pytest.raises(ValueError, match="positions"):
        r(torch.zeros(1, 1, 2, 12))
    for shape in ((2,), (1, 2), (2, 2), (4, 2), (2, 3, 2)):      # of other numbers of axes, batches' positions on one
        with pytest.raises(ValueError, match="3 axes"):
            r(torch.zeros(1, 1, 2, 12), positions=torch.zeros(shape, dtype=torch.int64))


def test_modules_refuse_other_forms_and_keep_float32():
    for args in ((0,), (4, -1), (4, 0, 0.0), (4, 0, math.inf), (4, 0, math.nan)):
        with pytest.raises(ValueError):
            TempoWindowAttention(*args)
    with pytest.raises(ValueError, match="post"):
        TempoResidualNorm(8, post="batch")
    n = TempoResidualNorm(8, "layer", "rms", gate=0.1).bfloat16()
    assert {k: (v.dtype, float(v[0])) for k, v in n.state_dict().items()} == {
        "gate": (torch.float32, float(torch.tensor(0.1))), "post_weight": (torch.float32, 1.0), "post_bias": (torch.float32, 0.0),
        "pre_weight": (torch.float32, 1.0)}
    assert not list(TempoResidualNorm(8, "layer", "layer", affine=False).parameters())
    x = torch.zeros(2, 3, 8)
    for message, args in (("own", (x, x, x[0, 0])), ("must be", (x, x[:1])), ("must be", (x[..., :4], x[..., :4]))):
        with pytest.raises(ValueError, match=message):
            n(*args)
    n = TempoResidualNorm(8)
    for shape in ((1, 3, 8), (2, 3, 1), (3, 1, 8), (2, 1, 1, 8), (), (3, 8), (4, 8)):
        with pytest.raises(ValueError):
            n(x, x, torch.zeros(shape))
