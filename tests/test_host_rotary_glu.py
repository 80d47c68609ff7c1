"""Refusals of rotary positions and the gated unit, which need no GPU: the C ABI's and the binding's."""
import ctypes

import pytest
import torch

from paper_2210_10246_amd import binding as B

INVALID, UNSUPPORTED, WORKSPACE = 1, 2, 3
f32, bf16 = torch.float32, torch.bfloat16


def heads(x=32, y=32, n=2, x_strides=(64, 16, 8), y_strides=(64, 16, 8)):
    return B._RotaryHeads(x, y, n, (ctypes.c_int64 * 3)(*x_strides), (ctypes.c_int64 * 3)(*y_strides))


def positions(p=None, bits=64, strides=(0, 1), start=0):
    return B._RotaryPositions(p, bits, (ctypes.c_int64 * 2)(*strides), start)


def rotary(q=None, k=None, freqs=32, at=None, B_=2, S=4, D=8, R=8, layout=0, dt=0, way="fwd"):
    call = getattr(B.load(), "tempo_rotary_" + way)
    return call(ctypes.byref(q) if q else None, ctypes.byref(k) if k else None, freqs,
                ctypes.byref(at) if at is not None else None, B_, S, D, R, layout, 1.0, dt, None)


@pytest.mark.parametrize("way", ["fwd", "bwd"])
def test_rotary_arguments_are_checked_before_any_launch(way):
    ok = positions()
    refused = [
        dict(q=None, at=ok), dict(q=heads(), at=None), dict(q=heads(), at=ok, B_=-1), dict(q=heads(), at=ok, S=-1),
        dict(q=heads(n=-1), at=ok), dict(q=heads(), k=heads(n=-1), at=ok), dict(q=heads(), at=ok, dt=2), dict(q=heads(), at=ok, layout=2),
        dict(q=heads(), at=ok, layout=-1), dict(q=heads(), at=ok, R=0), dict(q=heads(), at=ok, R=3), dict(q=heads(), at=ok, R=10),
        dict(q=heads(), at=ok, B_=1 << 20, S=1 << 20), dict(q=heads(n=1 << 24), at=ok), dict(q=heads(n=1 << 62), at=ok, D=1 << 62, R=2),
        dict(q=heads(), k=heads(n=1 << 21), at=ok), dict(q=heads(x_strides=(-1, 1, 1)), at=ok), dict(q=heads(y_strides=(64, -16, 8)), at=ok),
        dict(q=heads(y_strides=(0, 16, 8)), at=ok), dict(q=heads(y_strides=(64, 0, 8)), at=ok), dict(q=heads(y_strides=(64, 16, 0)), at=ok),
        dict(q=heads(x_strides=(1 << 50, 16, 8)), at=ok), dict(q=heads(), k=heads(y_strides=(64, 16, 0)), at=ok),
        dict(q=heads(), at=positions(32, bits=16)), dict(q=heads(), at=positions(32, strides=(-1, 1))),
        dict(q=heads(), at=positions(32, strides=(0, -1))), dict(q=heads(), at=positions(32, strides=(1 << 50, 1))),
        dict(q=heads(y_strides=(64, 8, 16)), at=ok), dict(q=heads(), at=positions(start=2 ** 53 + 1)),
        dict(q=heads(), at=positions(start=-2 ** 53 - 1)),
        dict(q=heads(x=None), at=ok), dict(q=heads(y=None), at=ok), dict(q=heads(), k=heads(x=None), at=ok), dict(q=heads(), at=ok, freqs=None),
    ]
    for args in refused:
        assert rotary(way=way, **args) == INVALID, args
    for args in (dict(q=heads(x=34), at=ok), dict(q=heads(y=33), at=ok, dt=1), dict(q=heads(), k=heads(y=34), at=ok),
                 dict(q=heads(), at=ok, freqs=36), dict(q=heads(), at=positions(36)), dict(q=heads(), at=positions(34, bits=32))):
        assert rotary(way=way, **args) == UNSUPPORTED, args
    for args in (dict(B_=0), dict(S=0)):
        assert rotary(q=heads(x=None, y=None), at=ok, freqs=None, way=way, **args) == 0
    assert rotary(q=heads(x=None, y=None, n=0), at=ok, freqs=None, way=way) == 0
    assert rotary(q=heads(x=None, y=None, n=0), k=heads(x=None, y=None, n=0), at=ok, freqs=None, way=way) == 0


def glu_fwd(x=16, w=16, bias=None, gu=16, h=16, ws=None, size=0, T=2, H=8, F=8, kind=0, dt=0):
    return B.load().tempo_glu_fwd(x, w, bias, gu, h, ws, size, T, H, F, kind, dt, None)


def glu_bwd(dh=16, gu=16, x=16, w=16, dgu=16, h=None, dx=16, dw=16, dbias=None, ws=None, size=0, T=2, H=8, F=8, kind=0, dt=0):
    return B.load().tempo_glu_bwd(dh, gu, x, w, dgu, h, dx, dw, dbias, ws, size, T, H, F, kind, dt, None)


def test_glu_arguments_are_checked_before_any_launch():
    big = 1 << 62
    for call in (glu_fwd, glu_bwd):
        for args in (dict(T=-1), dict(H=-1), dict(F=-1), dict(kind=3), dict(kind=-1), dict(dt=2), dict(T=big), dict(H=big), dict(F=big),
                     dict(T=1 << 21, F=1 << 21), dict(H=1 << 21, F=1 << 20)):
            assert call(**args) == INVALID, args
        for args in (dict(x=8), dict(w=24), dict(gu=8), dict(h=8), dict(ws=8), dict(T=(1 << 30) + 1, H=1, F=1), dict(T=1, H=1, F=(1 << 29) + 1),
                     dict(T=1 << 19, F=1 << 17, H=8)):
            assert call(**args) == UNSUPPORTED, args
    # a workspace that is too small, or none where one is needed
    sizes = dict(T=8, H=4096, F=64, dt=1)
    assert B.load().tempo_glu_fwd_workspace_bytes(8, 4096, 64, 1) > 15
    assert glu_fwd(**sizes) == WORKSPACE and glu_fwd(ws=16, size=15, **sizes) == WORKSPACE
    assert glu_bwd(dbias=16, **sizes) == WORKSPACE and glu_bwd(dbias=16, ws=16, size=15, **sizes) == WORKSPACE
    for args in (dict(x=None), dict(w=None), dict(h=None)):
        assert glu_fwd(**args) == INVALID, args
    for args in (dict(dh=None), dict(gu=None), dict(dgu=None), dict(x=None), dict(w=None)):
        assert glu_bwd(**args) == INVALID, args
    for args in (dict(bias=8),):
        assert glu_fwd(**args) == UNSUPPORTED
    for args in (dict(dh=8), dict(dgu=8), dict(dx=8), dict(dw=8), dict(dbias=8)):
        assert glu_bwd(**args) == UNSUPPORTED


def test_sizes_of_zero_need_no_pointers():
    nothing = dict(x=None, w=None, gu=None, h=None)
    assert glu_fwd(T=0, **nothing) == 0 and glu_fwd(F=0, **nothing) == 0
    back = dict(dh=None, dgu=None, dx=None, dw=None, **nothing)
    assert glu_bwd(T=0, **back) == 0 and glu_bwd(F=0, **back) == 0 and glu_bwd(T=0, H=0, F=0, **back) == 0
    lib = B.load()
    for size in (lib.tempo_glu_fwd_workspace_bytes, lib.tempo_glu_bwd_workspace_bytes):
        assert size(0, 0, 0, 0) == 0 and size(-1, 8, 8, 0) == 0 and size(8, 8, 8, 5) == 0 and size(1 << 40, 1 << 40, 8, 0) == 0


def test_binding_refuses_what_the_rotary_call_would_misread():
    q, k = torch.zeros(2, 3, 4, 8), torch.zeros(2, 3, 1, 8)
    f, p = torch.ones(4, dtype=torch.float64), torch.zeros(2, 3, dtype=torch.int64)

    def refused(match, q=q, k=k, freqs=f, positions=p, q_out=q, k_out=k, layout="half"):
        for call in (B.tempo_rotary_fwd, B.tempo_rotary_bwd):
            with pytest.raises(ValueError, match=match):
                call(q, k, freqs, positions, q_out, k_out, layout)
    refused("float32 or bfloat16", q=q.half())
    refused("freqs must be torch.float64", freqs=f.float())
    refused("layout", layout="quarter")
    refused("CUDA")
    for start in (2 ** 53 + 1, -2 ** 70):
        with pytest.raises(ValueError, match="start"):
            B.tempo_rotary_fwd(q, None, f, None, q, None, "half", 1.0, start)
    refused("q must be", q=q[0])
    refused("q must be", q=q.transpose(2, 3))
    refused("q_out must be", q_out=q[..., ::2])
    refused("q_out must have shape", q_out=q[:1])
    refused("q_out must be torch.float32", q_out=q.bfloat16())
    refused("k must be torch.float32", k=k.bfloat16(), k_out=k.bfloat16())
    refused("k must have the batch", k=k[:, :2], k_out=k[:, :2])
    refused("k must have the batch", k=k[..., :6], k_out=k[..., :6])
    refused("go together", k=None)
    refused("go together", k_out=None)
    refused("freqs must have 1 to 4", freqs=torch.ones(5, dtype=torch.float64))
    refused("freqs must have 1 to 4", freqs=f[:0])
    refused("positions must be int32", positions=p.float())
    refused("positions must be", positions=p[:, :2])
    refused("positions must be", positions=p[:, :, None])
    refused("positions must be", positions=torch.zeros(3, 3, dtype=torch.int64))


def test_binding_refuses_what_the_glu_calls_would_misread():
    x, w, b = torch.zeros(5, 8), torch.zeros(12, 8), torch.zeros(12)
    gu, h = torch.zeros(5, 12), torch.zeros(5, 6)

    def refused(match, x=x, w=w, bias=b, gu=gu, h=h, kind="silu"):
        with pytest.raises(ValueError, match=match):
            B.tempo_glu_fwd(x, w, bias, gu, h, kind)
    refused("float32 or bfloat16", x=x.half())
    refused("kind", kind="relu")
    refused("w must be", w=w[:11])
    refused("w must be", w=w.flatten())
    refused("x must be", x=x[:, :7])
    refused("w must be torch.float32", w=w.bfloat16())
    refused("bias must be torch.float32", bias=b.double())
    refused("bias must have 12", bias=b[:6])
    refused("gu must have 60", gu=gu[:4])
    refused("h must be", h=h.bfloat16())
    refused("h must have 30", h=gu)
    refused("CUDA")

    def back_refused(match, **other):
        args = dict(dh=h, gu=gu, x=x, w=w, dgu=gu, h=h, dx=x, dw=w, dbias=b, kind="silu") | other
        with pytest.raises(ValueError, match=match):
            B.tempo_glu_bwd(**args)
    back_refused("kind", kind="gelu")
    back_refused("dh must have 30", dh=gu)
    back_refused("dgu must have 60", dgu=h)
    back_refused("dx must be torch.float32", dx=x.bfloat16())
    back_refused("dw must have 96", dw=w[:6])
    back_refused("dbias must have 12", dbias=b[:6])
    back_refused("x must be torch.float32", x=x.bfloat16())
    back_refused("CUDA")
