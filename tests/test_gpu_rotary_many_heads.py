"""Rotary positions of as many tokens as make a lane take several heads, below and above the size from which what is written is not
kept in a cache: heads that are no multiple of a lane's, lanes whose heads are of q and of k, workgroups that are no multiple of 8.

The limits of csrc/rotary.hip are restated here, so that each case is where it is meant to be (what is written is not kept in a cache at
heads of 128 and 160, of neighbours at 64 and of 64 in float32 too); tolerance: test_gpu_rotary's."""
import pytest
import torch

from paper_2210_10246_amd import binding as B
from test_gpu_rotary import DT, check, freqs_of, normal

pytestmark = pytest.mark.gpu


def pieces_of(tokens, heads, D, half, layout, dtype, in_place=False):
    """16-byte pieces (two of them in the half layout) that lanes own, and the workgroups they make at several heads a lane."""
    V = 4 if dtype == "f32" else 8
    pairs = V if layout == "half" else V // 2
    units = -(-half // pairs) + (0 if in_place else -(-(D - 2 * half) // V))
    per_lane = 4 if layout == "half" else 8
    at_once = min(256 // min(units, 256), tokens)
    return tokens * units * heads, -(-tokens // at_once) * -(-heads // per_lane) * -(-units // 256)


def tokens_for(streamed, heads, D, half, layout, dtype):
    """The fewest tokens [3, S] of several heads a lane, below and above the streaming limit, in workgroups that are no multiple of 8.
    In place there may be fewer pieces: of several heads a lane there too."""
    cus = torch.cuda.get_device_properties(0).multi_processor_count
    several = cus * 8192 // ((4 if dtype == "f32" else 8) // (1 if layout == "half" else 2))
    stream = (48 << 20) // (32 if layout == "half" else 16)
    S = 1
    while True:
        pieces, blocks = pieces_of(3 * S, heads, D, half, layout, dtype)
        least, _ = pieces_of(3 * S, heads, D, half, layout, dtype, True)
        if least >= several and (pieces > stream) == streamed and blocks % 8 and S % 2:
            return S
        assert streamed or pieces <= stream
        S += 1


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("layout", ["half", "interleaved"])
@pytest.mark.parametrize("streamed", [False, True])
@pytest.mark.parametrize("A,K,D,half", [(9, 4, 83, 33), (9, 4, 64, 32), (5, 2, 40, 19), (11, 0, 18, 9), (9, 4, 128, 64),
                                         (5, 2, 160, 64)])
def test_several_heads_a_lane(A, K, D, half, streamed, layout, dtype):
    S = tokens_for(streamed, A + K, D, half, layout, dtype)
    freqs = freqs_of(half)
    positions = torch.randint(0, 5000, (3, S), device="cuda")
    qkv = normal(3, S, A + K + 1, D, dtype=dtype)      # a projection: q and k out of it, and by head
    q, k = qkv[:, :, :A], qkv[:, :, A:A + K] if K else None
    for call, back in ((B.tempo_rotary_fwd, False), (B.tempo_rotary_bwd, True)):
        out = [None if t is None else torch.full((3, t.shape[2], S, D), float("nan"), device="cuda", dtype=DT[dtype]).transpose(1, 2)
               for t in (q, k)]
        call(q, k, freqs, positions, *out, layout, 1.25)
        for x, y in zip((q, k), out):
            if x is not None:
                check(y, x, positions, freqs, layout, 1.25, back)
    place = qkv.clone()
    sides = [place[:, :, :A], place[:, :, A:A + K] if K else None]
    B.tempo_rotary_bwd(*sides, freqs, positions, *sides, layout, 1.25)
    assert all(x is None or torch.equal(x, y) for x, y in zip(sides, out)) and torch.equal(place[:, :, A + K:], qkv[:, :, A + K:])


@pytest.mark.parametrize("layout", ["half", "interleaved"])
def test_one_of_both_in_place(layout):
    """q in its own place and k elsewhere, and the other way round, of several heads a lane and of one."""
    for S in (tokens_for(False, 13, 83, 33, layout, "bf16"), 5):
        freqs, positions = freqs_of(33), torch.arange(S, device="cuda")
        q, k = normal(3, S, 9, 83, dtype="bf16"), normal(3, S, 4, 83, dtype="bf16", seed=1)
        want = [torch.empty_like(q), torch.empty_like(k)]
        B.tempo_rotary_fwd(q, k, freqs, positions, *want, layout)
        for i in range(2):
            sides, out = [q.clone(), k.clone()], [torch.empty_like(q), torch.empty_like(k)]
            out[i] = sides[i]
            B.tempo_rotary_fwd(*sides, freqs, positions, *out, layout)
            assert torch.equal(out[0], want[0]) and torch.equal(out[1], want[1])
