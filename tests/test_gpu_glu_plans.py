"""The gated unit with every tile that its calls can take, at sizes that fill none of them: outputs, what lies behind them, and the same
bits whichever gradients are wanted.  Which tile a size takes is checked without a GPU in test_glu_plan.py; tolerances: test_gpu_glu's."""
import pytest
import torch

from paper_2210_10246_amd import binding as B
from test_gpu_glu import DT, both_ways, inputs, normal

pytestmark = pytest.mark.gpu

# T, H, F, type, forward, backward on 256 compute units.  R: any type and address, A: whole pieces, P: copied to whole pieces; the tile's
# edge (few rows: columns); +: a sum in parts (of the backward: dx, dw).
CASES = [
    (8190, 1016, 4092, "bf16", "A256", "A256"),
    (8190, 1023, 4095, "bf16", "P256", "P256"),
    (2050, 4088, 4100, "bf16", "A128", "A256"),
    (5277, 1760, 8, "bf16", "A64+", "A256 dw+"),
    (300, 4000, 5004, "bf16", "A128", "A256 dx+"),
    (6503, 144, 6716, "bf16", "A256", "A256 dx+ dw+"),
    (338, 3976, 4893, "bf16", "A128", "P256 dx+"),
    (436, 4648, 188, "bf16", "A64+", "A128"),
    (246, 632, 3392, "bf16", "A64", "A128 dx+"),
    (4474, 416, 300, "bf16", "A64", "A128 dw+"),
    (7777, 8, 2752, "bf16", "A256", "A128 dx+ dw+"),
    (1259, 3648, 1714, "bf16", "A128", "P128"),
    (270, 4453, 321, "bf16", "R64+", "R128"),
    (386, 4433, 846, "bf16", "R128+", "R128"),
    (5298, 5640, 172, "bf16", "A128+", "A128"),
    (6907, 1850, 3586, "bf16", "P128", "P256"),
    (2788, 10, 2891, "bf16", "R128", "R128 dx+ dw+"),
    (840, 8, 16, "bf16", "A64", "A64 dw+"),
    (1467, 8, 272, "bf16", "A64", "A64 dx+ dw+"),
    (416, 10, 557, "bf16", "R64", "R64 dx+ dw+"),
    (43, 2840, 11012, "bf16", "few 128", "A256 dx+"),
    (13, 520, 2052, "bf16", "few 16", "A64 dx+"),
    (50, 520, 2052, "bf16", "few 64", "A64 dx+"),
    (6567, 13, 4176, "bf16", "R128", "P64"),
    (1801, 1003, 13, "bf16", "R64+", "R64 dw+"),
    (753, 2520, 344, "f32", "R64+", "R128"),
    (1682, 2576, 100, "f32", "R128+", "R64"),
    (2170, 67, 820, "f32", "R64", "R128 dx+ dw+"),
    (126, 1856, 2924, "f32", "R64", "R128 dx+"),
    (7925, 16, 512, "f32", "R128", "R64 dw+"),
    (680, 15, 2049, "f32", "R64", "R64 dx+ dw+"),
]


@pytest.mark.parametrize("T,H,F,dtype", [c[:4] for c in CASES])
def test_every_tile_both_ways(T, H, F, dtype):
    both_ways(T, H, F, dtype, "silu", True)


@pytest.mark.parametrize("T,H,F,dtype", [c[:4] for c in CASES])
def test_left_out_gradients_leave_the_others(T, H, F, dtype):
    x, w, b = inputs(T, H, F, dtype)
    gu, dh = normal(T, 2 * F, dtype=dtype, seed=5), normal(T, F, dtype=dtype, seed=6)
    like = (torch.empty_like(gu), torch.empty_like(dh), torch.empty_like(x), torch.empty_like(w), torch.empty_like(b))
    B.tempo_glu_bwd(dh, gu, x, w, *like)
    for left in ((1,), (2,), (3,), (4,), (2, 3), (1, 4)):
        outs = [None if i in left else torch.empty_like(t) for i, t in enumerate(like)]
        B.tempo_glu_bwd(dh, gu, x, w, *outs)
        assert all(a is None or torch.equal(a, c) for a, c in zip(outs, like)), left
    assert x.dtype == DT[dtype]
