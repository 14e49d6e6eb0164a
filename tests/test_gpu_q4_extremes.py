"""4-bit KV cache at the ends of its range, against the fp64 oracle."""
import numpy as np
import pytest
import torch

import oracle
from oracle import q4
from test_gpu_q4 import P, attend, check_attention, random_cache

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def bf16_of(x):
    return int(oracle.f32_to_bf16_bits(np.array([x], np.float32))[0])


@pytest.mark.parametrize("Hq,d", [(4, 128), (8, 128), (4, 64), (8, 64)])
@pytest.mark.parametrize("first_scale", [0.0, 2.0 ** -90])
@pytest.mark.parametrize("value", [1e3, 2.0 ** 26, -2.0 ** 31, 1e20, -2.0 ** 99])
def test_constant_rows_after_rows_of_tiny_scale(Hq, d, first_scale, value):
    """64 tokens with V = 0 (or tiny scales), then 64 whose V rows are constant (scale 0, all in the minimum) and whose logits
    are lower by three log2 units; then the other way round."""
    import paper_2609_35158_b200 as pd

    lens = np.array([128], np.int32)
    kv4, table, NP = random_cache(lens, 1, d, 200)
    scale = 0.125
    low = -3 * np.log(2) / (scale * d)                      # K = low everywhere with q = 1: a logit of -3 ln 2
    for t in range(128):
        rec = kv4[table[0, t // P], 0, 16 * d:].view(np.uint16).reshape(P, d // 64, 4)
        rec[t % P] = [0, 0, bf16_of(first_scale), 0] if t < 64 else [0, bf16_of(low), 0, bf16_of(value)]
    q = torch.ones((1, Hq, d), dtype=torch.bfloat16)
    for order in (np.arange(8), np.r_[4:8, 0:4], np.array([0, 4, 1, 5, 2, 6, 3, 7])):
        tab = table[:, order].copy()
        ref = q4.decode_attn(oracle.bf16_bits(q), kv4, tab, lens, scale)
        for split in (100000, 8, 3, 0):
            out, lse = attend(pd, Hq, 1, d, q.to(DEV), kv4, tab, lens, NP, scale, split)
            check_attention(out, lse, ref, f"order {order.tolist()} split {split}")
