"""4-bit KV cache at the ends of its range, against the fp64 oracle."""
import numpy as np
import pytest
import torch

import oracle
from oracle import q4
from pd_testlib import Ctx
from test_gpu_q4 import P, attend, bf16_dev, check_attention, dev, random_cache, table_for

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


@pytest.mark.parametrize("d", [128, 64])
def test_groups_next_to_the_largest_value_read_back_finite(d):
    """The scale of such a group is rounded so that no value leaves bf16; everything is within scale / 2 of its input."""
    import paper_2609_35158_b200 as pd

    n = 64
    rng = np.random.default_rng(210)
    x = np.zeros((n, 1, d), np.uint16)
    x[0, 0, :3] = [0x7F7F, bf16_of(-0.5 * 2.0 ** 120), 0]
    x[1, 0, :2] = [0x7F7F, 0x0000]
    x[2, 0, :] = 0x7F7F
    x[3, 0, :] = rng.integers(0x7F00, 0x7F80, d)
    x[4, 0, :2] = [0xFF7F, 0x0000]                                      # the smallest value is exact: nothing to round
    for t in range(5, n):                                               # ranges up to fp32's end around the largest values
        x[t, 0] = rng.integers(0x7C00, 0x7F80, d)
        x[t, 0, rng.integers(0, d, d // 4)] = 0
        x[t, 0, rng.integers(0, d, 2)] = [0x7F7F, bf16_of(-2.0 ** float(rng.uniform(60, 119)))]
    table, NP = table_for([n], 211)
    want = np.zeros((NP, 1, 18 * d), np.uint8)
    q4.append_tokens(x, x, np.array([0, n]), want, table, np.zeros(1, np.int32))
    kv4 = torch.zeros((NP, 1, 18 * d), dtype=torch.uint8, device=DEV)
    kp, vp = (torch.zeros((NP, 1, P, d), dtype=torch.bfloat16, device=DEV) for _ in range(2))
    with Ctx(1, 1, d, 1, table.shape[1], NP) as ctx:
        L, t = dev(np.zeros(1, np.int32)), dev(table)
        pd.pd_kv_append_tokens_q4(ctx.h, bf16_dev(x), bf16_dev(x), dev(np.array([0, n], np.int32)), kv4, t, L, n)
        pd.pd_kv_dequantize_q4(ctx.h, kv4, t, None, L, kp, vp, t)
        torch.cuda.synchronize()
    back = kp.float().cpu().numpy().astype(np.float64)[table[0, np.arange(n) // P], 0, np.arange(n) % P]
    given = oracle.bf16_bits_to_f64(x[:, 0])
    assert np.isfinite(back).all()
    assert np.array_equal(kv4.cpu().numpy(), want) and torch.equal(kp, vp)
    step = np.repeat(np.stack([oracle.bf16_bits_to_f64(kv4.cpu().numpy()[table[0, i // P], 0, 16 * d:].view(np.uint16).reshape(P, d // 64, 4)[i % P, :, 0])
                               for i in range(n)]), 64, -1)
    # half a step of the code, and the rounding of the value read back to bf16
    assert np.all(np.abs(back - given) <= step / 2 * (1 + 2.0 ** -20) + 2.0 ** -8 * np.abs(back))
