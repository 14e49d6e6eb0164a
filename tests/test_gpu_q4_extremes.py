"""4-bit KV cache at the ends of its range, against the fp64 oracle."""
import numpy as np
import pytest
import torch

import oracle
from oracle import q4
import workloads as wl
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


def test_a_key_group_with_a_nan_reaches_every_row_of_its_kv_head_only():
    """A NaN in K makes the logit NaN, and with it the softmax of every query head that reads that KV head."""
    import paper_2609_35158_b200 as pd

    for Hq, d in ((8, 128), (16, 64)):
        Hkv, G = 2, Hq // 2
        lens = np.array([40, 700], np.int32)
        kv4, table, NP = random_cache(lens, Hkv, d, 220)
        q = wl.random_bf16((2, Hq, d), 221, "cpu")
        ref = q4.decode_attn(oracle.bf16_bits(q), kv4, table, lens, 0.1)
        bad = kv4.copy()
        bad[table[1, 1], 1, 16 * d:].view(np.uint16).reshape(P, d // 64, 4)[3, 0, :2] = [0x7FC0, 0]
        for split in (0, 1, 100000):
            out, lse = attend(pd, Hq, Hkv, d, q.to(DEV), bad, table, lens, NP, 0.1, split)
            assert torch.isnan(out[1, G:].float()).all() and torch.isnan(lse[1, G:]).all()
            for sel in ((0, slice(None)), (1, slice(0, G))):
                check_attention(out[sel], lse[sel], [x[sel] for x in ref], f"{Hq} {d} split {split}")


@pytest.mark.parametrize("gain", [2.0 ** 95, 2.0 ** -90])
@pytest.mark.parametrize("Hq,d", [(8, 128), (16, 64)])
def test_attention_at_the_documented_ends_of_q_and_v(gain, Hq, d):
    """q and V some binades below 2^100 and as far down, over a K that leaves the logits as they are."""
    import paper_2609_35158_b200 as pd

    lens = np.array([40, 900, 1], np.int32)
    kv4, table, NP = random_cache(lens, 2, d, 230, scale_k=0.3 / gain, scale_v=0.3 * gain)
    q = (wl.random_bf16((3, Hq, d), 231, "cpu").float() * gain).to(torch.bfloat16)
    ref = q4.decode_attn(oracle.bf16_bits(q), kv4, table, lens, 0.1)
    for split in (0, 1, 100000):
        out, lse = attend(pd, Hq, 2, d, q.to(DEV), kv4, table, lens, NP, 0.1, split)
        check_attention(out, lse, ref, f"gain {gain} split {split}")


@pytest.mark.parametrize("small", [0, 1])
@pytest.mark.parametrize("Hq", [4, 8])
def test_the_smaller_of_two_v_groups_keeps_its_accuracy(Hq, small):
    """V groups of one head that differ by 2^8. Beside the usual bound, a weight may be off by half of fp16's smallest step,
    2^-25, where the head's largest is at least 2^2, times a code of up to 15."""
    import paper_2609_35158_b200 as pd

    d, lens = 128, np.array([1500, 33], np.int32)
    kv4, table, NP = random_cache(lens, 1, d, 240, poison=False)
    rec = kv4[..., 16 * d:].view(np.uint16).reshape(NP, 1, P, 2, 4)
    rec[..., small, 2:] = oracle.f32_to_bf16_bits((oracle.bf16_bits_to_f64(rec[..., small, 2:]) / 256).astype(np.float32))
    q = wl.random_bf16((2, Hq, d), 241, "cpu")
    out_, lse_, tol, tol_lse = q4.decode_attn(oracle.bf16_bits(q), kv4, table, lens, 0.1)
    for b in range(2):
        k, _, steps = q4.sequence_values(kv4, table, b, int(lens[b]), 0, d)
        z = np.float64(np.float32(0.1)) * (k @ oracle.bf16_bits_to_f64(oracle.bf16_bits(q[b])).T)     # [n, Hq]
        largest = (np.exp(z - z.max(0)) / np.exp(z - z.max(0)).sum(0) * (steps[0].max(1) / 15)[:, None]).max(0)
        tol[b] += (lens[b] * 15 * 2.0 ** -27 * largest)[:, None]
    assert np.abs(out_[0][:, 64 * small:64 * small + 64]).max() < 0.1 * np.abs(out_[0]).max()
    for split in (0, 7, 100000):
        out, lse = attend(pd, Hq, 1, d, q.to(DEV), kv4, table, lens, NP, 0.1, split)
        check_attention(out, lse, (out_, lse_, tol, tol_lse), f"split {split}")


def ragged_case(seed):
    """(Hq, Hkv, d, lengths, split_pages): every sequence draws its own length, empty ones and thousands of tokens among them."""
    rng = np.random.default_rng(2000 + seed)
    d, Hkv = [64, 128][seed % 2], int(rng.choice([1, 2, 3]))
    n = int(rng.integers(3, 9))
    lens = np.where(rng.random(n) < 0.2, 0, np.exp(rng.uniform(0, 8.6, n)) + rng.integers(0, 17, n)).astype(np.int32)
    lens[rng.integers(0, n)] = int(rng.integers(2500, 6000))
    return Hkv * [1, 2, 4, 8][(seed // 2) % 4], Hkv, d, lens, int(rng.choice([0, 0, 2, 7]))


@pytest.mark.parametrize("seed", range(12))
def test_ragged_random_batches(seed):
    import paper_2609_35158_b200 as pd

    Hq, Hkv, d, lens, split = ragged_case(seed)
    assert len(set(lens.tolist())) > 1 and lens.max() >= 2500
    rng = np.random.default_rng(2100 + seed)
    kv4, table, NP = random_cache(lens, Hkv, d, 2200 + seed, scale_k=float(10 ** rng.uniform(-3, 0.5)), scale_v=float(10 ** rng.uniform(-3, 3)))
    q = wl.random_bf16((len(lens), Hq, d), 2300 + seed, "cpu")
    scale = float(rng.uniform(0.02, 0.3))
    ref = q4.decode_attn(oracle.bf16_bits(q), kv4, table, lens, scale)
    out, lse = attend(pd, Hq, Hkv, d, q.to(DEV), kv4, table, lens, NP, scale, split)
    check_attention(out, lse, ref, f"seed {seed}: {Hq}/{Hkv} d={d} {lens.tolist()}")


def test_ragged_cases_are_ragged():
    cases = [ragged_case(s) for s in range(12)]
    assert sum((c[3] == 0).any() for c in cases) >= 3 and {(c[0] // c[1], c[2]) for c in cases} >= {(g, d) for g in (1, 2, 4, 8) for d in (64, 128)}
