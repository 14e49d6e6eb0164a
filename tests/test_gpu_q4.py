"""GPU parity of the 4-bit KV cache through the C ABI against the fp64 oracle: writing is bit-exact over whole pools,
reading back too, attention is within the bounds the oracle derives beside its result (one bf16 rounding, fp16 weights,
fp32 sums) on the same cache."""
import numpy as np
import pytest
import torch

import oracle
from oracle import q4
import workloads as wl
from pd_testlib import Ctx

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
P = 16


def dev(a):
    return torch.from_numpy(np.ascontiguousarray(a)).to(DEV)


def bf16_dev(bits):
    return torch.from_numpy(np.ascontiguousarray(bits).view(np.int16)).to(DEV).view(torch.bfloat16)


def table_for(lens, seed, slack=3, cols=None):
    """Scattered pages; unused entries are -1. (table [B, MP], pages in the pool)."""
    need = (np.asarray(lens) + P - 1) // P
    NP = int(need.sum()) + slack
    perm = np.random.default_rng(seed).permutation(NP)
    table = np.full((len(lens), max(1, int(need.max())) if cols is None else cols), -1, np.int32)
    at = 0
    for b, n in enumerate(need):
        table[b, :n] = perm[at:at + n]
        at += n
    return table, NP


def random_cache(lens, Hkv, d, seed, scale_k=0.3, scale_v=0.3, poison=True):
    """Blocks of random codes, log-normal scales and minima around -7.5 scales; empty slots and pages hold NaN records."""
    rng = np.random.default_rng(seed)
    table, NP = table_for(lens, seed + 1)
    kv4 = rng.integers(0, 256, (NP, Hkv, 18 * d)).astype(np.uint8)
    s = np.exp(0.5 * rng.standard_normal((NP, Hkv, P, d // 64, 2))) * np.array([scale_k, scale_v])
    rec = np.stack([s[..., 0], -7.5 * s[..., 0] * rng.uniform(0.5, 1.5, s.shape[:-1]), s[..., 1],
                    -7.5 * s[..., 1] * rng.uniform(0.5, 1.5, s.shape[:-1])], -1)
    rec = oracle.f32_to_bf16_bits(rec.astype(np.float32))
    if poison:
        used = np.zeros((NP, P), bool)
        for b, L in enumerate(lens):
            for t in range(int(L)):
                used[table[b, t // P], t % P] = True
        rec[~np.broadcast_to(used[:, None], (NP, Hkv, P))] = 0xFFFF
    kv4[..., 16 * d:] = rec.reshape(NP, Hkv, -1).view(np.uint8)
    return kv4, table, NP


def check_attention(out, lse, ref, what=""):
    want, want_lse, tol, tol_lse = ref
    got = out.float().cpu().numpy().astype(np.float64)
    assert np.isfinite(got).all(), what
    over = np.abs(got - want) - tol
    assert over.max() <= 0, f"{what}: {over.max()} past the bound at {np.unravel_index(over.argmax(), over.shape)}"
    if lse is not None:
        got = lse.cpu().numpy().astype(np.float64)
        live = np.isfinite(want_lse)
        assert np.array_equal(np.isneginf(got), ~live), what
        assert np.all(np.abs(got[live] - want_lse[live]) <= tol_lse[live]), what


def attend(pd, Hq, Hkv, d, q, kv4, table, lens, NP, scale, split_pages=0, want_lse=True):
    B = len(lens)
    out = torch.full((B, Hq, d), float("nan"), dtype=torch.bfloat16, device=DEV)
    lse = torch.full((B, Hq), float("nan"), dtype=torch.float32, device=DEV) if want_lse else None
    with Ctx(Hq, Hkv, d, B, table.shape[1], NP) as ctx:
        pd.pd_decode_attn_q4(ctx.h, q, dev(kv4), dev(table), dev(lens), out, lse, sm_scale=scale, split_pages=split_pages)
        torch.cuda.synchronize()
        assert pd.pd_device_status(ctx.h)[0] == 0
    return out, lse


@pytest.mark.parametrize("d", [128, 64])
def test_append_tokens_is_bit_exact(d):
    import paper_2609_35158_b200 as pd

    Hkv = 2
    before = np.array([0, 5, 16, 31, 40, 0, 7], np.int32)
    new = np.array([1, 30, 16, 0, 3, 50, 9], np.int32)
    rng = np.random.default_rng(10)
    table, NP = table_for(before + new, 11)
    total = int(new.sum())
    indptr = np.concatenate([[0], np.cumsum(new)]).astype(np.int32)
    k = (rng.standard_normal((total, Hkv, d)) * 10.0 ** rng.integers(-6, 6, (total, Hkv, 1))).astype(np.float32)
    v = np.rint(rng.standard_normal((total, Hkv, d)) * 20).astype(np.float32)  # small integers: many exact ties
    k, v = oracle.f32_to_bf16_bits(k), oracle.f32_to_bf16_bits(v)
    k[3, 0, :] = 0                          # all zero
    k[4, 0, :] = 0x4049                     # all equal
    k[5, 0, 7] = 0x7FC0                     # NaN: its group only
    k[6, 1, d - 1] = 0x7F80                 # inf
    k[7, 0, :2] = [0x7F7F, 0xFF7F]          # the range leaves fp32
    k[8, 0, :4] = [0x7E80, 0xFE80, 0x7000, 0x6F81]  # range 1.7e38: the scale is above 2^64
    k[9, 0, :] = rng.integers(0, 128, d)    # subnormals count as zero
    k[10, 0, :] = 0x8000                    # -0
    k[11, 0, :] = oracle.f32_to_bf16_bits((rng.standard_normal(d) * 1e-31).astype(np.float32))  # scale below 2^-100
    k[12, 0, :] = oracle.f32_to_bf16_bits((1.0 + 2.0 ** -7 * rng.integers(0, 3, d)).astype(np.float32))
    want = np.full((NP, Hkv, 18 * d), 0x55, np.uint8)
    lens = q4.append_tokens(k, v, indptr, want, table, before)
    kv4 = torch.full((NP, Hkv, 18 * d), 0x55, dtype=torch.uint8, device=DEV)
    with Ctx(Hkv, Hkv, d, len(new), table.shape[1], NP) as ctx:
        L = dev(before)
        pd.pd_kv_append_tokens_q4(ctx.h, bf16_dev(k), bf16_dev(v), dev(indptr), kv4, dev(table), L, int(new.max()),
                                  call_flags=pd.PD_APPEND_NO_ADVANCE)
        torch.cuda.synchronize()
        assert pd.pd_device_status(ctx.h)[0] == 0
        assert np.array_equal(kv4.cpu().numpy(), want)
        assert np.array_equal(L.cpu().numpy(), before)
        kv4.fill_(0x55)
        n0 = pd.pd_launch_count(ctx.h)
        pd.pd_kv_append_tokens_q4(ctx.h, bf16_dev(k), bf16_dev(v), dev(indptr), kv4, dev(table), L, 64)  # a loose bound
        torch.cuda.synchronize()
        assert pd.pd_launch_count(ctx.h) == n0 + 2
        assert np.array_equal(kv4.cpu().numpy(), want)
        assert np.array_equal(L.cpu().numpy(), lens)


def test_many_random_rows_quantise_to_the_exact_code():
    """4096 rows across 200 binades, ties included: the codes of the two-part reciprocal are those of exact division."""
    import paper_2609_35158_b200 as pd

    d, n = 128, 4096
    rng = np.random.default_rng(20)
    x = rng.standard_normal((n, 1, d)) * 2.0 ** rng.integers(-90, 90, (n, 1, 1))
    x[::3] = np.rint(x[::3] / 2.0 ** np.floor(np.log2(np.abs(x[::3]).max(-1, keepdims=True))) * rng.integers(1, 90, (len(x[::3]), 1, 1)))
    x[1::3] += rng.integers(-4, 4, x[1::3].shape[:-1] + (1,)) * np.abs(x[1::3]).max(-1, keepdims=True)
    k = oracle.f32_to_bf16_bits(x.astype(np.float32))
    table, NP = table_for([n], 21)
    kv4 = torch.zeros((NP, 1, 18 * d), dtype=torch.uint8, device=DEV)
    with Ctx(1, 1, d, 1, table.shape[1], NP) as ctx:
        kd = bf16_dev(k)
        pd.pd_kv_append_tokens_q4(ctx.h, kd, kd, dev(np.array([0, n], np.int32)), kv4, dev(table), dev(np.array([0], np.int32)), n)
        torch.cuda.synchronize()
    # the oracle's quantiser, all groups at once
    v = oracle.bf16_bits_to_f64(k).reshape(n, d // 64, 64)
    lo = v.min(-1)
    s = (np.float32(v.max(-1) - lo).astype(np.float64) / 15).astype(np.float32)
    s = oracle.bf16_bits_to_f64(((s.view(np.uint32).astype(np.uint64) + 0xFFFF) >> 16).astype(np.uint16))
    codes = np.rint((v - lo[..., None]).astype(np.float32).astype(np.float64) / s[..., None])
    got, _, _ = q4.sequence_values(kv4.cpu().numpy(), table, 0, n, 0, d)
    assert np.array_equal(got.reshape(v.shape), codes * s[..., None] + lo[..., None])


@pytest.mark.parametrize("d,Hkv", [(128, 8), (64, 3), (128, 1)])
def test_one_token_append_is_bit_exact_and_advances(d, Hkv):
    import paper_2609_35158_b200 as pd

    before = np.array([0, 1, 15, 16, 31, 100], np.int32)
    B, steps = len(before), 3
    rng = np.random.default_rng(30)
    table, NP = table_for(before + steps, 31)
    want = np.full((NP, Hkv, 18 * d), 0xAA, np.uint8)
    kv4 = torch.full((NP, Hkv, 18 * d), 0xAA, dtype=torch.uint8, device=DEV)
    lens = before
    with Ctx(Hkv, Hkv, d, B, table.shape[1], NP) as ctx:
        L = dev(before)
        for _ in range(steps):
            k, v = (oracle.f32_to_bf16_bits(rng.standard_normal((B, Hkv, d)).astype(np.float32)) for _ in range(2))
            lens = q4.append_tokens(k, v, np.arange(B + 1), want, table, lens)
            pd.pd_kv_append_q4(ctx.h, bf16_dev(k), bf16_dev(v), kv4, dev(table), L, call_flags=pd.PD_APPEND_NO_ADVANCE)
            pd.pd_kv_append_q4(ctx.h, bf16_dev(k), bf16_dev(v), kv4, dev(table), L)
        torch.cuda.synchronize()
        assert pd.pd_device_status(ctx.h)[0] == 0
    assert np.array_equal(kv4.cpu().numpy(), want)
    assert np.array_equal(L.cpu().numpy(), lens)


def test_append_errors_are_reported_and_skipped():
    import paper_2609_35158_b200 as pd

    d, Hkv = 128, 2
    table = np.array([[0, 1], [2, 99], [3, -1], [4, 5]], np.int32)
    before = np.array([31, 16, 17, 3], np.int32)       # full after one; bad page; bad page; fine
    kn = wl.random_bf16((8, Hkv, d), 40, DEV)
    indptr = dev(np.array([0, 2, 4, 6, 8], np.int32))
    with Ctx(Hkv, Hkv, d, 4, 2, 6) as ctx:
        for single in (False, True):
            kv4 = torch.zeros((6, Hkv, 18 * d), dtype=torch.uint8, device=DEV)
            L = dev(before)
            if single:
                pd.pd_kv_append_q4(ctx.h, kn[:4], kn[4:], kv4, dev(table), L)
            else:
                pd.pd_kv_append_tokens_q4(ctx.h, kn, kn, indptr, kv4, dev(table), L, 2)
            code, seq, detail = pd.pd_device_status(ctx.h)
            assert code == pd.PD_ERR_DEVICE_FAULT and seq in ((1, 2) if single else (0, 1, 2))
            assert L.cpu().tolist() == ([32, 16, 17, 4] if single else [31, 18, 19, 5])
            touched = kv4.flatten(1).any(1).cpu().tolist()
            assert touched == [False, single, False, False, True, False]
            assert pd.pd_device_status(ctx.h)[0] == 0  # cleared


@pytest.mark.parametrize("d", [128, 64])
def test_reading_back_is_exact_and_leaves_other_slots(d):
    import paper_2609_35158_b200 as pd

    Hkv = 3
    lens = np.array([0, 1, 16, 17, 50, 64, 200], np.int32)
    first = np.array([0, 0, 3, 16, 33, 64, 5], np.int32)
    kv4, table, NP = random_cache(lens, Hkv, d, 50)
    dst, _ = table_for(lens, 52)
    for f in (None, first):
        want = np.full((2, NP, Hkv, P, d), 0x1234, np.uint16)
        for b, L in enumerate(lens):
            for h in range(Hkv):
                k, v, _ = q4.sequence_values(kv4, table, b, int(L), h, d)
                for t in range(0 if f is None else int(f[b]), int(L)):
                    for i, x in enumerate((k, v)):
                        # the product is exact in fp32, the sum is rounded to fp32 and then to bf16
                        want[i, dst[b, t // P], h, t % P] = oracle.f32_to_bf16_bits(x[t].astype(np.float32))
        kp = bf16_dev(np.full((NP, Hkv, P, d), 0x1234, np.uint16))
        vp = kp.clone()
        with Ctx(Hkv, Hkv, d, len(lens), table.shape[1], NP) as ctx:
            pd.pd_kv_dequantize_q4(ctx.h, dev(kv4), dev(table), None if f is None else dev(f), dev(lens), kp, vp, dev(dst))
            torch.cuda.synchronize()
            assert pd.pd_device_status(ctx.h)[0] == 0
        assert np.array_equal(oracle.bf16_bits(kp), want[0]) and np.array_equal(oracle.bf16_bits(vp), want[1])


def test_reading_back_reports_bad_pages_and_lengths():
    import paper_2609_35158_b200 as pd

    d, Hkv, NP = 64, 1, 6
    lens = np.array([20, 33, 8], np.int32)             # the second is past its table row of two pages
    kv4 = np.zeros((NP, Hkv, 18 * d), np.uint8)
    kv4[..., 16 * d:] = np.tile(oracle.f32_to_bf16_bits(np.array([1, 2, 1, 2], np.float32)).view(np.uint8), 32 * d // 64 // 2)
    src = dev(np.array([[0, 77], [1, 2], [3, -1]], np.int32))
    dst = dev(np.array([[0, 1], [2, 3], [-5, 0]], np.int32))
    kp = torch.zeros((NP, Hkv, P, d), dtype=torch.bfloat16, device=DEV)
    vp = torch.zeros_like(kp)
    with Ctx(Hkv, Hkv, d, 3, 2, NP) as ctx:
        pd.pd_kv_dequantize_q4(ctx.h, dev(kv4), src, None, dev(lens), kp, vp, dst)
        assert pd.pd_device_status(ctx.h)[0] == pd.PD_ERR_DEVICE_FAULT
        assert kp[:, 0, 0, 0].tolist() == [2.0, 0, 0, 0, 0, 0] and (vp[0] == 2).all()
        pd.pd_kv_dequantize_q4(ctx.h, dev(kv4), dev(np.zeros((3, 2), np.int32)), dev(np.array([-1, 40, 9], np.int32)),
                               dev(np.array([20, 32, 8], np.int32)), kp, vp, dev(np.full((3, 2), 5, np.int32)))
        assert pd.pd_device_status(ctx.h) == (pd.PD_ERR_DEVICE_FAULT, 0, -1)
        assert (kp[5] == 0).all()                      # nothing lies between first_token and the length


GEOMS = [(32, 8), (32, 4), (8, 8), (4, 2), (16, 2), (1, 1)]


@pytest.mark.parametrize("split_pages", [0, 1, 3, 100000])
@pytest.mark.parametrize("d", [128, 64])
@pytest.mark.parametrize("Hq,Hkv", GEOMS)
def test_attention_small_ragged_poisoned(Hq, Hkv, d, split_pages):
    import paper_2609_35158_b200 as pd

    lens = np.array([1, 15, 16, 17, 31, 33, 64, 300, 0, 801], np.int32)
    kv4, table, NP = random_cache(lens, Hkv, d, 60 + Hq)
    q = wl.random_bf16((len(lens), Hq, d), 61, "cpu")
    scale = d ** -0.5
    ref = q4.decode_attn(oracle.bf16_bits(q), kv4, table, lens, scale)
    out, lse = attend(pd, Hq, Hkv, d, q.to(DEV), kv4, table, lens, NP, scale, split_pages)
    check_attention(out, lse, ref, f"{Hq}/{Hkv} d={d} split {split_pages}")
    again, _ = attend(pd, Hq, Hkv, d, q.to(DEV), kv4, table, lens, NP, scale, split_pages, want_lse=False)
    assert torch.equal(out.view(torch.int16), again.view(torch.int16))  # bit-reproducible, lse or not
    assert (out[8] == 0).all()


@pytest.mark.parametrize("gain", [1e-25, 1e-6, 1e4, 1e20])
def test_attention_takes_any_magnitude_of_q_and_scales(gain):
    """q times gain over a cache whose K is divided by it: the logits stay, fp16's range does not show."""
    import paper_2609_35158_b200 as pd

    Hq, Hkv, d = 8, 2, 128
    lens = np.array([40, 500, 3], np.int32)
    kv4, table, NP = random_cache(lens, Hkv, d, 70, scale_k=0.3 / gain, scale_v=0.3 * gain)
    q = (wl.random_bf16((3, Hq, d), 71, "cpu").float() * gain).to(torch.bfloat16)
    q[:, :, 5] = 0
    q[0, 0, :] = 0
    ref = q4.decode_attn(oracle.bf16_bits(q), kv4, table, lens, 0.1)
    for split in (0, 1):
        out, lse = attend(pd, Hq, Hkv, d, q.to(DEV), kv4, table, lens, NP, 0.1, split)
        check_attention(out, lse, ref, f"gain {gain} split {split}")


@pytest.mark.parametrize("d", [128, 64])
@pytest.mark.parametrize("late", [False, True])
def test_a_token_of_huge_scale_and_vanishing_weight_hides_nothing(d, late):
    """One token's V is 2^30 times the others' and its probability about 2^-60: it must not push the rest out of fp16."""
    import paper_2609_35158_b200 as pd

    Hq, Hkv = 4, 1
    lens = np.array([200], np.int32)
    kv4, table, NP = random_cache(lens, Hkv, d, 80)
    where = 190 if late else 2
    rec = kv4[table[0, where // P], 0, 16 * d:].view(np.uint16).reshape(P, d // 64, 4)
    rec[where % P, :, 2] = oracle.f32_to_bf16_bits(np.array([0.3 * 2.0 ** 30], np.float32))[0]
    rec[where % P, :, 3] = oracle.f32_to_bf16_bits(np.array([-2.0 * 2.0 ** 30], np.float32))[0]
    rec[where % P, :, 0] = 0
    rec[where % P, :, 1] = oracle.f32_to_bf16_bits(np.array([-50.0], np.float32))[0]   # K = -50 everywhere
    q = (wl.random_bf16((1, Hq, d), 81, "cpu").abs().float() * 0.1 + 0.2).to(torch.bfloat16)
    ref = q4.decode_attn(oracle.bf16_bits(q), kv4, table, lens, 0.05)
    for split in (0, 1, 100000):
        out, lse = attend(pd, Hq, Hkv, d, q.to(DEV), kv4, table, lens, NP, 0.05, split)
        check_attention(out, lse, ref, f"late {late} split {split}")


@pytest.mark.parametrize("at", [0, 15, 16, 37, 99])
def test_a_dominant_key_anywhere(at):
    """Logits that jump by about 290 log2 units at one token: the row is that token's V."""
    import paper_2609_35158_b200 as pd

    Hq, Hkv, d = 8, 2, 128
    lens = np.array([100], np.int32)
    kv4, table, NP = random_cache(lens, Hkv, d, 90)
    for h in range(Hkv):
        rec = kv4[table[0, at // P], h, 16 * d:].view(np.uint16).reshape(P, d // 64, 4)
        rec[at % P, :, 0], rec[at % P, :, 1] = 0, 0x41A0   # K = 20 everywhere
    q = torch.full((1, Hq, d), 1.0, dtype=torch.bfloat16)
    ref = q4.decode_attn(oracle.bf16_bits(q), kv4, table, lens, 0.08)
    out, lse = attend(pd, Hq, Hkv, d, q.to(DEV), kv4, table, lens, NP, 0.08)
    check_attention(out, lse, ref, f"at {at}")
    v = q4.sequence_values(kv4, table, 0, 100, 0, d)[1][at]
    assert np.abs(out[0, 0].float().cpu().numpy() - v).max() <= 2.0 ** -8 * np.abs(v).max() + 2.0 ** -11 * 15


def test_attention_closed_form():
    """Two tokens whose logits differ by one and whose V are +1 and -1: every output is tanh(1/2)."""
    import paper_2609_35158_b200 as pd

    d = 128
    one = int(oracle.f32_to_bf16_bits(np.array([1.0], np.float32))[0])
    kv4 = np.full((3, 1, 18 * d), 0xFF, np.uint8)
    rec = kv4[1, 0, 16 * d:].view(np.uint16).reshape(P, 2, 4)
    rec[0], rec[1] = [0, one, 0, one], [0, 0, 0, one | 0x8000]      # K = 1, 0; V = 1, -1; all scales zero
    q = torch.zeros((1, 4, d), dtype=torch.bfloat16, device=DEV)
    q[..., 0] = 8.0
    out, lse = attend(pd, 4, 1, d, q, kv4, np.array([[1, 2]], np.int32), np.array([2], np.int32), 3, 0.125)
    # fp32 statistics, exact products, one rounding to bf16
    assert np.abs(out.float().cpu().numpy() - np.tanh(0.5)).max() <= 2.0 ** -8 * np.tanh(0.5) + 1e-6
    assert np.abs(lse.cpu().numpy() - np.log(1 + np.e)).max() <= 1e-5


def test_a_group_with_a_nan_reaches_its_own_rows_only():
    import paper_2609_35158_b200 as pd

    Hq, Hkv, d = 8, 2, 128
    lens = np.array([40, 40], np.int32)
    kv4, table, NP = random_cache(lens, Hkv, d, 100)
    rec = kv4[table[1, 0], 1, 16 * d:].view(np.uint16).reshape(P, 2, 4)
    rec[3, 0, 2] = 0x7FC0                              # V scale of one token, first half of KV head 1 of sequence 1
    q = wl.random_bf16((2, Hq, d), 101, "cpu")
    clean = kv4.copy()
    clean[table[1, 0], 1, 16 * d:].view(np.uint16).reshape(P, 2, 4)[3, 0, 2] = 0x3E80
    ref = q4.decode_attn(oracle.bf16_bits(q), clean, table, lens, 0.1)
    out, lse = attend(pd, Hq, Hkv, d, q.to(DEV), kv4, table, lens, NP, 0.1)
    nan = torch.isnan(out.float()).cpu().numpy()
    assert nan[1, 4:, :64].all() and not nan[0].any() and not nan[1, :4].any()
    for sel in ((0, slice(None)), (1, slice(0, 4))):
        check_attention(out[sel], lse[sel], [x[sel] for x in ref])


def test_step_is_append_then_attention_and_can_be_captured():
    import paper_2609_35158_b200 as pd

    Hq, Hkv, d = 16, 2, 64
    before = np.array([0, 15, 16, 300, 31], np.int32)
    steps = 9
    B = len(before)
    kv4, _, _ = random_cache(before, Hkv, d, 110, poison=False)
    table, NP = table_for(before + 1 + 2 * steps, 111)
    rng = np.random.default_rng(112)
    kv4 = rng.integers(0, 256, (NP, Hkv, 18 * d)).astype(np.uint8)
    rec = np.broadcast_to(oracle.f32_to_bf16_bits(np.array([0.2, -1.5, 0.2, -1.5], np.float32)), (NP, Hkv, P, 4))
    kv4[..., 16 * d:] = np.ascontiguousarray(rec).view(np.uint8).reshape(NP, Hkv, -1)
    q = wl.random_bf16((B, Hq, d), 113, DEV)
    kn, vn = wl.random_bf16((B, Hkv, d), 114, DEV), wl.random_bf16((B, Hkv, d), 115, DEV)
    t = dev(table)
    with Ctx(Hq, Hkv, d, B, table.shape[1], NP) as ctx:
        a, La = dev(kv4), dev(before)
        out_a = torch.empty((B, Hq, d), dtype=torch.bfloat16, device=DEV)
        lse_a = torch.empty((B, Hq), dtype=torch.float32, device=DEV)
        for _ in range(1 + 2 * steps):
            pd.pd_kv_append_q4(ctx.h, kn, vn, a, t, La)
            pd.pd_decode_attn_q4(ctx.h, q, a, t, La, out_a, lse_a, sm_scale=0.125)
        b, Lb = dev(kv4), dev(before)
        out_b, lse_b = torch.empty_like(out_a), torch.empty_like(lse_a)
        step = lambda s: pd.pd_decode_step_q4(ctx.h, q, kn, vn, b, t, Lb, out_b, lse_b, sm_scale=0.125, stream=s)
        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):
            step(side)
            graph = torch.cuda.CUDAGraph()
            with torch.cuda.graph(graph, stream=side):
                for _ in range(steps):
                    step(torch.cuda.current_stream())
            graph.replay()
            graph.replay()
        torch.cuda.synchronize()
        assert pd.pd_device_status(ctx.h)[0] == 0
        assert torch.equal(La, Lb) and La.cpu().tolist() == (before + 1 + 2 * steps).tolist()
        assert torch.equal(a, b)
        assert torch.equal(out_a.view(torch.int16), out_b.view(torch.int16)) and torch.equal(lse_a, lse_b)
        ref = q4.decode_attn(oracle.bf16_bits(q), a.cpu().numpy(), table, La.cpu().numpy(), 0.125)
        check_attention(out_b, lse_b, ref)


def test_an_empty_batch_and_rows_behind_the_last_sequence():
    """All contexts empty; and a batch argument below the tensors' rows leaves the others as they were."""
    import paper_2609_35158_b200 as pd

    Hq, Hkv, d = 8, 2, 64
    lens = np.array([0, 0, 40], np.int32)
    kv4, table, NP = random_cache(lens, Hkv, d, 140)
    q = wl.random_bf16((3, Hq, d), 141, DEV)
    out = torch.full((3, Hq, d), 5.0, dtype=torch.bfloat16, device=DEV)
    lse = torch.full((3, Hq), 5.0, device=DEV)
    with Ctx(Hq, Hkv, d, 3, table.shape[1], NP) as ctx:
        pd.pd_decode_attn_q4(ctx.h, q, dev(kv4), dev(table), dev(lens), out, lse, batch=2, sm_scale=0.1)
        torch.cuda.synchronize()
        assert (out[:2] == 0).all() and torch.isneginf(lse[:2]).all() and (out[2] == 5).all() and (lse[2] == 5).all()
        pool, L = torch.zeros((NP, Hkv, 18 * d), dtype=torch.uint8, device=DEV), dev(np.array([3, 0, 8], np.int32))
        rows = dev(np.array([[0], [1], [2]], np.int32).repeat(table.shape[1], 1))
        kn = wl.random_bf16((3, Hkv, d), 142, DEV)
        pd.pd_kv_append_q4(ctx.h, kn, kn, pool, rows, L, batch=2)
        torch.cuda.synchronize()
        assert pd.pd_device_status(ctx.h)[0] == 0
        assert L.cpu().tolist() == [4, 1, 8] and pool.flatten(1).any(1).cpu().tolist()[:3] == [True, True, False]


def test_more_tokens_than_announced_are_refused_on_the_device():
    import paper_2609_35158_b200 as pd

    Hkv, d = 2, 128
    kn = wl.random_bf16((3, Hkv, d), 150, DEV)
    pool, L = torch.zeros((2, Hkv, 18 * d), dtype=torch.uint8, device=DEV), dev(np.zeros(2, np.int32))
    with Ctx(Hkv, Hkv, d, 2, 1, 2) as ctx:
        pd.pd_kv_append_tokens_q4(ctx.h, kn, kn, dev(np.array([0, 2, 3], np.int32)), pool, dev(np.array([[0], [1]], np.int32)), L, 1)
        assert pd.pd_device_status(ctx.h)[:2] == (pd.PD_ERR_DEVICE_FAULT, 0)
        assert L.cpu().tolist() == [0, 1] and pool.flatten(1).any(1).cpu().tolist() == [False, True]


def test_two_contexts_on_two_streams_at_once():
    import paper_2609_35158_b200 as pd

    Hq, Hkv, d = 32, 8, 128
    runs = []
    for seed, lens in ((160, [3000, 17, 900]), (170, [1, 5000, 0, 64])):
        lens = np.array(lens, np.int32)
        kv4, table, NP = random_cache(lens, Hkv, d, seed)
        q = wl.random_bf16((len(lens), Hq, d), seed + 1, DEV)
        runs.append((q, kv4, table, lens, NP, *attend(pd, Hq, Hkv, d, q, kv4, table, lens, NP, 0.09)))
    streams = [torch.cuda.Stream() for _ in runs]
    with Ctx(Hq, Hkv, d, 4, runs[0][2].shape[1], runs[0][4]) as a, Ctx(Hq, Hkv, d, 4, runs[1][2].shape[1], runs[1][4]) as b:
        inputs = [(r[0], dev(r[1]), dev(r[2]), dev(r[3]), torch.empty_like(r[5]), torch.empty_like(r[6])) for r in runs]
        torch.cuda.synchronize()
        for _ in range(20):
            for ctx, s, (q, kv, t, L, out, lse) in zip((a, b), streams, inputs):
                pd.pd_decode_attn_q4(ctx.h, q, kv, t, L, out, lse, sm_scale=0.09, stream=s)
        torch.cuda.synchronize()
        for r, x in zip(runs, inputs):
            assert torch.equal(r[5].view(torch.int16), x[4].view(torch.int16)) and torch.equal(r[6], x[5])


@pytest.mark.parametrize("seed", range(10))
def test_attention_random_cases(seed):
    import paper_2609_35158_b200 as pd

    rng = np.random.default_rng(1000 + seed)
    d, Hkv = int(rng.choice([64, 128])), int(rng.choice([1, 2, 3, 5]))
    Hq = Hkv * int(rng.choice([1, 2, 4, 8]))
    lens = np.minimum(np.exp(rng.uniform(0, 7.5, int(rng.integers(1, 9)))).astype(np.int32) * rng.integers(0, 2, 1)[0] + rng.integers(0, 70), 2000).astype(np.int32)
    kv4, table, NP = random_cache(lens, Hkv, d, 1100 + seed, scale_k=float(10 ** rng.uniform(-3, 1)), scale_v=float(10 ** rng.uniform(-3, 3)))
    q = wl.random_bf16((len(lens), Hq, d), 1200 + seed, "cpu")
    scale = float(rng.uniform(0.02, 0.3))
    ref = q4.decode_attn(oracle.bf16_bits(q), kv4, table, lens, scale)
    out, lse = attend(pd, Hq, Hkv, d, q.to(DEV), kv4, table, lens, NP, scale, int(rng.choice([0, 0, 2, 7])))
    check_attention(out, lse, ref, f"seed {seed}: {Hq}/{Hkv} d={d} {lens.tolist()}")


def test_blocks_past_four_gigabytes():
    """Pages at the far end of a pool of 5 GB: block offsets need 64 bits."""
    import paper_2609_35158_b200 as pd

    Hq, Hkv, d = 8, 8, 128
    NP = 5 * (1 << 30) // (Hkv * 18 * d)
    pool = torch.zeros((NP, Hkv, 18 * d), dtype=torch.uint8, device=DEV)
    table = np.array([[NP - 1, 1, NP - 2]], np.int32)
    k, v = (oracle.f32_to_bf16_bits(np.random.default_rng(s).standard_normal((40, Hkv, d)).astype(np.float32)) for s in (120, 121))
    small = np.zeros((3, Hkv, 18 * d), np.uint8)
    flat = np.array([[0, 1, 2]], np.int32)
    lens = q4.append_tokens(k, v, [0, 40], small, flat, np.zeros(1, np.int32))
    q = wl.random_bf16((1, Hq, d), 122, "cpu")
    ref = q4.decode_attn(oracle.bf16_bits(q), small, flat, lens, 0.1)
    with Ctx(Hq, Hkv, d, 1, 3, NP) as ctx:
        L, t = dev(np.zeros(1, np.int32)), dev(table)
        pd.pd_kv_append_tokens_q4(ctx.h, bf16_dev(k), bf16_dev(v), dev(np.array([0, 40], np.int32)), pool, t, L, 40)
        assert np.array_equal(pool[torch.from_numpy(table[0].astype(np.int64)).to(DEV)].cpu().numpy(), small)
        out, lse = torch.empty((1, Hq, d), dtype=torch.bfloat16, device=DEV), torch.empty((1, Hq), device=DEV)
        pd.pd_decode_attn_q4(ctx.h, q.to(DEV), pool, t, L, out, lse, sm_scale=0.1)
        torch.cuda.synchronize()
        assert pd.pd_device_status(ctx.h)[0] == 0
    check_attention(out, lse, ref)


def test_attention_reports_bad_pages_and_lengths():
    import paper_2609_35158_b200 as pd

    Hq, Hkv, d = 4, 2, 128
    lens = np.array([20, 20], np.int32)
    kv4, table, NP = random_cache(lens, Hkv, d, 130, poison=False)
    q = wl.random_bf16((2, Hq, d), 131, DEV)
    out = torch.empty_like(q)
    with Ctx(Hq, Hkv, d, 2, 2, NP) as ctx:
        bad = table.copy()
        bad[1, 1] = NP
        pd.pd_decode_attn_q4(ctx.h, q, dev(kv4), dev(bad), dev(lens), out, sm_scale=0.1)
        assert pd.pd_device_status(ctx.h) == (pd.PD_ERR_DEVICE_FAULT, 1, NP)
        pd.pd_decode_attn_q4(ctx.h, q, dev(kv4), dev(table), dev(np.array([20, 33], np.int32)), out, sm_scale=0.1)
        assert pd.pd_device_status(ctx.h)[:2] == (pd.PD_ERR_DEVICE_FAULT, 1)


def test_refusals():
    import paper_2609_35158_b200 as pd

    d, Hkv = 64, 2
    x = torch.zeros(65536, dtype=torch.uint8, device=DEV)
    off = x[1:]
    with Ctx(4, Hkv, d, 2, 4, 8) as ctx:
        h = ctx.h
        n0 = pd.pd_launch_count(h)
        bad = [
            lambda: pd.pd_kv_append_q4(h, x, x, off, x, x, batch=1),
            lambda: pd.pd_kv_append_q4(h, x, x, x, x, x, batch=3),
            lambda: pd.pd_kv_append_q4(h, x, x, x, x, x, batch=-1),
            lambda: pd.pd_kv_append_q4(h, x, x, x, x, x, batch=1, call_flags=2),
            lambda: pd.pd_kv_append_q4(h, off, x, x, x, x, batch=1),
            lambda: pd.pd_kv_append_tokens_q4(h, x, x, None, x, x, x, 1, batch=1),
            lambda: pd.pd_kv_append_tokens_q4(h, x, x, x, x, x, x, -1, batch=1),
            lambda: pd.pd_kv_append_tokens_q4(h, x, None, x, x, x, x, 1, batch=1),
            lambda: pd.pd_kv_dequantize_q4(h, x, x, None, x, x, off, x, batch=1),
            lambda: pd.pd_kv_dequantize_q4(h, x, x, None, x, x, x, None, batch=1),
            lambda: pd.pd_kv_dequantize_q4(h, x, x, None, x, x, x, x, batch=5),
            lambda: pd.pd_decode_attn_q4(h, x, x, x, x, off, batch=1),
            lambda: pd.pd_decode_attn_q4(h, x, None, x, x, x, batch=1),
            lambda: pd.pd_decode_attn_q4(h, x, x, x, x, x, batch=1, sm_scale=0.0),
            lambda: pd.pd_decode_attn_q4(h, x, x, x, x, x, batch=1, sm_scale=float("nan")),
            lambda: pd.pd_decode_attn_q4(h, x, x, x, x, x, batch=1, split_pages=-1),
            lambda: pd.pd_decode_step_q4(h, x, x, x, x, x, x, x, batch=1, sm_scale=float("inf")),
            lambda: pd.pd_decode_step_q4(h, x, None, x, x, x, x, x, batch=1),
        ]
        for i, call in enumerate(bad):
            with pytest.raises(pd.PdError) as e:
                call()
            assert e.value.code == pd.PD_ERR_INVALID_ARG, i
        assert pd.pd_launch_count(h) == n0             # nothing was enqueued
        pd.pd_decode_attn_q4(h, x, x, x, x, x, batch=0)
        pd.pd_kv_append_tokens_q4(h, x, x, x, x, x, x, 0, batch=1)
        assert pd.pd_launch_count(h) == n0
