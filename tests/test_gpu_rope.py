"""Rotary positions through the C ABI: against the fp64 oracle (extended-precision angles), the fused appends against
the rotation followed by the append, bit for bit, and a multi-turn run of the write and read paths together."""
import numpy as np
import pytest
import torch

import oracle
from oracle import q4
import workloads as wl
from pd_testlib import Ctx
from test_gpu_q4 import bf16_dev, check_attention, dev, table_for

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
P = 16


def frequencies(rot, base=10000.0):
    return (base ** (-np.arange(rot // 2) * 2.0 / rot)).astype(np.float32)


def check_rotated(got, x, positions, freq, axis, rot, adjacent, magnitude=1.0):
    want, tol = q4.rope(oracle.bf16_bits_to_f64(oracle.bf16_bits(x)), positions, freq, axis, rot, adjacent, magnitude)
    got = oracle.bf16_bits_to_f64(oracle.bf16_bits(got))
    assert np.all(np.abs(got - want) <= 2.0 ** -8 * np.abs(want) + 2 * tol)  # one rounding to bf16 of an fp32 result
    return want


@pytest.mark.parametrize("d,rot,adjacent,axes", [(128, 128, False, 1), (128, 128, True, 3), (128, 64, False, 2), (64, 64, False, 4),
                                                 (64, 16, True, 1), (64, 32, False, 3), (128, 112, False, 3), (128, 48, True, 2)])
@pytest.mark.parametrize("total", [1, 5, 67])
def test_rotation(d, rot, adjacent, axes, total):
    import paper_2609_35158_b200 as pd

    Hq, Hkv = 8, 2
    rng = np.random.default_rng(rot + axes + total)
    axis = rng.integers(0, axes, rot // 2)
    freq = frequencies(rot)
    pos = rng.integers(0, 40000, (axes, total)).astype(np.int32)
    pos[:, 0] = 0
    q, k = wl.random_bf16((total, Hq, d), 1, DEV), wl.random_bf16((total, Hkv, d), 2, DEV)
    qo, ko = torch.full_like(q, float("nan")), torch.full_like(k, float("nan"))
    rope = pd.rope_config(rot, freq, axis, axes, adjacent, 1.25)
    with Ctx(Hq, Hkv, d, 1, 1, 1) as ctx:
        pd.pd_rope_tokens(ctx.h, rope, dev(pos), q, k, qo, ko)
        torch.cuda.synchronize()
        check_rotated(qo, q, pos, freq, axis, rot, adjacent, 1.25)
        check_rotated(ko, k, pos, freq, axis, rot, adjacent, 1.25)
        assert torch.equal(qo[..., rot:], q[..., rot:])
        pd.pd_rope_tokens(ctx.h, rope, dev(pos), q, k, q, k)  # in place
        torch.cuda.synchronize()
    assert torch.equal(q.view(torch.int16), qo.view(torch.int16)) and torch.equal(k.view(torch.int16), ko.view(torch.int16))


def test_far_and_negative_positions_keep_their_angle():
    import paper_2609_35158_b200 as pd

    d = 128
    pos = np.array([[0, 1, -1, 10 ** 6, 10 ** 6 + 1, 123456789, -123456789, 2 ** 31 - 1, -2 ** 31]], np.int32)
    n = pos.shape[1]
    q, k = wl.random_bf16((n, 4, d), 3, DEV), wl.random_bf16((n, 4, d), 4, DEV)
    for freq in (frequencies(d), frequencies(d, 1e6), -frequencies(d), frequencies(d) * 7):
        qo, ko = torch.empty_like(q), torch.empty_like(k)
        with Ctx(4, 4, d, 1, 1, 1) as ctx:
            pd.pd_rope_tokens(ctx.h, pd.rope_config(d, freq), dev(pos), q, k, qo, ko)
            torch.cuda.synchronize()
        check_rotated(qo, q, pos, freq, [0] * 64, d, False)


def inv_two_pi(bits):
    """floor(2^bits / (2 pi)) by Machin's formula in integers."""
    n = bits + 64

    def atan_inverse(x):
        term = (1 << n) // x
        total, k, sign = term, 1, -1
        while term:
            term //= x * x
            k += 2
            total, sign = total + sign * (term // k), -sign
        return total

    return (1 << (n + bits)) // (8 * (4 * atan_inverse(5) - atan_inverse(239)))


def test_the_largest_frequencies_keep_their_angle_at_far_positions():
    """Rotating (1, 0) gives cosine and sine alone; where one of them is near 0, bf16 shows its absolute error. The tolerance:
    2^-31 turns and the rounding of the angle to fp32 (2^-26 turns) are below 2^-23 radians, sine and cosine of CUDA
    are within 2 units of 2^-24; together below 2^-21. Then one rounding to bf16."""
    import paper_2609_35158_b200 as pd

    d, n, bits = 64, 500, 320
    rng = np.random.default_rng(5)
    freq = rng.uniform(50, 400, d // 2).astype(np.float32) * rng.choice([-1, 1], d // 2).astype(np.float32)
    pos = rng.integers(-2 ** 31, 2 ** 31, (1, n)).astype(np.int32)
    unit = inv_two_pi(bits)
    want = np.empty((n, d))
    for i, f in enumerate(freq):
        num, den = float(f).as_integer_ratio()
        for t in range(n):
            whole = den << bits
            turn = (num * unit * int(pos[0, t])) % whole
            angle = 2 * np.pi * (((turn << 60) // whole) / 2.0 ** 60 - (turn * 2 >= whole))
            want[t, i], want[t, i + d // 2] = np.cos(angle), np.sin(angle)
    assert (np.abs(want) < 1e-3).sum() > 10
    q = torch.zeros((n, 1, d), dtype=torch.bfloat16, device=DEV)
    q[..., :d // 2] = 1
    qo, ko = torch.empty_like(q), torch.empty_like(q)
    with Ctx(1, 1, d, 1, 1, 1) as ctx:
        pd.pd_rope_tokens(ctx.h, pd.rope_config(d, freq), dev(pos), q, q, qo, ko)
        torch.cuda.synchronize()
    got = qo[:, 0].float().cpu().numpy().astype(np.float64)
    assert np.all(np.abs(got - want) <= 2.0 ** -8 * np.abs(want) + 2.0 ** -21)


def packed(before, new, seed, Hq, Hkv, d, axes):
    rng = np.random.default_rng(seed)
    total = int(new.sum())
    indptr = np.concatenate([[0], np.cumsum(new)]).astype(np.int32)
    pos = rng.integers(0, 5000, (axes, total)).astype(np.int32)
    return (indptr, pos, wl.random_bf16((total, Hq, d), seed + 1, DEV), wl.random_bf16((total, Hkv, d), seed + 2, DEV),
            wl.random_bf16((total, Hkv, d), seed + 3, DEV))


@pytest.mark.parametrize("d,rot,adjacent,Hkv", [(128, 128, False, 8), (64, 32, True, 2), (128, 64, False, 1), (64, 64, False, 40), (128, 128, False, 112)])
@pytest.mark.parametrize("new", [[1] * 7, [1, 0, 1, 1, 0, 0, 1], [0, 70, 1, 16, 3, 33, 5], [0, 0, 0, 0, 0, 0, 300]])
@pytest.mark.parametrize("with_positions", [True, False])
def test_fused_appends_are_the_two_calls(d, rot, adjacent, Hkv, new, with_positions):
    import paper_2609_35158_b200 as pd

    Hq = Hkv if Hkv > 100 else 2 * Hkv
    before, new = np.array([0, 5, 16, 31, 47, 3, 8], np.int32), np.array(new, np.int32)
    after = before + new
    indptr, pos, q, k, v = packed(before, new, 20, Hq, Hkv, d, 3)
    if not with_positions:
        pos = np.repeat(np.concatenate([np.arange(b, a) for b, a in zip(before, after)])[None], 3, 0).astype(np.int32)
    table, NP = table_for(after, 21)
    rope = pd.rope_config(rot, frequencies(rot), np.arange(rot // 2) % 3, 3, adjacent)
    B, most = len(new), int(new.max())
    t, ip, ps = dev(table), dev(indptr), dev(pos)
    with Ctx(Hq, Hkv, d, B, table.shape[1], NP) as ctx:
        qa, ka = torch.empty_like(q), torch.empty_like(k)
        pd.pd_rope_tokens(ctx.h, rope, ps, q, k, qa, ka)
        pools = [torch.full((NP, Hkv, P, d), 3.0, dtype=torch.bfloat16, device=DEV) for _ in range(4)]
        four = [torch.full((NP, Hkv, 18 * d), 7, dtype=torch.uint8, device=DEV) for _ in range(2)]
        lens = [dev(before) for _ in range(4)]
        pd.pd_kv_append_tokens(ctx.h, ka, v, ip, pools[0], pools[1], t, lens[0], most)
        pd.pd_kv_append_tokens_q4(ctx.h, ka, v, ip, four[0], t, lens[1], most)
        qb, qc = torch.empty_like(q), q.clone()
        arg = ps if with_positions else None
        for flags in (pd.PD_APPEND_NO_ADVANCE, 0):
            pd.pd_rope_append_tokens(ctx.h, rope, arg, q, k, v, ip, qb, pools[2], pools[3], t, lens[2], most, call_flags=flags)
        pd.pd_rope_append_tokens_q4(ctx.h, rope, arg, qc, k, v, ip, qc, four[1], t, lens[3], most)
        torch.cuda.synchronize()
        assert pd.pd_device_status(ctx.h)[0] == 0
    same = lambda a, b: torch.equal(a.view(torch.int16), b.view(torch.int16))
    assert same(qa, qb) and same(qa, qc)
    assert same(pools[0], pools[2]) and same(pools[1], pools[3]) and torch.equal(four[0], four[1])
    assert all(x.cpu().tolist() == after.tolist() for x in lens)


def test_fused_append_reports_and_skips():
    import paper_2609_35158_b200 as pd

    d, Hq, Hkv = 128, 4, 2
    table = np.array([[0, 1], [2, 99], [3, -1], [4, 5]], np.int32)
    before, new = np.array([31, 16, 17, 3], np.int32), np.array([2, 2, 2, 2], np.int32)
    indptr, pos, q, k, v = packed(before, new, 30, Hq, Hkv, d, 1)
    freq = frequencies(d)
    rope = pd.rope_config(d, freq)
    with Ctx(Hq, Hkv, d, 4, 2, 6) as ctx:
        for four in (False, True):
            L, qo = dev(before), torch.full_like(q, float("nan"))
            if four:
                kv = torch.zeros((6, Hkv, 18 * d), dtype=torch.uint8, device=DEV)
                pd.pd_rope_append_tokens_q4(ctx.h, rope, dev(pos), q, k, v, dev(indptr), qo, kv, dev(table), L, 2)
                touched = kv.flatten(1).any(1)
            else:
                kp, vp = (torch.zeros((6, Hkv, P, d), dtype=torch.bfloat16, device=DEV) for _ in range(2))
                pd.pd_rope_append_tokens(ctx.h, rope, dev(pos), q, k, v, dev(indptr), qo, kp, vp, dev(table), L, 2)
                touched = (kp != 0).flatten(1).any(1) | (vp != 0).flatten(1).any(1)
            code, seq, _ = pd.pd_device_status(ctx.h)
            assert code == pd.PD_ERR_DEVICE_FAULT and seq in (0, 1, 2)
            assert L.cpu().tolist() == [31, 18, 19, 5]
            assert touched.cpu().tolist() == [False, False, False, False, True, False]
            check_rotated(qo, q, pos, freq, [0] * 64, d, False)  # queries are rotated all the same


@pytest.mark.parametrize("new", [[1, 1, 1], [40, 30, 30], [0, 3, 2]])
@pytest.mark.parametrize("four", [False, True])
@pytest.mark.parametrize("rows_short", [0, 1])
def test_fused_append_leaves_out_sequences_without_positions(new, four, rows_short):
    """Positions for all rows but the last: the sequence that holds it keeps its pages, length and queries."""
    import paper_2609_35158_b200 as pd

    d, Hq, Hkv, axes = 128, 4, 2, 2
    before, new = np.array([3, 0, 7], np.int32), np.array(new, np.int32)
    table = np.arange(15, dtype=np.int32).reshape(3, 5)
    indptr, pos, q, k, v = packed(before, new, 60, Hq, Hkv, d, axes)
    held = int(indptr[3]) - rows_short
    freq, axis = frequencies(d), [i % axes for i in range(d // 2)]
    rope = pd.rope_config(d, freq, axis, num_axes=axes)
    with Ctx(Hq, Hkv, d, 3, 5, 15) as ctx:
        L, qo, given = dev(before), torch.full_like(q, float("nan")), dev(pos[:, :held].copy())
        if four:
            kv = torch.zeros((15, Hkv, 18 * d), dtype=torch.uint8, device=DEV)
            pd.pd_rope_append_tokens_q4(ctx.h, rope, given, q, k, v, dev(indptr), qo, kv, dev(table), L, int(new.max()))
            touched = kv.flatten(1).any(1)
        else:
            kp, vp = (torch.zeros((15, Hkv, P, d), dtype=torch.bfloat16, device=DEV) for _ in range(2))
            pd.pd_rope_append_tokens(ctx.h, rope, given, q, k, v, dev(indptr), qo, kp, vp, dev(table), L, int(new.max()))
            touched = (kp != 0).flatten(1).any(1) & (vp != 0).flatten(1).any(1)
        if rows_short:
            assert pd.pd_device_status(ctx.h) == (pd.PD_ERR_DEVICE_FAULT, 2, int(indptr[3]))
        else:
            assert pd.pd_device_status(ctx.h)[0] == 0
        served = 2 if rows_short else 3
        after = before.copy()
        after[:served] += new[:served]
        assert L.cpu().tolist() == after.tolist()
        want = np.zeros(15, bool)
        for b in range(served):
            for t in range(int(before[b]), int(after[b])):
                want[table[b, t // P]] = True
        assert touched.cpu().tolist() == want.tolist()
        n = int(indptr[served])
        check_rotated(qo[:n], q[:n], pos[:, :n], freq, axis, d, False)
        assert torch.isnan(qo[n:].float()).all()


def test_refusals():
    import paper_2609_35158_b200 as pd

    x = torch.zeros(65536, dtype=torch.uint8, device=DEV)
    off, ps, many = x[1:], torch.zeros((2, 64), dtype=torch.int32, device=DEV), torch.zeros((8, 64), dtype=torch.int32, device=DEV)

    def cfg(**kw):
        c = pd.rope_config(32, np.ones(16))
        for name, value in kw.items():
            setattr(c, name, value)
        return c

    ok, nan_freq, axis9, far = cfg(), cfg(), cfg(), cfg()
    nan_freq.inv_freq[3] = float("nan")
    axis9.axis_of_pair[15] = 1
    far.inv_freq[0] = 403.0
    with Ctx(4, 2, 64, 2, 4, 8) as ctx, Ctx(113, 113, 128, 1, 1, 1) as wide:
        h = ctx.h
        n0 = pd.pd_launch_count(h)
        for c in (cfg(rot_dim=0), cfg(rot_dim=80), cfg(num_axes=0), cfg(num_axes=5), cfg(adjacent=2), cfg(magnitude=float("inf")),
                  cfg(magnitude=float("nan")), nan_freq, axis9, far):
            for call in (lambda: pd.pd_rope_tokens(h, c, many, x, x, x, x, total=1),
                         lambda: pd.pd_rope_append_tokens(h, c, None, x, x, x, x, x, x, x, x, x, 1, batch=1),
                         lambda: pd.pd_rope_append_tokens_q4(h, c, None, x, x, x, x, x, x, x, x, 1, batch=1)):
                with pytest.raises(pd.PdError) as e:
                    call()
                assert e.value.code == pd.PD_ERR_INVALID_ARG
        for call in (lambda: pd.pd_rope_tokens(h, cfg(rot_dim=24), ps[0], x, x, x, x, total=1),
                     lambda: pd.pd_rope_append_tokens_q4(wide.h, ok, None, x, x, x, x, x, x, x, x, 1, batch=1)):
            with pytest.raises(pd.PdError) as e:
                call()
            assert e.value.code == pd.PD_ERR_UNSUPPORTED
        for i, call in enumerate((
                lambda: pd.pd_rope_tokens(h, ok, None, x, x, x, x, total=1),
                lambda: pd.pd_rope_tokens(h, ok, ps[0], x, x, off, x, total=1),
                lambda: pd.pd_rope_tokens(h, ok, ps[0], x, x, x, x, total=-1),
                lambda: pd.pd_rope_tokens(h, ok, ps[0], x, x, x, x, total=65),
                lambda: pd.pd_rope_append_tokens(h, ok, ps[0], x, x, x, None, x, x, x, x, x, 1, batch=1),
                lambda: pd.pd_rope_append_tokens(h, ok, ps[0], x, x, x, x, x, x, None, x, x, 1, batch=1),
                lambda: pd.pd_rope_append_tokens(h, ok, ps[0], x, x, x, x, x, x, x, x, x, 1, batch=3),
                lambda: pd.pd_rope_append_tokens(h, ok, ps[0], x, x, x, x, x, x, x, x, x, -1, batch=1),
                lambda: pd.pd_rope_append_tokens(h, ok, ps[0], x, x, x, x, x, x, x, x, x, 1, batch=1, call_flags=4),
                lambda: pd.pd_rope_append_tokens_q4(h, ok, ps[0], x, x, x, x, x, None, x, x, 1, batch=1),
                lambda: pd.pd_rope_append_tokens_q4(h, ok, ps[0], x, x, x, x, x, off, x, x, 1, batch=1))):
            with pytest.raises(pd.PdError) as e:
                call()
            assert e.value.code == pd.PD_ERR_INVALID_ARG, i
        with pytest.raises(ValueError):
            pd.pd_rope_tokens(h, cfg(num_axes=2), ps[0], x, x, x, x, total=1)
        assert pd.pd_launch_count(h) == n0
        pd.pd_rope_tokens(h, ok, ps[0], x, x, x, x, total=0)
        assert pd.pd_launch_count(h) == n0


@pytest.mark.parametrize("Hq,Hkv,d", [(8, 2, 128), (4, 4, 64)])
def test_a_multi_turn_run_over_the_4bit_cache(Hq, Hkv, d):
    """Two turns as an engine runs them: prompts rotated and written in 4 bits, the cache read back and prefilled over,
    then decode steps on the 4-bit cache. Everything is compared with the oracle on the cache's own values."""
    import paper_2609_35158_b200 as pd

    turns = [np.array([20, 3, 37], np.int32), np.array([5, 18, 1], np.int32)]
    steps, B, scale = 4, 3, d ** -0.5
    lens = np.zeros(B, np.int32)
    table, NP = table_for(sum(turns) + steps * len(turns), 40)
    freq = frequencies(d)
    rope = pd.rope_config(d, freq, np.arange(d // 2) % 3, 3)
    t = dev(table)
    kv4 = torch.zeros((NP, Hkv, 18 * d), dtype=torch.uint8, device=DEV)
    kp, vp = (torch.zeros((NP, Hkv, P, d), dtype=torch.bfloat16, device=DEV) for _ in range(2))
    with Ctx(Hq, Hkv, d, B, table.shape[1], NP) as ctx:
        L = dev(lens)
        for n, new in enumerate(turns):
            indptr, pos, q, k, v = packed(lens, new, 50 + n, Hq, Hkv, d, 3)
            ip, qo = dev(indptr), torch.empty_like(q)
            pd.pd_rope_append_tokens_q4(ctx.h, rope, dev(pos), q, k, v, ip, qo, kv4, t, L, int(new.max()))
            pd.pd_kv_dequantize_q4(ctx.h, kv4, t, None, L, kp, vp, t)
            out = torch.empty_like(q)
            pd.pd_prefill_attn(ctx.h, qo, ip, kp, vp, t, L, out, max_q_len=int(new.max()), sm_scale=scale)
            torch.cuda.synchronize()
            assert pd.pd_device_status(ctx.h)[0] == 0
            lens = lens + new
            assert L.cpu().tolist() == lens.tolist()
            # every prefill query is a decode query over its own prefix of the bf16 pages
            qb = oracle.bf16_bits(qo)
            for b in range(B):
                for i in range(int(new[b])):
                    at = np.array([lens[b] - new[b] + i + 1], np.int32)
                    row = int(indptr[b]) + i
                    want, _ = oracle.decode_attn(qb[row:row + 1], oracle.bf16_bits(kp), oracle.bf16_bits(vp), table[b:b + 1], at, scale)
                    got = out[row].float().cpu().numpy()
                    # P and the result are rounded to bf16, the weights sum to one
                    assert np.abs(got - want[0]).max() <= 2.0 ** -7 * max(1.0, np.abs(vp.float().cpu().numpy()).max())
            for _ in range(steps):
                indptr, pos, q, k, v = packed(lens, np.ones(B, np.int32), 70 + int(lens[0]), Hq, Hkv, d, 3)
                qo = torch.empty_like(q)
                pd.pd_rope_append_tokens_q4(ctx.h, rope, dev(pos), q, k, v, dev(indptr), qo, kv4, t, L, 1)
                out, lse = torch.empty_like(q), torch.empty((B, Hq), dtype=torch.float32, device=DEV)
                pd.pd_decode_attn_q4(ctx.h, qo, kv4, t, L, out, lse, sm_scale=scale)
                torch.cuda.synchronize()
                lens = lens + 1
                ref = q4.decode_attn(oracle.bf16_bits(qo), kv4.cpu().numpy(), table, lens, scale)
                check_attention(out, lse, ref)
        assert pd.pd_device_status(ctx.h)[0] == 0 and L.cpu().tolist() == lens.tolist()


@pytest.mark.parametrize("four", [False, True])
@pytest.mark.parametrize("d", [64, 128])
def test_more_tokens_than_announced_are_treated_as_by_the_two_calls(four, d):
    """max_q_len 1 and a sequence of two tokens: the append to 4-bit pages leaves it out, the bf16 one takes it; queries are
    rotated in any case."""
    import paper_2609_35158_b200 as pd

    Hq, Hkv = 8, 2
    before, new = np.array([3, 15, 0], np.int32), np.array([1, 2, 1], np.int32)
    indptr, pos, q, k, v = packed(before, new, 70, Hq, Hkv, d, 1)
    rope, table = pd.rope_config(d, frequencies(d)), dev(np.arange(6, dtype=np.int32).reshape(3, 2))
    ip, ps = dev(indptr), dev(pos)
    with Ctx(Hq, Hkv, d, 3, 2, 6) as ctx:
        def pools():
            if four:
                return [torch.full((6, Hkv, 18 * d), 7, dtype=torch.uint8, device=DEV)]
            return [torch.full((6, Hkv, P, d), 3.0, dtype=torch.bfloat16, device=DEV) for _ in range(2)]

        a, b, La, Lb = pools(), pools(), dev(before), dev(before)
        qa, ka, qb = torch.empty_like(q), torch.empty_like(k), torch.full_like(q, float("nan"))
        pd.pd_rope_tokens(ctx.h, rope, ps, q, k, qa, ka)
        (pd.pd_kv_append_tokens_q4 if four else pd.pd_kv_append_tokens)(ctx.h, ka, v, ip, *a, table, La, 1)
        one = pd.pd_device_status(ctx.h)
        (pd.pd_rope_append_tokens_q4 if four else pd.pd_rope_append_tokens)(ctx.h, rope, ps, q, k, v, ip, qb, *b, table, Lb, 1)
        two = pd.pd_device_status(ctx.h)
    assert one == two == ((pd.PD_ERR_DEVICE_FAULT, 1, 15) if four else (0, one[1], one[2]))
    assert La.cpu().tolist() == Lb.cpu().tolist() == ([4, 15, 1] if four else [4, 17, 1])
    assert torch.equal(qa.view(torch.int16), qb.view(torch.int16))
    assert all(torch.equal(x.view(torch.uint8), y.view(torch.uint8)) for x, y in zip(a, b))


@pytest.mark.parametrize("length", [2 ** 31 - 1, 2 ** 31 - 4, 2 ** 31 - 17, -2 ** 31, 65])
def test_appends_of_several_tokens_refuse_lengths_whose_sum_passes_32_bits(length):
    """Lengths past the table row, some so far that length plus tokens wraps: latched, length and pools as they were."""
    import paper_2609_35158_b200 as pd

    Hq, Hkv, d = 4, 2, 64
    before, new = np.array([5, length, 0], np.int64).astype(np.int32), np.array([3, 20, 4], np.int32)
    indptr, pos, q, k, v = packed(before, new, 80, Hq, Hkv, d, 1)
    rope, table = pd.rope_config(d, frequencies(d)), dev(np.arange(12, dtype=np.int32).reshape(3, 4))
    ip, qo = dev(indptr), torch.empty_like(q)
    with Ctx(Hq, Hkv, d, 3, 4, 12) as ctx:
        for form in range(4):
            L, kv = dev(before), torch.zeros((12, Hkv, 18 * d), dtype=torch.uint8, device=DEV)
            kp, vp = (torch.zeros((12, Hkv, P, d), dtype=torch.bfloat16, device=DEV) for _ in range(2))
            if form == 0:
                pd.pd_kv_append_tokens(ctx.h, k, v, ip, kp, vp, table, L, 20)
            elif form == 1:
                pd.pd_kv_append_tokens_q4(ctx.h, k, v, ip, kv, table, L, 20)
            elif form == 2:
                pd.pd_rope_append_tokens(ctx.h, rope, None, q, k, v, ip, qo, kp, vp, table, L, 20)
            else:
                pd.pd_rope_append_tokens_q4(ctx.h, rope, None, q, k, v, ip, qo, kv, table, L, 20)
            assert pd.pd_device_status(ctx.h) == (pd.PD_ERR_DEVICE_FAULT, 1, int(before[1])), form
            assert L.cpu().tolist() == [8, int(before[1]), 4], form
            touched = (kp != 0).flatten(1).any(1) if form % 2 == 0 else kv.flatten(1).any(1)
            assert torch.nonzero(touched).flatten().tolist() == [0, 8], form
