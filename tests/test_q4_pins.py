"""CPU pins of the 4-bit format's oracle, and what the new entry points refuse without a device."""
import ctypes

import numpy as np
import pytest
import torch

import oracle
from oracle import q4


def bits(x):
    return oracle.f32_to_bf16_bits(np.asarray(x, np.float32))


def test_layout_covers_every_nibble_and_record_once():
    for d in (64, 128):
        seen = set()
        for slot in range(16):
            for i in range(d):
                o, s = q4.nibble_at(d, slot, i)
                assert 0 <= o < 8 * d
                seen.add((o, s))
        assert len(seen) == 16 * d
        recs = sorted(q4.record_at(d, s, g, w, e) for s in range(16) for g in range(d // 64) for w in range(2) for e in range(2))
        assert recs == list(range(16 * d, 18 * d, 2))


def test_piece_order_spreads_eight_rows_over_all_banks():
    for d in (64, 128):
        for half in (0, 8):
            for piece in range(d // 32):
                banks = {(q4.nibble_at(d, half + r, piece * 32)[0] // 16) % 8 for r in range(8)}
                assert len(banks) == 8


def test_quantiser_properties():
    rng = np.random.default_rng(0)
    for trial in range(300):
        x = (rng.standard_normal(64) * 10.0 ** rng.integers(-20, 20)).astype(np.float32)
        if trial % 3 == 0:
            x = np.rint(x / np.abs(x).max() * 30)  # many exact ties
        b = bits(x)
        v = oracle.bf16_bits_to_f64(b)
        codes, s, m, bad = q4.quantize_group(b)
        assert not bad
        scale, least = oracle.bf16_bits_to_f64(np.array([s, m], np.uint16))
        assert least == v.min() and codes.min() == 0 and codes.max() in (14, 15)
        err = np.abs(codes * scale + least - v)
        assert err.max() <= scale / 2 * (1 + 1e-6)
        span = v.max() - v.min()
        assert span / 15 <= scale * (1 + 1e-6) and scale <= span / 15 * (1 + 2.0 ** -7) * (1 + 1e-6)


def test_quantiser_by_hand():
    # 0 .. 15 repeated: scale 1, codes the values themselves; halves in between tie to even
    codes, s, m, bad = q4.quantize_group(bits(list(range(16)) * 4))
    assert codes.tolist() == list(range(16)) * 4 and s == 0x3F80 and m == 0 and not bad
    x = [0.0, 15.0] + [k + 0.5 for k in range(15)] + [0.0] * 47
    codes, s, m, bad = q4.quantize_group(bits(x))
    assert s == 0x3F80 and codes[2:17].tolist() == [0, 2, 2, 4, 4, 6, 6, 8, 8, 10, 10, 12, 12, 14, 14]
    codes, s, m, bad = q4.quantize_group(bits([7.0] * 64))
    assert s == 0 and not codes.any() and m == 0x40E0
    for w in (np.nan, np.inf, -np.inf):
        assert q4.quantize_group(bits([w] + [1.0] * 63))[3]
    assert q4.quantize_group(np.array([0x7F7F, 0xFF7F] + [0] * 62, np.uint16))[3]  # the range leaves fp32
    assert q4.quantize_group(np.array([0x0001, 0x8001] + [0] * 62, np.uint16))[1:] == (0, 0, False)


def test_groups_next_to_the_largest_value_stay_finite():
    largest = 255 * 2.0 ** 120
    rng = np.random.default_rng(7)
    rows = [[0x7F7F, int(bits([-0.5 * 2.0 ** 120])[0])] + [0] * 62, [0x7F7F] + [0] * 63]
    for _ in range(200):
        low = int(bits([-2.0 ** rng.uniform(60, 119.9)])[0])
        rows.append([0x7F7F, low] + rng.integers(0x7000, 0x7F80, 62).tolist())
    down = 0
    for row in rows:
        b = np.array(row, np.uint16)
        v = oracle.bf16_bits_to_f64(b)
        codes, s, m, bad = q4.quantize_group(b)
        scale, least = oracle.bf16_bits_to_f64(np.array([s, m], np.uint16))
        got = codes * scale + least
        assert not bad and least == v.min() and got.max() < largest + 2.0 ** 119     # rounds to a finite bf16
        assert np.abs(got - v).max() <= scale / 2 * (1 + 2.0 ** -20)
        down += scale < (v.max() - v.min()) / 15
    assert down > 20


def test_pack_and_unpack_agree():
    rng = np.random.default_rng(1)
    for d in (64, 128):
        blk = np.zeros(18 * d, np.uint8)
        want = np.zeros((2, 16, d))
        for slot in rng.permutation(16):
            for which in range(2):
                row = bits(rng.standard_normal(d))
                q4.store_row(blk, which, int(slot), row)
                for g in range(d // 64):
                    c, s, m, _ = q4.quantize_group(row[g * 64:(g + 1) * 64])
                    sf, mf = oracle.bf16_bits_to_f64(np.array([s, m], np.uint16))
                    want[which, slot, g * 64:(g + 1) * 64] = c * sf + mf
        k, v = q4.block_values(blk, d)
        assert np.array_equal(k, want[0]) and np.array_equal(v, want[1])


def test_attention_oracle_agrees_with_the_bf16_oracle_on_values_bf16_holds():
    """Scales that are powers of two and minima that are multiples of them make every value a bf16 number."""
    rng = np.random.default_rng(2)
    d, Hq, Hkv, n = 64, 4, 2, 37
    kv4 = np.zeros((4, Hkv, 18 * d), np.uint8)
    table = np.array([[2, 0, 3]], np.int32)
    for page in range(4):
        for h in range(Hkv):
            kv4[page, h, :16 * d] = rng.integers(0, 256, 16 * d)
            rec = kv4[page, h, 16 * d:].view(np.uint16).reshape(16, 1, 4)
            rec[..., 0::2] = bits(2.0 ** rng.integers(-3, 1, (16, 1, 2)))
            rec[..., 1::2] = bits(-rng.integers(0, 8, (16, 1, 2)) / 8.0)
    k, v = np.zeros((4, Hkv, 16, d), np.uint16), np.zeros((4, Hkv, 16, d), np.uint16)
    for page in range(4):
        for h in range(Hkv):
            bk, bv = q4.block_values(kv4[page, h], d)
            k[page, h], v[page, h] = bits(bk), bits(bv)
            assert np.array_equal(oracle.bf16_bits_to_f64(k[page, h]), bk)
    q = bits(rng.standard_normal((1, Hq, d)))
    lens = np.array([n], np.int32)
    want, want_lse = oracle.decode_attn(q, k, v, table, lens, 0.125)
    out, lse, _, _ = q4.decode_attn(q, kv4, table, lens, 0.125)
    assert np.abs(out - want).max() < 1e-12 and np.abs(lse - want_lse).max() < 1e-12


def test_rope_oracle_by_hand():
    x = np.arange(1, 33, dtype=np.float64).reshape(1, 1, 32)
    axis, freq = [0] * 4 + [1] * 4, [np.pi / 2] * 8
    y, _ = q4.rope(x, np.array([[1], [2]]), freq, axis, 16, False)
    # a quarter turn: (a, b) -> (-b, a); a half turn: (-a, -b); the rest stays
    assert np.allclose(y[0, 0, :4], -x[0, 0, 8:12], atol=1e-6) and np.allclose(y[0, 0, 8:12], x[0, 0, :4], atol=1e-6)
    assert np.allclose(y[0, 0, 4:8], -x[0, 0, 4:8], atol=1e-5) and np.array_equal(y[0, 0, 16:], x[0, 0, 16:])
    y, _ = q4.rope(x, np.array([[1], [2]]), freq, axis, 16, True)
    assert np.allclose(y[0, 0, 0:8:2], -x[0, 0, 1:8:2], atol=1e-6) and np.allclose(y[0, 0, 1:8:2], x[0, 0, 0:8:2], atol=1e-6)


def test_fixed_point_turns_wrap_like_whole_turns():
    """The kernels' angle: position times a 64-bit fraction of a turn, modulo 2^64."""
    rng = np.random.default_rng(3)
    for f in np.float32(10000.0) ** (-np.arange(64, dtype=np.float64) / 64):
        turns = float(np.float32(f)) * 0.15915494309189533577
        fixed = int((turns - int(turns)) * 2.0 ** 64)
        for pos in [0, 1, -1, 2 ** 31 - 1, -2 ** 31, *rng.integers(-2 ** 31, 2 ** 31, 20).tolist()]:
            got = ((pos * fixed) % 2 ** 64) / 2.0 ** 64
            want = np.longdouble(pos) * np.longdouble(np.float32(f)) / (2 * np.arctan2(np.longdouble(0), np.longdouble(-1)))
            diff = float((np.longdouble(got) - want) - np.rint(np.longdouble(got) - want))
            assert abs(diff) < 2.0 ** -24, (f, pos, diff)


def test_entry_points_refuse_a_null_context():
    import paper_2609_35158_b200 as pd

    x = torch.zeros(64, dtype=torch.int32)
    rope = pd.rope_config(64, np.ones(32))
    calls = {
        "pd_kv_append_q4": (x, x, x, x, x, 1),
        "pd_kv_append_tokens_q4": (x, x, x, x, x, x, 1, 1),
        "pd_kv_dequantize_q4": (x, x, None, x, x, x, x, 1),
        "pd_decode_attn_q4": (x, x, x, x, x, x, 1, 1.0, 0),
        "pd_decode_step_q4": (x, x, x, x, x, x, x, x, 1, 1.0, 0),
        "pd_rope_tokens": (rope, x, x, x, x, x, 1),
        "pd_rope_append_tokens": (rope, x, x, x, x, x, x, x, x, x, x, 1, 1),
        "pd_rope_append_tokens_q4": (rope, x, x, x, x, x, x, x, x, x, 1, 1),
    }
    for name, args in calls.items():
        with pytest.raises(pd.PdError) as e:
            getattr(pd, name)(None, *args, stream=0)
        assert e.value.code == pd.PD_ERR_INVALID_ARG, name


def test_rope_config_checks_its_sequences():
    import paper_2609_35158_b200 as pd

    for bad in (dict(rot_dim=64, inv_freq=np.ones(31)), dict(rot_dim=256, inv_freq=np.ones(128)), dict(rot_dim=0, inv_freq=[]),
                dict(rot_dim=32, inv_freq=np.ones(16), axis_of_pair=[0] * 15), dict(rot_dim=32, inv_freq=np.ones(16), axis_of_pair=[-1] * 16)):
        with pytest.raises(ValueError):
            pd.rope_config(**bad)
    c = pd.rope_config(32, np.ones(16), axis_of_pair=[0] * 8 + [1] * 8, num_axes=2, adjacent=True, magnitude=0.5)
    assert (c.rot_dim, c.num_axes, c.adjacent, c.magnitude) == (32, 2, 1, 0.5) and list(c.axis_of_pair)[:16] == [0] * 8 + [1] * 8
    assert ctypes.sizeof(c) == 16 + 64 + 256
    with pytest.raises(ValueError):  # two axes, one row of positions
        pd.pd_rope_tokens(None, c, torch.zeros(4, dtype=torch.int32), *[torch.zeros(64)] * 4, total=4, stream=0)


def test_empty_tensors_do_not_pass_for_arguments_left_out():
    """The address of an empty tensor is null, which the library reads as an argument that was not given."""
    import paper_2609_35158_b200 as pd

    x, none = torch.zeros(64, dtype=torch.int32), torch.zeros(0, dtype=torch.int32)
    rope = pd.rope_config(64, np.ones(32), num_axes=2)
    rows = torch.zeros((2, 8), dtype=torch.int32)
    for positions in (rows[:, :0], torch.empty((2, 0), dtype=torch.int32)):
        with pytest.raises(ValueError):
            pd.pd_rope_append_tokens(None, rope, positions, x, x, x, x, x, x, x, x, x, 1, batch=1, stream=0)
        with pytest.raises(ValueError):
            pd.pd_rope_append_tokens_q4(None, rope, positions, x, x, x, x, x, x, x, x, 1, batch=1, stream=0)
    with pytest.raises(ValueError):
        pd.pd_kv_dequantize_q4(None, x, x, none, x, x, x, x, batch=1, stream=0)
    for call in (lambda: pd.pd_decode_attn_q4(None, x, x, x, x, x, none, batch=1, stream=0),
                 lambda: pd.pd_decode_step_q4(None, x, x, x, x, x, x, x, none, batch=1, stream=0)):
        with pytest.raises(ValueError):
            call()
    # a step without sequences or without tokens may come with empty tensors: the library answers
    for call in (lambda: pd.pd_rope_append_tokens(None, rope, rows[:, :0], x, x, x, x, x, x, x, x, x, 1, batch=0, stream=0),
                 lambda: pd.pd_rope_append_tokens_q4(None, rope, rows[:, :0], x, x, x, x, x, x, x, x, 0, batch=1, stream=0),
                 lambda: pd.pd_kv_dequantize_q4(None, x, x, none, x, x, x, x, batch=0, stream=0)):
        with pytest.raises(pd.PdError):
            call()


def test_frequencies_are_converted_to_turns_exactly():
    """The library's own conversion against integers: any sign and size, and the angle at any int32 position."""
    from test_gpu_rope import inv_two_pi
    import paper_2609_35158_b200 as pd

    bits_ = 400
    unit, rng = inv_two_pi(bits_), np.random.default_rng(8)
    freqs = [0.0, -0.0, 1.0, -1.0, 2.0 ** -126, 2.0 ** -149, -2.0 ** -140, 2.0 ** -40, 402.0, -402.0, np.pi, 2 * np.pi, 6.2831855, 1e-38]
    freqs += (2.0 ** rng.uniform(-130, 8.6, 300) * rng.choice([-1, 1], 300)).tolist()
    freqs += (10000.0 ** (-np.arange(64) / 64)).tolist()
    for f in np.array(freqs, np.float32):
        num, den = float(f).as_integer_ratio()
        got = pd.pd_rope_turns(float(f))
        assert 0 <= got < 2 ** 64
        for pos in [1, -1, 2 ** 31 - 1, -2 ** 31, *rng.integers(-2 ** 31, 2 ** 31, 5).tolist()]:
            whole = den << bits_                                              # one turn, in units of 2^-bits / den
            off = ((got * pos << bits_) * den - (num * unit * pos << 64)) % (whole << 64)
            off = min(off, (whole << 64) - off)                               # the shorter way round
            assert off <= abs(pos) * whole * 2, (f, pos)                      # 2^-63 turns for each position
    for bad in (float("nan"), float("inf"), 403.0, -403.0):
        with pytest.raises(pd.PdError):
            pd.pd_rope_turns(bad)
