"""The cache of shared latent vectors through the C ABI: append and absorbed decode attention against the fp64 oracle."""
import numpy as np
import pytest
import torch

import oracle
from oracle import latent as ol
import workloads as wl
from test_gpu_q4 import dev, table_for

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
P = 16
SCALE = 192 ** -0.5


def f64(t):
    return oracle.bf16_bits_to_f64(oracle.bf16_bits(t))


class Latent:
    """Context manager around a PD_FLAG_LATENT context."""

    def __init__(self, heads, max_batch, MP, NP):
        import paper_2609_35158_b200 as pd

        self.pd = pd
        self.h = pd.pd_create(heads, 1, 512, P, max_batch, MP, NP, 0, pd.PD_FLAG_LATENT)

    def __enter__(self):
        return self

    def __exit__(self, *exc):
        self.pd.pd_destroy(self.h)
        return False


def cache_for(lens, seed, slack=3, cols=None, poison=True):
    """(pages bf16 [NP][16][576], table): NaN in every slot that holds no token."""
    table, NP = table_for(lens, seed, slack, cols)
    pages = wl.random_bf16((NP, P, ol.ROW), seed + 100, DEV)
    if poison:
        free = torch.ones((NP, P), dtype=torch.bool)
        for b, n in enumerate(lens):
            for t0 in range(0, int(n), P):
                free[table[b, t0 // P], :min(P, int(n) - t0)] = False
        pages[free.to(DEV)] = float("nan")
    return pages, table


def queries(shape, seed):
    return wl.random_bf16(shape, seed, DEV)


def decode(ctx, q, pages, table, lens, scale=SCALE, split=0, lse=True, stream=None):
    out = torch.full(q.shape[:2] + (512,), float("nan"), dtype=torch.bfloat16, device=DEV)
    l = torch.full(q.shape[:2], float("nan"), dtype=torch.float32, device=DEV) if lse else None
    ctx.pd.pd_decode_attn_latent(ctx.h, q, pages, dev(table), dev(np.asarray(lens, np.int32)), out, l, sm_scale=scale, split_pages=split,
                                 stream=stream)
    torch.cuda.synchronize()
    return out, l


def check(out, lse, ref):
    want, wlse, bound, lbound = ref
    got = f64(out)
    assert np.all(np.abs(got - want) <= bound), np.max(np.abs(got - want) / np.maximum(bound, 1e-30))
    if lse is not None:
        got = lse.double().cpu().numpy()
        empty = np.isinf(wlse)
        assert np.array_equal(np.isneginf(got), empty)
        assert np.all(np.abs(got[~empty] - wlse[~empty]) <= lbound[~empty])


RAGGED = [0, 1, 15, 16, 17, 63, 64, 65, 0, 129, 300, 1000]


@pytest.mark.parametrize("heads", [1, 7, 16, 20, 32, 33, 64, 65, 100, 128])
@pytest.mark.parametrize("split", [0, 1, 3, 40])
def test_decode_ragged(heads, split):
    pages, table = cache_for(RAGGED, heads)
    q = queries((len(RAGGED), heads, 576), heads + 1)
    scale = float(np.float32(SCALE))
    with Latent(heads, len(RAGGED), table.shape[1], pages.shape[0]) as ctx:
        out, lse = decode(ctx, q, pages, table, RAGGED, split=split)
        assert ctx.pd.pd_device_status(ctx.h)[0] == 0
    check(out, lse, ol.decode(f64(q), np.nan_to_num(f64(pages)), table, RAGGED, scale))


def test_one_token_returns_its_latent():
    """p = 1 whatever the logit: the weight's rounding cancels against the sum of rounded weights."""
    lens = [1, 1, 1]
    pages, table = cache_for(lens, 5)
    q = queries((3, 24, 576), 6) * 3
    with Latent(24, 3, 1, pages.shape[0]) as ctx:
        out, lse = decode(ctx, q, pages, table, lens)
    rows = pages[torch.from_numpy(table[:, 0].astype(np.int64)).to(DEV), 0]
    assert torch.equal(out, rows[:, None, :512].expand(3, 24, 512))
    want = SCALE * (q.double() @ rows.double()[:, :, None])[..., 0]
    assert torch.all((lse.double() - want).abs() <= 2.0 ** -15 * SCALE * (q.double().abs() @ rows.double().abs()[:, :, None])[..., 0] + 1e-5)


def test_results_do_not_depend_on_pages_or_time():
    lens = [700, 33, 5000, 64]
    pages, table = cache_for(lens, 7)
    q = queries((4, 40, 576), 8)
    with Latent(40, 4, table.shape[1], pages.shape[0]) as ctx:
        out, lse = decode(ctx, q, pages, table, lens)
        for seed in range(3):
            perm = np.random.default_rng(seed).permutation(pages.shape[0])
            moved = torch.empty_like(pages)
            moved[torch.from_numpy(perm).to(DEV)] = pages
            out2, lse2 = decode(ctx, q, moved, np.where(table >= 0, perm[table], -1).astype(np.int32), lens)
            assert torch.equal(out, out2) and torch.equal(lse, lse2)


@pytest.mark.parametrize("heads", [5, 64, 128])
def test_logits_that_rise_fall_and_jump(heads):
    """The running reference is raised in the middle of a segment, by a little and by hundreds, for some heads and not for others."""
    n = 2000
    rng = np.random.default_rng(heads)
    for name in ("rise", "fall", "jump"):
        pages, table = cache_for([n], 9)
        t = np.arange(n)
        drift = {"rise": t / 12.0, "fall": (n - t) / 12.0, "jump": np.where(t == 1500, 290.0, 0.0)}[name]
        rows = f64(pages)[table[0]].reshape(-1, 576)
        rows[:n, 512] = drift                      # the last part of the key carries the drift
        flat = torch.from_numpy(rows.astype(np.float32)).to(torch.bfloat16).view(-1, P, 576).to(DEV)
        pages[torch.from_numpy(table[0].astype(np.int64)).to(DEV)] = flat
        q = queries((1, heads, 576), 10).float() * 0.3
        q[..., 512] = torch.from_numpy(rng.choice([-1.0, 0.0, 1.0, 2.0], heads)).to(DEV)
        q = q.to(torch.bfloat16)
        with Latent(heads, 1, table.shape[1], pages.shape[0]) as ctx:
            for split in (0, 1000):
                out, lse = decode(ctx, q, pages, table, [n], scale=1.0, split=split)
                check(out, lse, ol.decode(f64(q), np.nan_to_num(f64(pages)), table, [n], 1.0))


def test_long_contexts():
    lens = [65536, 40001, 7, 33333]
    pages, table = cache_for(lens, 11)
    q = queries((4, 12, 576), 12)
    with Latent(12, 4, table.shape[1], pages.shape[0]) as ctx:
        for split in (0, 4096):
            out, lse = decode(ctx, q, pages, table, lens, split=split)
            check(out, lse, ol.decode(f64(q), np.nan_to_num(f64(pages)), table, lens, float(np.float32(SCALE))))


def test_many_sequences():
    """More sequences than workers: whole ones, cut ones and empty ones in one range."""
    rng = np.random.default_rng(13)
    lens = rng.integers(0, 200, 700)
    lens[::9] = 0
    pages, table = cache_for(lens, 13)
    q = queries((700, 8, 576), 14)
    with Latent(8, 700, table.shape[1], pages.shape[0]) as ctx:
        for split in (0, 5):
            out, lse = decode(ctx, q, pages, table, lens, split=split)
            check(out, lse, ol.decode(f64(q), np.nan_to_num(f64(pages)), table, lens, float(np.float32(SCALE))))


@pytest.mark.parametrize("batch", [31, 128, 129, 300])
def test_batches_around_the_plan_by_one_warp(batch):
    """Up to 128 sequences every warp derives the ranges, beyond that the block: empty sequences first, last and between."""
    rng = np.random.default_rng(batch)
    lens = rng.integers(1, 400, batch)
    lens[[0, 1, batch // 2, batch - 1]] = 0
    pages, table = cache_for(lens, batch)
    q = queries((batch, 9, 576), batch + 1)
    with Latent(9, batch, table.shape[1], pages.shape[0]) as ctx:
        ref = ol.decode(f64(q), np.nan_to_num(f64(pages)), table, lens, float(np.float32(SCALE)))
        for split in (0, 17, 2 ** 31 - 1):
            out, lse = decode(ctx, q, pages, table, lens, split=split)
            check(out, lse, ref)
        plan = ctx.pd.pd_last_plan(ctx.h)
        assert plan["total_units"] == int(((lens + P - 1) // P).sum()) and plan["num_ranges"] == 1


def test_rows_behind_the_last_sequence_stay():
    import paper_2609_35158_b200 as pd

    lens = [70, 9, 300]
    pages, table = cache_for(lens, 27, poison=False)
    q = queries((3, 20, 576), 28)
    out = torch.full((3, 20, 512), 5.0, dtype=torch.bfloat16, device=DEV)
    lse = torch.full((3, 20), 5.0, device=DEV)
    with Latent(20, 8, table.shape[1], pages.shape[0]) as ctx:
        want, _ = decode(ctx, q[:2].contiguous(), pages, table[:2], lens[:2])
        pd.pd_decode_attn_latent(ctx.h, q, pages, dev(table), dev(np.asarray(lens, np.int32)), out, lse, batch=2, sm_scale=SCALE)
        torch.cuda.synchronize()
        assert torch.equal(out[:2], want) and torch.all(out[2] == 5.0) and torch.all(lse[2] == 5.0) and torch.isfinite(lse[:2]).all()
        # an append of the first two sequences' rows: the third one's, its length and its queries stay
        kv_new, q_rope = wl.random_bf16((6, 576), 29, DEV), wl.random_bf16((6, 20, 64), 30, DEV)
        q_out, before, n = torch.full_like(q_rope, 5.0), pages.clone(), dev(np.array([60, 3, 290], np.int32))
        pd.pd_rope_append_tokens_latent(ctx.h, pd.rope_config(64, frequencies(64)), None, q_rope, kv_new, None, 0.0, dev(indptr_of([2, 1, 3])), q_out,
                                        pages, dev(table), n, 2, batch=2)
        torch.cuda.synchronize()
        assert n.cpu().tolist() == [62, 4, 290] and torch.all(q_out[3:] == 5.0) and not torch.any(q_out[:3] == 5.0)
        used = torch.from_numpy(table[2][table[2] >= 0].astype(np.int64)).to(DEV)
        assert torch.equal(pages[used], before[used])


def test_all_empty_and_no_lse():
    pages, table = cache_for([0, 0], 15)
    q = queries((2, 33, 576), 16)
    with Latent(33, 2, 1, pages.shape[0]) as ctx:
        out, lse = decode(ctx, q, pages, table, [0, 0])
        assert torch.all(out == 0) and torch.all(torch.isneginf(lse))
        pages, table = cache_for([9, 3], 15)
        with Latent(33, 2, 1, pages.shape[0]) as ctx2:
            out, lse = decode(ctx2, q, pages, table, [9, 3])
            out2, _ = decode(ctx2, q, pages, table, [9, 3], lse=False)
            assert torch.equal(out, out2)


def test_a_nan_row_reaches_its_sequence_only():
    lens = [100, 300, 50]
    pages, table = cache_for(lens, 17)
    pages[table[1, 9], 3, 17] = float("nan")
    q = queries((3, 20, 576), 18)
    with Latent(20, 3, table.shape[1], pages.shape[0]) as ctx:
        out, lse = decode(ctx, q, pages, table, lens)
    assert torch.isnan(out[1]).all() and torch.isnan(lse[1]).all()
    assert torch.isfinite(out[0].float()).all() and torch.isfinite(out[2].float()).all()


def test_bad_pages_and_lengths_are_latched():
    lens = [100, 40]
    pages, table = cache_for(lens, 19, cols=8)
    q = queries((2, 20, 576), 20)
    with Latent(20, 2, 8, pages.shape[0]) as ctx:
        good, _ = decode(ctx, q, pages, table, lens)
        bad = table.copy()
        bad[0, 2] = pages.shape[0] + 7
        out, _ = decode(ctx, q, pages, bad, lens)
        code, seq, detail = ctx.pd.pd_device_status(ctx.h)
        assert code == ctx.pd.PD_ERR_DEVICE_FAULT and seq == 0 and detail == pages.shape[0] + 7
        assert torch.equal(out[1], good[1])
        out, _ = decode(ctx, q, pages, table, [-5, 40])
        code, seq, detail = ctx.pd.pd_device_status(ctx.h)
        assert code == ctx.pd.PD_ERR_DEVICE_FAULT and seq == 0 and detail == -5
        # (the lengths decide where the other sequence is cut, so not bit for bit)
        check(out, None, ol.decode(f64(q), np.nan_to_num(f64(pages)), table, [0, 40], float(np.float32(SCALE))))
        again, _ = decode(ctx, q, pages, table, lens)
        assert torch.equal(again, good) and ctx.pd.pd_device_status(ctx.h)[0] == 0


def test_pages_past_4_gb():
    NP = 250000                                     # 4.6 GB
    lens = [200, 77]
    pages = torch.empty((NP, P, 576), dtype=torch.bfloat16, device=DEV)
    small, table = cache_for(lens, 21)
    n = small.shape[0]
    pages[NP - n:] = small
    high = np.where(table >= 0, table + NP - n, -1).astype(np.int32)
    q = queries((2, 64, 576), 22)
    with Latent(64, 2, table.shape[1], NP) as ctx, Latent(64, 2, table.shape[1], n) as near:
        a, b = decode(ctx, q, pages, high, lens), decode(near, q, small, table, lens)
    assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1])


def test_capture_replay_and_two_streams():
    lens = [900, 31, 2500]
    pages, table = cache_for(lens, 23)
    q, q2 = queries((3, 48, 576), 24), queries((3, 48, 576), 25)
    t, n = dev(table), dev(np.asarray(lens, np.int32))
    with Latent(48, 3, table.shape[1], pages.shape[0]) as one, Latent(48, 3, table.shape[1], pages.shape[0]) as two:
        want, want2 = decode(one, q, pages, table, lens)[0], decode(one, q2, pages, table, lens)[0]
        a, b = torch.empty_like(want), torch.empty_like(want)
        s1, s2 = torch.cuda.Stream(), torch.cuda.Stream()
        for _ in range(5):
            one.pd.pd_decode_attn_latent(one.h, q, pages, t, n, a, sm_scale=SCALE, stream=s1)
            two.pd.pd_decode_attn_latent(two.h, q2, pages, t, n, b, sm_scale=SCALE, stream=s2)
        torch.cuda.synchronize()
        assert torch.equal(a, want) and torch.equal(b, want2)
        a.zero_()
        g = torch.cuda.CUDAGraph()
        torch.cuda.synchronize()
        with torch.cuda.graph(g):
            one.pd.pd_decode_attn_latent(one.h, q, pages, t, n, a, sm_scale=SCALE)
        g.replay()
        torch.cuda.synchronize()
        assert torch.equal(a, want)
        q.copy_(q2)
        g.replay()
        torch.cuda.synchronize()
        assert torch.equal(a, want2)


# ---------------------------------------------------------------- append

def frequencies(rot, base=10000.0):
    return (base ** (-np.arange(rot // 2) * 2.0 / rot)).astype(np.float32)


def indptr_of(new):
    return np.concatenate([[0], np.cumsum(new)]).astype(np.int32)


@pytest.mark.parametrize("heads,rot,adjacent,axes,norm,given", [(5, 64, False, 1, True, True), (20, 64, True, 1, True, False), (64, 32, False, 3, False, True),
                                                                (128, 16, True, 2, True, True), (1, 48, False, 4, True, True)])
@pytest.mark.parametrize("new", [[1, 1, 1], [0, 37, 300, 5]])
def test_append(heads, rot, adjacent, axes, norm, given, new):
    import paper_2609_35158_b200 as pd

    new = np.asarray(new)
    rng = np.random.default_rng(heads + rot)
    before = rng.integers(0, 90, len(new))
    total, indptr = int(new.sum()), indptr_of(new)
    pages, table = cache_for(before + new, heads, poison=False)
    start = pages.clone()
    wide = wl.random_bf16((total, 640), heads + 2, DEV) * 2
    kv_new = wide[:, 64:]                                            # a row stride of 640
    q = wl.random_bf16((total, heads, 192), heads + 3, DEV)
    q_out = torch.full((total, heads, 576), 7.0, dtype=torch.bfloat16, device=DEV)
    weight = (1 + 0.2 * torch.randn(512, device=DEV)).to(torch.bfloat16) if norm else None
    axis = rng.integers(0, axes, rot // 2)
    own = np.concatenate([b + np.arange(n) for b, n in zip(before, new)])
    pos = rng.integers(-2000000, 2000000, (axes, total)).astype(np.int32) if given else np.broadcast_to(own, (axes, total)).astype(np.int32)
    lens = dev(before.astype(np.int32))
    rope = pd.rope_config(rot, frequencies(rot), axis, axes, adjacent, 1.5)
    with Latent(heads, len(new), table.shape[1], pages.shape[0]) as ctx:
        pd.pd_rope_append_tokens_latent(ctx.h, rope, dev(pos) if given else None, q[..., 128:], kv_new, weight, 1e-5, dev(indptr), q_out[..., 512:],
                                        pages, dev(table), lens, int(new.max()))
        torch.cuda.synchronize()
        assert pd.pd_device_status(ctx.h)[0] == 0
        assert np.array_equal(lens.cpu().numpy(), before + new)
        # in place
        q2, pages2 = q.clone(), start.clone()
        lens2 = dev(before.astype(np.int32))
        pd.pd_rope_append_tokens_latent(ctx.h, rope, dev(pos) if given else None, q2[..., 128:], kv_new, weight, 1e-5, dev(indptr), q2[..., 128:],
                                        pages2, dev(table), lens2, int(new.max()), call_flags=pd.PD_APPEND_NO_ADVANCE)
        torch.cuda.synchronize()
        assert np.array_equal(lens2.cpu().numpy(), before)
    assert torch.equal(pages2, pages) and torch.equal(q2[..., :128], q[..., :128]) and torch.equal(q2[..., 128:], q_out[..., 512:])
    assert torch.all(q_out[..., :512] == 7.0)
    want, tol = ol.append_rows(f64(kv_new), None if weight is None else f64(weight), float(np.float32(1e-5)), pos, frequencies(rot), axis, rot, adjacent, 1.5)
    at = np.concatenate([table[b, (before[b] + np.arange(n)) // P] * P + (before[b] + np.arange(n)) % P for b, n in enumerate(new)])
    got = f64(pages).reshape(-1, 576)
    assert np.all(np.abs(got[at] - want) <= tol + ol.BF16 * (np.abs(want) + tol))
    rest = np.ones(len(got), bool)
    rest[at] = False
    assert np.array_equal(got[rest], f64(start).reshape(-1, 576)[rest])
    if not norm:
        assert np.array_equal(got[at][:, :512], f64(kv_new)[:, :512])
    qw, qtol = ol.q4.rope(f64(q)[..., 128:], pos, frequencies(rot), axis, rot, adjacent, 1.5)
    assert np.all(np.abs(f64(q_out)[..., 512:] - qw) <= qtol + ol.BF16 * (np.abs(qw) + qtol))


def test_append_edges():
    """No queries; a sequence without room and one with a bad page are latched, the others written; rows past the positions."""
    import paper_2609_35158_b200 as pd

    new, before = np.array([3, 2, 4]), np.array([0, 31, 10])
    indptr = indptr_of(new)
    table = np.array([[0, 1], [2, 3], [-1, 5]], np.int32)
    kv_new = wl.random_bf16((9, 576), 31, DEV)
    rope = pd.rope_config(64, frequencies(64))
    q = wl.random_bf16((9, 4, 64), 32, DEV)
    with Latent(4, 3, 2, 6) as ctx:
        pages, lens, q_out = torch.zeros((6, P, 576), dtype=torch.bfloat16, device=DEV), dev(before.astype(np.int32)), torch.zeros_like(q)
        pd.pd_rope_append_tokens_latent(ctx.h, rope, None, q, kv_new, None, 0.0, dev(indptr), q_out, pages, dev(table), lens, 4)
        torch.cuda.synchronize()
        code, seq, _ = pd.pd_device_status(ctx.h)
        assert code == pd.PD_ERR_DEVICE_FAULT and seq in (1, 2)
        assert lens.cpu().tolist()[:2] == [3, 31]
        assert torch.equal(pages[0, :3, :512], kv_new[:3, :512]) and not pages[1:].any()
        assert q_out.view(9, -1).any(1).all()                    # every sequence's queries are rotated
        pages2, lens2 = torch.zeros_like(pages), dev(np.array([0, 0, 0], np.int32))
        table2 = np.array([[0, 1], [2, 3], [4, 5]], np.int32)
        pd.pd_rope_append_tokens_latent(ctx.h, rope, None, None, kv_new, None, 0.0, dev(indptr), None, pages2, dev(table2), lens2, 4)
        torch.cuda.synchronize()
        assert pd.pd_device_status(ctx.h)[0] == 0 and lens2.cpu().tolist() == [3, 2, 4]
        assert torch.equal(pages2[4, :4, :512], kv_new[5:, :512])
        short = dev(np.zeros((1, 5), np.int32))
        pages3, lens3 = torch.zeros_like(pages), dev(np.array([0, 0, 0], np.int32))
        pd.pd_rope_append_tokens_latent(ctx.h, rope, short, None, kv_new, None, 0.0, dev(indptr), None, pages3, dev(table2), lens3, 4)
        torch.cuda.synchronize()
        code, seq, _ = pd.pd_device_status(ctx.h)
        assert code == pd.PD_ERR_DEVICE_FAULT and seq == 2 and lens3.cpu().tolist() == [3, 2, 0] and not pages3[4:].any()


def test_refusals():
    import paper_2609_35158_b200 as pd

    pages, table = cache_for([40], 33)
    q, out = queries((1, 20, 576), 34), torch.empty((1, 20, 512), dtype=torch.bfloat16, device=DEV)
    t, n, ip = dev(table), dev(np.array([40], np.int32)), dev(np.array([0, 1], np.int32))
    rope, kv_new = pd.rope_config(64, frequencies(64)), wl.random_bf16((1, 576), 35, DEV)

    def refused(code, f, *a, **k):
        with pytest.raises(pd.PdError) as e:
            f(*a, **k)
        assert e.value.code == code

    with Latent(20, 1, 3, pages.shape[0]) as ctx:
        inv, uns = pd.PD_ERR_INVALID_ARG, pd.PD_ERR_UNSUPPORTED
        at = pd.pd_decode_attn_latent
        refused(inv, at, ctx.h, q, pages, t, n, out, sm_scale=0.0)
        refused(inv, at, ctx.h, q, pages, t, n, out, sm_scale=float("nan"))
        refused(inv, at, ctx.h, q, pages, t, n, out, split_pages=-1)
        refused(inv, at, ctx.h, q, pages, t, n, out, batch=2)
        refused(inv, at, ctx.h, q.view(-1)[1:], pages, t, n, out, batch=1)
        refused(inv, at, ctx.h, None, pages, t, n, out, batch=1)
        ap = pd.pd_rope_append_tokens_latent
        refused(inv, ap, ctx.h, rope, None, None, kv_new, None, -1.0, ip, None, pages, t, n, 1)
        refused(inv, ap, ctx.h, rope, None, q[..., 512:], kv_new, None, 0.0, ip, None, pages, t, n, 1)
        refused(inv, ap, ctx.h, rope, None, None, kv_new, None, 0.0, ip, None, pages, t, n, 1, call_flags=2)
        refused(inv, ap, ctx.h, pd.rope_config(128, frequencies(128)), None, None, kv_new, None, 0.0, ip, None, pages, t, n, 1)
        refused(uns, ap, ctx.h, pd.rope_config(24, frequencies(24)), None, None, kv_new, None, 0.0, ip, None, pages, t, n, 1)
        with pytest.raises(ValueError):
            ap(ctx.h, rope, None, None, kv_new[:, :512], None, 0.0, ip, None, pages, t, n, 1)
        # the other caches' calls refuse this context, and these calls any other
        k = torch.zeros((4, 8, P, 64), dtype=torch.bfloat16, device=DEV)
        qq = torch.zeros((1, 8, 64), dtype=torch.bfloat16, device=DEV)
        refused(uns, pd.pd_decode_attn, ctx.h, qq, k, k, t, n, qq)
        refused(uns, pd.pd_kv_append, ctx.h, qq, qq, k, k, t, n)
        refused(uns, pd.pd_prefill_attn, ctx.h, qq, ip, k, k, t, n, qq, max_q_len=1)
        refused(uns, pd.pd_rope_tokens, ctx.h, rope, n, qq, qq, qq, qq)
        refused(uns, pd.pd_kv_quantize_pages, ctx.h, k, k, n, k, k, k)
        plain = pd.pd_create(8, 8, 64, P, 1, 3, 4, 0)
        try:
            refused(uns, at, plain, q, pages, t, n, out)
            refused(uns, ap, plain, rope, None, None, kv_new, None, 0.0, ip, None, pages, t, n, 1)
        finally:
            pd.pd_destroy(plain)
        assert pd.pd_device_status(ctx.h)[0] == 0


def test_a_run_of_steps():
    """Append and attend as a program does, lengths growing on the device, against the oracle's own cache."""
    import paper_2609_35158_b200 as pd

    heads, steps, lens = 24, 20, np.array([0, 14, 100])
    pages, table = cache_for(lens + steps, 41, poison=False)
    rope, freq = pd.rope_config(64, frequencies(64), adjacent=True), frequencies(64)
    weight = (1 + 0.1 * torch.randn(512, device=DEV)).to(torch.bfloat16)
    ctx_lens, ip = dev(lens.astype(np.int32)), dev(np.arange(4, dtype=np.int32))
    q, out = torch.empty((3, heads, 576), dtype=torch.bfloat16, device=DEV), torch.empty((3, heads, 512), dtype=torch.bfloat16, device=DEV)
    mirror = f64(pages)
    with Latent(heads, 3, table.shape[1], pages.shape[0]) as ctx:
        for i in range(steps):
            kv_new = wl.random_bf16((3, 576), 50 + i, DEV)
            q.copy_(wl.random_bf16((3, heads, 576), 80 + i, DEV))
            pd.pd_rope_append_tokens_latent(ctx.h, rope, None, q[..., 512:], kv_new, weight, 1e-6, ip, q[..., 512:], pages, dev(table), ctx_lens, 1)
            pd.pd_decode_attn_latent(ctx.h, q, pages, dev(table), ctx_lens, out, sm_scale=SCALE)
            torch.cuda.synchronize()
            want, tol = ol.append_rows(f64(kv_new), f64(weight), float(np.float32(1e-6)), (lens + i)[None], freq, [0] * 32, 64, True)
            got = f64(pages)
            for b in range(3):
                at = (table[b, (lens[b] + i) // P], (lens[b] + i) % P)
                assert np.all(np.abs(got[at] - want[b]) <= tol[b] + ol.BF16 * (np.abs(want[b]) + tol[b]))
                mirror[at] = got[at]
            check(out, None, ol.decode(f64(q), mirror, table, lens + i + 1, float(np.float32(SCALE))))
        assert pd.pd_device_status(ctx.h)[0] == 0
    assert np.array_equal(f64(pages), mirror)
