"""Expanded K and V of shared latent vectors and the attention over them, through the C ABI, against the fp64 oracle."""
import numpy as np
import pytest
import torch

import oracle
from oracle import latent as ol
import workloads as wl
from test_gpu_latent import Latent, P, SCALE, cache_for, check, decode, f64, frequencies, indptr_of, queries
from test_gpu_q4 import dev, table_for

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
SCALE32 = float(np.float32(SCALE))


def weights(heads, seed):
    return (wl.random_bf16((heads, 256, 512), seed, DEV).float() * 512 ** -0.5).to(torch.bfloat16)


def expanded_pools(pages, heads, seed, fill):
    """K and V pools that start as `fill` (a number) or random values."""
    shape = (pages, heads, P, 128)
    if fill is None:
        return wl.random_bf16(shape, seed, DEV), wl.random_bf16(shape, seed + 1, DEV)
    return torch.full(shape, fill, dtype=torch.bfloat16, device=DEV), torch.full(shape, fill, dtype=torch.bfloat16, device=DEV)


def expand(ctx, w, pages, table, first, lens, k, v, to):
    ctx.pd.pd_kv_expand_latent(ctx.h, w, pages, dev(table), None if first is None else dev(np.asarray(first, np.int32)), dev(np.asarray(lens, np.int32)),
                               k, v, dev(to))
    torch.cuda.synchronize()


def check_expanded(k, v, to, ref, written_only=True, fill=7.0):
    got = [f64(k), f64(v)]
    touched = np.zeros(got[0].shape[:1] + (P,), bool)
    for b, (lo, kw, vw, ktol, vtol) in enumerate(ref):
        t = lo + np.arange(len(kw))
        page, slot = to[b, t // P], t % P
        touched[page, slot] = True
        for x, want, tol in ((got[0], kw, ktol), (got[1], vw, vtol)):
            assert np.all(np.abs(x[page, :, slot] - want) <= tol)
    for x in got:
        assert np.all(x.transpose(0, 2, 1, 3)[~touched] == fill)


@pytest.mark.parametrize("heads", [1, 5, 8, 33, 128])
@pytest.mark.parametrize("some_first", [False, True])
def test_expand_ragged(heads, some_first):
    lens = np.array([0, 1, 16, 17, 127, 128, 129, 0, 400, 300])
    first = np.minimum(np.array([0, 0, 3, 17, 100, 0, 127, 5, 130, 299]), lens) if some_first else None
    pages, table = cache_for(lens, heads)
    to, NP = table_for(lens, heads + 1)
    k, v = expanded_pools(NP, heads, 0, 7.0)
    w = weights(heads, heads + 2)
    with Latent(heads, len(lens), table.shape[1], pages.shape[0]) as ctx:
        expand(ctx, w, pages, table, first, lens, k, v, to)
        assert ctx.pd.pd_device_status(ctx.h)[0] == 0
    check_expanded(k, v, to, ol.expand(f64(w), np.nan_to_num(f64(pages)), table, lens, first))


def test_expand_many_and_long():
    rng = np.random.default_rng(1)
    for lens, heads in ((rng.integers(0, 60, 900), 3), (np.array([9000, 3, 4100]), 7)):
        pages, table = cache_for(lens, 2, poison=False)
        to, NP = table_for(lens, 3)
        k, v = expanded_pools(NP, heads, 0, 7.0)
        w = weights(heads, 4)
        with Latent(heads, len(lens), table.shape[1], pages.shape[0]) as ctx:
            expand(ctx, w, pages, table, None, lens, k, v, to)
        check_expanded(k, v, to, ol.expand(f64(w), f64(pages), table, lens))


def test_expand_skips_bad_pages_and_sequences():
    lens = [70, 50, 40, 33]
    pages, table = cache_for(lens, 5, cols=6)
    to, NP = table_for(lens, 6, cols=6)
    w = weights(4, 7)
    bad, bad_to = table.copy(), to.copy()
    bad[0, 1], bad_to[1, 2] = -4, NP + 3
    with Latent(4, 4, 6, pages.shape[0]) as ctx:
        k, v = expanded_pools(NP, 4, 0, 7.0)
        expand(ctx, w, pages, bad, None, lens, k, v, bad_to)
        code, seq, detail = ctx.pd.pd_device_status(ctx.h)
        assert code == ctx.pd.PD_ERR_DEVICE_FAULT and (seq, detail) in ((0, -4), (1, NP + 3))
        good_k, good_v = expanded_pools(NP, 4, 0, 7.0)
        expand(ctx, w, pages, table, None, lens, good_k, good_v, to)
        assert ctx.pd.pd_device_status(ctx.h)[0] == 0
        for x, y in ((k, good_k), (v, good_v)):
            y = y.clone()
            y[int(to[0, 1])] = y[int(to[1, 2])] = 7.0
            assert torch.equal(x, y)
        for first, ln, where in (([0, -1, 0, 0], lens, 1), (None, [70, 50, 97, 33], 2)):
            k, v = expanded_pools(NP, 4, 0, 7.0)
            expand(ctx, w, pages, table, first, ln, k, v, to)
            code, seq, _ = ctx.pd.pd_device_status(ctx.h)
            assert code == ctx.pd.PD_ERR_DEVICE_FAULT and seq == where
            y = good_k.clone()
            y[torch.from_numpy(to[where][to[where] >= 0].astype(np.int64)).to(DEV)] = 7.0
            assert torch.equal(k, y)


def poison_tails(pool, to, lens):
    for b, n in enumerate(lens):
        if n % P:
            pool[int(to[b, n // P]), :, n % P:] = float("nan")


def turn(before, new, heads, seed):
    """Inputs of one turn over random expanded pages, NaN in every slot past a context."""
    lens = np.asarray(before) + np.asarray(new)
    pages, table = cache_for(lens, seed)
    to, NP = table_for(lens, seed + 1)
    k, v = expanded_pools(NP, heads, seed + 2, None)
    for x in (k, v):
        poison_tails(x, to, lens)
        used = np.zeros(NP, bool)
        used[to[to >= 0]] = True
        x[torch.from_numpy(~used).to(DEV)] = float("nan")
    return lens, pages, table, to, k, v, queries((int(np.sum(new)), heads, 192), seed + 4)


def prefill(ctx, q, new, k, v, to, pages, table, lens, max_q=None, scale=SCALE, lse=True):
    out = torch.full(q.shape[:2] + (128,), float("nan"), dtype=torch.bfloat16, device=DEV)
    l = torch.full(q.shape[:2], float("nan"), dtype=torch.float32, device=DEV) if lse else None
    ctx.pd.pd_prefill_attn_latent(ctx.h, q, dev(indptr_of(new)), k, v, dev(to), pages, dev(table), dev(np.asarray(lens, np.int32)), out, l,
                                  max_q_len=int(max(new)) if max_q is None else max_q, sm_scale=scale)
    torch.cuda.synchronize()
    return out, l


@pytest.mark.parametrize("heads", [1, 5, 20])
@pytest.mark.parametrize("before,new", [([0, 5, 130], [1, 1, 1]), ([0, 0, 0, 0], [1, 127, 128, 129]), ([0, 1, 63, 200, 100], [300, 40, 256, 257, 0]),
                                        ([1000, 127, 128, 129], [1, 130, 128, 127]), ([2000], [777])])
def test_prefill_ragged(heads, before, new):
    lens, pages, table, to, k, v, q = turn(before, new, heads, heads + len(new))
    with Latent(heads, len(new), table.shape[1], pages.shape[0]) as ctx:
        out, lse = prefill(ctx, q, new, k, v, to, pages, table, lens)
        assert ctx.pd.pd_device_status(ctx.h)[0] == 0
        out2, _ = prefill(ctx, q, new, k, v, to, pages, table, lens, max_q=int(max(new)) + 600, lse=False)
        assert torch.equal(out, out2)
    check(out, lse, ol.prefill(f64(q), indptr_of(new), np.nan_to_num(f64(k)), np.nan_to_num(f64(v)), to, np.nan_to_num(f64(pages)), table, lens, SCALE32))


@pytest.mark.parametrize("batch", [32, 33, 70])
def test_prefill_many_sequences(batch):
    """Up to 32 sequences the blocks rank them by themselves, beyond that a small kernel does; rows behind the last one stay."""
    rng = np.random.default_rng(batch)
    before, new = rng.integers(0, 90, batch), rng.integers(0, 60, batch)
    new[0] = 200
    lens, pages, table, to, k, v, q = turn(before, new, 2, batch)
    used = batch - 3
    with Latent(2, batch, table.shape[1], pages.shape[0]) as ctx:
        out, lse = prefill(ctx, q, new, k, v, to, pages, table, lens)
        part, _ = prefill(ctx, q, new[:used], k, v, to, pages, table, lens)
    n = int(new[:used].sum())
    assert torch.equal(part[:n], out[:n]) and torch.isnan(part[n:]).all()
    check(out, lse, ol.prefill(f64(q), indptr_of(new), np.nan_to_num(f64(k)), np.nan_to_num(f64(v)), to, np.nan_to_num(f64(pages)), table, lens, SCALE32))


@pytest.mark.parametrize("batch", [20, 45])
def test_prefill_more_items_than_blocks(batch):
    """Long turns among single tokens and sequences without any; calls of other shapes of the same context in between."""
    rng = np.random.default_rng(batch)
    before, new = rng.integers(0, 200, batch), rng.integers(0, 3, batch)
    new[[3, 11]] = 600, 257
    lens, pages, table, to, k, v, q = turn(before, new, 40, batch)
    with Latent(40, batch, table.shape[1], pages.shape[0]) as ctx:
        out, lse = prefill(ctx, q, new, k, v, to, pages, table, lens)
        one, _ = prefill(ctx, q, new[:1], k, v, to, pages, table, lens)
        again, _ = prefill(ctx, q, new, k, v, to, pages, table, lens)
        assert ctx.pd.pd_device_status(ctx.h)[0] == 0
    assert torch.equal(out, again) and torch.equal(one[:new[0]], out[:new[0]])
    check(out, lse, ol.prefill(f64(q), indptr_of(new), np.nan_to_num(f64(k)), np.nan_to_num(f64(v)), to, np.nan_to_num(f64(pages)), table, lens, SCALE32))


@pytest.mark.parametrize("heads,before,new", [(1, [9000], [1]), (8, [6000], [300]), (32, [4000], [128]), (5, [5000, 0, 40], [130, 600, 0]),
                                              (3, [20000], [129]), (2, [1300, 2600, 10], [1, 1, 1]), (16, [0], [2304])])
def test_prefill_few_items_on_long_contexts(heads, before, new):
    """Contexts are cut into stretches whose partial results are joined: the same bits in every call, whatever ran in between."""
    lens, pages, table, to, k, v, q = turn(before, new, heads, heads)
    with Latent(heads, len(new), table.shape[1], pages.shape[0]) as ctx:
        out, lse = prefill(ctx, q, new, k, v, to, pages, table, lens)
        other = np.asarray(lens) - np.asarray(new) // 2
        prefill(ctx, q, np.asarray(new) - np.asarray(new) // 2, k, v, to, pages, table, other)
        again, lse2 = prefill(ctx, q, new, k, v, to, pages, table, lens, max_q=int(max(new)) + 5)
        assert torch.equal(out, again) and torch.equal(lse, lse2) and ctx.pd.pd_device_status(ctx.h)[0] == 0
    check(out, lse, ol.prefill(f64(q), indptr_of(new), np.nan_to_num(f64(k)), np.nan_to_num(f64(v)), to, np.nan_to_num(f64(pages)), table, lens, SCALE32))


def test_prefill_logits_that_rise_and_jump():
    new, before = [300], [500]
    for name in ("rise", "jump"):
        lens, pages, table, to, k, v, q = turn(before, new, 6, 11)
        t = np.arange(800)
        drift = t / 10.0 if name == "rise" else np.where(t % 97 == 96, 3.0 * t, 0.0)
        x = pages.view(-1, 576)
        at = torch.from_numpy((table[0].repeat(P) * P + np.tile(np.arange(P), table.shape[1]))[:800].astype(np.int64)).to(DEV)
        x[at, 575] = torch.from_numpy(drift).to(DEV).to(torch.bfloat16)
        q[..., 191] = torch.tensor([1.0, 0.0, -1.0, 2.0, 0.5, 0.25], device=DEV).to(torch.bfloat16)
        with Latent(6, 1, table.shape[1], pages.shape[0]) as ctx:
            out, lse = prefill(ctx, q, new, k, v, to, pages, table, lens, scale=0.2)
        ref = ol.prefill(f64(q), indptr_of(new), np.nan_to_num(f64(k)), np.nan_to_num(f64(v)), to, np.nan_to_num(f64(pages)), table, lens, float(np.float32(0.2)))
        check(out, lse, ref)


def test_prefill_faults_are_latched():
    lens, pages, table, to, k, v, q = turn([30, 20], [40, 50], 4, 13)
    with Latent(4, 2, table.shape[1], pages.shape[0]) as ctx:
        good, _ = prefill(ctx, q, [40, 50], k, v, to, pages, table, lens)
        for which, at, val in ((0, (0, 1), -9), (1, (0, 2), 10 ** 6)):
            tables = [table.copy(), to.copy()]
            tables[which][at] = val
            out, _ = prefill(ctx, q, [40, 50], k, v, tables[1], pages, tables[0], lens)
            code, seq, detail = ctx.pd.pd_device_status(ctx.h)
            assert code == ctx.pd.PD_ERR_DEVICE_FAULT and seq == 0 and detail == val
            assert torch.equal(out[40:], good[40:])
        out, _ = prefill(ctx, q, [40, 50], k, v, to, pages, table, [39, 70])     # the cache does not hold the new tokens
        code, seq, _ = ctx.pd.pd_device_status(ctx.h)
        assert code == ctx.pd.PD_ERR_DEVICE_FAULT and seq == 0 and torch.equal(out[40:], good[40:])


def test_prefill_capture():
    lens, pages, table, to, k, v, q = turn([300, 10], [200, 90], 8, 15)
    w = weights(8, 16)
    with Latent(8, 2, table.shape[1], pages.shape[0]) as ctx:
        t, u, n, ip = dev(table), dev(to), dev(lens.astype(np.int32)), dev(indptr_of([200, 90]))
        out = torch.empty((290, 8, 128), dtype=torch.bfloat16, device=DEV)

        def both():
            ctx.pd.pd_kv_expand_latent(ctx.h, w, pages, t, None, n, k, v, u)
            ctx.pd.pd_prefill_attn_latent(ctx.h, q, ip, k, v, u, pages, t, n, out, max_q_len=200, sm_scale=SCALE)

        both()
        torch.cuda.synchronize()
        want = out.clone()
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            both()
        out.zero_(), k.zero_(), v.zero_()
        g.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, want)


def test_two_contexts_on_two_streams():
    """Blocks of both calls share the SMs; neither waits for the other's."""
    H, sides = 8, []
    for n, (before, new) in enumerate((([7000, 20], [200, 300]), ([900, 0, 33], [130, 1, 513]))):
        lens, pages, table, to, k, v, q = turn(before, new, H, 40 + n)
        ctx = Latent(H, len(new), table.shape[1], pages.shape[0])
        out = torch.empty((int(np.sum(new)), H, 128), dtype=torch.bfloat16, device=DEV)
        args = (q, dev(indptr_of(new)), k, v, dev(to), pages, dev(table), dev(lens.astype(np.int32)), out)
        sides.append((ctx, args, int(max(new)), torch.cuda.Stream()))
    want = []
    for ctx, args, m, _ in sides:
        ctx.pd.pd_prefill_attn_latent(ctx.h, *args, max_q_len=m, sm_scale=SCALE)
        torch.cuda.synchronize()
        want.append(args[-1].clone())
        args[-1].zero_()
    torch.cuda.synchronize()
    for _ in range(20):
        for ctx, args, m, stream in sides:
            ctx.pd.pd_prefill_attn_latent(ctx.h, *args, max_q_len=m, sm_scale=SCALE, stream=stream)
    torch.cuda.synchronize()
    for (ctx, args, _, _), x in zip(sides, want):
        assert torch.equal(args[-1], x) and ctx.pd.pd_device_status(ctx.h)[0] == 0
        ctx.pd.pd_destroy(ctx.h)


def test_expanded_pages_past_4_gb():
    """The last pages of pools of 5.2 GB each give what the first ones do."""
    H, NP = 64, 20000
    lens, new = np.asarray([70, 300], np.int32), [20, 260]
    pages, table = cache_for(lens, 31)
    w, q = weights(H, 32), queries((280, H, 192), 33)
    k, v = (torch.empty((NP, H, P, 128), dtype=torch.bfloat16, device=DEV) for _ in range(2))
    got = []
    with Latent(H, 2, table.shape[1], pages.shape[0]) as ctx:
        for at in (0, NP - 2 * table.shape[1]):
            to = (at + np.arange(2 * table.shape[1], dtype=np.int32)).reshape(2, -1)
            expand(ctx, w, pages, table, None, lens, k, v, to)
            got.append(prefill(ctx, q, new, k, v, to, pages, table, lens))
        assert ctx.pd.pd_device_status(ctx.h)[0] == 0
    assert torch.equal(got[0][0], got[1][0]) and torch.equal(got[0][1], got[1][1]) and torch.isfinite(got[0][0]).all()


def test_refusals():
    import paper_2609_35158_b200 as pd

    lens, pages, table, to, k, v, q = turn([3], [5], 4, 17)
    w, t, u, n, ip = weights(4, 18), dev(table), dev(to), dev(lens.astype(np.int32)), dev(indptr_of([5]))
    out = torch.empty((5, 4, 128), dtype=torch.bfloat16, device=DEV)

    def refused(code, f, *a, **kw):
        with pytest.raises(pd.PdError) as e:
            f(*a, **kw)
        assert e.value.code == code

    with Latent(4, 1, table.shape[1], pages.shape[0]) as ctx:
        inv, uns = pd.PD_ERR_INVALID_ARG, pd.PD_ERR_UNSUPPORTED
        ex, pf = pd.pd_kv_expand_latent, pd.pd_prefill_attn_latent
        refused(inv, ex, ctx.h, None, pages, t, None, n, k, v, u)
        refused(inv, ex, ctx.h, w, pages, t, None, n, k, v.view(-1)[8:], u)
        refused(inv, ex, ctx.h, w, pages, t, None, n, k, v, None)
        refused(inv, ex, ctx.h, w, pages, t, None, n, k, v, u, batch=2)
        refused(inv, ex, ctx.h, w, pages, t, None, n, k[:0], v, u)
        refused(inv, pf, ctx.h, q, ip, k, v, u, pages, t, n, out, max_q_len=-1)
        refused(inv, pf, ctx.h, q, ip, k, v, u, pages, t, n, out, max_q_len=5, sm_scale=-1.0)
        refused(inv, pf, ctx.h, q, None, k, v, u, pages, t, n, out, max_q_len=5, batch=1)
        with pytest.raises(ValueError):
            ex(ctx.h, w, pages, t, n[:0], n, k, v, u)
        plain = pd.pd_create(8, 8, 64, P, 1, 3, 4, 0)
        try:
            refused(uns, ex, plain, w, pages, t, None, n, k, v, u)
            refused(uns, pf, plain, q, ip, k, v, u, pages, t, n, out, max_q_len=5)
        finally:
            pd.pd_destroy(plain)
        assert pd.pd_device_status(ctx.h)[0] == 0


def test_a_turn_and_steps_in_both_forms():
    """A turn as a program runs it: append, expand, prefill; then a decode step in the absorbed form, whose output times W_v is
    that of the expanded form over the same cache."""
    import paper_2609_35158_b200 as pd

    heads, before, new = 12, np.array([0, 37]), np.array([70, 140])
    lens = before + new
    pages, table = cache_for(lens + 1, 21, poison=False)
    to, NP = table_for(lens + 1, 22)
    k, v = expanded_pools(NP, heads, 0, 0.0)
    w = weights(heads, 23)
    rope = pd.rope_config(64, frequencies(64))
    total = int(new.sum())
    kv_new, q = wl.random_bf16((total, 576), 24, DEV), queries((total, heads, 192), 25)
    n, one = dev(before.astype(np.int32)), dev(np.arange(3, dtype=np.int32))
    t, u, ip = dev(table), dev(to), dev(indptr_of(new))
    out = torch.empty((total, heads, 128), dtype=torch.bfloat16, device=DEV)
    lse = torch.empty((total, heads), dtype=torch.float32, device=DEV)
    with Latent(heads, 2, table.shape[1], pages.shape[0]) as ctx:
        h = ctx.h
        pd.pd_rope_append_tokens_latent(h, rope, None, q[..., 128:], kv_new, None, 0.0, ip, q[..., 128:], pages, t, n, int(new.max()))
        pd.pd_kv_expand_latent(h, w, pages, t, None, n, k, v, u)
        pd.pd_prefill_attn_latent(h, q, ip, k, v, u, pages, t, n, out, lse, max_q_len=int(new.max()), sm_scale=SCALE)
        torch.cuda.synchronize()
        assert np.array_equal(n.cpu().numpy(), lens)
        check(out, lse, ol.prefill(f64(q), indptr_of(new), f64(k), f64(v), to, f64(pages), table, lens, SCALE32))
        # a decode step of one more token per sequence
        kv1, q1 = wl.random_bf16((2, 576), 26, DEV), queries((2, heads, 192), 27)
        absorbed = torch.zeros((2, heads, 576), dtype=torch.bfloat16, device=DEV)
        absorbed[..., :512] = torch.einsum("hdl,bhd->bhl", w[:, :128].float(), q1[..., :128].float()).to(torch.bfloat16)
        pd.pd_rope_append_tokens_latent(h, rope, None, q1[..., 128:], kv1, None, 0.0, one, absorbed[..., 512:], pages, t, n, 1)
        lat, lse1 = torch.empty((2, heads, 512), dtype=torch.bfloat16, device=DEV), torch.empty((2, heads), dtype=torch.float32, device=DEV)
        pd.pd_decode_attn_latent(h, absorbed, pages, t, n, lat, lse1, sm_scale=SCALE)
        torch.cuda.synchronize()
        assert pd.pd_device_status(h)[0] == 0
    want = ol.decode(f64(absorbed), f64(pages), table, lens + 1, SCALE32)
    check(lat, lse1, want)
    wf = f64(w)
    kx, vx = np.zeros((NP, heads, P, 128)), np.zeros((NP, heads, P, 128))
    for b, (_, kk, vv, _, _) in enumerate(ol.expand(wf, f64(pages), table, lens + 1)):
        pos = np.arange(len(kk))
        kx[to[b, pos // P], :, pos % P], vx[to[b, pos // P], :, pos % P] = kk, vv
    q64 = np.concatenate([f64(q1)[..., :128], f64(absorbed)[..., 512:]], -1)
    exp, lse2, _, _ = ol.prefill(q64, [0, 1, 2], kx, vx, to, f64(pages), table, lens + 1, SCALE32)
    # the absorbed query was rounded to bf16: its logits move by at most 2^-8 of the sum of magnitudes
    move = max(ol.BF16 * SCALE32 * (np.abs(f64(absorbed)[b, :, :512]) @ np.abs(ol.rows_of(f64(pages), table[b], lens[b] + 1)[:, :512]).T).max()
               for b in range(2))
    assert np.all(np.abs(lse1.double().cpu().numpy() - lse2) <= move + 1e-3)
    got = np.einsum("hdl,bhl->bhd", wf[:, 128:], f64(lat))
    spread = np.einsum("hdl,bhl->bhd", np.abs(wf[:, 128:]), np.maximum(want[2], 0)) + 2.1 * move * 2 * np.abs(vx).max()   # sum p |v - out| is at most 2 max |v|
    assert np.all(np.abs(got - exp) <= spread)
