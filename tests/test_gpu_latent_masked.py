"""Shared latent vectors whose first tokens have logits far below the others', as left padding or a mask in the key part gives them."""
import numpy as np
import pytest
import torch

from oracle import latent as ol
import workloads as wl
from test_gpu_latent import DEV, Latent, P, cache_for, check, decode, f64
from test_gpu_latent_prefill import prefill, turn

pytestmark = pytest.mark.gpu

# Logits are one product each, exact in fp32; what is left are the roundings of scale * log2(e), of differences below 2^5 and of 2^x: less
# than 2^-18 of a logit's unit.
SHIFT = 2.0 ** -18
FACTORS = (1.0, 0.5, 0.25)          # what the heads multiply every logit by
LOW_AND_BASE = [(-np.inf, 0), (-np.inf, 400), (-np.inf, -400), (-1e38, 0), (-1e38, 400), (-1e9, -400), (-1e8, 0), (-1e5, 0)]


def masked_rows(rows, n_low, low, base, seed):
    """Rows [n][576] whose first n_low tokens have the logit `low` and the others base plus one of -2, 0, 4, 6, through the key part alone."""
    n = rows.shape[0]
    logit = torch.from_numpy(base + np.random.default_rng(seed).choice([-2.0, 0.0, 4.0, 6.0], n)).to(rows.dtype)
    logit[:n_low] = low
    rows[:, 512:] = 0.0
    rows[:, 512] = logit.to(rows.device)
    return logit.double().numpy()


def factors(heads):
    return np.resize(FACTORS, heads)


def attend(z, v, own_sum):
    """(out, lse, out bound, lse bound) of one query's logits z [H][n], -inf not in every place, over v [n][D] or per head [H][n][D]."""
    out, lse, bound = [], [], []
    for h in range(len(z)):
        top = z[h].max()
        e = np.exp(z[h] - top)
        o, b = ol._attend((e / e.sum())[None], v if v.ndim == 2 else v[h], np.array([SHIFT]), own_sum)
        out.append(o[0]), bound.append(b[0]), lse.append(top + np.log(e.sum()))
    lse = np.array(lse)
    return np.array(out), lse, np.array(bound), SHIFT + 2.0 ** -18 + 2.0 ** -21 * np.abs(lse)


@pytest.mark.parametrize("heads", [3, 20, 40, 100])
@pytest.mark.parametrize("low,base", LOW_AND_BASE)
def test_decode_behind_low_logits(heads, low, base):
    n_low = [0, 1, 63, 64, 65, 130, 299]
    lens = [300] * len(n_low)
    pages, table = cache_for(lens, heads)
    q = torch.zeros((len(lens), heads, 576), dtype=torch.bfloat16, device=DEV)
    q[..., 512] = torch.from_numpy(factors(heads)).to(DEV)
    ref = []
    for b, k in enumerate(n_low):
        at = torch.from_numpy((table[b].repeat(P) * P + np.tile(np.arange(P), table.shape[1]))[:300].astype(np.int64)).to(DEV)
        rows = pages.view(-1, 576)[at]
        logit = masked_rows(rows, k, low, base, b)
        pages.view(-1, 576)[at] = rows
        ref.append(attend(factors(heads)[:, None] * logit[None], f64(rows)[:, :512], True))
    with Latent(heads, len(lens), table.shape[1], pages.shape[0]) as ctx:
        for split in (0, 4, 7, 19, 40):            # from one tile a segment to whole sequences
            out, lse = decode(ctx, q, pages, table, lens, scale=1.0, split=split)
            check(out, lse, tuple(np.stack(x) for x in zip(*ref)))
        assert ctx.pd.pd_device_status(ctx.h)[0] == 0


@pytest.mark.parametrize("before,n_low,new", [([200] * 6, [0, 79, 80, 81, 160, 199], [70] * 6), ([2100, 1500], [1900, 700], [33, 150])])
@pytest.mark.parametrize("low,base", LOW_AND_BASE)
def test_prefill_behind_low_logits(before, n_low, new, low, base):
    heads = 3
    lens, pages, table, to, k, v, q = turn(before, new, heads, 3)
    q.zero_()
    q[..., 128] = torch.from_numpy(factors(heads)).to(DEV)
    ref = []
    for b, n in enumerate(lens):
        at = torch.from_numpy((table[b].repeat(P) * P + np.tile(np.arange(P), table.shape[1]))[:n].astype(np.int64)).to(DEV)
        rows = pages.view(-1, 576)[at]
        logit = masked_rows(rows, n_low[b], low, base, b)
        pages.view(-1, 576)[at] = rows
        ids = torch.from_numpy(to[b, :-(-n // P)].astype(np.int64)).to(DEV)
        values = f64(v[ids].transpose(0, 1).reshape(heads, -1, 128)[:, :n].contiguous())
        for i in range(int(before[b]), n):
            ref.append(attend(factors(heads)[:, None] * logit[None, :i + 1], values[:, :i + 1], False))
    ref = tuple(np.stack(x) for x in zip(*ref))
    with Latent(heads, len(new), table.shape[1], pages.shape[0]) as ctx:
        for max_q in (max(new), 1000000):                   # the kernel that cuts contexts, and the one that does not
            out, lse = prefill(ctx, q, new, k, v, to, pages, table, lens, max_q=max_q, scale=1.0)
            check(out, lse, ref)
        assert ctx.pd.pd_device_status(ctx.h)[0] == 0


def huge_rows(rows, size, seed):
    """Rows whose logits are `size` or the next bf16 value below it (half of each), or `size` alone where the seed is even."""
    n = rows.shape[0]
    logit = torch.full((n,), size, dtype=rows.dtype)
    if seed % 2:
        logit[np.random.default_rng(seed).permutation(n)[:n // 2]] = size * (1 - np.sign(size) * 2.0 ** -7)
    rows[:, 512:] = 0.0
    rows[:, 512] = logit.to(rows.device)
    return logit.double().numpy()


@pytest.mark.parametrize("size", [-1e38, -1e30, -1e10, -3e9, 3e9, 1e10, 1e30, 1e38])
def test_decode_of_huge_logits(size):
    """Only their differences count: equal ones share the weight, however large they are."""
    heads, lens = 20, [300, 300, 50, 50, 1, 150]
    pages, table = cache_for(lens, heads)
    q = torch.zeros((len(lens), heads, 576), dtype=torch.bfloat16, device=DEV)
    q[..., 512] = torch.from_numpy(factors(heads)).to(DEV)
    ref = []
    for b, n in enumerate(lens):
        at = torch.from_numpy((table[b].repeat(P) * P + np.tile(np.arange(P), table.shape[1]))[:n].astype(np.int64)).to(DEV)
        rows = pages.view(-1, 576)[at]
        logit = huge_rows(rows, size, b)
        pages.view(-1, 576)[at] = rows
        ref.append(attend(factors(heads)[:, None] * logit[None], f64(rows)[:, :512], True))
    with Latent(heads, len(lens), table.shape[1], pages.shape[0]) as ctx:
        for split in (0, 7, 40):
            out, lse = decode(ctx, q, pages, table, lens, scale=1.0, split=split)
            check(out, lse, tuple(np.stack(x) for x in zip(*ref)))
        assert ctx.pd.pd_device_status(ctx.h)[0] == 0


@pytest.mark.parametrize("size", [-1e38, -1e30, -1e10, -3e9, 3e9, 1e10, 1e30, 1e38])
def test_prefill_of_huge_logits(size):
    heads, before, new = 3, [0, 50, 2500], [90, 140, 20]
    lens, pages, table, to, k, v, q = turn(before, new, heads, 5)
    q.zero_()
    q[..., 128] = torch.from_numpy(factors(heads)).to(DEV)
    ref = []
    for b, n in enumerate(lens):
        at = torch.from_numpy((table[b].repeat(P) * P + np.tile(np.arange(P), table.shape[1]))[:n].astype(np.int64)).to(DEV)
        rows = pages.view(-1, 576)[at]
        logit = huge_rows(rows, size, b)
        pages.view(-1, 576)[at] = rows
        ids = torch.from_numpy(to[b, :-(-n // P)].astype(np.int64)).to(DEV)
        values = f64(v[ids].transpose(0, 1).reshape(heads, -1, 128)[:, :n].contiguous())
        for i in range(int(before[b]), n):
            ref.append(attend(factors(heads)[:, None] * logit[None, :i + 1], values[:, :i + 1], False))
    ref = tuple(np.stack(x) for x in zip(*ref))
    with Latent(heads, len(new), table.shape[1], pages.shape[0]) as ctx:
        for max_q in (max(new), 1000000):
            out, lse = prefill(ctx, q, new, k, v, to, pages, table, lens, max_q=max_q, scale=1.0)
            check(out, lse, ref)
        assert ctx.pd.pd_device_status(ctx.h)[0] == 0


def test_decode_of_sequences_masked_altogether():
    """Every logit -inf: as an empty context, zeros and a logarithm of -inf; its neighbours are not touched."""
    heads, lens, gone = 20, [300, 40, 300, 1, 130], [True, False, False, True, True]
    pages, table = cache_for(lens, heads)
    q = torch.zeros((len(lens), heads, 576), dtype=torch.bfloat16, device=DEV)
    q[..., 512] = torch.from_numpy(factors(heads)).to(DEV)
    ref = []
    for b, n in enumerate(lens):
        at = torch.from_numpy((table[b].repeat(P) * P + np.tile(np.arange(P), table.shape[1]))[:n].astype(np.int64)).to(DEV)
        rows = pages.view(-1, 576)[at]
        logit = masked_rows(rows, n if gone[b] else 0, -np.inf, 0, b)
        pages.view(-1, 576)[at] = rows
        zeros = (np.zeros((heads, 512)), np.full(heads, -np.inf), np.zeros((heads, 512)), np.zeros(heads))
        ref.append(zeros if gone[b] else attend(factors(heads)[:, None] * logit[None], f64(rows)[:, :512], True))
    with Latent(heads, len(lens), table.shape[1], pages.shape[0]) as ctx:
        for split in (0, 1, 7, 40):
            out, lse = decode(ctx, q, pages, table, lens, scale=1.0, split=split)
            check(out, lse, tuple(np.stack(x) for x in zip(*ref)))
        assert ctx.pd.pd_device_status(ctx.h)[0] == 0


@pytest.mark.parametrize("before,n_low,new", [([0, 0, 100], [30, 200, 0], [90, 200, 5]), ([2000, 0], [2300, 10], [300, 20])])
def test_prefill_of_rows_masked_altogether(before, n_low, new):
    """Rows that see -inf alone, ahead of rows that see more: zeros and a logarithm of -inf."""
    heads = 3
    lens, pages, table, to, k, v, q = turn(before, new, heads, 7)
    q.zero_()
    q[..., 128] = torch.from_numpy(factors(heads)).to(DEV)
    ref = []
    for b, n in enumerate(lens):
        at = torch.from_numpy((table[b].repeat(P) * P + np.tile(np.arange(P), table.shape[1]))[:n].astype(np.int64)).to(DEV)
        rows = pages.view(-1, 576)[at]
        logit = masked_rows(rows, n_low[b], -np.inf, 0, b)
        pages.view(-1, 576)[at] = rows
        ids = torch.from_numpy(to[b, :-(-n // P)].astype(np.int64)).to(DEV)
        values = f64(v[ids].transpose(0, 1).reshape(heads, -1, 128)[:, :n].contiguous())
        zeros = (np.zeros((heads, 128)), np.full(heads, -np.inf), np.zeros((heads, 128)), np.zeros(heads))
        for i in range(int(before[b]), n):
            ref.append(zeros if i < n_low[b] else attend(factors(heads)[:, None] * logit[None, :i + 1], values[:, :i + 1], False))
    ref = tuple(np.stack(x) for x in zip(*ref))
    with Latent(heads, len(new), table.shape[1], pages.shape[0]) as ctx:
        for max_q in (max(new), 1000000):
            out, lse = prefill(ctx, q, new, k, v, to, pages, table, lens, max_q=max_q, scale=1.0)
            check(out, lse, ref)
        assert ctx.pd.pd_device_status(ctx.h)[0] == 0
