"""Lengths that the page table cannot hold, in the latent calls: the sequence is left out and latched, its neighbours are right."""
import numpy as np
import pytest
import torch

import workloads as wl
from test_gpu_latent import DEV, Latent, cache_for, frequencies, indptr_of
from test_gpu_latent_prefill import prefill, turn
from test_gpu_q4 import dev

pytestmark = pytest.mark.gpu


def bad_lengths(columns):
    return [16 * columns + 1, 2 ** 31 - 1, 2 ** 31 - 5, -1, -2 ** 31]


@pytest.mark.parametrize("batch", [3, 40])
@pytest.mark.parametrize("which", range(5))
def test_prefill(batch, which):
    before, new = np.full(batch, 20), np.full(batch, 30)
    lens, pages, table, to, k, v, q = turn(before, new, 2, batch)
    bad = lens.copy()
    bad[1] = bad_lengths(table.shape[1])[which]
    with Latent(2, batch, table.shape[1], pages.shape[0]) as ctx:
        want, wlse = prefill(ctx, q, new, k, v, to, pages, table, lens)
        assert ctx.pd.pd_device_status(ctx.h)[0] == 0
        out, lse = prefill(ctx, q, new, k, v, to, pages, table, bad)
        code, seq, detail = ctx.pd.pd_device_status(ctx.h)
    assert code == ctx.pd.PD_ERR_DEVICE_FAULT and seq == 1 and detail == bad[1]
    rest = torch.ones(len(q), dtype=torch.bool, device=DEV)
    rest[30:60] = False
    assert torch.equal(out[rest], want[rest]) and torch.equal(lse[rest], wlse[rest])
    assert torch.isnan(out[~rest]).all() and torch.isnan(lse[~rest]).all()


@pytest.mark.parametrize("which", range(5))
def test_append(which):
    import paper_2609_35158_b200 as pd

    before, new, heads = np.array([5, 0, 9]), np.array([3, 20, 4]), 4
    table = np.arange(6, dtype=np.int32).reshape(3, 2)
    lens = before.copy()
    lens[1] = bad_lengths(2)[which]
    kv_new, q = wl.random_bf16((27, 576), 1, DEV), wl.random_bf16((27, heads, 64), 2, DEV)
    pages, n, out = torch.zeros((6, 16, 576), dtype=torch.bfloat16, device=DEV), dev(lens.astype(np.int32)), torch.zeros_like(q)
    with Latent(heads, 3, 2, 6) as ctx:
        pd.pd_rope_append_tokens_latent(ctx.h, pd.rope_config(64, frequencies(64)), None, q, kv_new, None, 0.0, dev(indptr_of(new)), out, pages, dev(table),
                                        n, 20)
        assert pd.pd_device_status(ctx.h) == (pd.PD_ERR_DEVICE_FAULT, 1, int(lens[1]))
    assert n.cpu().tolist() == [8, int(lens[1]), 13]
    assert torch.nonzero(pages.flatten(1).any(1)).flatten().tolist() == [0, 4]
    assert out.view(27, -1).any(1).all()                         # its queries are rotated all the same
