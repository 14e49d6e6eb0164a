"""max_q_len as a caller gives it who knows no bound: results are those of the exact one."""
import numpy as np
import pytest
import torch

import workloads as wl
from pd_testlib import Ctx
from test_gpu_latent import Latent, cache_for, frequencies
from test_gpu_latent_prefill import prefill, turn
from test_gpu_q4 import dev, table_for
from test_gpu_rope import packed

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
P = 16
BOUNDS = [2 ** 31 - 1, 2 ** 31 - 7, 2 ** 31 - 200, 2 ** 30]


@pytest.mark.parametrize("bound", BOUNDS)
def test_latent_append(bound):
    import paper_2609_35158_b200 as pd

    heads, before, new = 5, np.array([3, 40, 0]), np.array([20, 1, 33])
    pages, table = cache_for(before + new, 1, poison=False)
    total, indptr = int(new.sum()), np.concatenate([[0], np.cumsum(new)]).astype(np.int32)
    kv_new, q = wl.random_bf16((total, 576), 2, DEV), wl.random_bf16((total, heads, 64), 3, DEV)
    rope = pd.rope_config(64, frequencies(64))
    got = []
    with Latent(heads, 3, table.shape[1], pages.shape[0]) as ctx:
        for most in (33, bound):
            kv, lens, out = pages.clone(), dev(before.astype(np.int32)), torch.empty_like(q)
            pd.pd_rope_append_tokens_latent(ctx.h, rope, None, q, kv_new, None, 0.0, dev(indptr), out, kv, dev(table), lens, most)
            torch.cuda.synchronize()
            got.append((kv, lens, out))
        assert pd.pd_device_status(ctx.h)[0] == 0
    assert all(torch.equal(a, b) for a, b in zip(*got)) and got[1][1].cpu().tolist() == [23, 41, 33]


@pytest.mark.parametrize("bound", BOUNDS)
@pytest.mark.parametrize("four", [False, True])
def test_rotary_append(bound, four):
    import paper_2609_35158_b200 as pd

    Hq, Hkv, d, before, new = 8, 2, 128, np.array([3, 40, 0], np.int32), np.array([20, 1, 33], np.int32)
    indptr, pos, q, k, v = packed(before, new, 4, Hq, Hkv, d, 1)
    table, NP = table_for(before + new, 5)
    rope, got = pd.rope_config(d, frequencies(d)), []
    with Ctx(Hq, Hkv, d, 3, table.shape[1], NP) as ctx:
        for most in (33, bound):
            lens, out = dev(before), torch.empty_like(q)
            if four:
                pools = [torch.zeros((NP, Hkv, 18 * d), dtype=torch.uint8, device=DEV)]
                pd.pd_rope_append_tokens_q4(ctx.h, rope, dev(pos), q, k, v, dev(indptr), out, pools[0], dev(table), lens, most)
            else:
                pools = [torch.zeros((NP, Hkv, P, d), dtype=torch.bfloat16, device=DEV) for _ in range(2)]
                pd.pd_rope_append_tokens(ctx.h, rope, dev(pos), q, k, v, dev(indptr), out, *pools, dev(table), lens, most)
            torch.cuda.synchronize()
            got.append((*pools, lens, out))
        assert pd.pd_device_status(ctx.h)[0] == 0
    assert all(torch.equal(a, b) for a, b in zip(*got)) and got[1][-2].cpu().tolist() == [23, 41, 33]


@pytest.mark.parametrize("bound", BOUNDS)
def test_latent_prefill(bound):
    lens, pages, table, to, k, v, q = turn([100, 0], [40, 300], 3, 6)
    with Latent(3, 2, table.shape[1], pages.shape[0]) as ctx:
        want = prefill(ctx, q, [40, 300], k, v, to, pages, table, lens)
        got = prefill(ctx, q, [40, 300], k, v, to, pages, table, lens, max_q=bound)
        assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1]) and ctx.pd.pd_device_status(ctx.h)[0] == 0
