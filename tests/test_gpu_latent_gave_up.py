"""What a latent prefill that gave up a wait leaves in the workspace does not reach the calls that follow."""
import numpy as np
import pytest
import torch

from oracle import latent as ol
from test_gpu_latent import Latent, check, f64, indptr_of
from test_gpu_latent_prefill import SCALE32, prefill, turn

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("heads,before,new", [(8, [6000], [300]), (1, [9000], [1]), (5, [5000, 0, 40], [130, 600, 0])])
def test_prefill_after_a_call_that_gave_up(heads, before, new):
    lens, pages, table, to, k, v, q = turn(before, new, heads, heads)
    ref = ol.prefill(f64(q), indptr_of(new), np.nan_to_num(f64(k)), np.nan_to_num(f64(v)), to, np.nan_to_num(f64(pages)), table, lens, SCALE32)
    with Latent(heads, len(new), table.shape[1], pages.shape[0]) as ctx:
        pd = ctx.pd
        for stretches, before_any in ((2, True), (1, False), (3, False), (65535, False)):
            pd.pd_leave_arrivals(ctx.h, stretches)
            if stretches == 3:                                   # an earlier fault that nobody has read yet
                bad = table.copy()
                bad[0, 0] = -7
                prefill(ctx, q, new, k, v, to, pages, bad, lens)
                pd.pd_leave_arrivals(ctx.h, stretches)
            out, lse = prefill(ctx, q, new, k, v, to, pages, table, lens)
            check(out, lse, ref)
            if before_any:
                want, wlse = out, lse
            assert torch.equal(out, want) and torch.equal(lse, wlse)
        assert pd.pd_device_status(ctx.h)[0] == pd.PD_ERR_DEVICE_FAULT and pd.pd_device_status(ctx.h)[0] == 0


def test_refusals():
    import paper_2609_35158_b200 as pd

    with Latent(4, 1, 1, 1) as ctx:
        with pytest.raises(pd.PdError) as e:
            pd.pd_leave_arrivals(ctx.h, -1)
        assert e.value.code == pd.PD_ERR_INVALID_ARG
    plain = pd.pd_create(8, 8, 64, 16, 1, 3, 4, 0)
    try:
        with pytest.raises(pd.PdError) as e:
            pd.pd_leave_arrivals(plain, 0)
        assert e.value.code == pd.PD_ERR_UNSUPPORTED
    finally:
        pd.pd_destroy(plain)
