"""Cut contexts of the latent prefill whose last stretch only the second tile of an item sees."""
import numpy as np
import pytest
import torch

from oracle import latent as ol
from test_gpu_latent import Latent, check, f64, indptr_of
from test_gpu_latent_prefill import SCALE32, prefill, turn

BLOCK, ITEM, TILE = 80, 256, 128


def stretches(before, new, heads, sms):
    """The plan of the kernel that cuts contexts, restated: (sequence, head, first token, stretch, blocks of both tiles) of every item."""
    before, new = [int(x) for x in before], [int(x) for x in new]
    assert len(new) <= 32 and -(-max(new) // ITEM) * heads * len(new) <= 2 * sms          # else no context is cut
    blocks = lambda b, start: (before[b] + min(start + ITEM, new[b]) - 1) // BLOCK + 1
    tiles = [(b, start) for b in range(len(new)) for start in range(0, new[b], ITEM)]
    longest, chunk = max(blocks(*x) for x in tiles), 0
    if longest >= 16:
        fair, whole = -(-sum(blocks(*x) for x in tiles) * heads // sms), len(tiles) * heads
        best, c = longest if whole <= sms else max(longest, fair + longest // 2), max(fair, 8)
        while c < longest:
            pieces = sum(-(-blocks(*x) // c) for x in tiles) * heads
            est = max(c, 0 if pieces <= sms else fair + c // 2 + 4) + 4 + longest // c
            if pieces <= 2 * sms and est < best:
                best, chunk = est, c
            if c > best:
                break
            c += (c + 3) // 4
    items = []
    for b, start in tiles:
        nb = blocks(b, start)
        parts = -(-nb // chunk) if chunk else 1
        size, n_tok = -(-nb // parts), min(ITEM, new[b] - start)
        for left in range(parts):
            first = (before[b] + start + min(n_tok, TILE) - 1) // BLOCK + 1 - left * size
            nb0, nb1 = min(max(first, 0), size), min(max(nb - left * size, 0), size) if n_tok > TILE else 0
            assert nb0 or nb1
            items += [(b, h, start, left, nb0, nb1) for h in range(heads)]
    return items


SHAPES = [(1, [4300], [200]), (2, [6192], [417]), (2, [4339, 931], [151, 418])]


def test_the_shapes_have_such_a_stretch():
    for heads, before, new in SHAPES:
        items = stretches(before, new, heads, 148)
        assert any(nb0 == 0 and nb1 > 0 for *_, nb0, nb1 in items) and any(nb0 > 0 and nb1 > 0 for *_, nb0, nb1 in items)


@pytest.mark.gpu
def test_cut_contexts_replayed():
    """A captured call and eager ones of the same context in turn: each counts its stretches afresh."""
    heads, before, new = SHAPES[1]
    lens, pages, table, to, k, v, q = turn(before, new, heads, 9)
    args = [torch.from_numpy(np.ascontiguousarray(x, dtype=np.int32)).to(q.device) for x in (indptr_of(new), to, table, lens)]
    out = torch.empty(q.shape[:2] + (128,), dtype=torch.bfloat16, device=q.device)
    with Latent(heads, 1, table.shape[1], pages.shape[0]) as ctx:
        want, _ = prefill(ctx, q, new, k, v, to, pages, table, lens)
        few, _ = prefill(ctx, q, [33], k, v, to, pages, table, [5000])

        def call():
            ctx.pd.pd_prefill_attn_latent(ctx.h, q, args[0], k, v, args[1], pages, args[2], args[3], out, max_q_len=new[0], sm_scale=SCALE32)

        call()
        torch.cuda.synchronize()
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            call()
            call()
        for i in range(5):
            out.zero_()
            g.replay()
            if i % 2:
                assert torch.equal(prefill(ctx, q, [33], k, v, to, pages, table, [5000])[0][:33], few[:33])
            torch.cuda.synchronize()
            assert torch.equal(out, want)
        assert ctx.pd.pd_device_status(ctx.h)[0] == 0


@pytest.mark.gpu
@pytest.mark.parametrize("heads,before,new", SHAPES)
def test_a_stretch_that_only_the_second_tile_sees(heads, before, new):
    """The first tile's barriers and parities are left alone in it, and what it contributes to the join is nothing."""
    items = stretches(before, new, heads, torch.cuda.get_device_properties(0).multi_processor_count)
    assert any(nb0 == 0 and nb1 > 0 for *_, nb0, nb1 in items)
    lens, pages, table, to, k, v, q = turn(before, new, heads, heads)
    with Latent(heads, len(new), table.shape[1], pages.shape[0]) as ctx:
        out, lse = prefill(ctx, q, new, k, v, to, pages, table, lens)
        shorter = [max(n - 70, 0) for n in new]                  # a call with other stretches in between
        prefill(ctx, q, shorter, k, v, to, pages, table, np.asarray(before) + shorter)
        again, lse2 = prefill(ctx, q, new, k, v, to, pages, table, lens)
        assert torch.equal(out, again) and torch.equal(lse, lse2) and ctx.pd.pd_device_status(ctx.h)[0] == 0
    check(out, lse, ol.prefill(f64(q), indptr_of(new), np.nan_to_num(f64(k)), np.nan_to_num(f64(v)), to, np.nan_to_num(f64(pages)), table, lens, SCALE32))
