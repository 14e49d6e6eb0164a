"""Decode attention over 4-bit pages: plans with more ranges than workers, whose ranges are claimed while the kernel runs, the
largest automatic plans, long contexts. Against a plain reference in 64 bits with bounds that shrink with the length."""
import math

import numpy as np
import pytest
import torch

import oracle
from oracle import q4
import workloads as wl
from pd_testlib import Ctx
from test_gpu_q4 import P, check_attention, dev, random_cache

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def reference(q, kv4, table, lens, sm_scale):
    """(out, lse, tol_out, tol_lse, rms) in 64 bits for q bf16 [B, Hq, d] over blocks uint8 [NP, Hkv, 18 d].

    The bounds are those of ``oracle.q4.decode_attn`` but for the weights p * v_scale, each rounded to fp16 (off by at most
    2^-11 of itself) and multiplied by codes up to 15. There it is the sum over tokens, here the roundings are taken as
    independent (the tokens of a sequence are distinct) and zero in the mean: by Hoeffding, a sum of terms within +-c_t passes sqrt(2 ln(2 N / e) sum c_t^2) in one of
    N outputs with probability e = 1e-6 at most. For n tokens of equal weight that is sqrt(n) / 7 times tighter. The same for
    the errors of the logits, which multiply V rows that are drawn apart from them, and
    for the fp32 sums of p and p * v_min, at most n / 8 additions per lane, each off by at most 2^-24 of the sum. The sums of
    the codes' products are covered by the 2^-18: a tensor core cuts at most 2^-23 of a sum off per product, and an
    accumulator takes 32 products before it is rounded to nearest.

    rms: what the errors of a head's d outputs can come to, in the root of the mean square: a rounding is uniform within its
    bound, which makes 1 / sqrt(3) of it, and the rest counts in full."""
    B, Hq, d = q.shape
    NP, Hkv = kv4.shape[:2]
    G, groups = Hq // Hkv, d // 64
    byte, shift = (torch.from_numpy(x).to(DEV) for x in q4._tables(d))
    rec = kv4[..., 16 * d:].contiguous().view(torch.bfloat16).view(NP, Hkv, P, groups, 4).double()
    kv = []
    for which in range(2):
        code = ((kv4[:, :, 8 * d * which:][:, :, byte].long() >> shift) & 15).double().unflatten(-1, (groups, 64))
        kv.append((code * rec[..., 2 * which, None] + rec[..., 2 * which + 1, None]).flatten(-2))
    qd, scale = q.double(), float(np.float32(sm_scale))
    out = torch.zeros((B, Hq, d), dtype=torch.float64, device=DEV)
    tol = torch.zeros_like(out)
    lse = torch.full((B, Hq), -math.inf, dtype=torch.float64, device=DEV)
    tol_lse = torch.zeros_like(lse)
    rms = torch.zeros_like(lse)
    spread = math.sqrt(2 * math.log(2 * out.numel() / 1e-6))
    for b, n in enumerate(lens.tolist()):
        if n == 0:
            continue
        pages = torch.from_numpy(table[b, :-(-n // P)].astype(np.int64)).to(DEV)
        k, v = (x[pages].transpose(0, 1).flatten(1, 2)[:, :n] for x in kv)                    # [Hkv, n, d]
        r = rec[pages].transpose(0, 1).flatten(1, 2)[:, :n].abs()                             # [Hkv, n, groups, 4]
        qb = qd[b].view(Hkv, G, d)
        z = scale * (qb @ k.transpose(1, 2))
        top = torch.logsumexp(z, -1)
        p = torch.exp(z - top[..., None])                                                     # [Hkv, G, n]
        o = p @ v
        size = (p @ (15 * r[..., 2] + r[..., 3])).repeat_interleave(64, -1)
        noise = torch.sqrt((p * p) @ (15 * r[..., 2]) ** 2).repeat_interleave(64, -1)
        sums = 2.0 ** -18 + spread * math.sqrt(n / 8) * 2.0 ** -24
        qa = qb.abs().unflatten(-1, (groups, 64)).sum(-1)
        delta = 2.0 ** -19 * scale * (qa @ (15 * r[..., 0] + r[..., 1]).transpose(1, 2)).amax(-1)   # [Hkv, G]
        out[b], lse[b] = o.view(Hq, d), top.view(Hq)
        rest = sums * size
        noise = 2.0 ** -11 * noise + 2 * delta[..., None] * torch.sqrt((p * p) @ (15 * r[..., 2] + r[..., 3]) ** 2).repeat_interleave(64, -1)
        tol[b] = (2.0 ** -8 * o.abs() + spread * noise + rest).view(Hq, d)
        tol_lse[b] = (delta + 4e-6 * (1 + top.abs()) + spread * math.sqrt(n / 8) * 2.0 ** -24).view(Hq)
        rms[b] = torch.sqrt((((2.0 ** -8 * o) ** 2 + noise ** 2) / 3).mean(-1)).add(torch.sqrt((rest ** 2).mean(-1))).view(Hq)
    return [x.cpu().numpy() for x in (out, lse, tol, tol_lse, rms)]


def check_tight(out, lse, ref, what=""):
    check_attention(out, lse, ref[:4], what)
    error = np.sqrt(((out.float().cpu().numpy() - ref[0]) ** 2).mean(-1))
    assert np.all(error <= 1.25 * ref[4]), f"{what}: {(error / np.maximum(ref[4], 1e-300)).max()}"  # 64 or 128 outputs: their mean square scatters


def bits(x):
    return x.view(torch.int16) if x.dtype == torch.bfloat16 else x


@pytest.mark.parametrize("Hq,Hkv,d", [(8, 2, 128), (16, 2, 128), (8, 2, 64), (16, 2, 64)])
def test_more_ranges_than_workers(Hq, Hkv, d):
    """Ranges of one page: workers claim most of them. The counters are left as the next call needs them: three calls in a
    row, one with a plan of few ranges between, one of the bf16 kernel that claims from the same counters."""
    import paper_2609_35158_b200 as pd

    lens = np.array([4000, 6001, 0, 3999, 1, 4016, 4200, 3500, 5000], np.int32)
    kv4, table, NP = random_cache(lens, Hkv, d, 300 + Hq)
    q = wl.random_bf16((len(lens), Hq, d), 301, DEV)
    kv, t, L = dev(kv4), dev(table), dev(lens)
    ref = reference(q, kv, table, lens, 0.1)
    k16, v16 = (wl.random_bf16((NP, Hkv, P, d), 302 + i, DEV) for i in range(2))
    outs = []
    with Ctx(Hq, Hkv, d, len(lens), table.shape[1], NP) as ctx:
        def call(split):
            out = torch.full((len(lens), Hq, d), float("nan"), dtype=torch.bfloat16, device=DEV)
            lse = torch.full((len(lens), Hq), float("nan"), device=DEV)
            pd.pd_decode_attn_q4(ctx.h, q, kv, t, L, out, lse, sm_scale=0.1, split_pages=split)
            plan = pd.pd_last_plan(ctx.h)
            check_tight(out, lse, ref, f"split {split}")
            return plan, out, lse

        for split in (1, 1, 0, 1):
            plan, out, lse = call(split)
            if split == 1:
                assert plan["num_ranges"] == Hkv * int(((lens + P - 1) // P).sum()) > plan["num_workers"]
                outs.append((out, lse))
            else:
                assert plan["num_ranges"] <= plan["num_workers"]
        a, b = torch.empty_like(q), torch.empty_like(q)
        pd.pd_decode_attn(ctx.h, q, k16, v16, t, L, a, sm_scale=0.1, split_pages=1)
        _, out, lse = call(1)
        pd.pd_decode_attn(ctx.h, q, k16, v16, t, L, b, sm_scale=0.1, split_pages=1)
        outs.append((out, lse))
        torch.cuda.synchronize()
        assert pd.pd_device_status(ctx.h)[0] == 0
    assert torch.equal(bits(a), bits(b))
    for out, lse in outs[1:]:  # who claims a range changes nothing
        assert torch.equal(bits(out), bits(outs[0][0])) and torch.equal(lse, outs[0][1])


def test_more_ranges_than_workers_captured_and_replayed():
    import paper_2609_35158_b200 as pd

    Hq, Hkv, d = 8, 2, 128
    lens = np.array([7000, 9001, 40, 5000], np.int32)
    kv4, table, NP = random_cache(lens, Hkv, d, 310)
    q = wl.random_bf16((len(lens), Hq, d), 311, DEV)
    kv, t, L = dev(kv4), dev(table), dev(lens)
    out, again = (torch.empty_like(q) for _ in range(2))
    with Ctx(Hq, Hkv, d, len(lens), table.shape[1], NP) as ctx:
        pd.pd_decode_attn_q4(ctx.h, q, kv, t, L, out, sm_scale=0.1, split_pages=1)
        plan = pd.pd_last_plan(ctx.h)
        assert plan["num_ranges"] > plan["num_workers"]
        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):
            graph = torch.cuda.CUDAGraph()
            with torch.cuda.graph(graph, stream=side):
                for _ in range(3):
                    pd.pd_decode_attn_q4(ctx.h, q, kv, t, L, again, sm_scale=0.1, split_pages=1)
            for _ in range(3):
                again.fill_(float("nan"))
                graph.replay()
        torch.cuda.synchronize()
        assert pd.pd_device_status(ctx.h)[0] == 0
    assert torch.equal(bits(out), bits(again))
    check_tight(out, None, reference(q, kv, table, lens, 0.1))


@pytest.mark.parametrize("Hq,d,longest", [(32, 128, 17000), (8, 64, 22000)])
def test_a_batch_of_256_long_contexts(Hq, d, longest):
    """More than 1024 pages per worker under the automatic plan, over a pool whose pages the sequences share."""
    import paper_2609_35158_b200 as pd

    Hkv, B, NP = 8, 256, 1400
    rng = np.random.default_rng(320)
    lens = rng.integers(longest - 1500, longest, B).astype(np.int32)
    lens[[3, 100, 255]] = [0, 1, 17]
    kv4, _, _ = random_cache([NP * P], Hkv, d, 321, poison=False)
    kv4 = kv4[:NP]
    table = np.stack([rng.permutation(NP)[:(longest + P - 1) // P] for _ in range(B)]).astype(np.int32)
    q = wl.random_bf16((B, Hq, d), 322, DEV)
    kv, t, L = dev(kv4), dev(table), dev(lens)
    out = torch.full((B, Hq, d), float("nan"), dtype=torch.bfloat16, device=DEV)
    lse = torch.full((B, Hq), float("nan"), device=DEV)
    out2, lse2 = torch.empty_like(out), torch.empty_like(lse)
    with Ctx(Hq, Hkv, d, B, table.shape[1], NP) as ctx:
        pd.pd_decode_attn_q4(ctx.h, q, kv, t, L, out, lse, sm_scale=0.1)
        plan = pd.pd_last_plan(ctx.h)
        pd.pd_decode_attn_q4(ctx.h, q, kv, t, L, out2, lse2, sm_scale=0.1)
        torch.cuda.synchronize()
        assert pd.pd_device_status(ctx.h)[0] == 0
    units = Hkv * int(((lens + P - 1) // P).sum())
    assert units > 1024 * plan["num_workers"] >= 1024 * plan["num_ranges"]  # one long range per worker
    check_tight(out, lse, reference(q, kv, table, lens, 0.1))
    assert torch.equal(bits(out), bits(out2)) and torch.equal(lse, lse2)


@pytest.mark.parametrize("Hq,Hkv,d", [(32, 8, 128), (16, 2, 64), (8, 1, 128)])
def test_long_contexts_under_the_tight_bound(Hq, Hkv, d):
    import paper_2609_35158_b200 as pd

    lens = np.array([20000, 0, 33001, 9000, 65536], np.int32)
    NP = 4200
    rng = np.random.default_rng(330)
    kv4, _, _ = random_cache([NP * P], Hkv, d, 331, scale_k=0.1, poison=False)
    kv4 = kv4[:NP]
    table = np.stack([rng.permutation(NP)[:4096] for _ in lens]).astype(np.int32)
    q = wl.random_bf16((len(lens), Hq, d), 332, DEV)
    kv, t, L = dev(kv4), dev(table), dev(lens)
    ref = reference(q, kv, table, lens, 0.09)
    with Ctx(Hq, Hkv, d, len(lens), table.shape[1], NP) as ctx:
        for split in (0, 100000, 1024, 128, 5):
            out = torch.full((len(lens), Hq, d), float("nan"), dtype=torch.bfloat16, device=DEV)
            lse = torch.full((len(lens), Hq), float("nan"), device=DEV)
            pd.pd_decode_attn_q4(ctx.h, q, kv, t, L, out, lse, sm_scale=0.09, split_pages=split)
            torch.cuda.synchronize()
            assert pd.pd_device_status(ctx.h)[0] == 0
            check_tight(out, lse, ref, f"split {split}")


def test_the_two_references_agree():
    lens = np.array([1, 40, 0, 333], np.int32)
    for Hq, Hkv, d in ((8, 2, 64), (4, 4, 128)):
        kv4, table, NP = random_cache(lens, Hkv, d, 340, poison=False)
        q = wl.random_bf16((len(lens), Hq, d), 341, "cpu")
        a = q4.decode_attn(oracle.bf16_bits(q), kv4, table, lens, 0.1)
        b = reference(q.to(DEV), dev(kv4), table, lens, 0.1)
        assert np.allclose(a[0], b[0], rtol=0, atol=1e-12) and np.allclose(a[1], b[1], rtol=0, atol=1e-12) and np.all(b[3] >= a[3])
