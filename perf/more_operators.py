"""Latent attention: a cache of one shared latent vector a token, measured against its plain forms.

A token's row of the cache is 576 bf16 values: a latent c of 512 and a rotated key part r of 64, shared by all heads; pages
are [pages][16][576]. Four kinds of pass:

* ``append``: packed new tokens written to the cache, the latent normalised and the key part rotated on the way, the
  queries' 64 rotated values with them;
* ``decode``: one new query token per sequence in the absorbed form, q [B][H][576] = (query times the key expansion,
  rotated part): logits q . (c, r), output sum p c;
* ``expand``: a cached context's K and V of every head, K_h = W_h[:128] c and V_h = W_h[128:] c, into bf16 pages
  [pages][H][16][128];
* ``prefill``: the new tokens of a turn in the expanded form, q [T][H][192] = (128 against K_h, 64 against r), causal.
"""
import math

import numpy as np
import torch

own = False

PAGE = 16
LATENT = 512
ROPE = 64
ROW = LATENT + ROPE
HEAD = 128
SCALE = float(np.float32((HEAD + ROPE) ** -0.5))
DEV = "cuda"


# ---------------------------------------------------------------- cases

def listed():
    return [
        # one decode step's tokens of 64 sequences, queries rotated into the absorbed rows
        dict(name="append_b64_one_token", op="append", batch=64, h=64, qlo=1, qhi=1, clo=2048, chi=16384, norm=True, adjacent=True, width=576, far=0, lens_seed=1),
        # one turn of a multi-turn rollout per sequence, queries rotated into the expanded rows
        dict(name="append_b16_turns", op="append", batch=16, h=32, qlo=256, qhi=2048, clo=0, chi=4096, norm=True, adjacent=False, width=192, far=0, lens_seed=2),
        # one short sequence on a shard of 8 heads: the latency of a call
        dict(name="decode_b1_short_h8", op="decode", batch=1, h=8, lo=300, hi=300, dist="uniform", lens_seed=3),
        # a mixed batch with empty and one-token contexts, an odd number of heads
        dict(name="decode_b37_ragged_h20", op="decode", batch=37, h=20, lo=0, hi=5001, dist="uniform", lens_seed=4),
        # a rollout batch of 2K-16K contexts on a shard of 16 heads
        dict(name="decode_b64_2k_16k_h16", op="decode", batch=64, h=16, lo=2048, hi=16384, dist="uniform", lens_seed=5),
        # lognormal contexts, 64 heads
        dict(name="decode_b64_lognormal_h64", op="decode", batch=64, h=64, lo=1024, hi=32768, dist="lognormal", lens_seed=6),
        # all 128 heads on one GPU
        dict(name="decode_b64_2k_16k_h128", op="decode", batch=64, h=128, lo=2048, hi=16384, dist="uniform", lens_seed=7),
        # low decode concurrency: few long contexts
        dict(name="decode_b4_32k_64k_h32", op="decode", batch=4, h=32, lo=32768, hi=65536, dist="uniform", lens_seed=8),
        # short odd contexts expanded for 5 heads
        dict(name="expand_b9_odd_h5", op="expand", batch=9, h=5, lo=0, hi=1000, lens_seed=9),
        # the cached prefixes of a batch of turns
        dict(name="expand_b16_2k_8k_h32", op="expand", batch=16, h=32, lo=2048, hi=8192, lens_seed=10),
        # short odd turns
        dict(name="prefill_b9_odd_h20", op="prefill", batch=9, h=20, qlo=1, qhi=333, clo=0, chi=1000, lens_seed=11),
        # one turn of a multi-turn rollout per sequence
        dict(name="prefill_b8_turns_h32", op="prefill", batch=8, h=32, qlo=256, qhi=2048, clo=0, chi=16384, lens_seed=12),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["append", "decode", "decode", "decode", "expand", "prefill"])
    seed = rng.randrange(1 << 30)
    h = rng.choice([8, 16, 32, 64, 128, rng.randint(1, 128)])
    if op == "decode":
        hi = _log(rng, 1, 65536)
        lo = min(hi, rng.choice([0, 1, _log(rng, 1, hi), hi]))
        most = max(1, min(256, (1 << 26) // (hi * max(h, 16))))
        return dict(op=op, batch=_log(rng, 1, most), h=h, lo=lo, hi=hi, dist="uniform", lens_seed=seed)
    if op == "expand":
        h = rng.choice([4, 8, 32, rng.randint(1, 40)])
        hi = _log(rng, 1, 16384)
        lo = min(hi, rng.choice([0, _log(rng, 1, hi), hi]))
        most = max(1, min(128, 2500000 // (hi * h)))
        return dict(op=op, batch=_log(rng, 1, most), h=h, lo=lo, hi=hi, lens_seed=seed)
    if op == "append":
        qhi = _log(rng, 1, 16384)
        qlo = min(qhi, rng.choice([1, _log(rng, 1, qhi), qhi]))
        batch = _log(rng, 1, max(1, min(256, 500000 // (qhi * h))))
        return dict(op=op, batch=batch, h=h, qlo=qlo, qhi=qhi, clo=0, chi=_log(rng, 1, 4096), norm=rng.choice([True, False]),
                    adjacent=rng.choice([True, False]), width=rng.choice([192, 576]), far=rng.choice([0, 0, _log(rng, 1000, 2000000)]), lens_seed=seed)
    h = rng.choice([4, 8, 32, rng.randint(1, 40)])
    qhi = _log(rng, 1, 4096)
    qlo = min(qhi, rng.choice([1, _log(rng, 1, qhi), qhi]))
    chi = _log(rng, 1, 8192)
    batch = _log(rng, 1, max(1, min(64, 1500000000 // (qhi * (qhi + chi) * h))))
    return dict(op=op, batch=batch, h=h, qlo=qlo, qhi=qhi, clo=0, chi=chi, lens_seed=seed)


def _lengths(case):
    """(lengths before the new tokens, new tokens) of every sequence; decode and expand have no new tokens."""
    r = np.random.RandomState(case["lens_seed"] % (1 << 31))
    b = case["batch"]
    if case["op"] in ("decode", "expand"):
        if case.get("dist") == "lognormal":
            n = np.clip(np.rint(np.exp(math.log(8192.0) + 0.7 * r.standard_normal(b))), case["lo"], case["hi"]).astype(np.int64)
        else:
            n = r.randint(case["lo"], case["hi"] + 1, b)
            if case["lo"] <= 1 and b >= 8:  # an empty context and a one-token one always come along
                n[1], n[2] = case["lo"], 1
            n[0] = max(n[0], 1)
        return n, np.zeros(b, np.int64)
    return r.randint(case["clo"], case["chi"] + 1, b), r.randint(case["qlo"], case["qhi"] + 1, b)


def work(case):
    before, new = _lengths(case)
    b, h = case["batch"], case["h"]
    t, ctx = int(new.sum()), int(before.sum())
    pages = 4 * int(((before + new + PAGE - 1) // PAGE).sum())
    if case["op"] == "append":
        return {"bytes": t * (2 * ROW * 2 + 2 * h * ROPE * 2 + 4) + 4 * b, "flops": t * (4 * LATENT + 3 * (h + 1) * ROPE)}
    if case["op"] == "decode":
        return {"bytes": ctx * ROW * 2 + b * h * ((ROW + LATENT) * 2 + 4) + pages, "flops": 2 * ctx * h * (ROW + LATENT)}
    if case["op"] == "expand":
        return {"bytes": ctx * (LATENT + 2 * h * HEAD) * 2 + 2 * h * HEAD * LATENT * 2 + pages, "flops": 2 * ctx * LATENT * 2 * h * HEAD}
    pairs = int((new * before + new * (new + 1) // 2).sum())
    read = (ctx + t) * (2 * h * HEAD + ROPE) * 2
    return {"bytes": read + t * h * ((HEAD + ROPE + HEAD) * 2 + 4) + 2 * pages, "flops": 2 * pairs * h * (HEAD + ROPE + HEAD)}


# ---------------------------------------------------------------- inputs

def _randn(shape, g):
    return torch.randn(shape, generator=g, device=DEV)


def _bf16(x):
    return x.to(torch.bfloat16)


def _rows(n, g):
    """Cached rows: normalised latents with a few strong channels, rotated keys."""
    x = _randn((n, ROW), g)
    x[:, 7:LATENT:64] *= 3.0
    x[:, LATENT::8] *= 2.0
    return _bf16(x)


def _table(case, lens, seed, salt):
    """A scattered page table with room for `lens` tokens: (table int32 [B, MP], pages in the pool)."""
    need = (lens + PAGE - 1) // PAGE
    pool = int(need.sum()) + 1 + int(need.sum()) // 16
    perm = np.random.RandomState((case["lens_seed"] * 31 + seed + salt) % (1 << 31)).permutation(pool)
    table = np.full((case["batch"], max(1, int(need.max()))), -1, np.int32)
    at = 0
    for b, n in enumerate(need):
        table[b, :n] = perm[at:at + n]
        at += n
    return torch.from_numpy(table).to(DEV), pool


def prepare(case, seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(int(seed) * 1000003 + case["lens_seed"] % 65521)
    before, new = _lengths(case)
    after = before + new
    b, h = case["batch"], case["h"]
    table, pool = _table(case, after, int(seed), 0)
    s = dict(case=dict(case), table=table, pool=pool, before=torch.from_numpy(before.astype(np.int32)).to(DEV),
             after=torch.from_numpy(after.astype(np.int32)).to(DEV), max_q=int(new.max()) if b else 0)
    t = int(new.sum())
    indptr = np.concatenate([[0], np.cumsum(new)]).astype(np.int32)
    s["indptr"] = torch.from_numpy(indptr).to(DEV)
    if case["op"] == "append":
        seq = np.repeat(np.arange(b), new)
        pos = before[seq] + np.arange(t) - indptr[seq]
        s["seq"], s["pos"] = torch.from_numpy(seq).to(DEV), torch.from_numpy(pos).to(DEV)
        s["kv_new"] = _bf16(_randn((t, ROW), g) * (0.3 + 3.0 * torch.rand((t, 1), generator=g, device=DEV)))  # as it leaves its projection
        s["weight"] = _bf16(1.0 + 0.2 * _randn((LATENT,), g)) if case["norm"] else None
        s["eps"] = 1e-6
        s["q"] = _bf16(_randn((t, h, HEAD + ROPE), g))
        s["q_out"] = torch.zeros((t, h, case["width"]), dtype=torch.bfloat16, device=DEV)
        s["kv"] = torch.zeros((pool, PAGE, ROW), dtype=torch.bfloat16, device=DEV)
        s["inv_freq"] = (10000.0 ** (-np.arange(ROPE // 2) * 2.0 / ROPE)).astype(np.float32)
        s["positions"] = torch.from_numpy((pos + case["far"]).astype(np.int32)).to(DEV)
        return s
    s["kv"] = _rows(pool * PAGE, g).view(pool, PAGE, ROW)
    if case["op"] == "decode":
        s["q"] = _bf16(_randn((b, h, ROW), g))
        s["out"] = torch.empty((b, h, LATENT), dtype=torch.bfloat16, device=DEV)
        s["lse"] = torch.empty((b, h), dtype=torch.float32, device=DEV)
        return s
    s["kv_table"], s["kv_pool"] = _table(case, after, int(seed), 7)      # the expanded pages, a pool of their own
    shape = (s["kv_pool"], h, PAGE, HEAD)
    if case["op"] == "expand":
        s["w"] = _bf16(_randn((h, 2 * HEAD, LATENT), g) * LATENT ** -0.5)
        s["k_pages"] = torch.zeros(shape, dtype=torch.bfloat16, device=DEV)
        s["v_pages"] = torch.zeros(shape, dtype=torch.bfloat16, device=DEV)
        return s
    s["k_pages"], s["v_pages"] = _bf16(_randn(shape, g)), _bf16(_randn(shape, g))
    s["q"] = _bf16(_randn((t, h, HEAD + ROPE), g))
    s["out"] = torch.empty((t, h, HEAD), dtype=torch.bfloat16, device=DEV)
    s["lse"] = torch.empty((t, h), dtype=torch.float32, device=DEV)
    return s


# ---------------------------------------------------------------- one pass

_handles = {}


def _handle(pd, s):
    """The library context of this geometry, kept for the life of the program."""
    c = s["case"]
    key = (c["h"], c["batch"], s["table"].shape[1], s["pool"])
    if key not in _handles:
        _handles[key] = pd.pd_create(c["h"], 1, LATENT, PAGE, key[1], key[2], key[3], 0, pd.PD_FLAG_LATENT)
    return _handles[key]


def run(state):
    s, op = state, state["case"]["op"]
    if own:
        import paper_2609_35158_b200 as pd

        h = _handle(pd, s)
        if op == "append":
            if "rope" not in s:
                s["rope"] = pd.rope_config(ROPE, s["inv_freq"], adjacent=s["case"]["adjacent"])
            pd.pd_rope_append_tokens_latent(h, s["rope"], s["positions"], s["q"][..., HEAD:], s["kv_new"], s["weight"], s["eps"], s["indptr"],
                                            s["q_out"][..., -ROPE:], s["kv"], s["table"], s["before"], s["max_q"],
                                            call_flags=pd.PD_APPEND_NO_ADVANCE)
            return s["q_out"], s["kv"]
        if op == "decode":
            pd.pd_decode_attn_latent(h, s["q"], s["kv"], s["table"], s["after"], s["out"], s["lse"], sm_scale=SCALE)
            return s["out"], s["lse"]
        if op == "expand":
            pd.pd_kv_expand_latent(h, s["w"], s["kv"], s["table"], None, s["after"], s["k_pages"], s["v_pages"], s["kv_table"])
            return s["k_pages"], s["v_pages"]
        pd.pd_prefill_attn_latent(h, s["q"], s["indptr"], s["k_pages"], s["v_pages"], s["kv_table"], s["kv"], s["table"], s["after"],
                                  s["out"], s["lse"], max_q_len=s["max_q"], sm_scale=SCALE)
        return s["out"], s["lse"]
    return {"append": _plain_append, "decode": _plain_decode, "expand": _plain_expand, "prefill": _plain_prefill}[op](s)


def _rotate(x, cos, sin, adjacent):
    x = x.float()
    a, b = (x[..., 0::2], x[..., 1::2]) if adjacent else (x[..., :ROPE // 2], x[..., ROPE // 2:])
    y, z = a * cos - b * sin, a * sin + b * cos
    return _bf16(torch.stack((y, z), -1).flatten(-2) if adjacent else torch.cat((y, z), -1))


def _plain_append(s):
    c = s["case"]
    angle = s["positions"].double()[:, None] * torch.from_numpy(s["inv_freq"]).to(DEV).double()   # far positions need 64 bits
    cos, sin = torch.cos(angle).float(), torch.sin(angle).float()
    lat = s["kv_new"][:, :LATENT].float()
    if s["weight"] is not None:
        lat = lat * torch.rsqrt((lat * lat).mean(-1, keepdim=True) + s["eps"]) * s["weight"].float()
    page, slot = s["table"][s["seq"], s["pos"] // PAGE].long(), s["pos"] % PAGE
    s["kv"][page, slot] = torch.cat((_bf16(lat), _rotate(s["kv_new"][:, LATENT:], cos, sin, c["adjacent"])), -1)
    s["q_out"][..., -ROPE:] = _rotate(s["q"][..., HEAD:], cos[:, None], sin[:, None], c["adjacent"])
    return s["q_out"], s["kv"]


def _plain_decode(s):
    rows = s["kv"][s["table"].clamp(min=0).long()].flatten(1, 2).float()             # [B, tokens, 576]
    logits = SCALE * torch.einsum("bhd,btd->bht", s["q"].float(), rows)
    dead = torch.arange(rows.shape[1], device=DEV)[None, :] >= s["after"][:, None]
    logits = logits.masked_fill(dead[:, None, :], -math.inf)
    top = logits.amax(-1, keepdim=True)
    top = torch.where(torch.isfinite(top), top, torch.zeros_like(top))
    p = torch.exp(logits - top)
    total = p.sum(-1, keepdim=True)
    out = torch.einsum("bht,btd->bhd", p, rows[..., :LATENT]) / torch.where(total > 0, total, torch.ones_like(total))
    lse = torch.where(total > 0, top + torch.log(total), torch.full_like(total, -math.inf))
    return _bf16(out), lse.squeeze(-1)


def _plain_expand(s):
    h = s["case"]["h"]
    w = s["w"].float().reshape(-1, LATENT)
    for b, n in enumerate(s["after"].tolist()):
        t = torch.arange(n, device=DEV)
        lat = s["kv"][s["table"][b, t // PAGE].long(), t % PAGE, :LATENT].float()
        both = _bf16(lat @ w.T).view(n, h, 2, HEAD)
        to = s["kv_table"][b, t // PAGE].long()
        s["k_pages"][to, :, t % PAGE] = both[:, :, 0]
        s["v_pages"][to, :, t % PAGE] = both[:, :, 1]
    return s["k_pages"], s["v_pages"]


def _plain_prefill(s):
    h = s["case"]["h"]
    start = s["indptr"].tolist()
    for b, n in enumerate(s["after"].tolist()):
        m = start[b + 1] - start[b]
        t = torch.arange(n, device=DEV)
        at, slot = s["kv_table"][b, t // PAGE].long(), t % PAGE
        k, v = s["k_pages"][at, :, slot].float(), s["v_pages"][at, :, slot].float()     # [n, H, 128]
        r = s["kv"][s["table"][b, t // PAGE].long(), slot, LATENT:].float()
        q = s["q"][start[b]:start[b + 1]].float()
        hidden = t[None, :] > (n - m + torch.arange(m, device=DEV))[:, None]
        step = max(1, min(h, (1 << 28) // max(1, m * n)))
        for i in range(0, h, step):
            z = torch.einsum("mhd,nhd->hmn", q[:, i:i + step, :HEAD], k[:, i:i + step]) + torch.einsum("mhd,nd->hmn", q[:, i:i + step, HEAD:], r)
            z = (SCALE * z).masked_fill(hidden, -math.inf)
            top = z.amax(-1, keepdim=True)
            p = torch.exp(z - top)
            total = p.sum(-1, keepdim=True)
            s["out"][start[b]:start[b + 1], i:i + step] = _bf16(torch.einsum("hmn,nhd->mhd", p / total, v[:, i:i + step]))
            s["lse"][start[b]:start[b + 1], i:i + step] = (top + torch.log(total)).squeeze(-1).T
    return s["out"], s["lse"]


# ---------------------------------------------------------------- the definitions in 64 bits

def exact(case, seed):
    s = prepare(case, seed)
    return {"append": _exact_append, "decode": _exact_decode, "expand": _exact_expand, "prefill": _exact_prefill}[case["op"]](s)


def _slots_of(table, b, n):
    """Flat slot numbers of tokens 0 .. n - 1 of sequence b."""
    pages = table[b, :-(-n // PAGE)].long()
    return (pages[:, None] * PAGE + torch.arange(PAGE, device=DEV)).flatten()[:n]


def _exact_append(s):
    c = s["case"]
    turn = torch.exp(1j * torch.outer(s["positions"].double(), torch.from_numpy(s["inv_freq"].astype(np.float64)).to(DEV)))

    def turned(x, by):
        pairs = x.double().unflatten(-1, (-1, 2) if c["adjacent"] else (2, -1))
        if not c["adjacent"]:
            pairs = pairs.transpose(-1, -2)
        z = torch.view_as_real(torch.view_as_complex(pairs.contiguous()) * by)
        return (z if c["adjacent"] else z.transpose(-1, -2)).flatten(-2)

    x = s["kv_new"].double()
    lat = x[:, :LATENT]
    if s["weight"] is not None:
        size = torch.sqrt(lat.square().sum(-1) / LATENT + s["eps"])
        lat = lat / size[:, None] * s["weight"].double()
    kv = torch.zeros((s["pool"] * PAGE, ROW), dtype=torch.float64, device=DEV)
    start = s["indptr"].tolist()
    for b, n in enumerate(s["after"].tolist()):
        to = _slots_of(s["table"], b, n)[n - (start[b + 1] - start[b]):]
        kv[to, :LATENT] = lat[start[b]:start[b + 1]]
        kv[to, LATENT:] = turned(x[start[b]:start[b + 1], LATENT:], turn[start[b]:start[b + 1]])
    q = torch.zeros(s["q_out"].shape, dtype=torch.float64, device=DEV)
    q[..., c["width"] - ROPE:] = turned(s["q"][..., HEAD:], turn[:, None])
    return q, kv.view(s["pool"], PAGE, ROW)


def _exact_decode(s):
    c = s["case"]
    out = torch.zeros((c["batch"], c["h"], LATENT), dtype=torch.float64, device=DEV)
    lse = torch.full((c["batch"], c["h"]), -math.inf, dtype=torch.float64, device=DEV)
    flat = s["kv"].view(-1, ROW)
    for b, n in enumerate(s["after"].tolist()):
        if n == 0:
            continue
        rows = flat[_slots_of(s["table"], b, n)].double()
        z = SCALE * (s["q"][b].double() @ rows.T)
        lse[b] = torch.logsumexp(z, -1)
        out[b] = torch.softmax(z, -1) @ rows[:, :LATENT]
    return out, lse


def _exact_expand(s):
    h = s["case"]["h"]
    done = [torch.zeros((s["kv_pool"], h, PAGE, HEAD), dtype=torch.float64, device=DEV) for _ in range(2)]
    flat = s["kv"].view(-1, ROW)
    for b, n in enumerate(s["after"].tolist()):
        if n == 0:
            continue
        lat = flat[_slots_of(s["table"], b, n), :LATENT].double()
        to = _slots_of(s["kv_table"], b, n)
        for i in range(h):
            for x, w in zip(done, s["w"][i].double().split(HEAD)):
                x[to // PAGE, i, to % PAGE] = lat @ w.T
    return tuple(done)


def _exact_prefill(s):
    h = s["case"]["h"]
    out = torch.zeros(s["out"].shape, dtype=torch.float64, device=DEV)
    lse = torch.zeros(s["lse"].shape, dtype=torch.float64, device=DEV)
    start, flat = s["indptr"].tolist(), s["kv"].view(-1, ROW)
    for b, n in enumerate(s["after"].tolist()):
        lo, hi = start[b], start[b + 1]
        r = flat[_slots_of(s["table"], b, n), LATENT:].double()
        at = _slots_of(s["kv_table"], b, n)
        for i in range(h):
            k = torch.cat((s["k_pages"][at // PAGE, i, at % PAGE].double(), r), -1)
            v = s["v_pages"][at // PAGE, i, at % PAGE].double()
            z = SCALE * (s["q"][lo:hi, i].double() @ k.T)
            z += torch.full_like(z, -math.inf).triu(n - (hi - lo) + 1)
            lse[lo:hi, i] = torch.logsumexp(z, -1)
            out[lo:hi, i] = torch.softmax(z, -1) @ v
    return out, lse
