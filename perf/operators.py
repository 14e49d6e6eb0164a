"""The 4-bit KV cache and the rotary write path, measured against their plain forms.

Three kinds of pass:

* ``decode``: attention of one new query token per sequence over a cache held in 4 bits;
* ``store``: packed new tokens quantised into the 4-bit cache and read back into bf16 pages;
* ``rope``: packed new tokens rotated (one to four position axes) and appended to the bf16 cache.

A 4-bit page of one KV head is a block of 18 * D bytes: 16 rows of D / 2 bytes of K codes, 16 of V codes, then
per token and group of 64 values four bf16 numbers {k_scale, k_min, v_scale, v_min}; a value is
scale * code + min. A row's 16-byte piece c (values 32 c .. 32 c + 31, low nibble first) is stored at piece
position c ^ swizzle(slot): (slot >> 1) & 3 for D = 128, (slot >> 2) & 1 for D = 64.
"""
import math

import numpy as np
import torch

own = False

PAGE = 16
GROUP = 64
DEV = "cuda"


# ---------------------------------------------------------------- cases

def listed():
    return [
        # one short sequence at the tiny geometry: the latency of a call
        dict(name="decode_b1_short_d64", op="decode", batch=1, hq=8, hkv=2, d=64, lo=256, hi=256, dist="uniform", lens_seed=1),
        # a mixed batch at head_dim 64 with fresh (empty) sequences and one-token contexts in it
        dict(name="decode_b37_ragged_d64", op="decode", batch=37, hq=16, hkv=2, d=64, lo=0, hi=5001, dist="uniform", lens_seed=2),
        # a rollout batch of 2K-16K contexts
        dict(name="decode_b64_2k_16k", op="decode", batch=64, hq=32, hkv=8, d=128, lo=2048, hi=16384, dist="uniform", lens_seed=3),
        # eight query heads per KV head, lognormal contexts
        dict(name="decode_b64_gqa8_lognormal", op="decode", batch=64, hq=32, hkv=4, d=128, lo=1024, hi=32768, dist="lognormal", lens_seed=4),
        # low decode concurrency: few long contexts
        dict(name="decode_b8_32k_64k", op="decode", batch=8, hq=32, hkv=8, d=128, lo=32768, hi=65536, dist="uniform", lens_seed=5),
        # one decode step's tokens written and read back
        dict(name="store_b64_one_token", op="store", batch=64, hkv=8, d=128, qlo=1, qhi=1, clo=2048, chi=16384, lens_seed=6),
        # short odd turns at head_dim 64
        dict(name="store_b9_odd_d64", op="store", batch=9, hkv=2, d=64, qlo=1, qhi=333, clo=0, chi=1000, lens_seed=7),
        # one turn of a multi-turn rollout per sequence
        dict(name="store_b16_turns", op="store", batch=16, hkv=8, d=128, qlo=256, qhi=2048, clo=0, chi=16384, lens_seed=8),
        # whole long prompts
        dict(name="store_b4_32k", op="store", batch=4, hkv=8, d=128, qlo=32768, qhi=32768, clo=0, chi=0, lens_seed=9),
        # one decode step's tokens, text positions
        dict(name="rope_b64_one_token", op="rope", batch=64, hq=32, hkv=8, d=128, axes=1, rot=128, adjacent=False, qlo=1, qhi=1, clo=2048, chi=16384, far=0, lens_seed=10),
        # turns with images and video in them: time, height, width
        dict(name="rope_b16_turns_3axes", op="rope", batch=16, hq=32, hkv=8, d=128, axes=3, rot=128, adjacent=False, qlo=256, qhi=2048, clo=0, chi=4096, far=0, lens_seed=11),
        # half of each head rotated in adjacent pairs, positions past a million
        dict(name="rope_b3_far_partial_d64", op="rope", batch=3, hq=16, hkv=2, d=64, axes=2, rot=32, adjacent=True, qlo=1001, qhi=9001, clo=0, chi=77, far=1000003, lens_seed=12),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["decode", "decode", "store", "rope"])
    d = rng.choice([64, 128, 128])
    hkv = rng.choice([1, 2, 4, 8])
    hq = hkv * rng.choice([1, 2, 4, 8])
    seed = rng.randrange(1 << 30)
    if op == "decode":
        hi = _log(rng, 1, 65536)
        lo = min(hi, rng.choice([0, 1, _log(rng, 1, hi), hi]))
        most = max(1, min(256, (1 << 19) * 8 // (max(hi, 1) * hkv)))  # at most the largest listed work
        return dict(op="decode", batch=_log(rng, 1, most), hq=hq, hkv=hkv, d=d, lo=lo, hi=hi, dist="uniform", lens_seed=seed)
    qhi = _log(rng, 1, 32768)
    qlo = min(qhi, rng.choice([1, _log(rng, 1, qhi), qhi]))
    most = max(1, min(256, 131072 // qhi))
    batch = _log(rng, 1, most)
    if op == "store":
        return dict(op="store", batch=batch, hkv=hkv, d=d, qlo=qlo, qhi=qhi, clo=0, chi=_log(rng, 1, 4096), lens_seed=seed)
    qhi = min(qhi, 16384)
    qlo = min(qlo, qhi)
    return dict(op="rope", batch=max(1, min(batch, 16384 // qhi)), hq=min(hq, 32), hkv=hkv, d=d, axes=rng.choice([1, 2, 3, 4]),
                rot=rng.choice([d, d, d // 2, d // 4]), adjacent=rng.choice([False, True]), qlo=qlo, qhi=qhi, clo=0,
                chi=_log(rng, 1, 4096), far=rng.choice([0, 0, _log(rng, 1000, 2000000)]), lens_seed=seed)


def _lengths(case):
    """(lengths before the new tokens, new tokens) of every sequence; decode cases have no new tokens."""
    r = np.random.RandomState(case["lens_seed"] % (1 << 31))
    b = case["batch"]
    if case["op"] == "decode":
        if case["dist"] == "lognormal":
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
    d, hkv = case["d"], case["hkv"]
    per_token4 = hkv * (d + 8 * d // GROUP)            # codes and records of one token, K and V
    per_token16 = 2 * hkv * d * 2
    t = int(new.sum())
    if case["op"] == "decode":
        b, hq = case["batch"], case["hq"]
        return {"bytes": int(before.sum()) * per_token4 + 2 * b * hq * d * 2 + b * hq * 4 + 4 * int(((before + PAGE - 1) // PAGE).sum()),
                "flops": 4 * hq * d * int(before.sum())}
    if case["op"] == "store":                          # bf16 tokens in; codes, records and the bf16 read-back out
        return {"bytes": t * (2 * per_token16 + per_token4), "flops": 8 * t * 2 * hkv * d}
    rows = case["hq"] + hkv
    return {"bytes": t * (2 * rows * d * 2 + 2 * hkv * d * 2 + 4 * case["axes"]), "flops": 3 * t * rows * case["rot"]}


# ---------------------------------------------------------------- the 4-bit format, in torch operations

def _piece_index(d, device):
    """[16, pieces]: which piece of the row lies at each piece position of a slot."""
    slot = torch.arange(PAGE, device=device)[:, None]
    pos = torch.arange(d // 32, device=device)[None, :]
    return pos ^ (((slot >> 1) & 3) if d == 128 else ((slot >> 2) & 1))


def _quantize(x):
    """x [..., D] bf16 -> codes uint8 [..., D], scale and min bf16 [..., D / 64]."""
    g = x.float().unflatten(-1, (-1, GROUP))
    g = torch.where(g.abs() < 2.0 ** -126, torch.zeros_like(g), g)
    lo, hi = g.amin(-1, keepdim=True), g.amax(-1, keepdim=True)
    s = (hi - lo) / torch.full_like(lo, 15.0)                               # a number as the divisor becomes its reciprocal on the GPU
    up = ((s.view(torch.int32) + 0xFFFF) & -65536).view(torch.float32)     # the next bf16 at or above
    s = torch.where(s < 2.0 ** -100, torch.zeros_like(s), torch.where(torch.isfinite(s), up, torch.full_like(s, math.nan)))
    code = torch.where(s > 0, torch.round((g - lo) / torch.where(s > 0, s, torch.ones_like(s))), torch.zeros_like(g)).clamp(0, 15)
    return code.to(torch.uint8).flatten(-2), s.squeeze(-1).to(torch.bfloat16), lo.squeeze(-1).to(torch.bfloat16)


def _dequantize(code, scale, lo):
    """The inverse, in 32 bits."""
    g = code.float().unflatten(-1, (-1, GROUP))
    return (scale.float().unsqueeze(-1) * g + lo.float().unsqueeze(-1)).flatten(-2)


def _pack_blocks(k, v):
    """k, v [pages, hkv, 16, D] bf16 -> blocks uint8 [pages, hkv, 18 D]."""
    d = k.shape[-1]
    parts, recs = [], []
    for x in (k, v):
        code, s, lo = _quantize(x)
        b = (code[..., 0::2] | (code[..., 1::2] << 4)).unflatten(-1, (-1, 16))
        idx = _piece_index(d, x.device)[None, None, :, :, None].expand(*b.shape)
        parts.append(torch.gather(b, 3, idx).flatten(2))
        recs += [s, lo]
    rec = torch.stack(recs, -1).contiguous().view(torch.uint8).flatten(2)     # [pages, hkv, 16, groups, 4] bf16
    return torch.cat(parts + [rec], -1)


def _unpack_blocks(blocks, d):
    """blocks uint8 [..., 18 D] -> K and V in 32 bits [..., 16, D]."""
    out = []
    rec = blocks[..., 16 * d:].contiguous().view(torch.bfloat16).unflatten(-1, (PAGE, d // GROUP, 4))
    for i in range(2):
        b = blocks[..., 8 * d * i:8 * d * (i + 1)].unflatten(-1, (PAGE, d // 32, 16))
        idx = _piece_index(d, blocks.device)[:, :, None].expand(b.shape)
        b = torch.gather(b, -2, idx).flatten(-2)      # piece positions are an involution of the pieces
        code = torch.stack((b & 15, b >> 4), -1).flatten(-2)
        out.append(_dequantize(code, rec[..., 2 * i], rec[..., 2 * i + 1]))
    return out


# ---------------------------------------------------------------- inputs

def _randn(shape, g):
    return torch.randn(shape, generator=g, device=DEV)


def _keys(shape, g):
    """Keys with a few strong channels, as they come out of a projection."""
    x = _randn(shape, g)
    x[..., ::16] *= 4.0
    x[..., 5::32] += 6.0
    return x.to(torch.bfloat16)


def _table(case, lens, seed):
    """A scattered page table with room for `lens` tokens: (table int32 [B, MP], pages in the pool)."""
    need = (lens + PAGE - 1) // PAGE
    pool = int(need.sum()) + 1 + int(need.sum()) // 16
    perm = np.random.RandomState((case["lens_seed"] * 31 + seed) % (1 << 31)).permutation(pool)
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
    d, hkv, b = case["d"], case["hkv"], case["batch"]
    table, pool = _table(case, after, int(seed))
    s = dict(case=dict(case), table=table, pool=pool, scale=float(np.float32(d ** -0.5)),
             before=torch.from_numpy(before.astype(np.int32)).to(DEV), after=torch.from_numpy(after.astype(np.int32)).to(DEV),
             max_q=int(new.max()) if b else 0)
    if case["op"] == "decode":
        s["kv4"] = torch.empty((pool, hkv, 18 * d), dtype=torch.uint8, device=DEV)
        step = max(1, (1 << 25) // (hkv * PAGE * d))
        for p in range(0, pool, step):
            n = min(step, pool - p)
            s["kv4"][p:p + n] = _pack_blocks(_keys((n, hkv, PAGE, d), g), _randn((n, hkv, PAGE, d), g).to(torch.bfloat16))
        s["q"] = _randn((b, case["hq"], d), g).to(torch.bfloat16)
        s["out"] = torch.empty_like(s["q"])
        s["lse"] = torch.empty((b, case["hq"]), dtype=torch.float32, device=DEV)
        return s
    t = int(new.sum())
    indptr = np.concatenate([[0], np.cumsum(new)]).astype(np.int32)
    s["indptr"] = torch.from_numpy(indptr).to(DEV)
    # where every packed row lands
    seq = np.repeat(np.arange(b), new)
    pos = before[seq] + np.arange(t) - indptr[seq]
    s["seq"], s["pos"] = torch.from_numpy(seq).to(DEV), torch.from_numpy(pos).to(DEV)
    s["k"], s["v"] = _keys((t, hkv, d), g), _randn((t, hkv, d), g).to(torch.bfloat16)
    s["k_pages"] = torch.zeros((pool, hkv, PAGE, d), dtype=torch.bfloat16, device=DEV)
    s["v_pages"] = torch.zeros_like(s["k_pages"])
    if case["op"] == "store":
        s["kv4"] = torch.zeros((pool, hkv, 18 * d), dtype=torch.uint8, device=DEV)
        return s
    s["q"] = _randn((t, case["hq"], d), g).to(torch.bfloat16)
    s["q_out"] = torch.empty_like(s["q"])
    half = case["rot"] // 2
    s["inv_freq"] = (10000.0 ** (-np.arange(half) * 2.0 / case["rot"])).astype(np.float32)
    s["axis"] = (np.arange(half) * case["axes"] // half).astype(np.uint8)          # contiguous sections
    p = pos + case["far"]
    grid = np.stack([p] + [case["far"] + (pos // (7 + 4 * a)) % 97 for a in range(1, case["axes"])])
    s["positions"] = torch.from_numpy(np.ascontiguousarray(grid.astype(np.int32))).to(DEV)
    return s


# ---------------------------------------------------------------- one pass

_handles = {}


def _handle(pd, s):
    """The library context of this geometry, kept for the life of the program."""
    c = s["case"]
    key = (c.get("hq", c["hkv"]), c["hkv"], c["d"], c["batch"], s["table"].shape[1], s["pool"])
    if key not in _handles:
        _handles[key] = pd.pd_create(key[0], key[1], key[2], PAGE, key[3], key[4], key[5], 0)
    return _handles[key]


def run(state):
    op = state["case"]["op"]
    if own:
        import paper_2609_35158_b200 as pd

        h = _handle(pd, state)
        if op == "decode":
            pd.pd_decode_attn_q4(h, state["q"], state["kv4"], state["table"], state["after"], state["out"], state["lse"],
                                 sm_scale=state["scale"])
            return state["out"], state["lse"]
        if op == "store":
            pd.pd_kv_append_tokens_q4(h, state["k"], state["v"], state["indptr"], state["kv4"], state["table"], state["before"],
                                      state["max_q"], call_flags=pd.PD_APPEND_NO_ADVANCE)
            pd.pd_kv_dequantize_q4(h, state["kv4"], state["table"], state["before"], state["after"], state["k_pages"],
                                   state["v_pages"], state["table"])
            return state["k_pages"], state["v_pages"]
        c = state["case"]
        if "rope" not in state:
            state["rope"] = pd.rope_config(c["rot"], state["inv_freq"], axis_of_pair=state["axis"], num_axes=c["axes"], adjacent=c["adjacent"])
        pd.pd_rope_append_tokens(h, state["rope"], state["positions"], state["q"], state["k"], state["v"], state["indptr"],
                                 state["q_out"], state["k_pages"], state["v_pages"], state["table"], state["before"], state["max_q"],
                                 call_flags=pd.PD_APPEND_NO_ADVANCE)
        return state["q_out"], state["k_pages"], state["v_pages"]
    return {"decode": _plain_decode, "store": _plain_store, "rope": _plain_rope}[op](state)


def _plain_decode(s):
    c = s["case"]
    b, hq, hkv, d = c["batch"], c["hq"], c["hkv"], c["d"]
    k, v = _unpack_blocks(s["kv4"][s["table"].clamp(min=0).long()], d)               # [B, MP, hkv, 16, D]
    k, v = k.transpose(2, 3).flatten(1, 2), v.transpose(2, 3).flatten(1, 2)          # [B, tokens, hkv, D]
    q = s["q"].float().view(b, hkv, hq // hkv, d)
    logits = s["scale"] * torch.einsum("bhgd,bthd->bhgt", q, k)
    dead = torch.arange(k.shape[1], device=DEV)[None, :] >= s["after"][:, None]
    logits = logits.masked_fill(dead[:, None, None, :], -math.inf)
    top = logits.amax(-1, keepdim=True)
    top = torch.where(torch.isfinite(top), top, torch.zeros_like(top))
    p = torch.exp(logits - top)
    total = p.sum(-1, keepdim=True)
    out = torch.einsum("bhgt,bthd->bhgd", p, v) / torch.where(total > 0, total, torch.ones_like(total))
    lse = torch.where(total > 0, top + torch.log(total), torch.full_like(total, -math.inf))
    return out.reshape(b, hq, d).to(torch.bfloat16), lse.reshape(b, hq)


def _slots(s):
    return s["table"][s["seq"], s["pos"] // PAGE].long(), s["pos"] % PAGE


def _plain_store(s):
    page, slot = _slots(s)
    for x, pages in ((s["k"], s["k_pages"]), (s["v"], s["v_pages"])):
        pages[page, :, slot] = _dequantize(*_quantize(x)).to(torch.bfloat16)
    return s["k_pages"], s["v_pages"]


def _rotate(x, cos, sin, rot, adjacent):
    x = x.float()
    r = x[..., :rot]
    a, b = (r[..., 0::2], r[..., 1::2]) if adjacent else (r[..., :rot // 2], r[..., rot // 2:])
    y, z = a * cos - b * sin, a * sin + b * cos
    r = torch.stack((y, z), -1).flatten(-2) if adjacent else torch.cat((y, z), -1)
    return torch.cat((r, x[..., rot:]), -1).to(torch.bfloat16)


def _plain_rope(s):
    c = s["case"]
    where = torch.from_numpy(s["axis"].astype(np.int64)).to(DEV)
    angle = s["positions"].double()[where].T * torch.from_numpy(s["inv_freq"]).to(DEV).double()   # [T, pairs]: far positions need 64 bits
    cos, sin = torch.cos(angle).float()[:, None], torch.sin(angle).float()[:, None]
    page, slot = _slots(s)
    s["k_pages"][page, :, slot] = _rotate(s["k"], cos, sin, c["rot"], c["adjacent"])
    s["v_pages"][page, :, slot] = s["v"]
    return _rotate(s["q"], cos, sin, c["rot"], c["adjacent"]), s["k_pages"], s["v_pages"]


# ---------------------------------------------------------------- the definitions in 64 bits

def exact(case, seed):
    s = prepare(case, seed)
    return {"decode": _exact_decode, "store": _exact_store, "rope": _exact_rope}[case["op"]](s)


def _exact_decode(s):
    c = s["case"]
    hq, hkv, d = c["hq"], c["hkv"], c["d"]
    lens, table = s["after"].tolist(), s["table"].cpu().numpy()
    out = torch.zeros((c["batch"], hq, d), dtype=torch.float64, device=DEV)
    lse = torch.full((c["batch"], hq), -math.inf, dtype=torch.float64, device=DEV)
    # byte of value j in slot i's row: its piece j // 32 lies at (j // 32) ^ swizzle(i)
    i, j = np.meshgrid(np.arange(PAGE), np.arange(d), indexing="ij")
    turn = (i // 2) % 4 if d == 128 else (i // 4) % 2
    byte = torch.from_numpy(i * (d // 2) + ((j // 32) ^ turn) * 16 + (j % 32) // 2).to(DEV)
    odd = torch.from_numpy(j % 2).to(DEV)
    for b, n in enumerate(lens):
        if n == 0:
            continue
        pages = torch.from_numpy(table[b, :-(-n // PAGE)].astype(np.int64)).to(DEV)
        blk = s["kv4"][pages]                                                         # [pages, hkv, 18 D]
        words = blk[:, :, 16 * d:].cpu().numpy().view(np.uint16).astype(np.uint32) << 16    # bf16 is the upper half of a float32
        nums = torch.from_numpy(words.view(np.float32).astype(np.float64)).to(DEV).view(len(pages), hkv, PAGE, d // GROUP, 4)
        got = []
        for m in range(2):
            raw = blk[:, :, 8 * d * m + byte].long()
            code = torch.where(odd > 0, raw // 16, raw % 16).double()
            x = code.view(len(pages), hkv, PAGE, d // GROUP, GROUP) * nums[..., 2 * m, None] + nums[..., 2 * m + 1, None]
            got.append(x.reshape(len(pages), hkv, PAGE, d).permute(1, 0, 2, 3).reshape(hkv, -1, d)[:, :n])
        q = s["q"][b].double().view(hkv, hq // hkv, d)
        z = float(np.float32(s["scale"])) * (q @ got[0].transpose(1, 2))              # [hkv, group, n]
        lse[b] = torch.logsumexp(z, -1).view(-1)
        out[b] = (torch.softmax(z, -1) @ got[1]).reshape(hq, d)
    return out, lse


def _exact_store(s):
    d, hkv = s["case"]["d"], s["case"]["hkv"]
    page = s["table"].cpu().numpy()[s["seq"].cpu().numpy(), s["pos"].cpu().numpy() // PAGE]
    at = torch.from_numpy(page.astype(np.int64)).to(DEV) * PAGE + s["pos"] % PAGE
    done = []
    for x in (s["k"], s["v"]):
        y = torch.zeros((s["pool"] * PAGE, hkv, d), dtype=torch.float64, device=DEV)
        step = max(1, (1 << 25) // (hkv * d))
        for t in range(0, x.shape[0], step):
            w = x[t:t + step].double().reshape(-1, GROUP)
            least = w.min(1).values[:, None]
            span = ((w.max(1).values[:, None] - least).float().double() / 15).float()   # the scale is a bf16 at or above span / 15
            mant, ex = torch.frexp(span.double())
            scale = torch.ldexp(torch.ceil(mant * 256), ex - 8)
            scale = torch.where(span.double() < 2.0 ** -100, torch.zeros_like(scale), scale)
            diff = (w - least).float().double()
            code = torch.where(scale > 0, torch.round(diff / torch.where(scale > 0, scale, torch.ones_like(scale))), torch.zeros_like(diff))
            y[at[t:t + step]] = (code * scale + least).view(-1, hkv, d)
        done.append(y.view(s["pool"], PAGE, hkv, d).transpose(1, 2).contiguous())
    return tuple(done)


def _exact_rope(s):
    c = s["case"]
    d, hkv, rot = c["d"], c["hkv"], c["rot"]
    pos, freq, axis = s["positions"].cpu().numpy().astype(np.float64), s["inv_freq"].astype(np.float64), s["axis"]
    at = s["table"][s["seq"], s["pos"] // PAGE].long() * PAGE + s["pos"] % PAGE
    turn = [torch.polar(torch.ones(1, dtype=torch.float64, device=DEV), torch.from_numpy(pos[axis[i]] * freq[i]).to(DEV)) for i in range(rot // 2)]

    def rotated(x):
        y = x.double()
        for i in range(rot // 2):
            a, b = (2 * i, 2 * i + 1) if c["adjacent"] else (i, i + rot // 2)
            z = torch.complex(x[..., a].double(), x[..., b].double()) * turn[i][:, None]
            y[..., a], y[..., b] = z.real, z.imag
        return y

    done = [rotated(s["q"])]
    for x in (rotated(s["k"]), s["v"].double()):
        y = torch.zeros((s["pool"] * PAGE, hkv, d), dtype=torch.float64, device=DEV)
        y[at] = x
        done.append(y.view(s["pool"], PAGE, hkv, d).transpose(1, 2).contiguous())
    return tuple(done)
