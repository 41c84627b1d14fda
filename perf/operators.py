"""What is measured of the operators around the 8-bit KV cache: multi-axis rotary positions (`rope`), block tables and
slot maps (`plan`), the write into the cache (`write`) and attention over it (`attend`).

`run` computes a case in elementary torch operations in 32 bits (angles in 64) or, where `own` is set, through the
package's entry points.  `exact` computes the same from the definitions in 64 bits.
"""
import math
import random

import torch

own = False

DEV = "cuda"
E_MIN, E_MAX = -48, 48            # exponents that a block's scale may take
Q_MAX = {"e4m3": 448.0, "i8": 127.0}
CACHE_DTYPE = {"e4m3": torch.float8_e4m3fn, "i8": torch.int8}


# ------------------------------------------------------------------------------------------------ cases
def listed():
    return [
        # one decode step of 32 sequences, 28 query and 4 key heads: the smallest call, latency
        dict(name="rope_step", op="rope", dtype="bf16", batch=32, seq=1, hq=28, hk=4, d=128, rot=128, planes=3,
             layout="blocks", pairing="halves", inverse=False, fused=True, far=20000),
        # the prompt of four long videos before Stage 2, views of one fused projection
        dict(name="rope_prompt", op="rope", dtype="bf16", batch=4, seq=2176, hq=28, hk=4, d=128, rot=128, planes=3,
             layout="blocks", pairing="halves", inverse=False, fused=True, far=20000),
        # the gradient of a vision encoder's two-axis positions over 16384 patches, 32 bits
        dict(name="rope_encoder_grad", op="rope", dtype="f32", batch=2, seq=16384, hq=16, hk=16, d=80, rot=80, planes=2,
             layout="per_axis", pairing="adjacent", inverse=True, fused=False, far=32),
        # 256 requests grow by a token each
        dict(name="plan_step", op="plan", batch=256, block=16, past_lo=195, past_hi=300, new_lo=1, new_hi=1, ending=0, mix=1),
        # a busy server: prompts arrive, running requests grow or shrink, others end
        dict(name="plan_prompts", op="plan", batch=1024, block=32, past_lo=1, past_hi=4000, new_lo=1, new_hi=700, ending=300, mix=2),
        # 256 sequences of the 11 % schedule append one token
        dict(name="write_step", op="write", dtype="bf16", cache="e4m3", batch=256, hk=32, d=128, block=16, past_lo=195,
             past_hi=259, new_lo=1, new_hi=1, padded=False, mix=3),
        # the survivors of Stage 2 at the 2880-token shape go into the cache as the prune call lays them out
        dict(name="write_survivors", op="write", dtype="bf16", cache="e4m3", batch=32, hk=32, d=128, block=16, past_lo=0,
             past_hi=0, new_lo=259, new_hi=259, padded=True, mix=4),
        # long videos from a 32-bit model, 64-token blocks of integers, rows of ragged length
        dict(name="write_frames_f32", op="write", dtype="f32", cache="i8", batch=4, hk=4, d=128, block=64, past_lo=0,
             past_hi=100, new_lo=12000, new_hi=16512, padded=False, mix=5),
        # one chat sequence, one token: latency
        dict(name="attend_one", op="attend", dtype="bf16", cache="e4m3", batch=1, hq=32, hk=32, d=128, block=16, past_lo=107,
             past_hi=107, new_lo=1, new_hi=1, causal=True, tail=0, mix=6),
        # a full decode batch
        dict(name="attend_step", op="attend", dtype="bf16", cache="e4m3", batch=256, hq=32, hk=32, d=128, block=16,
             past_lo=195, past_hi=300, new_lo=1, new_hi=1, causal=True, tail=0, mix=7),
        # a few long videos that were not pruned, grouped heads, 64-token blocks of integers
        dict(name="attend_frames", op="attend", dtype="bf16", cache="i8", batch=4, hq=28, hk=4, d=128, block=64,
             past_lo=9000, past_hi=16512, new_lo=1, new_hi=1, causal=True, tail=3, mix=8),
        # a chunk of a long prompt behind what the cache holds already
        dict(name="attend_chunk", op="attend", dtype="bf16", cache="e4m3", batch=2, hq=28, hk=4, d=128, block=64,
             past_lo=15000, past_hi=16384, new_lo=900, new_hi=1024, causal=True, tail=0, mix=9),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi + 0.49)))))


def draw(rng):
    op = rng.choice(["rope", "plan", "write", "attend", "attend"])
    mix = rng.randrange(1 << 30)
    if op == "rope":
        hk = rng.choice([1, 2, 4, 8, 16, 32])
        hq = hk * rng.choice([1, 1, 2, 4, 7, 8]) if hk <= 8 else hk
        d = rng.choice([32, 64, 72, 80, 96, 128, 128, 256])
        rot = rng.choice([d, d, d // 2])
        dtype = rng.choice(["bf16", "bf16", "f32"])
        rows = 70_000_000 // ((hq + hk) * d * (2 if dtype == "f32" else 1))
        batch = _log(rng, 1, min(256, rows))
        return dict(op=op, dtype=dtype, batch=batch, seq=_log(rng, 1, max(1, min(16384, rows // batch))), hq=hq, hk=hk, d=d, rot=rot,
                    planes=rng.choice([1, 2, 3, 3, 4]), layout=rng.choice(["blocks", "cycled", "per_axis"]),
                    pairing=rng.choice(["halves", "adjacent"]), inverse=rng.random() < 0.4, fused=rng.random() < 0.5,
                    far=_log(rng, 16, 500000))
    if op == "plan":
        batch = _log(rng, 1, 1024)
        decode = rng.random() < 0.4
        return dict(op=op, batch=batch, block=rng.choice([16, 32, 64, 128]), past_lo=1, past_hi=_log(rng, 2, 4000), new_lo=1,
                    new_hi=1 if decode else _log(rng, 1, 700), ending=rng.randrange(0, batch // 2 + 1), mix=mix)
    if op == "write":
        hk, d = rng.choice([1, 2, 4, 8, 16, 32]), rng.choice([64, 80, 96, 128, 128, 256])
        rows = 16_000_000 // (hk * d)
        batch = _log(rng, 1, min(256, rows))
        past = rng.choice([0, _log(rng, 1, 2000)])
        new = _log(rng, 1, max(1, min(16384, rows // batch)))
        return dict(op=op, dtype=rng.choice(["bf16", "bf16", "f32"]), cache=rng.choice(["e4m3", "i8"]), batch=batch, hk=hk, d=d,
                    block=rng.choice([16, 32, 64, 128]), past_lo=past // 2, past_hi=past, new_lo=max(1, new // 2), new_hi=new,
                    padded=rng.random() < 0.4, mix=mix)
    hk = rng.choice([1, 2, 4, 8, 32])
    hq = hk * rng.choice([1, 2, 4, 7, 8]) if hk <= 8 else hk
    d = rng.choice([64, 80, 96, 128, 128, 128, 256])
    kind = rng.choice(["one", "step", "few", "prompt"])
    dtype = rng.choice(["bf16", "bf16", "bf16", "f32"])
    new = {"one": 1, "step": 1, "few": rng.randint(2, 16), "prompt": _log(rng, 17, 1024)}[kind]
    batch = 1 if kind == "one" else _log(rng, 1, 4 if kind == "prompt" else 256)
    tokens = 60_000_000 // (hk * d)                                        # of the whole cache
    if new > 1:
        tokens = min(tokens, 600_000_000 // (new * hq))                    # scores that the plain form holds
    if dtype == "f32" and new > 16:
        tokens = min(tokens, 30_000_000_000 // (new * hq * d))
    past = _log(rng, 1, max(2, min(30000, tokens // batch)))
    return dict(op=op, dtype=dtype, cache=rng.choice(["e4m3", "i8"]), batch=batch, hq=hq, hk=hk, d=d, block=rng.choice([16, 32, 64, 128]),
                past_lo=past // 2, past_hi=past, new_lo=1 if kind == "few" else new, new_hi=new, causal=rng.random() < 0.8,
                tail=rng.choice([0, 0, 3]), mix=mix)


def _lengths(case, seed=0):
    """(past, new) of each sequence: the same set for every seed, in another order.  A `plan` case lets `ending` of its
    sequences shrink or end, and a few of the others start from nothing."""
    r = random.Random(case["mix"])
    pairs = []
    for i in range(case["batch"]):
        past, new = r.randint(case["past_lo"], case["past_hi"]), r.randint(case["new_lo"], case["new_hi"])
        if case["op"] == "plan":
            if i < case["ending"]:
                new = -past if r.random() < 0.7 else -r.randint(0, past)
            elif r.random() < 0.1:
                past = 0
        pairs.append((past, new))
    random.Random(seed).shuffle(pairs)
    return pairs


def work(case):
    es = 4 if case.get("dtype") == "f32" else 2
    if case["op"] == "rope":
        elems = case["batch"] * case["seq"] * (case["hq"] + case["hk"]) * case["d"]
        return {"bytes": 2 * elems * es + 4 * case["planes"] * case["batch"] * case["seq"] + 8 * (case["rot"] // 2),
                "flops": 3 * elems * case["rot"] // case["d"]}
    pairs, bs = _lengths(case), case["block"]
    rows = sum(max(n, 0) for _, n in pairs)
    if case["op"] == "plan":
        moved = sum(abs(-(-(p + n) // bs) - -(-p // bs)) for p, n in pairs)
        return {"bytes": 8 * len(pairs) + 4 * (2 * len(pairs) + 1) + 12 * rows + 8 * moved + 48, "flops": rows}
    blocks = sum(-(-(p + n) // bs) - p // bs for p, n in pairs)
    if case["op"] == "write":
        per = case["hk"] * case["d"]
        return {"bytes": 2 * rows * per * (es + 1) + 8 * blocks * case["hk"] + 4 * (blocks + 2 * len(pairs)), "flops": 6 * rows * per}
    tokens = sum(p + n for p, n in pairs)
    seen = sum(n * p + n * (n + 1) // 2 if case["causal"] else n * (p + n) for p, n in pairs)
    table = sum(-(-(p + n) // bs) for p, n in pairs)
    return {"bytes": 2 * tokens * case["hk"] * case["d"] + 8 * table * case["hk"] + 4 * table + rows * case["hq"] * (2 * case["d"] * es + 4),
            "flops": 4 * seen * case["hq"] * case["d"]}


# ------------------------------------------------------------------------------------------------ inputs
def _dtype(case):
    return torch.float32 if case["dtype"] == "f32" else torch.bfloat16


def _gen(seed):
    return torch.Generator(device=DEV).manual_seed(seed)


def _i32(values):
    return torch.tensor(values, dtype=torch.int32, device=DEV)


def _sections(pairs, planes):
    """Pairs of each axis: the first (time) has about half of the others' share, as three-axis models have it."""
    if planes == 1:
        return [pairs]
    first = max(1, pairs // (2 * planes - 1))
    rest = [(pairs - first) // (planes - 1)] * (planes - 1)
    rest[-1] += pairs - first - sum(rest)
    return [first] + rest


def _ladder(case):
    """(inv_freq, axis) of each pair."""
    n, sizes, base = case["rot"] // 2, _sections(case["rot"] // 2, case["planes"]), 10000.0
    if case["layout"] == "cycled":
        left, axis, a = list(sizes), [], 0
        while len(axis) < n:
            if left[a] > 0:
                left[a] -= 1
                axis.append(a)
            a = (a + 1) % len(left)
    else:
        axis = [a for a, s in enumerate(sizes) for _ in range(s)]
    if case["layout"] == "per_axis":
        freq = [base ** (-j / s) for s in sizes for j in range(s)]
    else:
        freq = [base ** (-i / n) for i in range(n)]
    return torch.tensor(freq, dtype=torch.float64).float().to(DEV), _i32(axis)


def _quantise_blocks(x, cache):
    """Quantises a pool [blocks, heads, block, d] with a power-of-two scale for each block and head."""
    e = _exponent(x.abs().amax((2, 3)), cache)
    scale = torch.exp2(e)
    y = x * torch.exp2(-e)[:, :, None, None]
    return (y if cache == "e4m3" else y.round()).to(CACHE_DTYPE[cache]), scale


def _pool(case, g, blocks, gain):
    """A cache whose blocks are all filled, keys with a few strong channels."""
    shape = (blocks, case["hk"], case["block"], case["d"])
    out = []
    for _ in range(2):
        x = torch.randn(shape, device=DEV, generator=g)
        x *= gain[:, None, :]
        out += list(_quantise_blocks(x, case["cache"]))
        gain = torch.ones_like(gain)
    kc, ks, vc, vs = out
    return kc, vc, ks, vs


def prepare(case, seed):
    g = _gen(seed)
    if case["op"] == "rope":
        B, S, H, d, dt = case["batch"], case["seq"], case["hq"] + case["hk"], case["d"], _dtype(case)
        if case["fused"]:       # one projection's output [B, S, q heads | k heads | v heads, d]
            x = torch.randn((B, S, H + case["hk"], d), device=DEV, generator=g).to(dt)
            q, k = x[:, :, :case["hq"]].transpose(1, 2), x[:, :, case["hq"]:H].transpose(1, 2)
        else:
            q = torch.randn((B, case["hq"], S, d), device=DEV, generator=g).to(dt)
            k = torch.randn((B, case["hk"], S, d), device=DEV, generator=g).to(dt)
        pos = torch.randint(0, case["far"], (case["planes"], B, S), device=DEV, generator=g, dtype=torch.int32)
        inv_freq, axis = _ladder(case)
        return {"case": case, "q": q, "k": k, "pos": pos, "inv_freq": inv_freq, "axis": axis,
                "q_out": torch.zeros((B, case["hq"], S, d), device=DEV, dtype=dt),
                "k_out": torch.zeros((B, case["hk"], S, d), device=DEV, dtype=dt)}
    pairs, bs, B = _lengths(case, seed), case["block"], case["batch"]
    past, new = [p for p, _ in pairs], [n for _, n in pairs]
    have = [-(-p // bs) for p in past]
    need = [-(-(p + n) // bs) for p, n in pairs]
    held = have if case["op"] == "plan" else need
    columns = max(1, max(max(a, b) for a, b in zip(have, need))) + 3
    blocks = sum(max(a, b) for a, b in zip(have, need)) + 5
    ids = torch.randperm(blocks, device=DEV, generator=g).to(torch.int32)
    col = torch.arange(columns, device=DEV)
    h = torch.tensor(held, device=DEV)
    first = torch.cumsum(h, 0) - h
    at = (first[:, None] + col).clamp(max=blocks - 1)
    table = torch.where(col < h[:, None], ids[at], torch.full_like(ids[at], -1)).contiguous()
    rows = sum(max(n, 0) for n in new)
    if case["op"] == "plan":
        used = sum(have)
        head = int(torch.randint(0, 10 * blocks, (1,), generator=torch.Generator().manual_seed(seed)))
        ring = torch.full((blocks,), -1, dtype=torch.int32, device=DEV)
        place = (head + torch.arange(blocks - used, device=DEV)) % blocks
        ring[place] = ids[used:]
        return {"case": case, "past": _i32(past), "new": _i32(new), "table": table, "ring": ring, "rows": rows + 7,
                "ring_state": torch.tensor([head, head + blocks - used], dtype=torch.int64, device=DEV),
                "kv_len": _i32([0] * B), "row_offset": _i32([0] * (B + 1)),
                "slot_map": torch.full((rows + 7,), -1, dtype=torch.int64, device=DEV),
                "row_pos": torch.full((rows + 7,), -1, dtype=torch.int32, device=DEV),
                "ring_state_out": torch.zeros(2, dtype=torch.int64, device=DEV), "report": _i32([0] * 4)}
    offsets = [0]
    for n in new:
        offsets.append(offsets[-1] + n)
    gain = torch.exp2(2.0 * (torch.rand((case["hk"], case["d"]), device=DEV, generator=g) < 0.03))
    kc, vc, ks, vs = _pool(case, g, blocks, gain)
    st = {"case": case, "kv_len": _i32([p + n for p, n in pairs]), "row_offset": _i32(offsets), "table": table,
          "k_cache": kc, "v_cache": vc, "k_scale": ks, "v_scale": vs, "max_new": max(new)}
    if case["op"] == "write":
        # later tokens are a little larger than what the cache holds: some scales have to grow
        lead = (B, max(new)) if case["padded"] else (rows,)
        for name, ch in (("k", gain), ("v", torch.ones_like(gain))):
            x = torch.randn((*lead, case["hk"], case["d"]), device=DEV, generator=g) * ch
            x *= 1 + (torch.rand((*lead, case["hk"], 1), device=DEV, generator=g) < 0.1) * 1.0
            x = x.to(_dtype(case))
            st[name] = x.transpose(1, 2).contiguous() if case["padded"] else x       # padded: [B, heads, rows, d]
        return st
    q = 1.5 * torch.randn((rows + case["tail"], case["hq"], case["d"]), device=DEV, generator=g)
    st.update(q=q.to(_dtype(case)), scale=case["d"] ** -0.5, out=torch.zeros_like(q, dtype=_dtype(case)),
              lse=torch.zeros((rows + case["tail"], case["hq"]), device=DEV))
    return st


# ------------------------------------------------------------------------------------------------ one pass
def run(st):
    if own:
        return _run_own(st)
    return {"rope": _rope, "plan": _plan, "write": _write, "attend": _attend}[st["case"]["op"]](st)


def _run_own(st):
    import paper_2505_22654_b200 as vscan
    c = st["case"]
    if c["op"] == "rope":
        return vscan.vscan_rope(st["q"], st["k"], st["pos"], st["inv_freq"], st["axis"],
                                pairing=vscan.ROPE_HALVES if c["pairing"] == "halves" else vscan.ROPE_ADJACENT,
                                inverse=c["inverse"], q_out=st["q_out"], k_out=st["k_out"])
    if c["op"] == "plan":
        out = {n: st[n] for n in ("kv_len", "row_offset", "slot_map", "row_pos", "ring_state_out", "report")}
        vscan.vscan_kv_plan(st["past"], st["new"], st["table"], st["ring"], st["ring_state"], c["block"], out=out)
        return {**out, "table": st["table"], "ring": st["ring"]}
    cache = (st["k_cache"], st["v_cache"], st["k_scale"], st["v_scale"])
    if c["op"] == "write":
        vscan.vscan_kv_write(st["k"], st["v"], st["kv_len"], st["row_offset"], st["table"], *cache)
        return cache
    if "workspace" not in st:      # as a server keeps it from step to step
        st["workspace"] = vscan.vscan_kv_attention_workspace(st["q"], st["table"], st["k_cache"], max_q_len=st["max_new"])
    vscan.vscan_kv_attention(st["q"], st["kv_len"], st["row_offset"], st["table"], *cache, scale=st["scale"],
                             max_q_len=st["max_new"], causal=c["causal"], out=st["out"], lse=st["lse"], workspace=st["workspace"])
    return st["out"], st["lse"]


def _rope(st):
    c = st["case"]
    n, sign = c["rot"] // 2, -1.0 if c["inverse"] else 1.0
    angle = st["pos"].double()[st["axis"].long()] * st["inv_freq"].double()[:, None, None]     # [pairs, B, S]
    cos, sin = (t.permute(1, 2, 0)[:, None].float() for t in (torch.cos(angle), sign * torch.sin(angle)))
    a, b = (slice(0, n), slice(n, 2 * n)) if c["pairing"] == "halves" else (slice(0, 2 * n, 2), slice(1, 2 * n, 2))

    def turn(x, out):
        x = x.float()
        y = x.clone(memory_format=torch.contiguous_format)
        y[..., a] = x[..., a] * cos - x[..., b] * sin
        y[..., b] = x[..., b] * cos + x[..., a] * sin
        return y.to(out.dtype)

    return turn(st["q"], st["q_out"]), turn(st["k"], st["k_out"])


def _owner(row_offset, rows):
    """The sequence of each of `rows` packed rows and the row's number within it."""
    row = torch.arange(rows, device=DEV)
    seq = torch.searchsorted(row_offset[1:].contiguous().long(), row, right=True)
    return row, seq.clamp(max=row_offset.numel() - 2), row - row_offset.long()[seq.clamp(max=row_offset.numel() - 2)]


def _plan(st):
    bs, B, blocks = st["case"]["block"], st["case"]["batch"], st["ring"].numel()
    past, new = st["past"].long(), st["new"].long()
    grow = new.clamp(min=0)
    kv_len = past + new
    row_offset = torch.cat([torch.zeros(1, dtype=torch.int64, device=DEV), torch.cumsum(grow, 0)])
    have, need = (past + bs - 1) // bs, (kv_len + bs - 1) // bs
    take, give = (need - have).clamp(min=0), (have - need).clamp(min=0)
    head, tail = st["ring_state"][0], st["ring_state"][1]
    columns = torch.arange(st["table"].shape[1], device=DEV)
    taken = (columns >= have[:, None]) & (columns < need[:, None])
    place = head + (torch.cumsum(take, 0) - take)[:, None] + columns - have[:, None]
    table = torch.where(taken, st["ring"][(place % blocks).long()], st["table"])
    given = (columns >= need[:, None]) & (columns < have[:, None])
    place = torch.where(given, (tail + (torch.cumsum(give, 0) - give)[:, None] + columns - need[:, None]) % blocks, blocks)
    ring = torch.cat([st["ring"], st["ring"][:1]])
    ring[place.reshape(-1)] = st["table"].reshape(-1)       # the extra entry takes what is not given back
    row, seq, i = _owner(row_offset, st["rows"])
    live = row < row_offset[-1]
    pos = past[seq] + i
    col = (pos // bs).clamp(0, columns.numel() - 1)
    slot = table[seq, col].long() * bs + pos % bs
    return {"kv_len": kv_len.int(), "row_offset": row_offset.int(), "slot_map": torch.where(live, slot, st["slot_map"]),
            "row_pos": torch.where(live, pos, st["row_pos"].long()).int(),
            "ring_state_out": torch.stack([head + take.sum(), tail + give.sum()]),
            "report": torch.stack([torch.zeros_like(head), take.sum(), give.sum(), row_offset[-1]]).int(),
            "table": table, "ring": ring[:blocks]}


def _exponent(amax, cache):
    """The least e with amax <= qmax * 2^e, between E_MIN and E_MAX; NaN where amax is infinite or none."""
    m, e = torch.frexp(amax)                                   # amax = m * 2^e, m in [0.5, 1)
    top, bits = (0.875, 9) if cache == "e4m3" else (0.9921875, 7)
    e = (e - bits + (m > top)).float()
    e = torch.where(amax == 0, torch.full_like(e, E_MIN), e).clamp(E_MIN, E_MAX)
    return torch.where(torch.isfinite(amax), e, torch.full_like(e, math.nan))


def _code(x, cache):
    """32-bit values, already divided by their scale, to codes; NaN to the code of 0."""
    top = Q_MAX[cache]
    x = torch.where(torch.isnan(x), torch.zeros_like(x), x.clamp(-top, top))
    return (x if cache == "e4m3" else torch.round(x)).to(CACHE_DTYPE[cache]).view(torch.uint8)


def _write(st):
    c, bs = st["case"], st["case"]["block"]
    row_offset, kv_len, table = st["row_offset"].long(), st["kv_len"].long(), st["table"].long()
    new = row_offset[1:] - row_offset[:-1]
    if c["padded"]:
        B, H, n, d = st["k"].shape
        seq = torch.arange(B, device=DEV).repeat_interleave(n)
        i = torch.arange(n, device=DEV).repeat(B)
        sources = [t.transpose(1, 2).reshape(B * n, H, d).float() for t in (st["k"], st["v"])]
    else:
        _, seq, i = _owner(row_offset, st["k"].shape[0])
        sources = [st["k"].float(), st["v"].float()]
    live = (i < new[seq])[:, None]
    start = kv_len - new
    pos = (start[seq] + i).clamp(min=0)
    column = (pos // bs).clamp(max=table.shape[1] - 1)
    block = table[seq, column]
    blocks = st["k_cache"].shape[0]
    block = torch.where(live[:, 0], block, blocks)                         # an extra block takes the rows that are not there
    kept = start % bs                                                      # tokens that a sequence's first block already holds
    edge = torch.where((kept > 0) & (new > 0), table.gather(1, (start // bs).clamp(max=table.shape[1] - 1)[:, None])[:, 0], blocks)
    old_row = torch.arange(bs, device=DEV) < kept[:, None]                 # [B, bs]
    done = []
    for x, codes, scale in zip(sources, (st["k_cache"], st["v_cache"]), (st["k_scale"], st["v_scale"])):
        bad = ~torch.isfinite(x).all(-1)
        amax = torch.where(bad, torch.full_like(x[..., 0], math.inf), x.abs().amax(-1))
        peak = torch.full((blocks + 1, c["hk"]), -1.0, device=DEV).scatter_reduce(0, block[:, None].expand_as(amax), amax, "amax")
        wide = torch.cat([scale, torch.zeros_like(scale[:1])])
        carried = torch.zeros_like(wide)
        carried[edge] = wide[edge]
        fresh = torch.exp2(_exponent(peak.clamp(min=0), c["cache"]))
        now = torch.where(peak < 0, wide, torch.where(torch.isnan(carried), carried, torch.maximum(carried, fresh)))
        pool = torch.cat([codes.view(torch.uint8), codes[:1].view(torch.uint8)])
        held = pool[edge]                                                  # [B, heads, bs, d]
        ratio = (wide[edge] / now[edge])[:, :, None, None]
        again = _code(held.view(CACHE_DTYPE[c["cache"]]).float() * ratio, c["cache"])
        pool[edge] = torch.where(old_row[:, None, :, None], again, held)
        pool[block, :, pos % bs] = _code(x / now[block][..., None], c["cache"])
        done.append((pool[:blocks].view(CACHE_DTYPE[c["cache"]]), now[:blocks]))
    return done[0][0], done[1][0], done[0][1], done[1][1]


def _attend(st):
    c, bs = st["case"], st["case"]["block"]
    B, H, G, d = c["batch"], c["hk"], c["hq"] // c["hk"], c["d"]
    row_offset, kv_len, top = st["row_offset"].long(), st["kv_len"].long(), st["max_new"]
    new = row_offset[1:] - row_offset[:-1]
    i = torch.arange(top, device=DEV)
    live = i < new[:, None]                                                # [B, top]
    row = torch.where(live, row_offset[:-1, None] + i, 0)
    q = st["q"].float()[row].reshape(B, top, H, G, d).permute(0, 2, 3, 1, 4).reshape(B, H, G * top, d)
    ids = st["table"].long().clamp(min=0)
    T = ids.shape[1] * bs
    k, v = ((codes[ids].float() * scale[ids][..., None, None]).permute(0, 2, 1, 3, 4).reshape(B, H, T, d)
            for codes, scale in ((st["k_cache"], st["k_scale"]), (st["v_cache"], st["v_scale"])))
    s = torch.matmul(q, k.transpose(2, 3)).mul_(st["scale"]).view(B, H, G, top, T)
    key = torch.arange(T, device=DEV)
    last = kv_len[:, None] - new[:, None] + i if c["causal"] else (kv_len - 1)[:, None].expand(B, top)
    s.masked_fill_((key > last[..., None])[:, None, None], -math.inf)
    m = s.amax(-1, keepdim=True)
    p = s.sub_(torch.where(torch.isinf(m), torch.zeros_like(m), m)).exp_()
    total = p.sum(-1, keepdim=True)
    o = torch.matmul(p.view(B, H, G * top, T), v).view(B, H, G, top, d) / torch.where(total > 0, total, torch.ones_like(total))
    lse = (m + torch.log(total))[..., 0]
    rows = st["q"].shape[0]
    at = torch.where(live, row, rows).reshape(-1)                          # an extra row takes what is not there
    out, stats = torch.cat([st["out"], st["out"][:1]]), torch.cat([st["lse"], st["lse"][:1]])
    out[at] = o.permute(0, 3, 1, 2, 4).reshape(B * top, H * G, d).to(out.dtype)
    stats[at] = lse.permute(0, 3, 1, 2).reshape(B * top, H * G)
    return out[:rows], stats[:rows]


# ------------------------------------------------------------------------------------------------ 64 bits
def exact(case, seed):
    st = prepare(case, seed)
    return {"rope": _exact_rope, "plan": _exact_plan, "write": _exact_write, "attend": _exact_attend}[case["op"]](st)


def _exact_rope(st):
    c = st["case"]
    pairs = c["rot"] // 2
    done = []
    for x in (st["q"], st["k"]):
        y = x.double().contiguous()
        src = y.clone()
        for p in range(pairs):
            i, j = (p, p + pairs) if c["pairing"] == "halves" else (2 * p, 2 * p + 1)
            theta = st["pos"][int(st["axis"][p])].double() * st["inv_freq"][p].double()
            if c["inverse"]:
                theta = -theta
            z = torch.complex(src[..., i], src[..., j]) * torch.polar(torch.ones_like(theta), theta)[:, None]
            y[..., i], y[..., j] = z.real, z.imag
        done.append(y)
    return tuple(done)


def _exact_plan(st):
    bs, blocks = st["case"]["block"], st["ring"].numel()
    past, new, table, ring = (st[n].tolist() for n in ("past", "new", "table", "ring"))
    (head, tail), source = st["ring_state"].tolist(), st["ring"].tolist()
    slots, places = st["slot_map"].tolist(), st["row_pos"].tolist()
    offsets, lens, taken, given = [0], [], 0, 0
    for b, (p, n) in enumerate(zip(past, new)):
        lens.append(p + n)
        have, need = -(-p // bs), -(-(p + n) // bs)
        for j in range(have, need):
            table[b][j] = source[(head + taken) % blocks]
            taken += 1
        for j in range(need, have):
            ring[(tail + given) % blocks] = table[b][j]
            given += 1
        for t in range(p, p + n):
            r = offsets[-1] + t - p
            slots[r], places[r] = table[b][t // bs] * bs + t % bs, t
        offsets.append(offsets[-1] + max(n, 0))
    return {"kv_len": _i32(lens), "row_offset": _i32(offsets), "slot_map": torch.tensor(slots), "row_pos": _i32(places),
            "ring_state_out": torch.tensor([head + taken, tail + given]), "report": _i32([0, taken, given, offsets[-1]]),
            "table": _i32(table), "ring": _i32(ring)}


def _exact_code(x, cache):
    """Nearest value of the cache's type, ties to even."""
    if cache == "i8":
        return torch.round(x).clamp(-127, 127)
    _, e = torch.frexp(x)
    step = torch.exp2((e - 1).clamp(min=-6).double() - 3)
    return (torch.round(x / step) * step).clamp(-448, 448)


def _exact_write(st):
    c, bs = st["case"], st["case"]["block"]
    offsets, lens, table = st["row_offset"].tolist(), st["kv_len"].tolist(), st["table"].tolist()
    done = []
    for name, codes, scale in (("k", st["k_cache"], st["k_scale"]), ("v", st["v_cache"], st["v_scale"])):
        codes, scale = codes.float().double(), scale.double().clone()
        for b, end in enumerate(lens):
            n = offsets[b + 1] - offsets[b]
            x = st[name][b, :, :n] if c["padded"] else st[name][offsets[b]:offsets[b + 1]].transpose(0, 1)
            x, start = x.double(), end - n                                 # [heads, n, d]
            whole = -(-n // bs) + 1
            first = start // bs
            canvas = torch.zeros((c["hk"], whole * bs + bs, c["d"]), dtype=torch.float64, device=DEV)
            canvas[:, start - first * bs:start - first * bs + n] = x
            used = -(-end // bs) - first
            canvas = canvas[:, :used * bs].view(c["hk"], used, bs, c["d"])
            need = canvas.abs().amax((2, 3)) / Q_MAX[c["cache"]]           # [heads, used]
            grid = torch.exp2(torch.arange(E_MIN, E_MAX + 1, device=DEV, dtype=torch.float64))
            s = grid[torch.searchsorted(grid, need.contiguous()).clamp(max=grid.numel() - 1)]
            ids = torch.tensor(table[b][first:first + used], device=DEV)
            kept = start - first * bs
            old = codes[ids[0], :, :kept] if kept else None
            if kept:
                s[:, 0] = torch.maximum(s[:, 0], scale[ids[0]])
                old = _exact_code(old * (scale[ids[0]] / s[:, 0])[:, None, None], c["cache"])
            y = _exact_code(canvas / s[:, :, None, None], c["cache"])
            for j, lo, hi in {(0, kept, min(bs, kept + n)), (used - 1, kept if used == 1 else 0, end - (first + used - 1) * bs)}:
                codes[ids[j], :, lo:hi] = y[:, j, lo:hi]
            if used > 2:
                codes[ids[1:-1]] = y[:, 1:-1].transpose(0, 1)
            if kept:
                codes[ids[0], :, :kept] = old
            scale[ids] = s.transpose(0, 1)
        done.append((codes if c["cache"] == "e4m3" else codes.to(torch.int8), scale))
    return done[0][0], done[1][0], done[0][1], done[1][1]


def _exact_attend(st):
    c, bs = st["case"], st["case"]["block"]
    H, G, d = c["hk"], c["hq"] // c["hk"], c["d"]
    out, lse = st["out"].double(), st["lse"].double()
    offsets, lens = st["row_offset"].tolist(), st["kv_len"].tolist()
    for b, T in enumerate(lens):
        lo, hi = offsets[b], offsets[b + 1]
        n = hi - lo
        if n == 0:
            continue
        ids = st["table"][b, :-(-T // bs)].long()
        for h in range(H) if n * T * c["hq"] > 10_000_000 else (slice(None),):
            heads = slice(h, h + 1) if isinstance(h, int) else h
            k, v = ((codes[ids][:, heads].float().double() * scale[ids][:, heads, None, None].double()).transpose(0, 1).reshape(-1, len(ids) * bs, d)[:, :T]
                    for codes, scale in ((st["k_cache"], st["k_scale"]), (st["v_cache"], st["v_scale"])))
            q = st["q"][lo:hi].double().view(n, H, G, d)[:, heads].permute(1, 2, 0, 3)                # [heads, G, n, d]
            s = st["scale"] * torch.einsum("hgnd,htd->hgnt", q, k)
            if c["causal"]:
                hidden = torch.arange(T, device=DEV) > T - n + torch.arange(n, device=DEV)[:, None]
                s = s.masked_fill(hidden, -math.inf)
            z = torch.logsumexp(s, -1)
            o = torch.einsum("hgnt,htd->nhgd", torch.exp(s - z[..., None]), v)
            out[lo:hi].view(n, H, G, d)[:, heads] = o
            lse[lo:hi].view(n, H, G)[:, heads] = z.permute(2, 0, 1)
    return out, lse
