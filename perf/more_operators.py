"""What is measured of the operators around a prompt and of a cache that is kept short: attention over whole prompts in the model's
own type (`prompt`), attention weights gathered for each cached token (`weigh`), and the eviction of the tokens that
gathered least (`evict`).

`run` computes a case in elementary torch operations in 32 bits or, where `own` is set, through the package's entry points.
`exact` computes the same from the definitions in 64 bits.
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
        # the text and the survivors of one image, 28 query and 4 key heads: the smallest prompt, latency
        dict(name="prompt_one", op="prompt", dtype="bf16", batch=1, hq=28, hk=4, d=128, q_lo=197, q_hi=197, past_lo=0, past_hi=0,
             causal=True, padded=False, tail=0, mix=1),
        # four videos through the layers in front of Stage 2
        dict(name="prompt_videos", op="prompt", dtype="bf16", batch=4, hq=28, hk=4, d=128, q_lo=1700, q_hi=2176, past_lo=0, past_hi=0,
             causal=True, padded=False, tail=5, mix=2),
        # a layer of a vision encoder over 160 crops of 576 patches and a [CLS] token, every token sees every other
        dict(name="prompt_encoder", op="prompt", dtype="bf16", batch=160, hq=16, hk=16, d=64, q_lo=577, q_hi=577, past_lo=0, past_hi=0,
             causal=False, padded=True, tail=0, mix=3),
        # two long documents with many pages: the largest
        dict(name="prompt_long", op="prompt", dtype="bf16", batch=2, hq=28, hk=4, d=128, q_lo=9000, q_hi=12200, past_lo=0, past_hi=0,
             causal=True, padded=False, tail=0, mix=4),
        # questions behind long videos whose keys are in memory already, in the model's type
        dict(name="prompt_behind", op="prompt", dtype="bf16", batch=5, hq=32, hk=32, d=128, q_lo=20, q_hi=130, past_lo=2000, past_hi=5000,
             causal=True, padded=False, tail=0, mix=5),
        # an encoder with heads of 80 in 32 bits, images of any size
        dict(name="prompt_f32", op="prompt", dtype="f32", batch=3, hq=16, hk=16, d=80, q_lo=250, q_hi=1030, past_lo=0, past_hi=0,
             causal=False, padded=False, tail=3, mix=6),
        # one decode step of 256 sequences
        dict(name="weigh_step", op="weigh", dtype="bf16", cache="e4m3", batch=256, hq=32, hk=32, d=128, block=16, past_lo=195, past_hi=300,
             new_lo=1, new_hi=1, window=1, decay=1.0, causal=True, mix=7),
        # one decode step of a single sequence
        dict(name="weigh_one", op="weigh", dtype="bf16", cache="i8", batch=1, hq=28, hk=4, d=128, block=64, past_lo=700, past_hi=700,
             new_lo=1, new_hi=1, window=1, decay=0.98, causal=True, mix=8),
        # two long prompts, just written: what their last 512 rows look at
        dict(name="weigh_window", op="weigh", dtype="bf16", cache="e4m3", batch=2, hq=28, hk=4, d=128, block=32, past_lo=15000, past_hi=16000,
             new_lo=900, new_hi=1024, window=512, decay=1.0, causal=True, mix=9),
        # decode steps of long sequences: 256 sequences let go of a block's worth of tokens each
        dict(name="evict_step", op="evict", cache="e4m3", batch=256, hk=32, d=128, block=16, len_lo=240, len_hi=300, keep_lo=224, keep_hi=224,
             first=4, last=32, per_head=True, mix=10),
        # eight long prompts down to 2048 tokens a head
        dict(name="evict_prompt", op="evict", cache="i8", batch=8, hk=8, d=128, block=64, len_lo=12000, len_hi=16400, keep_lo=2048, keep_hi=2048,
             first=16, last=256, per_head=True, mix=11),
        # one sequence down to its half, all heads alike: latency
        dict(name="evict_one", op="evict", cache="e4m3", batch=1, hk=4, d=128, block=32, len_lo=2100, len_hi=2100, keep_lo=1000, keep_hi=1000,
             first=4, last=64, per_head=False, mix=12),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi + 0.49)))))


def draw(rng):
    op = rng.choice(["prompt", "prompt", "prompt", "weigh", "weigh", "evict", "evict"])
    mix = rng.randrange(1 << 30)
    hk = rng.choice([1, 2, 4, 8, 16, 32])
    group = rng.choice([1, 1, 2, 4, 7, 8]) if hk <= 8 else 1
    hq = hk * group
    if op == "prompt":
        dtype = rng.choice(["bf16", "bf16", "bf16", "f32"])
        d = rng.choice([32, 64, 64, 72, 80, 96, 128, 128, 128, 256])
        batch = _log(rng, 1, 128)
        pairs = 1_500_000_000 // hq                                        # (row, key) pairs that the plain form holds
        if dtype == "f32":
            pairs = min(pairs, 30_000_000_000 // (hq * d))
        q = _log(rng, 1, max(1, min(8192, math.isqrt(pairs // batch))))
        past = rng.choice([0, 0, _log(rng, 1, max(2, min(16000, pairs // (batch * q) - q)))]) if pairs // (batch * q) > q + 2 else 0
        past = min(past, 100_000_000 // (batch * hk * d))
        return dict(op=op, dtype=dtype, batch=batch, hq=hq, hk=hk, d=d, q_lo=max(1, q // 2), q_hi=q, past_lo=past // 2, past_hi=past,
                    causal=rng.random() < 0.7, padded=rng.random() < 0.4, tail=rng.choice([0, 0, 3]), mix=mix)
    cache, block = rng.choice(["e4m3", "i8"]), rng.choice([16, 32, 64, 128])
    d = rng.choice([64, 80, 96, 128, 128, 128, 256])
    batch = _log(rng, 1, 256)
    if op == "weigh":
        kind = rng.choice(["step", "few", "window"])
        batch = min(batch, 8) if kind == "window" else batch
        new = {"step": 1, "few": rng.randint(2, 16), "window": _log(rng, 17, 1024)}[kind]
        tokens = min(40_000_000 // (hk * d), 500_000_000 // (new * hq))
        past = _log(rng, 16, max(32, min(30000, tokens // batch)))
        return dict(op=op, dtype=rng.choice(["bf16", "bf16", "bf16", "f32"]), cache=cache, batch=batch, hq=hq, hk=hk, d=d, block=block,
                    past_lo=past // 2, past_hi=past, new_lo=1 if kind == "few" else new, new_hi=new,
                    window=new if kind != "window" else _log(rng, 1, new), decay=rng.choice([1.0, 1.0, 0.95, 0.0]), causal=rng.random() < 0.8,
                    mix=mix)
    tokens = 100_000_000 // (hk * d * batch)
    length = _log(rng, 8, max(16, min(20000, tokens)))
    keep = max(4, int(length * rng.uniform(0.05, 0.9)))
    return dict(op=op, cache=cache, batch=batch, hk=hk, d=d, block=block, len_lo=max(2, length // 2), len_hi=length, keep_lo=max(2, keep // 2),
                keep_hi=keep, first=rng.choice([0, 0, 4]), last=rng.choice([0, 1, keep // 8]), per_head=rng.random() < 0.6, mix=mix)


def _lengths(case, seed=0):
    """(before, new) of each sequence, or (length, kept) for an eviction: the same set for every seed, in another order."""
    r = random.Random(case["mix"])
    names = {"prompt": ("past", "q"), "weigh": ("past", "new"), "evict": ("len", "keep")}[case["op"]]
    pairs = [tuple(r.randint(case[n + "_lo"], case[n + "_hi"]) for n in names) for _ in range(case["batch"])]
    random.Random(seed).shuffle(pairs)
    return pairs


def work(case):
    pairs = _lengths(case)
    if case["op"] == "prompt":
        es = 4 if case["dtype"] == "f32" else 2
        rows, keys = sum(n for _, n in pairs), sum(p + n for p, n in pairs)
        seen = sum(n * p + n * (n + 1) // 2 if case["causal"] else n * (p + n) for p, n in pairs)
        return {"bytes": rows * case["hq"] * (2 * case["d"] * es + 4) + 2 * keys * case["hk"] * case["d"] * es + 8 * len(pairs),
                "flops": 4 * seen * case["hq"] * case["d"]}
    bs, per = case["block"], case["hk"] * case["d"]
    if case["op"] == "weigh":
        es, tokens = 4 if case["dtype"] == "f32" else 2, sum(p + n for p, n in pairs)
        used = [min(n, case["window"]) for _, n in pairs]
        seen = sum(u * (p + n) - (u * (u - 1) // 2 if case["causal"] else 0) for (p, n), u in zip(pairs, used))
        table = sum(-(-(p + n) // bs) for p, n in pairs)
        return {"bytes": tokens * (per + 4 * case["hk"]) + 4 * sum(p for p, _ in pairs) * case["hk"] + 4 * table * (1 + case["hk"]) +
                sum(used) * case["hq"] * (case["d"] * es + 4), "flops": 2 * seen * case["hq"] * case["d"]}
    kept = sum(min(n, k) for n, k in pairs)
    heads = case["hk"] if case["per_head"] else 1
    blocks = sum(-(-n // bs) + -(-min(n, k) // bs) for n, k in pairs)
    return {"bytes": 4 * sum(n for n, _ in pairs) * case["hk"] + 4 * kept * (heads + case["hk"]) + 4 * kept * per +
            8 * blocks * case["hk"] + 4 * blocks + 12 * len(pairs), "flops": 2 * kept * per}


# ------------------------------------------------------------------------------------------------ inputs
def _dtype(case):
    return torch.float32 if case["dtype"] == "f32" else torch.bfloat16


def _gen(seed):
    return torch.Generator(device=DEV).manual_seed(seed)


def _i32(values):
    return torch.tensor(values, dtype=torch.int32, device=DEV)


def _offsets(counts):
    offsets = [0]
    for n in counts:
        offsets.append(offsets[-1] + n)
    return offsets


def _rows(case, g, heads, counts, tail, gain):
    """Rows of every sequence: packed one after another, or [batch, heads, rows, d]."""
    if case["padded"]:
        x = torch.randn((case["batch"], heads, max(counts) + tail, case["d"]), device=DEV, generator=g) * gain[:, None]
    else:
        x = torch.randn((sum(counts) + tail, heads, case["d"]), device=DEV, generator=g) * gain
    return x.to(_dtype(case))


def _strong_channels(case, g):
    return torch.exp2(2.0 * (torch.rand((case["hk"], case["d"]), device=DEV, generator=g) < 0.03))


def _pool(case, g, blocks):
    """A cache whose blocks are all filled, keys with a few strong channels, a power-of-two scale for each block and head."""
    gain, out = _strong_channels(case, g), []
    for _ in range(2):
        x = torch.randn((blocks, case["hk"], case["block"], case["d"]), device=DEV, generator=g)
        x *= gain[:, None, :]
        e = _exponent(x.abs().amax((2, 3)), case["cache"])
        y = x * torch.exp2(-e)[:, :, None, None]
        out += [(y if case["cache"] == "e4m3" else y.round()).to(CACHE_DTYPE[case["cache"]]), torch.exp2(e)]
        gain = torch.ones_like(gain)
    return {"k_cache": out[0], "v_cache": out[2], "k_scale": out[1], "v_scale": out[3]}


def _table(case, g, lengths):
    """Blocks of a pool in any order for sequences of these lengths; columns behind them hold -1."""
    held = torch.tensor([-(-n // case["block"]) for n in lengths], device=DEV)
    columns, blocks = int(held.max()) + 3, int(held.sum()) + 5
    ids = torch.randperm(blocks, device=DEV, generator=g).to(torch.int32)
    col = torch.arange(columns, device=DEV)
    first = torch.cumsum(held, 0) - held
    at = (first[:, None] + col).clamp(max=blocks - 1)
    return torch.where(col < held[:, None], ids[at], torch.full_like(ids[at], -1)).contiguous(), blocks


def prepare(case, seed):
    g = _gen(seed)
    pairs = _lengths(case, seed)
    if case["op"] == "prompt":
        new, keys = [n for _, n in pairs], [p + n for p, n in pairs]
        q = _rows(case, g, case["hq"], new, case["tail"], torch.full((case["hq"], case["d"]), 1.5, device=DEV))
        gain = _strong_channels(case, g)
        return {"case": case, "q": q, "k": _rows(case, g, case["hk"], keys, case["tail"], gain),
                "v": _rows(case, g, case["hk"], keys, case["tail"], torch.ones_like(gain)), "row_offset": _i32(_offsets(new)),
                "kv_offset": _i32(_offsets(keys)), "max_new": max(new), "scale": case["d"] ** -0.5, "out": torch.zeros_like(q),
                "lse": torch.zeros(q.shape[:-1], device=DEV)}
    if case["op"] == "weigh":
        lengths, new = [p + n for p, n in pairs], [n for _, n in pairs]
        table, blocks = _table(case, g, lengths)
        st = {"case": case, "kv_len": _i32(lengths), "row_offset": _i32(_offsets(new)), "table": table, "max_new": max(new),
              "scale": case["d"] ** -0.5, **_pool(case, g, blocks)}
        del st["v_cache"], st["v_scale"]
        st["q"] = (1.5 * torch.randn((sum(new), case["hq"], case["d"]), device=DEV, generator=g)).to(_dtype(case))
        # what the attention of the step left: the logarithm of each row's sum (rows in front of the window are not asked for)
        s, row, live = _scores(st)
        lse = torch.zeros((sum(new) + 1, case["hq"]), device=DEV)
        at = torch.where(live, row, sum(new)).reshape(-1)
        lse[at] = torch.logsumexp(s, -1).permute(0, 3, 1, 2).reshape(at.numel(), case["hq"])
        st["lse"] = lse[:-1].contiguous()
        st["weight"] = torch.rand((blocks, case["hk"], case["block"]), device=DEV, generator=g) ** 8 * 20
        return st
    lengths, keep = [n for n, _ in pairs], [k for _, k in pairs]
    table, blocks = _table(case, g, lengths)
    # few tokens gather most of the weight, many none at all, and heads agree in part
    shape = (blocks, case["hk"], case["block"])
    w = torch.exp(1.5 * torch.randn((blocks, 1, case["block"]), device=DEV, generator=g) + 1.5 * torch.randn(shape, device=DEV, generator=g))
    w *= torch.rand((blocks, 1, case["block"]), device=DEV, generator=g) > 0.05
    return {"case": case, "kv_len": _i32(lengths), "budget": _i32(keep), "table": table, "weight": w, "weight_out": torch.zeros_like(w),
            "max_keep": max(keep), "delta": _i32([0] * len(pairs)),
            "kept": torch.full((len(pairs), case["hk"] if case["per_head"] else 1, max(keep)), -1, dtype=torch.int32, device=DEV),
            **_pool(case, g, blocks)}


# ------------------------------------------------------------------------------------------------ one pass
def run(st):
    if own:
        return _run_own(st)
    return {"prompt": _prompt, "weigh": _weigh, "evict": _evict}[st["case"]["op"]](st)


def _run_own(st):
    import paper_2505_22654_b200 as vscan
    c = st["case"]
    if c["op"] == "prompt":
        if "workspace" not in st:      # as a server keeps it from step to step
            st["workspace"] = vscan.vscan_attention_workspace(st["q"], st["k"], st["row_offset"], max_q_len=st["max_new"])
        vscan.vscan_attention(st["q"], st["k"], st["v"], st["row_offset"], scale=st["scale"], max_q_len=st["max_new"],
                              kv_offset=st["kv_offset"], causal=c["causal"], out=st["out"], lse=st["lse"], workspace=st["workspace"])
        return st["out"], st["lse"]
    if c["op"] == "weigh":
        vscan.vscan_kv_weigh(st["q"], st["lse"], st["kv_len"], st["row_offset"], st["table"], st["k_cache"], st["k_scale"], st["weight"],
                             scale=st["scale"], max_q_len=st["max_new"], decay=c["decay"], window=c["window"], causal=c["causal"])
        return st["weight"]
    cache = (st["k_cache"], st["v_cache"], st["k_scale"], st["v_scale"])
    if "workspace" not in st:
        st["workspace"] = vscan.vscan_kv_evict_workspace(st["table"], st["k_cache"], max_keep=st["max_keep"], per_head=c["per_head"])
    vscan.vscan_kv_evict(st["kv_len"], st["budget"], st["table"], st["weight"], *cache, max_keep=st["max_keep"], keep_first=c["first"],
                         keep_last=c["last"], per_head=c["per_head"], weight_out=st["weight_out"], kept=st["kept"], delta=st["delta"],
                         workspace=st["workspace"])
    return (*cache, st["weight_out"], st["kept"], st["delta"])


def _softmax_rows(s):
    """Weights that are not yet divided, their sums, and the logarithms; a row that sees nothing has sum 0 and -inf."""
    m = s.amax(-1, keepdim=True)
    p = s.sub_(torch.where(torch.isinf(m), torch.zeros_like(m), m)).exp_()
    total = p.sum(-1, keepdim=True)
    return p, total, (m + torch.log(total))[..., 0]


def _prompt(st):
    c = st["case"]
    B, H, G, d, top = c["batch"], c["hk"], c["hq"] // c["hk"], c["d"], st["max_new"]
    row_offset, kv_offset = st["row_offset"].long(), st["kv_offset"].long()
    new, length = row_offset[1:] - row_offset[:-1], kv_offset[1:] - kv_offset[:-1]
    i = torch.arange(top, device=DEV)
    live = i < new[:, None]                                                # [B, top]
    row = torch.where(live, row_offset[:-1, None] + i, 0)
    if c["padded"]:
        q, k, v = st["q"][:, :, :top].float(), st["k"].float(), st["v"].float()
        T = k.shape[2]
    else:
        T = st["k"].shape[0]
        T = min(T, int(c["q_hi"] + c["past_hi"]))
        at = (kv_offset[:-1, None] + torch.arange(T, device=DEV)).clamp(max=st["k"].shape[0] - 1)
        q, k, v = (x.float()[r].transpose(1, 2) for x, r in ((st["q"], row), (st["k"], at), (st["v"], at)))
    s = torch.matmul(q.reshape(B, H, G * top, d), k.transpose(2, 3)).mul_(st["scale"]).view(B, H, G, top, T)
    last = length[:, None] - new[:, None] + i if c["causal"] else (length - 1)[:, None].expand(B, top)
    s.masked_fill_((torch.arange(T, device=DEV) > last[..., None])[:, None, None], -math.inf)
    p, total, lse = _softmax_rows(s)
    o = torch.matmul(p.view(B, H, G * top, T), v).view(B, H, G, top, d) / torch.where(total > 0, total, torch.ones_like(total))
    o, lse = o.view(B, H * G, top, d).to(st["out"].dtype), lse.reshape(B, H * G, top)
    if c["padded"]:
        out, stats, on = st["out"].clone(), st["lse"].clone(), live[:, None]
        out[:, :, :top] = torch.where(on[..., None], o, out[:, :, :top])
        stats[:, :, :top] = torch.where(on, lse, stats[:, :, :top])
        return out, stats
    rows = st["q"].shape[0]
    at = torch.where(live, row, rows).reshape(-1)                          # an extra row takes what is not there
    out, stats = torch.cat([st["out"], st["out"][:1]]), torch.cat([st["lse"], st["lse"][:1]])
    out[at] = o.transpose(1, 2).reshape(B * top, H * G, d)
    stats[at] = lse.transpose(1, 2).reshape(B * top, H * G)
    return out[:rows], stats[:rows]


def _scores(st):
    """Scores [B, heads, group, rows of the window, tokens] of the window's rows against the cached keys, -inf where a row does
    not see; the packed row of each, and which of them are there."""
    c, bs = st["case"], st["case"]["block"]
    B, H, G, d = c["batch"], c["hk"], c["hq"] // c["hk"], c["d"]
    row_offset, kv_len = st["row_offset"].long(), st["kv_len"].long()
    new = row_offset[1:] - row_offset[:-1]
    top = min(st["max_new"], c["window"])
    i = new[:, None] - top + torch.arange(top, device=DEV)                 # the last `top` rows of each sequence
    live = i >= 0
    row = torch.where(live, row_offset[:-1, None] + i, 0)
    q = st["q"].float()[row].reshape(B, top, H, G, d).permute(0, 2, 3, 1, 4).reshape(B, H, G * top, d)
    ids = st["table"].long().clamp(min=0)
    T = ids.shape[1] * bs
    k = (st["k_cache"][ids].float() * st["k_scale"][ids][..., None, None]).permute(0, 2, 1, 3, 4).reshape(B, H, T, d)
    s = torch.matmul(q, k.transpose(2, 3)).mul_(st["scale"]).view(B, H, G, top, T)
    last = kv_len[:, None] - new[:, None] + i if c["causal"] else (kv_len - 1)[:, None].expand(B, top)
    last = torch.where(live, last, -1)
    return s.masked_fill_((torch.arange(T, device=DEV) > last[..., None])[:, None, None], -math.inf), row, live


def _weigh(st):
    c, bs = st["case"], st["case"]["block"]
    B, H = c["batch"], c["hk"]
    s, row, live = _scores(st)
    lse = st["lse"][row].reshape(B, row.shape[1], H, -1).permute(0, 2, 3, 1)          # [B, heads, group, rows]
    given = s.sub_(lse[..., None]).exp_().sum((2, 3))                                  # [B, heads, tokens]
    kv_len, new = st["kv_len"].long(), (st["row_offset"][1:] - st["row_offset"][:-1]).long()
    T = given.shape[-1]
    at = torch.arange(T, device=DEV)
    ids = st["table"].long()
    block = torch.where((at < kv_len[:, None]) & (new[:, None] > 0), ids[:, at // bs], st["weight"].shape[0])     # [B, T]
    pool = torch.cat([st["weight"], st["weight"][:1]])                                 # an extra block takes what is not there
    old = pool[block, :, at % bs].transpose(1, 2)
    now = torch.where((at < (kv_len - new)[:, None])[:, None], c["decay"] * old, torch.zeros_like(old)) + given
    pool[block, :, at % bs] = now.transpose(1, 2)
    st["weight"].copy_(pool[:-1])
    return st["weight"]


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


def _evict(st):
    c, bs = st["case"], st["case"]["block"]
    B, H, d, most = c["batch"], c["hk"], c["d"], st["max_keep"]
    kv_len, ids = st["kv_len"].long(), st["table"].long().clamp(min=0)
    T, blocks = ids.shape[1] * bs, st["weight"].shape[0]
    at = torch.arange(T, device=DEV)
    keep = torch.minimum(st["budget"].long(), kv_len).clamp(max=most)                  # [B]
    w = st["weight"][ids].permute(0, 2, 1, 3).reshape(B, H, T)
    rank = w if c["per_head"] else w.double().sum(1, keepdim=True).float()             # shared: one sum in 64 bits
    rank = torch.where(torch.isnan(rank), torch.full_like(rank, -math.inf), rank)
    safe = (at < c["first"]) | (at >= (kv_len - c["last"])[:, None])
    rank = torch.where(safe[:, None], torch.full_like(rank, math.inf), rank)
    there = (at < kv_len[:, None])[:, None].expand_as(rank)
    by_weight = torch.sort(rank, dim=-1, descending=True, stable=True)[1]                  # equal ones by their place
    by_weight = by_weight.gather(-1, torch.sort((~there).gather(-1, by_weight).int(), dim=-1, stable=True)[1])
    chosen = torch.zeros_like(there).scatter(-1, by_weight, (at < keep[:, None])[:, None].expand_as(there))
    j = torch.arange(most, device=DEV)
    src = torch.sort(torch.where(chosen, at, T + at), -1)[0]
    src = torch.cat([src, src[..., :1].expand(*src.shape[:2], max(0, most - T))], -1)[..., :most]
    on = (j < keep[:, None])[:, None]                                                  # [B, 1, most]
    st["kept"].copy_(torch.where(on, src, st["kept"].long()).int())
    st["delta"].copy_((keep - kv_len).int())
    src = torch.where(on, src, 0).expand(B, H, most)
    moved = on & (src != j)
    columns = (most + bs - 1) // bs
    moved = torch.cat([moved, moved.new_zeros(B, H, columns * bs - most)], -1).view(B, H, columns, bs).any(-1)
    moved = moved.repeat_interleave(bs, -1)[..., :most] & on                           # whole blocks are written anew
    head = torch.arange(H, device=DEV)[:, None]
    seq = torch.arange(B, device=DEV)[:, None, None]
    from_block, from_place = ids[seq, src // bs], src % bs
    to_block = torch.where(moved, ids[seq, j // bs], blocks)                           # an extra block takes what stays
    for codes, scale in ((st["k_cache"], st["k_scale"]), (st["v_cache"], st["v_scale"])):
        x = codes[from_block, head, from_place].float() * scale[from_block, head][..., None]           # [B, H, most, d]
        bad = ~torch.isfinite(x).all(-1)
        amax = torch.where(bad, torch.full_like(x[..., 0], math.inf), x.abs().amax(-1))
        peak = torch.full((blocks + 1, H), -1.0, device=DEV)
        peak = peak.view(-1).scatter_reduce(0, (to_block * H + head).reshape(-1), amax.reshape(-1), "amax").view(blocks + 1, H)
        now = torch.where(peak < 0, torch.cat([scale, scale[:1]]), torch.exp2(_exponent(peak.clamp(min=0), c["cache"])))
        pool = torch.cat([codes.view(torch.uint8), codes[:1].view(torch.uint8)])
        pool[to_block, head, j % bs] = _code(x / now[to_block, head][..., None], c["cache"])
        codes.view(torch.uint8).copy_(pool[:blocks])
        scale.copy_(now[:blocks])
    pool = torch.cat([st["weight_out"], st["weight_out"][:1]])
    pool[torch.where(on.expand_as(src), ids[seq, j // bs], blocks), head, j % bs] = st["weight"][from_block, head, from_place]
    st["weight_out"].copy_(pool[:blocks])
    return (st["k_cache"], st["v_cache"], st["k_scale"], st["v_scale"], st["weight_out"], st["kept"], st["delta"])


# ------------------------------------------------------------------------------------------------ 64 bits
def exact(case, seed):
    st = prepare(case, seed)
    return {"prompt": _exact_prompt, "weigh": _exact_weigh, "evict": _exact_evict}[case["op"]](st)


def _exact_prompt(st):
    c = st["case"]
    H, G, d = c["hk"], c["hq"] // c["hk"], c["d"]
    out, lse = st["out"].double(), st["lse"].double()
    rows, keys = st["row_offset"].tolist(), st["kv_offset"].tolist()
    for b in range(c["batch"]):
        n, T = rows[b + 1] - rows[b], keys[b + 1] - keys[b]
        if c["padded"]:
            q, k, v = st["q"][b, :, :n], st["k"][b, :, :T], st["v"][b, :, :T]
            to, to_lse = out[b, :, :n], lse[b, :, :n]
        else:
            q = st["q"][rows[b]:rows[b + 1]].transpose(0, 1)
            k, v = (x[keys[b]:keys[b + 1]].transpose(0, 1) for x in (st["k"], st["v"]))
            to, to_lse = out[rows[b]:rows[b + 1]].transpose(0, 1), lse[rows[b]:rows[b + 1]].transpose(0, 1)
        for h in range(c["hq"]) if n * T * c["hq"] > 20_000_000 else (slice(None),):
            heads = slice(h, h + 1) if isinstance(h, int) else h
            kv = slice(h // G, h // G + 1) if isinstance(h, int) else torch.arange(c["hq"], device=DEV) // G
            s = st["scale"] * (q[heads].double() @ k[kv].double().transpose(1, 2))
            if c["causal"]:
                s.masked_fill_(torch.arange(T, device=DEV) > T - n + torch.arange(n, device=DEV)[:, None], -math.inf)
            z = torch.logsumexp(s, -1)
            to[heads] = torch.exp(s - z[..., None]) @ v[kv].double()
            to_lse[heads] = z
    return out, lse


def _exact_weigh(st):
    c, bs = st["case"], st["case"]["block"]
    H, G, d = c["hk"], c["hq"] // c["hk"], c["d"]
    weight = st["weight"].double()
    offsets, lens = st["row_offset"].tolist(), st["kv_len"].tolist()
    for b, T in enumerate(lens):
        n = offsets[b + 1] - offsets[b]
        u = min(n, c["window"])
        ids = st["table"][b, :-(-T // bs)].long()
        k = (st["k_cache"][ids].float().double() * st["k_scale"][ids][..., None, None].double()).transpose(0, 1).reshape(H, len(ids) * bs, d)[:, :T]
        q = st["q"][offsets[b + 1] - u:offsets[b + 1]].double().view(u, H, G, d)
        z = st["lse"][offsets[b + 1] - u:offsets[b + 1]].double().view(u, H, G)
        given = torch.zeros((H, T), dtype=torch.float64, device=DEV)
        for h in range(H):
            s = st["scale"] * torch.einsum("ngd,td->ngt", q[:, h], k[h]) - z[:, h, :, None]
            if c["causal"]:
                s.masked_fill_((torch.arange(T, device=DEV) > T - u + torch.arange(u, device=DEV)[:, None])[:, None], -math.inf)
            given[h] = torch.exp(s).sum((0, 1))
        w = weight[ids].transpose(0, 1).reshape(H, -1)
        w[:, T - n:T] = 0
        w[:, :T] = w[:, :T] * c["decay"] + given
        weight[ids] = w.view(H, len(ids), bs).transpose(0, 1)
    return weight


def _exact_code(x, cache):
    """Nearest value of the cache's type, ties to even."""
    if cache == "i8":
        return torch.round(x).clamp(-127, 127)
    _, e = torch.frexp(x)
    step = torch.exp2((e - 1).clamp(min=-6).double() - 3)
    return (torch.round(x / step) * step).clamp(-448, 448)


def _exact_evict(st):
    c, bs = st["case"], st["case"]["block"]
    H, d = c["hk"], c["d"]
    lens, budget, kept, delta = st["kv_len"].tolist(), st["budget"].tolist(), st["kept"].clone(), []
    weight, weight_out = st["weight"].double(), st["weight_out"].double()
    pools = [[st[n + "_cache"].float().double(), st[n + "_scale"].double()] for n in "kv"]
    grid = torch.exp2(torch.arange(E_MIN, E_MAX + 1, device=DEV, dtype=torch.float64))
    for b, T in enumerate(lens):
        ids = st["table"][b, :-(-T // bs)].long()
        n = min(budget[b], T, st["max_keep"])
        delta.append(n - T)
        w = weight[ids].transpose(0, 1).reshape(H, -1)[:, :T]
        score = w.clone() if c["per_head"] else w.sum(0, keepdim=True).float().double()
        score[:, :c["first"]] = math.inf
        score[:, max(T - c["last"], 0):] = math.inf
        # a token stays if fewer than n are ahead of it: larger, or as large and earlier
        order = torch.argsort(-score, dim=-1, stable=True)
        src = torch.sort(order[:, :n], -1)[0]
        kept[b, :, :n] = src.int()
        src = src.expand(H, n)
        used = -(-n // bs)
        fill = used * bs - n
        for values, scale in pools:
            x = (values[ids] * scale[ids][..., None, None]).transpose(0, 1).reshape(H, -1, d)
            x = x.gather(1, src[..., None].expand(H, n, d))
            x = torch.cat([x, x.new_zeros(H, fill, d)], 1).view(H, used, bs, d)
            same = torch.cat([src == torch.arange(n, device=DEV), torch.ones((H, fill), dtype=torch.bool, device=DEV)], 1).view(H, used, bs).all(-1)
            need = x.abs().amax((2, 3)) / Q_MAX[c["cache"]]
            s = grid[torch.searchsorted(grid, need.contiguous()).clamp(max=grid.numel() - 1)]
            y = _exact_code(x / s[..., None, None], c["cache"])
            live = (torch.arange(used * bs, device=DEV) < n).view(used, bs)
            write = (~same[..., None] & live)[..., None]
            values[ids[:used]] = torch.where(write, y, values[ids[:used]].transpose(0, 1)).transpose(0, 1)
            scale[ids[:used]] = torch.where(same, scale[ids[:used]].T, s).T
        moved = torch.cat([w.gather(1, src), w.new_zeros(H, fill)], 1).view(H, used, bs)
        live = (torch.arange(used * bs, device=DEV) < n).view(used, bs)
        weight_out[ids[:used]] = torch.where(live, moved, weight_out[ids[:used]].transpose(0, 1)).transpose(0, 1)
    codes = [v if c["cache"] == "e4m3" else v.to(torch.int8) for v, _ in pools]
    return (codes[0], codes[1], pools[0][1], pools[1][1], weight_out, kept, _i32(delta))
