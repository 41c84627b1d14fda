"""vscan_kv_attention at the edges of its numbers, against the float64 oracle and for every kernel the calls choose from: scores
whose factor vanishes (scale 0, query rows and keys of zeros, negative scale) over partly masked 16-token groups; values of
neighbouring blocks many binades apart, and scales far above what a block holds; warps that run through many short sequences, and what they report; the cache's workspace and what it does where a
tensor is refused; queries and keys that are views of one buffer.

Tolerances as derived in test_gpu_cache_ops.py, and beside the tests that have their own.
"""
import numpy as np
import pytest
import torch

import paper_2505_22654_b200 as vs
from oracle import cache_oracle as co
from test_gpu_cache_ops import DT, KV, Cache, _offsets, _tables, attend_tol, gen, i32

pytestmark = pytest.mark.gpu


def _written(kv, H, bs, d, lens, ks, vals, seed=0):
    """A cache that holds these rows, its oracle copy, and the block tables."""
    blocks = sum(-(-n // bs) for n in lens) + 2
    c = Cache(kv, H, bs, d, blocks, seed)
    table = _tables(lens, bs, max(-(-n // bs) for n in lens) + 1, blocks, np.random.default_rng(seed))
    vs.vscan_kv_write(torch.cat(ks).cuda(), torch.cat(vals).cuda(), i32(lens), i32(_offsets(lens)), i32(table), *c.arrays)
    c.write(ks, vals, lens, table)
    c.same()
    return c, table


@pytest.mark.parametrize("kv", ["e4m3", "i8"])
@pytest.mark.parametrize("scale", [0.0, 0.125, -0.125])
@pytest.mark.parametrize("dtype,d,past,new", [
    ("bf16", 128, [0, 100], [40, 33]), ("bf16", 64, [5, 0], [70, 150]),       # many rows
    ("bf16", 128, [0, 100], [3, 2]), ("f32", 64, [0, 100], [40, 3])])
def test_attention_where_a_scores_factor_vanishes(kv, scale, dtype, d, past, new):
    H, hq, bs = 2, 4, 16
    g, lens = gen(d + len(kv)), [p + n for p, n in zip(past, new)]
    ks = [torch.randn((n, H, d), generator=g).to(DT[dtype]) for n in lens]
    vals = [torch.randn((n, H, d), generator=g).to(DT[dtype]) for n in lens]
    ks[0][:] = 0                                     # a sequence of padding: every key, and below every second query, is zero
    for x in ks[1:]:
        x[len(x) // 2 // bs * bs:] = 0               # ... or the later half of it, from a block's start on
    c, table = _written(kv, H, bs, d, lens, ks, vals)
    qs = [torch.randn((n, hq, d), generator=g).to(DT[dtype]) for n in new]
    for x in qs:
        x[::2] = 0
    q = torch.cat(qs).cuda()
    off = _offsets(new)
    for causal in (True, False):
        out, lse = torch.full_like(q, 7.0), torch.full(q.shape[:2], 7.0, device="cuda")
        vs.vscan_kv_attention(q, i32(lens), i32(off), i32(table), *c.arrays, scale, max_q_len=max(new), causal=causal, out=out, lse=lse)
        out, lse = out.double().cpu().numpy(), lse.double().cpu().numpy()
        for b, T in enumerate(lens):
            (k, there), (v, _) = (co.gather(c.codes[i], c.scale[i], table[b], T, bs, KV[kv][0]) for i in range(2))
            ref, ref_lse, weight, reach = co.attention(qs[b].double().numpy(), k, v, there, scale, causal, past[b])
            got, got_lse = out[off[b]:off[b + 1]], lse[off[b]:off[b + 1]]
            assert np.isfinite(got).all() and np.isfinite(got_lse).all(), (b, np.argwhere(~np.isfinite(got_lse))[:4])
            assert (np.abs(got - ref) <= attend_tol(dtype, d, T, ref, weight, reach, v)).all()
            e, sums = (d + 8) * 2.0 ** -24 * reach, (T / 4 + 16) * 2.0 ** -24
            assert (np.abs(got_lse - ref_lse) <= e + sums + np.abs(ref_lse) * 2.0 ** -22).all()


def _apart_check(kv, dtype, hq, H, d, past, new, v_exp, seed, q_gain=1.0):
    """Values of neighbouring blocks v_exp[j] binades from 1, and each row measured by what it sees alone: the tolerance of
    attend_tol, but the smallest step of a weight in 16 bits for a row of its own.  The row's largest product of weight and block
    scale is 2^8 or more in that form, each is off by at most half of 2^-24, so in all tokens 2^-33 of what the largest code times that
    largest product is.  Exponents that a block scale of up to 2^56 is part of are up to 256 in size with all that is added on the way:
    2^-16 of a weight."""
    bs, T, g = 16, past + new, gen(seed)
    grow = torch.tensor([v_exp[t // bs % len(v_exp)] for t in range(T)]).double()[:, None, None]
    k = torch.randn((T, H, d), generator=g).to(DT[dtype])
    v = (torch.randn((T, H, d), generator=g).double() * torch.exp2(grow)).to(DT[dtype])
    c, table = _written(kv, H, bs, d, [T], [k], [v])
    q = (q_gain * torch.randn((new, hq, d), generator=g)).to(DT[dtype])
    out, lse = torch.full_like(q, 7.0).cuda(), torch.full((new, hq), 7.0, device="cuda")
    vs.vscan_kv_attention(q.cuda(), i32([T]), i32([0, new]), i32(table), *c.arrays, 0.125, max_q_len=new, out=out, lse=lse)
    out, lse = out.double().cpu().numpy(), lse.double().cpu().numpy()
    (kk, there), (vv, _) = (co.gather(c.codes[i], c.scale[i], table[0], T, bs, KV[kv][0]) for i in range(2))
    ref, ref_lse, weight, reach = co.attention(q.double().numpy(), kk, vv, there, 0.125, True, past)
    tol = attend_tol(dtype, d, T, ref, weight, reach, np.zeros(1))
    wide = 2.0 ** -16 if dtype == "bf16" else 0.0
    tol += wide * weight
    if dtype == "bf16":
        s = np.stack([c.scale[1][table[0][t // bs]] for t in range(T)])        # [T, H]
        for i in range(new):
            for j in range(hq):
                x = 0.125 * (kk[:past + i + 1, j // (hq // H)] @ q[i, j].double().numpy())
                p = np.exp(x - ref_lse[i, j])
                tol[i, j] += T * 2.0 ** -33 * co.Q_MAX[KV[kv][0]] * (p * s[:past + i + 1, j // (hq // H)]).max()
    err = np.abs(out - ref)
    assert (err <= tol).all(), (float((err / tol).max()), np.argwhere(err > tol)[:4])
    e, sums = (d + 8) * 2.0 ** -24 * reach, (T / 4 + 16) * 2.0 ** -24
    assert (np.abs(lse - ref_lse) <= e + sums + wide + np.abs(ref_lse) * 2.0 ** -22).all()


@pytest.mark.parametrize("kv", ["e4m3", "i8"])
@pytest.mark.parametrize("dtype,hq,H,d,past,new", [("bf16", 4, 2, 64, 0, 150), ("bf16", 2, 2, 128, 130, 300), ("bf16", 14, 2, 48, 40, 37),
                                                     ("f32", 4, 2, 64, 20, 60)])
@pytest.mark.parametrize("v_exp", [[0, 33], [-30, 10, -20, 40, 0, 30, -40, 5, 20], [40, 0, -40]])
@pytest.mark.parametrize("q_gain", [1.0, 4.0])
def test_attention_rows_do_not_depend_on_the_values_behind_them(kv, dtype, hq, H, d, past, new, v_exp, q_gain):
    _apart_check(kv, dtype, hq, H, d, past, new, v_exp, seed=d + new, q_gain=q_gain)


@pytest.mark.parametrize("kv", ["e4m3", "i8"])
@pytest.mark.parametrize("new", [2, 40])
def test_attention_values_whose_scale_is_zero_weigh_but_give_nothing(kv, new):
    """V scales of 0 (blocks filled by hand) over codes that are not 0: 0 times the code, and the tokens count in the denominator.
    A sequence of such blocks alone gives exactly 0."""
    H, d, bs, T, g = 1, 64, 16, 100, gen(new)
    k, v = (torch.randn((T, H, d), generator=g).to(torch.bfloat16) for _ in range(2))
    c, table = _written(kv, H, bs, d, [T, T], [k, k], [v, v])
    zero = [table[0][1], table[0][4]] + table[1][:7]
    c.scale[1][zero] = 0.0
    c.dev_scale[1][zero] = 0.0
    q = torch.randn((2 * new, 2, d), generator=g).to(torch.bfloat16)
    out = vs.vscan_kv_attention(q.cuda(), i32([T, T]), i32([0, new, 2 * new]), i32(table), *c.arrays, 0.125, max_q_len=new)
    (kk, there), (vv, _) = (co.gather(c.codes[i], c.scale[i], table[0], T, bs, KV[kv][0]) for i in range(2))
    ref, _, weight, reach = co.attention(q[:new].double().numpy(), kk, vv, there, 0.125, True, T - new)
    assert (np.abs(out[:new].double().cpu().numpy() - ref) <= attend_tol("bf16", d, T, ref, weight, reach, vv)).all()
    assert (out[new:] == 0).all()


@pytest.mark.parametrize("kv", ["e4m3", "i8"])
@pytest.mark.parametrize("hq,H,d,past,new", [(2, 2, 64, 149, 1), (4, 1, 128, 1000, 1), (14, 2, 48, 77, 2), (4, 2, 256, 60, 5)])
@pytest.mark.parametrize("v_exp", [[0, 33], [-30, 10, -20, 40, 0, 30, -40, 5, 20], [40, 0, -40]])
@pytest.mark.parametrize("q_gain", [1.0, 4.0, 8.0])
def test_attention_of_few_rows_keeps_what_large_values_with_small_weights_add(kv, hq, H, d, past, new, v_exp, q_gain):
    _apart_check(kv, "bf16", hq, H, d, past, new, v_exp, seed=d + new, q_gain=q_gain)


@pytest.mark.parametrize("dtype,new,batch", [("bf16", 1, 2400), ("bf16", 17, 300), ("f32", 1, 2400)])
def test_attention_of_the_largest_values_before_a_block_of_zeros(dtype, new, batch):
    """100,000 tokens of values of 1.75 x 2^56, the largest that the cache holds, then a block of zeros, whose scale is the least: the
    sums stay inside float32.  Keys are zero, so every visible token weighs the same.  Many sequences read the same blocks, so that
    none is cut into short pieces."""
    H, d, bs, big = 1, 16, 256, 400 * 256
    T = big + new
    k, v = torch.zeros((T, H, d)).to(DT[dtype]), torch.full((T, H, d), 1.75 * 2.0 ** 56).to(DT[dtype])
    v[big:] = 0
    blocks = -(-T // bs)
    c = Cache("e4m3", H, bs, d, blocks, 0)
    table = i32([list(range(blocks))] * batch)
    vs.vscan_kv_write(k.cuda(), v.cuda(), i32([T]), i32([0, T]), table[:1], *c.arrays)
    q = torch.ones((new * batch, H, d), dtype=DT[dtype], device="cuda")
    out = vs.vscan_kv_attention(q, i32([T] * batch), i32(np.arange(batch + 1) * new), table, *c.arrays, 1.0, max_q_len=new).double().cpu()
    want = 1.75 * 2.0 ** 56 * big / (big + torch.arange(1, new + 1).double())[None, :, None, None].expand(batch, new, H, d).reshape(out.shape)
    # weights are equal (one rounding in common, which the denominator does not have); sums of T terms
    tol = torch.finfo(DT[dtype]).eps / 2 + (T / 4 + 16) * 2.0 ** -24 + (2.0 ** -11 if dtype == "bf16" else 0) + 2.0 ** -16
    assert ((out - want).abs() <= tol * want).all()


def test_attention_of_many_short_sequences_a_warp_each_after_the_other():
    """3,000 sequences of 0 to 40 tokens, a row each: a warp goes from sequence to sequence and head to head."""
    H, hq, d, bs, B = 2, 6, 64, 16, 3000
    rng, g = np.random.default_rng(3), gen(3)
    lens = [int(n) for n in rng.integers(0, 41, size=B)]
    ks, vals = ([torch.randn((n, H, d), generator=g).to(torch.bfloat16) for n in lens] for _ in range(2))
    c, table = _written("e4m3", H, bs, d, lens, ks, vals)
    q = torch.randn((B, hq, d), generator=g).to(torch.bfloat16)
    args = (q.cuda(), i32(lens), i32(np.arange(B + 1)), i32(table), *c.arrays, 0.125)
    out = vs.vscan_kv_attention(*args)
    for _ in range(30):
        assert torch.equal(vs.vscan_kv_attention(*args), out)
    got = out.double().cpu().numpy()
    for b, T in enumerate(lens):
        (k, there), (v, _) = (co.gather(c.codes[i], c.scale[i], table[b], T, bs, co.E4M3) for i in range(2))
        ref, _, weight, reach = co.attention(q[b:b + 1].double().numpy(), k, v, there, 0.125, True, T - 1)
        assert (np.abs(got[b:b + 1] - ref) <= attend_tol("bf16", d, T, ref, weight, reach, v)).all(), b


def test_attention_reports_a_bad_block_whichever_warp_meets_it():
    H, d, bs, B = 1, 64, 16, 2368                  # as many segments as warps
    c, g = Cache("e4m3", H, bs, d, 8, 5), gen(6)
    q = torch.randn((B, 1, d), generator=g).to(torch.bfloat16).cuda()
    good = np.zeros((B, 1), dtype=np.int32)
    ws = vs.vscan_kv_attention_workspace(q, i32(good), c.dev[0], 1)
    for at in list(range(16)) + [2367, 1111, 593]:
        bad = good.copy()
        bad[at] = 8
        for table, status in ((bad, 1), (good, 0)):
            vs.vscan_kv_attention(q, i32([16] * B), i32(np.arange(B + 1)), i32(table), *c.arrays, 0.1, workspace=ws)
            assert vs.vscan_check(ws) == status


def test_cache_holds_one_workspace_whatever_the_row_counts_are():
    """Packed prompts of 60 different row counts: memory grows by at most the two largest workspaces; a graph that was captured on a
    small one gives the same bits afterwards."""
    H, hq, d = 2, 4, 128
    cache = vs.VScanCache(num_blocks=200, block_size=16, kv_heads=H, head_dim=d, batch=2, max_blocks=100, rows=2000)
    g = gen(1)
    k, v = (torch.randn((1500, H, d), generator=g).to(torch.bfloat16).cuda() for _ in range(2))
    q = torch.randn((1500, hq, d), generator=g).to(torch.bfloat16).cuda()
    cache.plan(i32([300, 0]))
    cache.write(k[:300], v[:300])
    few, out = q[:1].contiguous(), torch.zeros((1, hq, d), dtype=torch.bfloat16, device="cuda")
    cache.plan(i32([1, 0]))
    cache.write(k[300:301], v[300:301])
    want = cache.attend(few, 0.1).clone()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        cache.attend(few, 0.1, out=out)
    before = torch.cuda.memory_allocated()
    for n in range(17, 77):
        cache.attend(q[:n * 20], 0.1, max_q_len=n * 20)
    assert cache.check() == (0, 0)
    assert torch.cuda.memory_allocated() - before < 160 << 20
    noise = [torch.full((8 << 20,), 255, dtype=torch.uint8, device="cuda") for _ in range(20)]      # over what has been let go
    out.zero_()
    graph.replay()
    assert torch.equal(out, want) and cache.check() == (0, 0)
    del noise


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("layout", ["tokens", "heads", "turns", "sides", "rows", "groups"])
@pytest.mark.parametrize("hq,hk", [(4, 4), (6, 2), (1, 1)])
def test_rope_in_place_on_views_of_one_buffer(dtype, layout, hq, hk):
    """Queries and keys side by side in a token, in a sequence, head by head in turn, as two halves, one behind the other in the rows
    of a head, and the tokens in front of the sequences: the same bits as out of place, and nothing else changed."""
    B, S, d, g = 2, 5, 64, gen(hq)
    if layout in ("turns", "rows") and hq != hk:
        pytest.skip("needs as many query as key heads")
    shape = {"tokens": (B, S, hq + 2 * hk, d), "heads": (B, hq + 2 * hk, S, d), "turns": (B, S, hq, 3, d), "sides": (hq + 2 * hk, B, S, d),
             "rows": (B, hq, 3 * S, d), "groups": (S, B, hq + 2 * hk, d)}[layout]
    buf = torch.randn(shape, generator=g).to(DT[dtype]).cuda()
    q, k, rest = {"tokens": lambda: [t.transpose(1, 2) for t in buf.split([hq, hk, hk], 2)], "heads": lambda: buf.split([hq, hk, hk], 1),
                  "turns": lambda: [buf[:, :, :, i].transpose(1, 2) for i in range(3)],
                  "sides": lambda: [t.transpose(0, 1) for t in buf.split([hq, hk, hk], 0)], "rows": lambda: buf.split(S, 2),
                  "groups": lambda: [t.permute(1, 2, 0, 3) for t in buf.split([hq, hk, hk], 2)]}[layout]()
    pos = torch.randint(0, 900, (2, B, S), generator=g, dtype=torch.int32).cuda()
    table, before = vs.rope_table(d, [20, 12]), rest.clone()
    want = vs.vscan_rope(q, k, pos, *table, q_out=torch.empty(q.shape, dtype=q.dtype, device="cuda"), k_out=torch.empty(k.shape, dtype=q.dtype, device="cuda"))
    vs.vscan_rope(q, k, pos, *table, q_out=q, k_out=k)
    assert torch.equal(q, want[0]) and torch.equal(k, want[1]) and torch.equal(rest, before)


def test_a_refused_step_leaves_the_cache_as_it_was():
    B, H, hq, d, g = 2, 2, 4, 64, gen(2)
    caches = [vs.VScanCache(num_blocks=20, block_size=16, kv_heads=H, head_dim=d, batch=B, max_blocks=6, rows=64) for _ in range(2)]
    t = lambda heads, n: torch.randn((B, heads, n, d), generator=g).to(torch.bfloat16).cuda()  # noqa: E731
    rope, pos = vs.rope_table(d, [32]), torch.zeros((1, B, 20), dtype=torch.int32, device="cuda")
    first, second = (t(hq, 20), t(H, 20), t(H, 20)), (t(hq, 3), t(H, 3), t(H, 3))
    for c in caches:
        c.step(*first, pos, rope, i32([20, 15]), 0.125)
    c, other = caches
    before = [c.kv_len.tolist(), c._plan["ring_state_out"].tolist()]
    p3, n3 = pos[:, :, :3].contiguous(), i32([3, -15])
    q, k, v = second
    for bad in ((q, k, v[:, :1]), (q, k, v.float()), (q, k, v[..., :48]), (q[..., :48], k[..., :48], v[..., :48]), (q[:, :3], k, v)):
        with pytest.raises((ValueError, TypeError, vs.VScanError)):
            c.step(*bad, p3, rope if bad[0].shape[-1] == d else vs.rope_table(48, [24]), n3, 0.125)
        assert [c.kv_len.tolist(), c._plan["ring_state_out"].tolist()] == before and c.row_offset.tolist() == [0] * (B + 1)
        assert (c.attend(q, 0.125, max_q_len=3) == 0).all()
    with pytest.raises((ValueError, vs.VScanError)):
        c.step(q, k, v, p3, rope, n3, 0.125, out=torch.zeros_like(q[:, :1]))
    outs = [x.step(q, k, v, p3, rope, n3, 0.125) for x in caches]
    assert torch.equal(*outs) and c.kv_len.tolist() == other.kv_len.tolist() == [23, 0]
    assert c._plan["ring_state_out"].tolist() == other._plan["ring_state_out"].tolist()
    n = [row[:2] for row in c.block_table.tolist()]
    assert n[0] == other.block_table.tolist()[0][:2]


def test_survivors_that_a_cache_does_not_take_leave_it_as_it_was():
    from synth import CONFIGS, stage2_inputs
    cfg = CONFIGS[2].with_(name="cache_run", B=2, C=1, k2=32, Hq=8, Hkv=4, d=64, Dh=256, pos_planes=3)
    d2 = stage2_inputs(cfg, 0, cfg.B)
    red = vs.VScanReducer.from_config(cfg)
    bf = lambda a: torch.from_numpy(np.ascontiguousarray(a)).cuda().to(torch.bfloat16)  # noqa: E731
    red.stage2(bf(d2["q_last"]), bf(d2["k"]), bf(d2["v"]), bf(d2["hidden"]), torch.from_numpy(np.ascontiguousarray(d2["pos_ids"])).cuda())
    cache = vs.VScanCache(num_blocks=40, block_size=16, kv_heads=2, head_dim=64, batch=2, max_blocks=20, rows=2 * red.S_out)
    with pytest.raises(ValueError):
        red.cache_survivors(cache)
    assert cache.kv_len.tolist() == [0, 0] and cache.row_offset.tolist() == [0, 0, 0]


@pytest.mark.parametrize("kv", ["e4m3", "i8"])
@pytest.mark.parametrize("dtype,hq,H,d,new", [("bf16", 2, 2, 64, 1), ("bf16", 4, 1, 128, 2), ("bf16", 4, 1, 256, 1), ("bf16", 4, 2, 64, 60), ("bf16", 2, 1, 128, 300),
                                                ("f32", 2, 2, 64, 3)])
@pytest.mark.parametrize("over", [12, 25, 50])
@pytest.mark.parametrize("q_gain", [0.1, 3.0])
def test_attention_beside_blocks_whose_scale_is_far_above_what_they_hold(kv, dtype, hq, H, d, new, over, q_gain):
    """A block keeps the scale of large tokens that were taken back. Every third block (many rows: every third step of 128 keys) has
    codes of 0 under a scale 2^over times the others'; what the other blocks add keeps the precision that it has without them."""
    T, bs, g = 700, 16, gen(over + new)
    few = new * (hq // H) <= 16
    k, v = torch.randn((T, H, d), generator=g).to(DT[dtype]), torch.randn((T, H, d), generator=g).to(DT[dtype])
    v *= 2.0 ** -20 if over == 50 else 1.0
    stale = [j for j in range(T // bs) if (j % 3 == 1 if few or dtype == "f32" else j // 8 % 3 == 1)]
    for j in stale:
        v[j * bs:(j + 1) * bs] = 0
    c, table = _written(kv, H, bs, d, [T], [k], [v])
    high = float(c.scale[1][table[0][0]].max()) * 2.0 ** over
    at = [table[0][j] for j in stale]
    c.scale[1][at], c.dev_scale[1][at] = high, high
    q = (q_gain * torch.randn((new, hq, d), generator=g)).to(DT[dtype])
    out = vs.vscan_kv_attention(q.cuda(), i32([T]), i32([0, new]), i32(table), *c.arrays, d ** -0.5, max_q_len=new).double().cpu().numpy()
    (kk, there), (vv, _) = (co.gather(c.codes[i], c.scale[i], table[0], T, bs, KV[kv][0]) for i in range(2))
    ref, _, weight, reach = co.attention(q.double().numpy(), kk, vv, there, d ** -0.5, True, T - new)
    err, tol = np.abs(out - ref), attend_tol(dtype, d, T, ref, weight, reach, vv)
    assert (err <= tol).all(), (float((err / tol).max()), np.argwhere(err > tol)[:4])


@pytest.mark.parametrize("dtype,new,batch", [("bf16", 1, 2400), ("bf16", 20, 160), ("f32", 1, 600)])
@pytest.mark.parametrize("over", [25, 50])
def test_attention_of_scales_that_come_and_go_while_scores_fall(dtype, new, batch, over):
    """Stretches of 128 keys, values of 1 and stale blocks (codes of 0 under a scale 2^over times the others') in turn, each 20 below the one
    before in score: the first stretch has all the weight, and what follows must not move its sums out of float32.  Many sequences read the same blocks,
    so that none is cut into short pieces."""
    H, d, bs, run, turns, g = 1, 16, 16, 128, 12, gen(over)
    T = 2 * run * turns
    k, v = torch.zeros((T, H, d)), torch.ones((T, H, d)) + torch.rand((T, H, d), generator=g)
    k[:, 0, 0] = -20.0 * (torch.arange(T) // run)
    v *= 2.0 ** -20 if over == 50 else 1.0
    stale = [j for j in range(T // bs) if j // 8 % 2 == 1]
    for j in stale:
        v[j * bs:(j + 1) * bs] = 0
    c, table = _written("e4m3", H, bs, d, [T], [k.to(DT[dtype])], [v.to(DT[dtype])])
    at = [table[0][j] for j in stale]
    high = float(c.scale[1][table[0][0]].max()) * 2.0 ** over
    c.scale[1][at], c.dev_scale[1][at] = high, high
    q = torch.zeros((batch * new, H, d), dtype=DT[dtype])
    q[..., 0] = 1.0
    out, lse = torch.zeros_like(q).cuda(), torch.zeros((batch * new, H), device="cuda")
    vs.vscan_kv_attention(q.cuda(), i32([T] * batch), i32(np.arange(batch + 1) * new), i32(table * batch), *c.arrays, 1.0, max_q_len=new, causal=False,
                          out=out, lse=lse)
    (kk, there), (vv, _) = (co.gather(c.codes[i], c.scale[i], table[0], T, bs, co.E4M3) for i in range(2))
    ref, ref_lse, weight, reach = co.attention(q[:1].double().numpy(), kk, vv, there, 1.0, False, 0)
    tol = attend_tol(dtype, d, T, ref, weight, np.full_like(reach, 20.0), vv)
    assert (np.abs(out.double().cpu().numpy() - ref) <= tol).all() and (np.abs(lse.double().cpu().numpy() - ref_lse) <= 1e-4).all()
