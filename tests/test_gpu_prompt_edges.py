"""vscan_attention, vscan_kv_weigh and vscan_kv_evict where they could go wrong beside what test_gpu_prompt_ops.py runs; tolerances are those of that
file."""
import numpy as np
import pytest
import torch

import paper_2505_22654_b200 as vs
from oracle import cache_oracle as co
from test_gpu_cache_ops import DT, _offsets, gen, i32
from test_gpu_prompt_ops import _evict_case, _random_cache, _weigh_case, check_attention

pytestmark = pytest.mark.gpu


# --------------------------------------------------------------------------- attention: tiles of an odd number of rows
@pytest.mark.parametrize("group", [5, 11, 13, 25])
@pytest.mark.parametrize("d,rows,hk", [(136, [2000, 300], 3), (192, [300, 300, 1], 4), (256, [2000, 2000], 4), (256, [6000], 2), (128, [2000], 2)])
def test_attention_of_groups_whose_tiles_have_an_odd_number_of_rows(group, d, rows, hk):
    """125, 121, 117 rows a tile above 128 channels, causal, long enough to be cut; `out` holds NaN, so that a row that is not written shows."""
    g, off, scale = gen(group + d), _offsets(rows), d ** -0.5
    q, k, v = (torch.randn((off[-1], H, d), generator=g).to(DT["bf16"]).cuda() for H in (hk * group, hk, hk))
    out, lse = torch.full_like(q, float("nan")), torch.full(q.shape[:2], float("nan"), device="cuda")
    ws = vs.vscan_attention_workspace(q, k, i32(off), max(rows))
    vs.vscan_attention(q, k, v, i32(off), scale, max(rows), out=out, lse=lse, workspace=ws)
    assert vs.vscan_check(ws) == 0
    for b, n in enumerate(rows):
        for h in range(hk):
            heads = slice(h * group, (h + 1) * group)
            for i in range(0, n, 1500):                       # rows i .. j - 1 see the first j keys at most
                j = min(i + 1500, n)
                mine, keys = slice(off[b] + i, off[b] + j), slice(off[b], off[b] + j)
                check_attention("bf16", out[mine, heads], lse[mine, heads], q[mine, heads], k[keys, h:h + 1], v[keys, h:h + 1], scale, True)


def test_attention_of_queries_and_keys_in_each_others_place_is_refused():
    q, k = torch.zeros((5, 4, 64), dtype=torch.bfloat16, device="cuda"), torch.zeros((5, 2, 64), dtype=torch.bfloat16, device="cuda")
    with pytest.raises(vs.VScanError, match="vscan_attention"):
        vs.vscan_attention(k, q, q, i32([0, 5]), 0.1, 5)


# --------------------------------------------------------------------------- attention: a visible score of -infinity
def _rest(scale):
    """What float32 leaves of scale * log2(e), as float32."""
    factor = float(np.float32(scale)) * 1.4426950408889634
    return float(np.float32(factor - float(np.float32(factor))))


SCALES = (0.125, 0.3, 9e-39, 0.1, -0.125, -0.1)


def test_the_scales_have_rests_of_every_sign():
    rests = [_rest(s) for s in SCALES]
    assert rests[0] > 0 and rests[2] == 0 and rests[3] < 0 and rests[4] < 0 < rests[5]


@pytest.mark.parametrize("scale", SCALES)
@pytest.mark.parametrize("dtype,shared", [("f32", False), ("bf16", False), ("bf16", True), ("f32", True)])
@pytest.mark.parametrize("d", [64, 80, 256])
def test_attention_gives_no_weight_to_a_score_of_minus_infinity(dtype, shared, scale, d):
    """Keys with a channel of -infinity (or infinity, for negative scales) that every query meets with a positive one: softmax gives them 0, the
    others as if they were not there.
    shared: the two heads of the keys are one (stride 0), which the CUDA cores take in bf16 too."""
    g, n, m = gen(d), 70, 300
    q, k, v = (torch.randn((rows, H, d), generator=g) for rows, H in ((n, 4), (m, 1 if shared else 2), (m, 2)))
    q[..., 3] = q[..., 3].abs() + 0.5
    gone = torch.zeros(m, dtype=torch.bool)
    gone[[0, 5, 64, 127, 128, 200, 299]] = True
    k[gone, :, 3] = float("-inf") if scale > 0 else float("inf")
    q, k, v = (x.to(DT[dtype]).cuda() for x in (q, k, v))
    k = k.expand(m, 2, d) if shared else k
    stay = (~gone).cuda()
    out, lse = torch.full_like(q, 7.0), torch.full(q.shape[:2], 7.0, device="cuda")
    vs.vscan_attention(q, k, v, i32([0, n]), scale, n, kv_offset=i32([0, m]), causal=False, out=out, lse=lse)
    check_attention(dtype, out, lse, q, k[stay], v[stay], scale, False)
    # causal, rows and keys alike: row 0 sees nothing but such a key
    gone[1:] = False
    k = k.clone()
    k[1:, :, 3] = 0.25
    vs.vscan_attention(q, k, v, i32([0, n]), scale, n, out=out, lse=lse)
    check_attention(dtype, out[1:], lse[1:], q[1:], k[1:n], v[1:n], scale, True)
    assert (out[0] == 0).all() and torch.isneginf(lse[0]).all()


def test_attention_gives_no_weight_to_a_score_that_leaves_float32():
    q, k, v = torch.full((3, 1, 64), 1e19, device="cuda"), torch.full((5, 1, 64), 1e-19, device="cuda"), torch.randn((5, 1, 64), device="cuda")
    k[2] = -1e19                                             # a sum of -6.4e39
    lse = torch.empty((3, 1), device="cuda")
    out = vs.vscan_attention(q, k, v, i32([0, 3]), 0.125, 3, kv_offset=i32([0, 5]), causal=False, lse=lse)
    stay = [0, 1, 3, 4]
    check_attention("f32", out, lse, q, k[stay], v[stay], 0.125, False)


# --------------------------------------------------------------------------- weigh: scores that leave float32
@pytest.mark.parametrize("kv", ["e4m3", "i8"])
@pytest.mark.parametrize("scale", [0.125, 0.1, -0.125, -0.1])
@pytest.mark.parametrize("rows", [1, 3])
def test_weigh_of_scores_of_minus_infinity_gives_nothing(kv, scale, rows):
    """float32 rows whose products with every key (codes above 0) sum to less than float32 holds: they add 0, the other row what it adds alone."""
    hk, d, T = 2, 32, 40
    kind, codes, sc, dev = _random_cache(kv, hk, 16, d, 4, 3)
    codes[0][:] = codes[0] % 63 + 64                         # above 0; e4m3: 2 and more
    dev[0].view(torch.uint8).copy_(torch.from_numpy(codes[0]))
    table, q = [[2, 0, 3]], torch.randn((rows, hk, d), generator=gen(1))
    q[-1] = -1e38 if scale > 0 else 1e38
    q[rows // 2 + 1:] = q[-1]
    lse = torch.full((rows, hk), 0.75)
    w = torch.rand((4, hk, 16), generator=gen(2))
    got, want = w.cuda(), w.double().numpy()
    vs.vscan_kv_weigh(q.cuda(), lse.cuda(), i32([T]), i32([0, rows]), i32(table), dev[0], dev[2], got, scale, max_q_len=rows, decay=0.5, causal=False)
    slack = co.weigh(want, [q.double().numpy()], [lse.double().numpy()], codes[0], sc[0], [T], table, 16, kind, float(np.float32(scale)), 0.5, None, False)
    tol = (d + 8) * 2.0 ** -24 * slack + (2.0 ** -21 + (rows / 4 + 16) * 2.0 ** -24 + 2.0 ** -23) * np.abs(want)
    assert (np.abs(got.double().cpu().numpy() - want) <= tol).all() and np.isfinite(want).all()


# --------------------------------------------------------------------------- evict: protected tokens and infinite weights
@pytest.mark.parametrize("per_head", [True, False])
@pytest.mark.parametrize("B,hk,bs,length", [(2, 2, 16, 120), (100, 4, 16, 100), (1, 2, 64, 1500), (1, 1, 16, 17000)])
def test_evict_keeps_protected_tokens_in_front_of_infinite_weights(per_head, B, hk, bs, length):
    """More tokens of infinite weight (or of weights whose sum over the heads is) than the budget; ranks by a CTA, by a warp, through memory."""
    def spoil(table, weight, scale, codes):
        weight[:] = np.inf
        weight[table[0][0]] = 3e38
    lens, budget = [length - b % 7 for b in range(B)], [(40, 11, 6, 3)[b % 4] for b in range(B)]
    for first, last in ((3, 5), (0, 8), (2, 0)):
        _evict_case("i8", hk, 16, bs, lens, budget, first, last, per_head, spoil=spoil)


@pytest.mark.parametrize("B", [1, 160])
def test_evict_sums_over_the_heads_that_leave_float32_rank_below_protected_tokens(B):
    def spoil(table, weight, scale, codes):
        weight[:] = 3e38
    _evict_case("e4m3", 2, 16, 16, [90] * B, [20] * B, 1, 12, False, spoil=spoil)


# --------------------------------------------------------------------------- offsets outside the buffers, streams, graphs
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("padded", [False, True])
def test_attention_of_offsets_that_leave_the_buffers(dtype, padded):
    """What is outside is not there, positions follow the offsets as given; rows that nobody owns hold what they held."""
    g = gen(4)
    q, k, v = (torch.randn((5, 1, 64), generator=g).to(DT[dtype]).cuda() for _ in range(3))
    views = [x.transpose(0, 1)[None] if padded else x for x in (q, k, v)]

    def call(off, koff, causal=True):
        out = torch.full_like(views[0], 7.0)
        lse = torch.full(out.shape[:-1], 7.0, device="cuda")
        vs.vscan_attention(*views, i32(off), 0.2, 9, kv_offset=i32(koff), causal=causal, out=out, lse=lse)
        return (out[0].transpose(0, 1), lse[0].T) if padded else (out, lse)

    out, lse = call([0, 9], [0, 5])                          # rows 5 .. 8 are not there; row 4 is at 0
    assert (out[:4] == 0).all() and torch.isneginf(lse[:4]).all()
    check_attention(dtype, out[4:], lse[4:], q[4:], k[:1], v[:1], 0.2, True)
    out, lse = call([0, 5], [0, 2 ** 31 - 1])                # rows stand behind all keys that there are
    check_attention(dtype, out, lse, q, k, v, 0.2, False)
    out, lse = call([0, 5], [5, 5])
    assert (out == 0).all() and torch.isneginf(lse).all()
    for off, koff in (([3, 1], [0, 5]),) + (() if padded else (([-2, 3], [-2, 3]), ([5, 9], [5, 9]))):
        out, lse = call(off, koff)
        assert (out == 7).all() and (lse == 7).all()
    out, lse = call([0, 3], [0, 5], False)
    check_attention(dtype, out[:3], lse[:3], q[:3], k, v, 0.2, False)
    assert (out[3:] == 7).all() and (lse[3:] == 7).all()


def test_attention_of_two_streams_at_once():
    """A workspace each: results as one after the other."""
    g = gen(22)
    sets = [[torch.randn((1500, 2, 128), generator=g).to(torch.bfloat16).cuda() for _ in range(3)] for _ in range(2)]
    off = i32([0, 700, 1500])
    want = [vs.vscan_attention(*s, off, 0.1, 800) for s in sets]
    for s, w in zip(sets, want):
        check_attention("bf16", w[:700], vs_lse(s, off)[:700], s[0][:700], s[1][:700], s[2][:700], 0.1, True)
    streams, spaces = [torch.cuda.Stream() for _ in sets], [vs.vscan_attention_workspace(s[0], s[1], off, 800) for s in sets]
    outs = [[torch.zeros_like(s[0]) for _ in range(8)] for s in sets]
    torch.cuda.synchronize()
    for n in range(8):
        for s, st, ws, out in zip(sets, streams, spaces, outs):
            with torch.cuda.stream(st):
                vs.vscan_attention(*s, off, 0.1, 800, out=out[n], workspace=ws)
    torch.cuda.synchronize()
    assert all(torch.equal(o, w) for out, w in zip(outs, want) for o in out) and [vs.vscan_check(w) for w in spaces] == [0, 0]


def vs_lse(s, off):
    lse = torch.empty(s[0].shape[:2], device="cuda")
    vs.vscan_attention(*s, off, 0.1, 800, lse=lse)
    return lse


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_a_captured_step_with_weights_and_an_eviction(dtype):
    """A decode step and an eviction of a cache in one graph, replayed: codes, weights and lengths as those of a cache that made the calls."""
    hq, hk, d, B, g = 4, 2, 64, 3, gen(31)
    rope, budget = vs.rope_table(d, [d // 2]), i32([20, 40, 9])
    make = [vs.VScanCache(num_blocks=40, block_size=16, kv_heads=hk, head_dim=d, batch=B, max_blocks=8, rows=200, weights=True) for _ in range(2)]
    q, k, v = (torch.randn((B, H, 60, d), generator=g).to(DT[dtype]).cuda() for H in (hq, hk, hk))
    pos = torch.arange(60, dtype=torch.int32, device="cuda").expand(1, B, -1).contiguous()
    for c in make:
        c.prompt(q, k, v, pos, rope, i32([60, 33, 5]), d ** -0.5)
    q1, k1, v1 = (torch.randn((B, H, 1, d), generator=g).to(DT[dtype]).cuda() for H in (hq, hk, hk))
    at, one, kept = i32([[[60], [33], [5]]]), i32([1, 1, 1]), torch.full((B, hk, 64), -1, dtype=torch.int32, device="cuda")

    def turn(c):
        out = c.step(q1, k1, v1, at, rope, one, d ** -0.5, decay=0.5)
        c.evict(budget, 64, 2, 3, kept=kept)
        return out
    plain, captured = make
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    spare = vs.VScanCache(num_blocks=40, block_size=16, kv_heads=hk, head_dim=d, batch=B, max_blocks=8, rows=200, weights=True)
    with torch.cuda.stream(side):
        turn(spare)
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = turn(captured)
    for n in range(4):
        q1.copy_(torch.randn(q1.shape, generator=gen(n)))
        k1.copy_(torch.randn(k1.shape, generator=gen(9 + n)))
        want = turn(plain).clone()
        want_kept = kept.clone()
        graph.replay()
        assert torch.equal(out, want) and torch.equal(kept, want_kept)
        for a, b in ((plain.k_scale, captured.k_scale), (plain.v_scale, captured.v_scale), (plain.kv_len, captured.kv_len), (plain.weight, captured.weight),
                     (plain.block_table, captured.block_table), (plain.k.view(torch.uint8), captured.k.view(torch.uint8)),
                     (plain.v.view(torch.uint8), captured.v.view(torch.uint8))):
            assert torch.equal(a, b)
        assert plain.check() == captured.check() == (0, 0)


# --------------------------------------------------------------------------- the most sequences, and what lies beyond 2^31 elements
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_the_most_sequences(dtype):
    """8,192 sequences of 0 to 3 rows behind 0 to 20 tokens, through all three calls."""
    B, hq, hk, d, g, rng = 8192, 2, 1, 32, gen(41), np.random.default_rng(3)
    new = [int(n) for n in rng.integers(0, 4, size=B)]
    keys = [n + int(p) for n, p in zip(new, rng.integers(0, 21, size=B))]
    off, koff = _offsets(new), _offsets(keys)
    q, k, v = (torch.randn((n, H, d), generator=g).to(DT[dtype]).cuda() for n, H in ((off[-1], hq), (koff[-1], hk), (koff[-1], hk)))
    out, lse = torch.full_like(q, float("nan")), torch.full(q.shape[:2], float("nan"), device="cuda")
    ws = vs.vscan_attention_workspace(q, k, i32(off), 3)
    vs.vscan_attention(q, k, v, i32(off), 0.2, 3, kv_offset=i32(koff), out=out, lse=lse, workspace=ws)
    assert vs.vscan_check(ws) == 0 and torch.isfinite(out).all() and torch.isfinite(lse).all()
    for b in [0, 1, B - 2, B - 1] + [int(x) for x in rng.integers(0, B, size=60)]:
        mine, theirs = slice(off[b], off[b + 1]), slice(koff[b], koff[b + 1])
        if new[b]:
            check_attention(dtype, out[mine], lse[mine], q[mine], k[theirs], v[theirs], 0.2, True)
    # each sequence has two blocks: the weights of its tokens, and of those 7 stay
    table = torch.randperm(2 * B, generator=g).view(B, 2).int().cuda()
    codes = torch.randint(-100, 101, (2, 2 * B, hk, 16, d), generator=g).to(torch.int8).cuda()
    scale = torch.full((2, 2 * B, hk), 2.0 ** -7, device="cuda")
    z = 2 + torch.rand(lse.shape, generator=g).cuda()
    w = torch.full((2 * B, hk, 16), 0.5, device="cuda")
    vs.vscan_kv_weigh(q, z, i32(keys), i32(off), table, codes[0], scale[0], w, 0.2, max_q_len=3, decay=0.5)
    first = codes.clone()
    ws = vs.vscan_kv_evict_workspace(table, codes[0], 7)
    kept = torch.full((B, hk, 7), -1, dtype=torch.int32, device="cuda")
    delta = vs.vscan_kv_evict(i32(keys), i32([7] * B), table, w, codes[0], codes[1], scale[0], scale[1], 7, 1, 1, kept=kept, workspace=ws)
    assert vs.vscan_check(ws) == 0 and delta.tolist() == [min(7, m) - m for m in keys]
    for b in [0, B - 1] + [int(x) for x in rng.integers(0, B, size=60)]:
        m, n = keys[b], new[b]
        ids = table[b].long()
        kk = first[0][ids].double().reshape(32, d)[:m] / 128
        got = w[ids].reshape(32)[:m].double()
        x, zz = q[off[b]:off[b] + n].double(), z[off[b]:off[b] + n].double()
        s = 0.2 * torch.einsum("nhd,td->hnt", x, kk) - zz.T[..., None]
        s.masked_fill_(torch.arange(m, device="cuda") > m - n + torch.arange(n, device="cuda")[:, None], -torch.inf)
        want = torch.where(torch.arange(m, device="cuda") < m - n, 0.25 if n else 0.5, 0.0).double() + s.exp().sum((0, 1))
        # scores of some ten units at most
        assert ((got - want).abs() <= (40 * 2.0 ** -24 * 64 + 2.0 ** -21 + 20 * 2.0 ** -24) * want).all()
        rank = got.clone()
        rank[:1] = rank[max(m - 1, 0):] = torch.inf
        stay = torch.sort(torch.sort(rank, descending=True, stable=True)[1][:7])[0]
        assert kept[b, 0].tolist() == stay.tolist() + [-1] * (7 - len(stay))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_attention_of_keys_beyond_two_to_the_31_elements(dtype):
    """A sequence whose keys and values begin 2.2 x 10^9 elements into their buffers, behind one that has no rows."""
    far, n, m, hk, d, g = 2_200_000, 20, 333, 8, 128, gen(51)
    q = torch.randn((n, 16, d), generator=g).to(DT[dtype]).cuda()
    k, v = (torch.zeros((far + m, hk, d), dtype=DT[dtype], device="cuda") for _ in range(2))
    for t in (k, v):
        t[far:] = torch.randn((m, hk, d), generator=g).to(DT[dtype]).cuda()
    out, lse = torch.full_like(q, 7.0), torch.full(q.shape[:2], 7.0, device="cuda")
    vs.vscan_attention(q, k, v, i32([0, 0, n]), 0.1, n, kv_offset=i32([0, far, far + m]), out=out, lse=lse)
    check_attention(dtype, out, lse, q, k[far:], v[far:], 0.1, True)


@pytest.mark.parametrize("dtype,rows", [("bf16", 1), ("bf16", 40), ("f32", 2)])
def test_weights_and_evictions_of_blocks_beyond_two_to_the_31_elements(dtype, rows):
    """Blocks that begin 2.3 x 10^9 codes into the cache."""
    blocks, hk, bs, d, T, g = 70_000, 8, 32, 128, 100, gen(52)
    k, v = (torch.zeros((blocks, hk, bs, d), dtype=torch.int8, device="cuda") for _ in range(2))
    ks, vsc, w = torch.full((blocks, hk), 2.0 ** -7, device="cuda"), torch.full((blocks, hk), 2.0 ** -7, device="cuda"), torch.full((blocks, hk, bs), 0.5, device="cuda")
    ids = torch.tensor([blocks - 1, blocks - 4, blocks - 2, blocks - 3], device="cuda")
    for t in (k, v):
        t[ids] = torch.randint(-100, 101, (4, hk, bs, d), generator=g).to(torch.int8).cuda()
    before = [t[ids].clone() for t in (k, v)]
    q, lse = torch.randn((rows, hk, d), generator=g).to(DT[dtype]).cuda(), 2 + torch.rand((rows, hk), generator=g).cuda()
    table = ids.int()[None]
    vs.vscan_kv_weigh(q, lse, i32([T]), i32([0, rows]), table, k, ks, w, 0.1, max_q_len=rows, causal=False)
    kk = before[0].double().transpose(0, 1).reshape(hk, -1, d)[:, :T] / 128
    want = torch.where(torch.arange(T, device="cuda") < T - rows, 0.5, 0.0) + (0.1 * torch.einsum("nhd,htd->hnt", q.double(), kk) - lse.double().T[..., None]).exp().sum(1)
    got = w[ids].transpose(0, 1).reshape(hk, -1)[:, :T].double()
    assert ((got - want).abs() <= (136 * 2.0 ** -24 * 64 + 2.0 ** -21 + (rows / 4 + 16) * 2.0 ** -24) * want).all()
    kept = torch.zeros((1, hk, 50), dtype=torch.int32, device="cuda")
    assert vs.vscan_kv_evict(i32([T]), i32([50]), table, w, k, v, ks, vsc, 50, kept=kept).tolist() == [50 - T]
    src = torch.sort(torch.sort(got.float(), dim=-1, descending=True, stable=True)[1][:, :50], dim=-1)[0]
    assert torch.equal(kept[0].long(), src)
    for now, sc, old in ((k, ks, before[0]), (v, vsc, before[1])):
        flat = lambda x: x.transpose(0, 1).reshape(hk, -1, d)  # noqa: E731
        values = flat(now[ids].double() * sc[ids][..., None, None].double())[:, :50]
        assert torch.equal(values, flat(old).double().gather(1, src[..., None].expand(hk, 50, d)) / 128)


# --------------------------------------------------------------------------- weigh: on both sides of the choice of a kernel
@pytest.mark.parametrize("hq,hk,d,new", [
    (1, 1, 128, [17, 40, 0]), (1, 1, 128, [64, 3, 50]), (1, 1, 128, [65, 3, 64]), (2, 2, 64, [64, 20]), (2, 2, 64, [66, 1]), (7, 1, 96, [9, 2]), (7, 1, 96, [10, 9]),
    (13, 1, 128, [5, 4]), (33, 1, 64, [2, 1]), (64, 1, 128, [1, 1]), (64, 1, 128, [2, 0]), (2, 1, 256, [24, 9]), (2, 1, 256, [25, 24]), (3, 1, 144, [16, 0]),
    (3, 1, 192, [17, 5]), (1, 1, 48, [129, 65]), (5, 1, 240, [10, 11])])
@pytest.mark.parametrize("kv", ["e4m3", "i8"])
def test_weigh_where_the_kernel_changes(kv, hq, hk, d, new):
    past = [150, 40, 7][:len(new)]
    for window, causal in ((None, True), (60, True), (None, False)):
        _weigh_case(kv, "bf16", hq, hk, d, 16, past, new, causal=causal, padded=len(new) % 2 == 1, window=window, decay=0.5, seed=d + hq, missing=[(0, 2), (1, 1)])


def test_evict_of_more_long_tables_than_ctas_stay_resident():
    """300 ranks of more than 4,096 tokens."""
    _evict_case("i8", 100, 16, 64, [4200, 4100, 130], [900, 4099, 64], 2, 9, ties=True)
