"""vscan_attention, vscan_kv_weigh and vscan_kv_evict against plain implementations in 64 bits: types, head layouts, lengths from nothing to long,
odd sizes, strides, rows that see nothing, what is not finite, and a run of them together.

Tolerances, fixed before the first run.  `h(t)` = finfo(t).eps / 2 is the one rounding of a result.
  attention  with A = sum p |v| and e = (head_dim + 8) 2^-24 max scale sum |q| |k| (error of a score, summed in 32 bits), each weight is off
             by 2 e + 2^-21 (exponential) + h(bf16) where the weights are rounded to 16 bits, the sums by (keys / 4 + 16) 2^-24: times A, plus
             h |result|.  lse: e + (keys / 4 + 16) 2^-24 + |lse| 2^-22.
  weigh      a weight exp(s - lse) is off by its exponent's error, (head_dim + 8) 2^-24 (|scale| sum |q| |k| + |lse|), and 2^-21 (exponential)
             of itself; the sum over rows x heads of the group by (rows x heads / 4 + 16) 2^-24, the older weight times decay by 2^-23.
  evict      everything exactly.
"""
import numpy as np
import pytest
import torch

import paper_2505_22654_b200 as vs
from oracle import cache_oracle as co
from test_gpu_cache_ops import DT, KV, Cache, _offsets, _tables, gen, h, i32

pytestmark = pytest.mark.gpu


# --------------------------------------------------------------------------- attention over whole prompts
def plain_attention(q, k, v, scale, causal):
    """q [n, Hq, d], k and v [m, Hkv, d] -> out, lse, sum p |v|, largest |scale| sum |q| |k|, all float64; only what a row sees counts."""
    n, hq, d = q.shape
    m, hk = k.shape[:2]
    q, k, v = (x.double().transpose(0, 1) for x in (q, k, v))
    k, v = (x.repeat_interleave(hq // hk, 0) for x in (k, v))
    on = torch.arange(m, device=q.device) <= m - n + torch.arange(n, device=q.device)[:, None] if causal else torch.ones((n, m), dtype=torch.bool, device=q.device)
    s = torch.where(on, scale * (q @ k.transpose(1, 2)), -torch.inf)
    top = s.amax(-1, keepdim=True) if m else torch.full((hq, n, 1), -torch.inf, dtype=torch.float64, device=q.device)
    p = torch.where(on, torch.exp(s - torch.where(torch.isinf(top) & (top < 0), 0.0, top)), 0.0)
    total = p.sum(-1, keepdim=True)
    p = torch.where(total > 0, p / total, torch.where(torch.isnan(total), total, torch.zeros_like(p)))
    finite = torch.where(torch.isfinite(v), v, 0.0)
    out = p @ finite
    for value in (torch.inf, -torch.inf, torch.nan):          # what is not finite reaches those who see it
        hit = torch.isnan(v) if value != value else v == value
        out = out + torch.where((on.double() @ hit.double()) > 0, value, 0.0)
    reach = torch.where(on, abs(scale) * (q.abs() @ k.abs().transpose(1, 2)), 0.0).amax(-1) if m else torch.zeros((hq, n), dtype=torch.float64, device=q.device)
    lse = (top + torch.log(total))[..., 0]
    return (x.transpose(0, 1) for x in (out, lse, p @ finite.abs(), reach))


def check_attention(dtype, got, got_lse, q, k, v, scale, causal):
    d, m = q.shape[2], k.shape[0]
    ref, ref_lse, weight, reach = plain_attention(q, k, v, scale, causal)
    e, sums = (d + 8) * 2.0 ** -24 * reach, (m / 4 + 16) * 2.0 ** -24
    tol = (2 * e + 2.0 ** -21 + (h("bf16") if dtype == "bf16" else 0) + sums)[..., None] * weight + h(dtype) * ref.abs()
    fine = torch.isfinite(ref)
    assert torch.equal(torch.nan_to_num(got.double()[~fine], nan=5.0), torch.nan_to_num(ref[~fine], nan=5.0))
    err = (got.double() - ref).abs()[fine]
    assert (err <= tol[fine]).all(), float((err / tol[fine].clamp(min=1e-30)).max())
    fine = torch.isfinite(ref_lse)
    assert torch.equal(torch.nan_to_num(got_lse.double()[~fine], nan=5.0), torch.nan_to_num(ref_lse[~fine], nan=5.0))
    err = (got_lse.double() - ref_lse).abs()[fine]
    assert (err <= (e + sums + ref_lse.abs() * 2.0 ** -22)[fine]).all(), float(err.max())


def run_attention(dtype, hq, hk, d, past, new, causal, padded, seed=0, scale=None, max_q=None, poison=True, same=False, touch=None):
    """One call on random sequences, NaN in everything that no row sees; rows that no sequence owns stay.  touch(b, q, k, v): changes a
    sequence's rows first."""
    g, B = gen(seed), len(new)
    keys = [max(p + n, 0) for p, n in zip(past, new)]
    scale = d ** -0.5 if scale is None else scale
    seqs = []
    for b, (n, m) in enumerate(zip(new, keys)):
        q, k, v = (torch.randn((r, H, d), generator=g).to(DT[dtype]) for r, H in ((n, hq), (m, hk), (m, hk)))
        if touch:
            touch(b, q, k, v)
        seqs.append((q, k, v))
    fill = float("nan") if poison else 0.0
    off, koff = _offsets(new), _offsets(keys)
    sent = []
    for i, (H, counts, at) in enumerate(((hq, new, off), (hk, keys, koff), (hk, keys, koff))):
        if padded:
            t = torch.full((B, H, max(counts) + 2, d), fill, dtype=DT[dtype])
            for b in range(B):
                t[b, :, :counts[b]] = seqs[b][i].transpose(0, 1)
            sent.append(t.cuda())
        else:                                                       # rows of a wider buffer
            t = torch.full((at[-1] + 3, 2 * H, d), fill, dtype=DT[dtype])
            t[:at[-1], :H] = torch.cat([s[i] for s in seqs])
            sent.append(t.cuda()[:, :H])
    q, k, v = sent
    top = max_q or max(max(new), 1)
    out, lse = torch.full(q.shape, 7.0, dtype=DT[dtype], device="cuda"), torch.full(q.shape[:-1], 7.0, device="cuda")
    ws = vs.vscan_attention_workspace(q, k, i32(off), top)
    ws.buf.fill_(0xEE)
    kv_offset = None if same else i32(koff)
    vs.vscan_attention(q, k, v, i32(off), scale, top, kv_offset=kv_offset, causal=causal, out=out, lse=lse, workspace=ws)
    assert vs.vscan_check(ws) == 0
    again = torch.full(q.shape, 7.0, dtype=DT[dtype], device="cuda")
    vs.vscan_attention(q, k, v, i32(off), scale, top, kv_offset=kv_offset, causal=causal, out=again, workspace=ws)
    assert torch.equal(out.nan_to_num(5.0), again.nan_to_num(5.0)), "the same call gives other bits"
    for b, n in enumerate(new):
        mine, mine_lse = (out[b, :, :n].transpose(0, 1), lse[b, :, :n].T) if padded else (out[off[b]:off[b + 1]], lse[off[b]:off[b + 1]])
        if n:
            check_attention(dtype, mine, mine_lse, *(x.cuda() for x in seqs[b]), scale, causal)
        if padded:
            assert (out[b, :, n:] == 7).all() and (lse[b, :, n:] == 7).all()
    if not padded:
        assert (out[off[-1]:] == 7).all() and (lse[off[-1]:] == 7).all()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("hq,hk,d,past,new", [
    (4, 4, 128, [0, 0, 0], [1, 128, 129]), (14, 2, 128, [0, 0, 0], [300, 1, 37]), (8, 1, 64, [0], [577]), (3, 3, 72, [0, 0], [64, 65]),
    (2, 1, 80, [0, 5, 0], [127, 130, 0]), (6, 3, 8, [0, 100], [20, 256]), (64, 1, 96, [3], [9]), (1, 1, 32, [0, 0], [513, 255]),
    (2, 2, 256, [0, 70], [70, 33]), (5, 1, 136, [10], [40]), (7, 1, 128, [1000, 3], [1, 2]), (1, 1, 128, [0], [1]), (40, 1, 128, [200], [17])])
def test_attention(dtype, hq, hk, d, past, new):
    for causal in (True, False):
        run_attention(dtype, hq, hk, d, past, new, causal, padded=len(new) % 2 == 0, seed=hq + d)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_attention_one_offset_for_rows_and_keys(dtype):
    run_attention(dtype, 4, 2, 64, [0, 0, 0], [200, 1, 90], True, padded=False, same=True)
    run_attention(dtype, 4, 2, 64, [0, 0], [20, 90], False, padded=True, same=True)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_attention_rows_that_see_nothing(dtype):
    # no keys; more rows than keys: the first rows stand before every key
    run_attention(dtype, 4, 2, 64, [0, -3, -200, 0], [0, 5, 300, 2], True, padded=True, seed=5)
    run_attention(dtype, 4, 2, 128, [-1, -40, -7], [1, 40, 300], True, padded=False, seed=6)
    run_attention(dtype, 4, 2, 128, [-1, -40, 9], [1, 40, 1], False, padded=False, seed=7)
    q = torch.randn((3, 2, 64), generator=gen(1)).to(DT[dtype]).cuda()
    none = torch.zeros((0, 2, 64), dtype=DT[dtype], device="cuda")
    lse = torch.zeros((3, 2), device="cuda")
    assert (vs.vscan_attention(q, none, none, i32([0, 3]), 0.1, 3, kv_offset=i32([0, 0]), lse=lse) == 0).all() and torch.isneginf(lse).all()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("hq,hk,d,past,new", [(1, 1, 128, [9000], [200]), (7, 1, 64, [5000, 3, 0], [1, 2, 900]), (2, 2, 72, [0, 2500, 0], [1400, 90, 5])])
def test_attention_of_cut_sequences(dtype, hq, hk, d, past, new):
    for causal in (True, False):
        run_attention(dtype, hq, hk, d, past, new, causal, padded=False, seed=3)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("scale", [0.0, -0.2, 1e-30])
def test_attention_scales(dtype, scale):
    def zeros(b, q, k, v):
        q[::2] = 0
        k[len(k) // 2:] = 0
    run_attention(dtype, 4, 2, 64, [0, 40], [150, 100], True, padded=False, scale=scale, touch=zeros)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("d", [64, 128])
def test_attention_what_is_not_finite_reaches_those_who_see_it(dtype, d):
    """Values of a token that rows in front of it do not see: they stay finite, the others get the infinity of its sign, or NaN."""
    inf, nan = float("inf"), float("nan")

    def touch(b, q, k, v):
        if b == 0:
            v[40, 0, 3], v[40, 1, 5], v[70, 0, 3] = inf, -inf, -inf           # one after the other: NaN
            v[299, 1, d - 1] = nan
        else:
            v[-1, 0, 0] = nan
            v[130, :, 7] = inf
            k[-2] = nan                                                        # the last two rows see it
    run_attention(dtype, 4, 2, d, [0, 10], [300, 290], True, padded=False, touch=touch)
    run_attention(dtype, 4, 2, d, [0, 10], [300, 290], True, padded=True, touch=touch)


@pytest.mark.parametrize("hq,hk,d,past,new", [
    (1, 1, 192, [0], [1]), (2, 2, 256, [0, 0, 700], [129, 128, 1]), (7, 1, 256, [0, 40], [300, 18]), (4, 2, 136, [0, 5, 0], [127, 130, 0]),
    (64, 1, 200, [3], [9]), (1, 1, 256, [9000], [200]), (14, 2, 192, [2500, 0], [90, 1400]), (3, 3, 248, [-1, -40, 9], [1, 200, 1]),
    (40, 1, 184, [600], [17]), (2, 1, 256, [0, -200], [577, 300])])
def test_attention_wide_heads(hq, hk, d, past, new):
    for causal in (True, False):
        run_attention("bf16", hq, hk, d, past, new, causal, padded=len(new) % 2 == 0, seed=hq + d)


@pytest.mark.parametrize("d", [136, 192, 256])
def test_attention_wide_heads_what_is_not_finite_reaches_those_who_see_it(d):
    inf, nan = float("inf"), float("nan")

    def touch(b, q, k, v):
        v[40, 0, 3], v[40, 1, d - 6], v[70, 0, 3] = inf, -inf, -inf
        v[len(v) - 1, 1, d - 1] = nan
        v[130, :, 130] = -inf
        k[-2] = nan
    run_attention("bf16", 4, 2, d, [0, 10], [300, 290], True, padded=False, touch=touch)
    run_attention("bf16", 2, 2, d, [0, 10], [300, 290], True, padded=True, touch=touch)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_attention_large_scores_and_one_hot_rows(dtype):
    """Scores of hundreds, whose running maximum is raised many times over: each row's weights are nearly one key's alone."""
    def ramp(b, q, k, v):
        q[:] = 4.0
        k *= torch.linspace(0.1, 6.0, len(k))[:, None, None].to(k.dtype)
    run_attention(dtype, 2, 1, 128, [0, 700], [600, 300], True, padded=False, touch=ramp)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_attention_shared_and_reversed_layouts(dtype):
    """Keys of one head expanded over two (stride 0), rows of one fused projection, and a token-major padded batch."""
    g = gen(9)
    fused = torch.randn((90, 8, 64), generator=g).to(DT[dtype]).cuda()
    q, k, v = fused[:, :4], fused[:, 4:5].expand(90, 2, 64), fused[:, 6:]
    off, out, lse = i32([0, 90]), torch.empty((90, 4, 64), dtype=DT[dtype], device="cuda"), torch.empty((4, 90), device="cuda").T
    vs.vscan_attention(q, k, v, off, 0.125, 90, out=out, lse=lse)
    check_attention(dtype, out, lse, q, k, v, 0.125, True)
    batch = torch.randn((2, 50, 6, 64), generator=g).to(DT[dtype]).cuda()
    q, k, v = (batch[:, :, i:j].transpose(1, 2) for i, j in ((0, 4), (4, 5), (5, 6)))
    lse = torch.empty((2, 4, 50), device="cuda")
    out = vs.vscan_attention(q, k, v, i32([0, 50, 100]), 0.125, 50, causal=False, lse=lse)
    for b in range(2):
        check_attention(dtype, out[b].transpose(0, 1), lse[b].T, q[b].transpose(0, 1), k[b].transpose(0, 1), v[b].transpose(0, 1), 0.125, False)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_attention_max_q_len_and_rows_outside_the_buffer(dtype):
    run_attention(dtype, 2, 1, 64, [10, 40], [2, 3], True, padded=True, seed=10, max_q=100)
    g = gen(4)
    q, k, v = (torch.randn((5, 1, 64), generator=g).to(DT[dtype]).cuda() for _ in range(3))
    full, part, more = (torch.full_like(q, 7.0) for _ in range(3))
    vs.vscan_attention(q, k, v, i32([0, 5]), 0.2, 5, out=full)
    vs.vscan_attention(q, k, v, i32([0, 5]), 0.2, 3, out=part)
    assert torch.equal(full[:3], part[:3]) and (part[3:] == 7).all()
    # offsets that leave the buffers, fall, or begin below 0: what is outside is not there
    for off, koff in (([0, 9], [0, 5]), ([3, 1], [0, 5]), ([-2, 3], [-2, 3]), ([0, 5], [0, 2 ** 31 - 1]), ([5, 9], [5, 9]), ([0, 5], [5, 5])):
        vs.vscan_attention(q, k, v, i32(off), 0.2, 9, kv_offset=i32(koff), out=more)
    torch.cuda.synchronize()


def test_attention_of_many_pieces_gives_the_same_bits_every_time():
    """Sequences of very different sizes on few CTAs: roles hand over to each other in every order that timing allows."""
    new, past = [130, 1, 66, 40, 1, 300, 1, 700, 5], [0, 500, 3, 700, 5, 3, 900, 0, 0]
    keys, g = [p + n for p, n in zip(past, new)], gen(13)
    q = torch.randn((sum(new), 4, 80), generator=g).to(torch.bfloat16).cuda()
    k, v = (torch.randn((sum(keys), 2, 80), generator=g).to(torch.bfloat16).cuda() for _ in range(2))
    off, koff = i32(_offsets(new)), i32(_offsets(keys))
    ws = vs.vscan_attention_workspace(q, k, off, 700)
    first = vs.vscan_attention(q, k, v, off, 0.1, 700, kv_offset=koff, workspace=ws).clone()
    for _ in range(60):
        assert torch.equal(vs.vscan_attention(q, k, v, off, 0.1, 700, kv_offset=koff, workspace=ws), first)
        assert vs.vscan_check(ws) == 0


def test_attention_in_a_graph_and_on_another_stream():
    g = gen(21)
    q, k, v = (torch.randn((400, 2, 128), generator=g).to(torch.bfloat16).cuda() for _ in range(3))
    off, out, ws = i32([0, 150, 400]), torch.zeros_like(q), vs.vscan_attention_workspace(q, k, i32([0, 150, 400]), 250)
    want = vs.vscan_attention(q, k, v, off, 0.1, 250, workspace=ws).clone()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        vs.vscan_attention(q, k, v, off, 0.1, 250, out=out, workspace=ws)
    q2 = torch.randn((400, 2, 128), generator=g).to(torch.bfloat16).cuda()
    for x in (q2, q.clone()):
        q.copy_(x)
        out.zero_()
        graph.replay()
        assert torch.equal(out, vs.vscan_attention(q, k, v, off, 0.1, 250))
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        q.copy_(q2)
        there = vs.vscan_attention(q, k, v, off, 0.1, 250)
    torch.cuda.current_stream().wait_stream(side)
    assert torch.equal(there, out) is False or torch.equal(q2, q)
    assert torch.equal(there, vs.vscan_attention(q2, k, v, off, 0.1, 250)) and not torch.equal(there, want)


# --------------------------------------------------------------------------- weights of cached tokens
def _random_cache(kv, hk, bs, d, blocks, seed):
    """Codes without NaN, scales of a few binades; the oracle's copy and the GPU's."""
    rng = np.random.default_rng(seed)
    kind, dt = KV[kv]
    codes = [rng.integers(0, 256, size=(blocks, hk, bs, d)).astype(np.uint8) for _ in range(2)]
    for c in codes:
        c[(c & 0x7F) == 0x7F] = 0x11 if kind == co.E4M3 else 0x7E
        c[c == 0x80] = 0
    scale = [2.0 ** rng.integers(-9, -5, size=(blocks, hk)).astype(np.float64) for _ in range(2)]
    dev = [torch.from_numpy(c.copy()).cuda().view(dt) for c in codes] + [torch.from_numpy(s).float().cuda() for s in scale]
    return kind, codes, scale, dev


def _weigh_case(kv, dtype, hq, hk, d, bs, past, new, causal=True, padded=False, window=None, decay=1.0, seed=0, missing=(), max_q=None):
    B, g, rng = len(new), gen(seed), np.random.default_rng(seed)
    lens = [p + n for p, n in zip(past, new)]
    cols, blocks = max(max(-(-n // bs) for n in lens), 1) + 1, sum(max(-(-n // bs), 0) for n in lens) + 2
    kind, codes, scale, dev = _random_cache(kv, hk, bs, d, blocks, seed)
    table = _tables(lens, bs, cols, blocks, rng)
    for b, j in missing:
        table[b][j] = (-1, blocks, 2 ** 31 - 1)[(b + j) % 3]
    qs = [torch.randn((n, hq, d), generator=g).to(DT[dtype]) for n in new]
    # lse as the step's attention leaves it
    zs = []
    for b in range(B):
        k, there = co.gather(codes[0], scale[0], table[b], lens[b], bs, kind)
        zs.append(co.attention(qs[b].double().numpy(), k, k, there, d ** -0.5, causal, lens[b] - new[b])[1].astype(np.float32))
    off = _offsets(new)
    if padded:
        q, z = torch.full((B, hq, max(new) + 2, d), float("nan"), dtype=DT[dtype]), torch.full((B, hq, max(new) + 2), float("nan"))
        for b in range(B):
            q[b, :, :new[b]], z[b, :, :new[b]] = qs[b].transpose(0, 1), torch.from_numpy(zs[b]).T
    else:
        q, z = torch.full((off[-1] + 3, hq, d), float("nan"), dtype=DT[dtype]), torch.full((off[-1] + 3, hq), float("nan"))
        q[:off[-1]], z[:off[-1]] = torch.cat(qs), torch.from_numpy(np.concatenate(zs))
    weight = rng.random((blocks, hk, bs)).astype(np.float32) * 3
    for b in range(B):                                   # what a new token's place held is not read
        for t in range(max(lens[b] - new[b], 0), lens[b]):
            blk = table[b][t // bs]
            if 0 <= blk < blocks:
                weight[blk, :, t % bs] = np.nan
    got = torch.from_numpy(weight.copy()).cuda()
    want = weight.astype(np.float64)
    slack = co.weigh(want, [x.double().numpy() for x in qs], [x.astype(np.float64) for x in zs], codes[0], scale[0], lens, table, bs, kind, d ** -0.5,
                     decay, window, causal)
    vs.vscan_kv_weigh(q.cuda(), z.cuda(), i32(lens), i32(off), i32(table), dev[0], dev[2], got, d ** -0.5, max_q_len=max_q or max(max(new), 1),
                      decay=decay, window=window, causal=causal)
    got = got.double().cpu().numpy()
    rows = max(new) * (hq // hk)
    tol = (d + 8) * 2.0 ** -24 * slack + (2.0 ** -21 + (rows / 4 + 16) * 2.0 ** -24 + 2.0 ** -23) * np.abs(want)
    np.testing.assert_array_equal(np.isnan(got), np.isnan(want))
    fine = ~np.isnan(want)
    err = np.abs(got - want)[fine]
    assert (err <= tol[fine] + 1e-37).all(), float((err / (tol[fine] + 1e-37)).max())


@pytest.mark.parametrize("kv", ["e4m3", "i8"])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("hq,hk,d,bs,past,new", [
    (4, 4, 128, 16, [0, 15, 16, 63, 200], [1, 1, 1, 1, 1]), (14, 2, 128, 64, [90, 0], [1, 1]), (8, 1, 64, 32, [129], [1]), (16, 1, 256, 16, [70], [1]),
    (2, 1, 80, 128, [100], [1]), (6, 3, 16, 256, [5, 300], [1, 1]), (40, 1, 96, 16, [33], [1]), (4, 2, 128, 16, [10, 0, 60], [0, 5, 3]),
    (7, 1, 128, 16, [50, 3], [16, 1]), (2, 2, 64, 16, [0], [70]), (3, 1, 48, 32, [40], [40]), (2, 1, 256, 16, [10], [30]), (1, 1, 128, 16, [300], [20]),
    (4, 1, 64, 16, [0, 200], [140, 33])])
def test_weigh(kv, dtype, hq, hk, d, bs, past, new):
    _weigh_case(kv, dtype, hq, hk, d, bs, past, new, padded=len(new) % 2 == 0, seed=d + hq)
    _weigh_case(kv, dtype, hq, hk, d, bs, past, new, causal=False, padded=len(new) % 2 == 1, window=2, decay=0.5, seed=d + hq)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("new", [[1, 1], [20, 2], [40, 90]])
def test_weigh_windows_missing_blocks_and_empty_sequences(dtype, new):
    _weigh_case("e4m3", dtype, 4, 2, 64, 16, [100, 50], new, window=17, decay=0.9, seed=1, missing=[(0, 0), (0, 3), (1, 1)])
    _weigh_case("i8", dtype, 4, 2, 128, 16, [-1, 50], new, seed=2, max_q=200)             # one more row than tokens: the first sees nothing
    _weigh_case("i8", dtype, 4, 2, 64, 16, [0, 0], [0, 0], seed=3)
    _weigh_case("i8", dtype, 2, 2, 64, 16, [30, 5], new, window=1, decay=0.0, seed=4)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_weigh_of_more_rows_than_max_q_len_and_long_windows(dtype):
    """Rows behind max_q_len are not there: tokens that only they would see get nothing."""
    for hq, hk, d, past, new, top in ((4, 2, 64, [30, 0], [400, 300], 20), (7, 1, 128, [500, 3], [90, 200], 1000), (1, 1, 32, [600], [300], 1000)):
        lens, off = [p + n for p, n in zip(past, new)], _offsets(new)
        kind, codes, scale, dev = _random_cache("e4m3", hk, 16, d, sum(-(-n // 16) for n in lens) + 2, d)
        table = _tables(lens, 16, -(-max(lens) // 16), len(codes[0]), np.random.default_rng(0))
        q = torch.randn((off[-1], hq, d), generator=gen(d)).to(DT[dtype]).cuda()
        lse = (5 + torch.rand((off[-1], hq), generator=gen(1))).cuda()
        got = torch.full((len(codes[0]), hk, 16), 2.0, device="cuda")
        vs.vscan_kv_weigh(q, lse, i32(lens), i32(off), i32(table), dev[0], dev[2], got, d ** -0.5, max_q_len=top, decay=0.5)
        want = torch.full(got.shape, 2.0, dtype=torch.float64, device="cuda")
        for b, T in enumerate(lens):
            ids, n, rows = torch.tensor(table[b][:-(-T // 16)], device="cuda"), new[b], min(new[b], top)
            k = (dev[0][ids].double() * dev[2][ids].double()[..., None, None]).transpose(0, 1).reshape(hk, -1, d)[:, :T]
            x = q[off[b]:off[b] + rows].double().view(rows, hk, hq // hk, d)
            s = d ** -0.5 * torch.einsum("nhgd,htd->hgnt", x, k) - lse[off[b]:off[b] + rows].double().view(rows, hk, -1).permute(1, 2, 0)[..., None]
            s.masked_fill_(torch.arange(T, device="cuda") > T - n + torch.arange(rows, device="cuda")[:, None], -torch.inf)
            w = torch.cat([torch.full((hk, T - n), 1.0, device="cuda", dtype=torch.float64), torch.zeros((hk, n), device="cuda", dtype=torch.float64)], 1)
            w = torch.nn.functional.pad(w + s.exp().sum((1, 2)), (0, len(ids) * 16 - T), value=2.0)
            want[ids] = w.view(hk, len(ids), 16).transpose(0, 1)
        # scores of a few units at most: (head_dim + 8) 2^-24 (|s| + |lse|) below 136 x 2^-24 x 64 of a weight, and the sums
        tol = (136 * 2.0 ** -24 * 64 + 2.0 ** -21 + (max(new) * hq / 4 + 16) * 2.0 ** -24) * want.abs()
        assert ((got.double() - want).abs() <= tol).all(), float(((got.double() - want).abs() / tol).max())


def test_weigh_over_many_short_and_one_long_sequence():
    _weigh_case("e4m3", "bf16", 2, 1, 64, 16, [3000] + [2] * 40, [1] * 41, seed=5)
    _weigh_case("e4m3", "bf16", 8, 8, 64, 16, [20] * 30, [1] * 30, seed=6)


@pytest.mark.parametrize("kv", ["e4m3", "i8"])
@pytest.mark.parametrize("hq,hk,d,bs,past,new,window,causal,padded", [
    (2, 1, 256, 16, [300, 0], [40, 200], None, True, False), (7, 1, 192, 64, [100, 513], [64, 3], 20, True, True), (4, 4, 144, 32, [500], [129], None, False, False),
    (40, 1, 224, 128, [90, 7], [5, 30], 17, True, False), (64, 2, 256, 16, [130], [9], None, True, True), (3, 3, 240, 256, [0, 1000, 20], [300, 0, 257], 250, True, False)])
def test_weigh_windows_of_wide_heads(kv, hq, hk, d, bs, past, new, window, causal, padded):
    _weigh_case(kv, "bf16", hq, hk, d, bs, past, new, causal=causal, padded=padded, window=window, decay=0.5, seed=hq + d, missing=[(0, 1)] if past[0] else ())


def test_weigh_rows_that_see_nothing_give_nothing_and_nan_reaches_its_own():
    c, n = Cache("i8", 2, 16, 32, 4, 0), 3
    q = torch.randn((n, 2, 32), generator=gen(2)).to(torch.bfloat16).cuda()
    lse = torch.full((n, 2), float("-inf"), device="cuda")
    w = torch.ones((4, 2, 16), device="cuda")
    args = (i32([20]), i32([0, n]), i32([[3, 1]]), c.dev[0], c.dev_scale[0], w)
    vs.vscan_kv_weigh(q, lse, *args, 0.2, max_q_len=n)
    want = torch.ones((4, 2, 16), device="cuda")
    want[1, :, 1:4] = 0                                # tokens 17, 18, 19 are new
    assert torch.equal(w, want)
    c.dev_scale[0][1, 0] = float("nan")                # tokens 16 .. 19 of head 0
    lse.fill_(0.5)
    vs.vscan_kv_weigh(q, lse, *args, 1e-6, max_q_len=n)
    assert torch.isnan(w[1, 0, :4]).all() and not torch.isnan(w[1, 0, 4:]).any() and not torch.isnan(w[[0, 2, 3]]).any() and not torch.isnan(w[:, 1]).any()


# --------------------------------------------------------------------------- eviction
def _evict_case(kv, hk, d, bs, lens, budget, first=0, last=0, per_head=True, max_keep=None, seed=0, ties=False, spoil=None, where="other"):
    rng = np.random.default_rng(seed)
    B = len(lens)
    cols, blocks = max(max(-(-n // bs) for n in lens), 0) + 2, sum(max(-(-n // bs), 0) for n in lens) + 2
    kind, codes, scale, dev = _random_cache(kv, hk, bs, d, blocks, seed)
    table = _tables(lens, bs, cols, blocks, rng)
    weight = rng.random((blocks, hk, bs)).astype(np.float32)
    if ties:
        weight = (weight * 4).astype(np.int64).astype(np.float32)
    if spoil:
        spoil(table, weight, scale, codes)
        for i in range(2):
            dev[2 + i].copy_(torch.from_numpy(scale[i]))
            dev[i].view(torch.uint8).copy_(torch.from_numpy(codes[i]))
    most = max(max(budget), 0) if max_keep is None else max_keep
    w = torch.from_numpy(weight.copy()).cuda()
    w_out = {"other": torch.full_like(w, 9.0), "same": w, "none": None}[where]
    kept = torch.full((B, hk if per_head else 1, most), -5, dtype=torch.int32, device="cuda")
    ref, delta, moved, wrong = co.evict(codes, scale, weight, lens, budget, table, bs, kind, most, first, last, per_head)
    ws = vs.vscan_kv_evict_workspace(i32(table), dev[0], most, per_head)
    ws.buf.fill_(0xEE)
    got = vs.vscan_kv_evict(i32(lens), i32(budget), i32(table), w, *dev, most, first, last, per_head, weight_out=w_out, kept=kept, workspace=ws)
    assert vs.vscan_check(ws) == (1 if wrong else 0)
    assert got.tolist() == delta
    for b in range(B):
        n = 0 if ref[b] is None else len(ref[b][0])
        for i in range(kept.shape[1]):
            assert kept[b, i].tolist() == ([] if n == 0 else ref[b][i]) + [-5] * (most - n)
    # places behind the tokens that stay may hold anything
    alive = np.ones((blocks, hk, bs), dtype=bool)
    used = np.ones((blocks, hk), dtype=bool)
    for b, T in enumerate(lens):
        if ref[b] is None:
            continue
        n = T + delta[b]
        for t in range(n, -(-max(T, 1) // bs) * bs):
            alive[table[b][t // bs], :, t % bs] = False
        for j in range(-(-n // bs), -(-T // bs)):
            used[table[b][j]] = False
    for i in range(2):
        np.testing.assert_array_equal(dev[2 + i].double().cpu().numpy()[used], scale[i][used])
        np.testing.assert_array_equal(dev[i].view(torch.uint8).cpu().numpy()[alive], codes[i][alive])
    if w_out is not None:
        want = np.full_like(weight, 9.0) if where == "other" else weight
        for at, x in moved.items():
            want[at] = x
        at = alive if where == "same" else np.ones_like(alive)
        np.testing.assert_array_equal(w_out.cpu().numpy()[at], want[at])


@pytest.mark.parametrize("kv", ["e4m3", "i8"])
@pytest.mark.parametrize("per_head", [True, False])
@pytest.mark.parametrize("hk,d,bs,lens,budget,first,last", [
    (2, 64, 16, [100, 33, 16, 1, 0], [50, 32, 16, 0, 3], 0, 0), (1, 128, 16, [300], [299], 4, 10), (4, 128, 32, [70, 200], [35, 64], 2, 20),
    (3, 80, 64, [500, 64], [130, 63], 0, 1), (2, 256, 16, [90], [48], 1, 1), (2, 16, 256, [700, 255], [300, 100], 3, 3), (1, 256, 256, [600], [512], 0, 0),
    (8, 96, 128, [400], [129], 10, 100), (2, 128, 64, [130], [1], 0, 0), (2, 48, 16, [40, 50], [30, 30], 20, 20)])
def test_evict(kv, per_head, hk, d, bs, lens, budget, first, last):
    for where in ("other", "same", "none"):
        _evict_case(kv, hk, d, bs, lens, budget, first, last, per_head, seed=d + bs, where=where)


@pytest.mark.parametrize("per_head", [True, False])
def test_evict_ties_protected_tokens_and_what_is_not_finite(per_head):
    _evict_case("e4m3", 2, 32, 16, [120, 90], [40, 89], per_head=per_head, ties=True)
    _evict_case("i8", 2, 32, 16, [120, 90], [10, 20], 8, 30, per_head, ties=True)                # more protected ones than the budget
    _evict_case("i8", 1, 32, 16, [120], [40], 2 ** 31 - 1, 2 ** 31 - 1, per_head)

    def spoil(table, weight, scale, codes):
        weight[table[0][1]] = np.nan
        weight[table[0][2], :, 3] = np.inf
        weight[table[0][3], 0, :4] = -np.inf
        weight[table[0][4], :, :5] = -1.5
        weight[table[0][4], :, 5:8] = -0.0
        weight[table[0][4], :, 8:10] = 0.0
        scale[0][table[0][5], 0] = np.nan
        scale[1][table[0][0]] = 2.0 ** 48
        scale[1][table[0][2]] = 2.0 ** -48
        scale[0][table[0][6]] = 0.0
        codes[1][table[0][6]] = 0
    for n in (60, 90, 110):
        _evict_case("e4m3", 2, 32, 16, [128], [n], 0, 5, per_head, spoil=spoil)
        _evict_case("i8", 2, 32, 16, [128], [n], 0, 5, per_head, spoil=spoil)


@pytest.mark.parametrize("per_head", [True, False])
def test_evict_budgets_beyond_max_keep_and_sequences_out_of_order(per_head):
    _evict_case("i8", 2, 32, 16, [120, 20, 50], [100, 30, -4], per_head=per_head, max_keep=40)
    _evict_case("i8", 2, 32, 16, [120, 20], [0, 0], per_head=per_head, max_keep=0)

    def bad(table, weight, scale, codes):
        table[0][2] = -1
        table[2][0] = 10 ** 6
    _evict_case("e4m3", 2, 32, 16, [120, 90, 40], [50, 50, 40], per_head=per_head, spoil=bad)
    _evict_case("e4m3", 2, 32, 16, [-3, 60], [50, 50], per_head=per_head)


@pytest.mark.parametrize("kv", ["e4m3", "i8"])
@pytest.mark.parametrize("hk,d,bs", [(24, 32, 16), (32, 128, 32), (40, 16, 64), (26, 256, 16), (32, 48, 32)])
def test_evict_of_many_heads(kv, hk, d, bs):
    """Enough heads and sequences for a warp each."""
    rng = np.random.default_rng(hk)
    B = -(-1100 // hk)
    lens = [int(n) for n in rng.integers(0, min(5 * bs, 400), size=B)]     # (tables of at most 512 tokens at blocks of 16 to 64)
    budget = [int(rng.integers(0, n + 1)) for n in lens]

    def spoil(table, weight, scale, codes):
        scale[0][table[1][0], 3] = np.nan
    for per_head, where in ((True, "other"), (True, "same"), (False, "none")):
        _evict_case(kv, hk, d, bs, lens, budget, 2, 3, per_head, where=where, seed=d, spoil=spoil, ties=where == "same")


def test_evict_of_many_short_sequences_out_of_order_and_of_no_finite_rank():
    rng = np.random.default_rng(5)
    lens = [int(n) for n in rng.integers(-1, 200, size=310)]
    budget = [int(n) for n in rng.integers(-2, 150, size=310)]

    def spoil(table, weight, scale, codes):
        weight[rng.random(weight.shape) < 0.3] = np.nan
        weight[rng.random(weight.shape) < 0.3] = -np.inf
        weight[rng.random(weight.shape) < 0.2] = np.inf
        weight[rng.random(weight.shape) < 0.2] = -0.0
        for b in range(0, 310, 9):
            if lens[b] > 0:
                table[b][(lens[b] - 1) // 16] = (-1, 10 ** 6)[b % 2]
    for per_head in (True, False):
        _evict_case("i8", 3, 16, 16, lens, budget, 1, 2, per_head, spoil=spoil, max_keep=120)


@pytest.mark.parametrize("per_head", [True, False])
@pytest.mark.parametrize("length,keep", [(5000, 1200), (20000, 9000), (20000, 19990)])
def test_evict_long_sequences(per_head, length, keep):
    """Beyond what shared memory holds of the keys, many units in a row that wait for those in front; against torch in 64 bits."""
    hk, d, bs, g = 2, 32, 16, gen(length + keep)
    cols = -(-length // bs)
    k, v = (torch.randn((1, hk, length, d), generator=g).cuda() for _ in range(2))
    c = vs.VScanCache(num_blocks=cols, block_size=bs, kv_heads=hk, head_dim=d, batch=1, max_blocks=cols, rows=length, kv_dtype="i8")
    c.plan(i32([length]))
    c.write(k, v)
    w = (torch.randint(0, 50, (cols, hk, bs), generator=g).float() ** 2).cuda()
    ids = c.block_table[0].long()

    def rows(codes, scale):
        return (codes[ids].double() * scale[ids][..., None, None].double()).transpose(0, 1).reshape(hk, cols * bs, d)[:, :length]
    before = [rows(c.k, c.k_scale), rows(c.v, c.v_scale)]
    flat = w[ids].transpose(0, 1).reshape(hk, -1)[:, :length].double()
    rank = flat if per_head else flat.sum(0, keepdim=True)
    order = torch.sort(rank, dim=-1, descending=True, stable=True)[1][:, :keep]
    src = torch.sort(order, -1)[0].expand(hk, keep)
    kept = torch.zeros((1, hk if per_head else 1, keep), dtype=torch.int32, device="cuda")
    delta = vs.vscan_kv_evict(c.kv_len, i32([keep]), c.block_table, w, *c.arrays, keep, per_head=per_head, kept=kept)
    assert delta.tolist() == [keep - length] and torch.equal(kept[0].long(), src[:kept.shape[1]])
    c.plan(delta)
    assert c.kv_len.tolist() == [keep] and int(c.report[2]) == cols - -(-keep // bs)
    used = -(-keep // bs)
    for old, (codes, scale) in zip(before, ((c.k, c.k_scale), (c.v, c.v_scale))):
        want = old.gather(1, src[..., None].expand(hk, keep, d))
        now = (codes[ids[:used]].double() * scale[ids[:used]][..., None, None].double()).transpose(0, 1).reshape(hk, -1, d)[:, :keep]
        step = scale[ids[:used]].double().T.repeat_interleave(bs, 1)[:, :keep, None]
        assert ((now - want).abs() <= step / 2).all()
        full = torch.cat([want, want.new_zeros(hk, used * bs - keep, d)], 1).view(hk, used, bs * d).abs().amax(-1)
        fits = full <= 127 * scale[ids[:used]].double().T
        assert fits.all()


def test_evict_in_a_graph_and_again():
    """Captured and replayed: the workspace of the call before says nothing."""
    kind, codes, scale, dev = _random_cache("i8", 2, 16, 32, 9, 0)
    table, w = i32([[0, 1, 2, 3, 4, 5, 6, 7]]), torch.rand((9, 2, 16), generator=gen(0)).cuda()
    first = [t.clone() for t in dev]
    args = (i32([125]), i32([60]), table, w, *dev, 60)
    ws = vs.vscan_kv_evict_workspace(table, dev[0], 60)
    vs.vscan_kv_evict(*args, workspace=ws)
    want = [t.clone() for t in dev]
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        vs.vscan_kv_evict(*args, workspace=ws)
    for _ in range(5):
        for t, u in zip(dev, first):
            t.copy_(u)
        graph.replay()
        assert all(torch.equal(t.view(torch.uint8) if t.element_size() == 1 else t, u.view(torch.uint8) if u.element_size() == 1 else u)
                   for t, u in zip(dev, want))
    assert vs.vscan_check(ws) == 0


# --------------------------------------------------------------------------- a run of them together
@pytest.mark.parametrize("kv", ["e4m3", "i8"])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("per_head", [True, False])
def test_a_layer_from_prompts_to_evictions(kv, dtype, per_head):
    """Prompts, decode steps, an eviction, decode steps, another one: each call's result against 64 bits from what the cache held before it."""
    hq, hk, d, bs, B, cols = 6, 2, 64, 16, 3, 12
    g, kind = gen(11), KV[kv][0]
    c = vs.VScanCache(num_blocks=B * cols, block_size=bs, kv_heads=hk, head_dim=d, batch=B, max_blocks=cols, rows=500, kv_dtype=kv, weights=True)
    rope, scale = vs.rope_table(d, [d // 2]), d ** -0.5
    weight = np.zeros((B * cols, hk, bs))

    def state():
        return [t.view(torch.uint8).cpu().numpy() for t in (c.k, c.v)], [t.double().cpu().numpy() for t in (c.k_scale, c.v_scale)], c.block_table.tolist()

    def sequence(codes, scales, table, i, b, T):
        return co.gather(codes[i], scales[i], table[b], T, bs, kind)

    def weights_follow(q, lse, new, lens, decay, window):
        codes, scales, table = state()
        slack = co.weigh(weight, [q[b, :, :n].transpose(0, 1).double().cpu().numpy() for b, n in enumerate(new)],
                         [lse[b][:n] for b, n in enumerate(new)], codes[0], scales[0], lens, table, bs, kind, scale, decay, window)
        # lse is that of 64 bits here: the calls' own is off by what test_attention allows, at most 1e-5 + (head_dim + 8) 2^-24 of the scores' size
        tol = (2 * (d + 8) * 2.0 ** -24) * slack + (1e-5 + 2.0 ** -21 + (max(new) * 3 / 4 + 16) * 2.0 ** -24) * np.abs(weight)
        got = c.weight.double().cpu().numpy()
        for b, T in enumerate(lens):
            for t in range(T):
                at = (table[b][t // bs], slice(None), t % bs)
                assert (np.abs(got[at] - weight[at]) <= tol[at] + 1e-30).all(), (b, t, got[at], weight[at])
        weight[:] = got

    new = [140, 17, 63]
    q, k, v = (torch.randn((B, H, max(new), d), generator=g).to(DT[dtype]).cuda() for H in (hq, hk, hk))
    pos = torch.arange(max(new), dtype=torch.int32, device="cuda").expand(1, B, -1).contiguous()
    out = c.prompt(q, k, v, pos, rope, i32(new), scale, window=8)
    tq, tk = vs.vscan_rope(q, k, pos, *rope)
    lse = []
    for b, n in enumerate(new):
        x = [t[b, :, :n].transpose(0, 1) for t in (tq, tk, v)]
        _, ref_lse, _, _ = plain_attention(*x, scale, True)
        got_lse = ref_lse.float()                                       # its own check is in test_attention
        check_attention(dtype, out[b, :, :n].transpose(0, 1), got_lse, *x, scale, True)
        lse.append(ref_lse.cpu().numpy())
    lens = list(new)
    weights_follow(tq, lse, new, lens, 1.0, 8)
    assert c.kv_len.tolist() == lens and c.check() == (0, 0)
    where = [pos[0, b, :n].tolist() for b, n in enumerate(new)]
    for turn in range(2):
        for _ in range(3):
            q, k, v = (torch.randn((B, H, 1, d), generator=g).to(DT[dtype]).cuda() for H in (hq, hk, hk))
            at = torch.tensor([[[w[-1] + 1] for w in where]], dtype=torch.int32, device="cuda")
            for w in where:
                w.append(w[-1] + 1)
            out = c.step(q, k, v, at, rope, i32([1] * B), scale, decay=0.75)
            lens = [n + 1 for n in lens]
            tq, _ = vs.vscan_rope(q, k, at, *rope)
            codes, scales, table = state()
            lse = []
            for b, T in enumerate(lens):
                (kk, there), (vv, _) = (sequence(codes, scales, table, i, b, T) for i in range(2))
                ref, ref_lse, size, reach = co.attention(tq[b].transpose(0, 1).double().cpu().numpy(), kk, vv, there, scale, True, T - 1)
                err = np.abs(out[b].transpose(0, 1).double().cpu().numpy() - ref)
                e = (d + 8) * 2.0 ** -24 * reach
                tol = (2 * e + 2.0 ** -21 + (2.0 ** -11 if dtype == "bf16" else 0) + (T / 4 + 16) * 2.0 ** -24)[..., None] * size + h(dtype) * np.abs(ref)
                assert (err <= tol + T * 2.0 ** -29 * np.abs(vv).max()).all()
                lse.append(ref_lse)
            weights_follow(tq, lse, [1] * B, lens, 0.75, None)
        codes, scales, table = state()
        budget = [60, 40, 30 + turn]
        ref, delta, moved, wrong = co.evict(codes, scales, weight.astype(np.float32), lens, budget, table, bs, kind, 64, 2, 5, per_head)
        kept = torch.full((B, hk if per_head else 1, 64), -1, dtype=torch.int32, device="cuda")
        assert c.evict(i32(budget), 64, keep_first=2, keep_last=5, per_head=per_head, kept=kept).tolist() == delta and not wrong
        for b in range(B):
            for i in range(kept.shape[1]):
                assert kept[b, i, :lens[b] + delta[b]].tolist() == ref[b][i]
        lens = [n + e for n, e in zip(lens, delta)]
        assert c.kv_len.tolist() == lens and c.check() == (0, 0)
        now, now_scales, _ = state()
        for b, T in enumerate(lens):
            for i in range(2):
                want, got = sequence(codes, scales, table, i, b, T), sequence(now, now_scales, table, i, b, T)
                np.testing.assert_array_equal(got[0], want[0])
            for t in range(T):
                weight[table[b][t // bs], :, t % bs] = [moved[table[b][t // bs], head, t % bs] for head in range(hk)]
        free = int(c._plan["ring_state_out"][1] - c._plan["ring_state_out"][0])
        assert free == B * cols - sum(-(-n // bs) for n in lens)
