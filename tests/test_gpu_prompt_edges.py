"""vscan_attention, vscan_kv_weigh and vscan_kv_evict where they could go wrong beside what test_gpu_prompt_ops.py runs; tolerances are those of that
file."""
import numpy as np
import pytest
import torch

import paper_2505_22654_b200 as vs
from oracle import cache_oracle as co
from test_gpu_cache_ops import DT, _offsets, gen, i32
from test_gpu_prompt_ops import _evict_case, _random_cache, check_attention

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
