"""vscan_attention, vscan_kv_weigh and vscan_kv_evict where they could go wrong beside what test_gpu_prompt_ops.py runs; tolerances are those of that
file."""
import pytest
import torch

import paper_2505_22654_b200 as vs
from test_gpu_cache_ops import DT, _offsets, gen, i32
from test_gpu_prompt_ops import check_attention

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
