"""vscan_kv_attention where a score's factor vanishes: scale 0, query rows of zeros, keys of zeros, negative scale; causal rows that
see part of a 16-token group.  Against the float64 oracle, for every kernel the calls choose from.

Tolerances as derived in test_gpu_cache_ops.py.
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
