"""vscan_rope and the vscan_kv_* calls against the float64 oracle: types, head layouts, lengths from nothing to long, odd
sizes, strides, masked and missing tokens, and a run of them together as a decode step uses them.

Tolerances, fixed before the first run.  `h(t)` = finfo(t).eps / 2 is the one rounding of a result.
  rope    cos and sin are off by at most 2^-25 pi (the angle's rounding) + 2^-24 (the function's), the products and the sum by
          2^-24 each: 5e-7 (|x| + |y|) in all, plus h |result|.
  attend  with A = sum p |v| and e = (head_dim + 8) 2^-24 max scale sum |q| |k| (error of a score, summed in 32 bits), each
          weight is off by 2 e + 2^-21 (exponential) + h(f16) where the weights are rounded to 16 bits (bf16 queries), the sums
          by (tokens / 4 + 16) 2^-24: times A, plus h |result|.  lse: e + (tokens / 4 + 16) 2^-24 + |lse| 2^-22.
          Weights in 16 bits also have a smallest step.  The largest weight of a row is at least 2^8 before its rounding, in units of
          a V scale that is at most 8 times a block's own, so each is off by at most half of 2^-24, 2^-33 of the largest; a code
          times that scale is at most 16 max |v| (a block's scale is at most twice what its values need): tokens 2^-29 max |v|
          in all, which is all there is of a result whose heavy keys have values of exactly 0.
"""
import numpy as np
import pytest
import torch

import paper_2505_22654_b200 as vs
from oracle import cache_oracle as co

pytestmark = pytest.mark.gpu

DT = {"f32": torch.float32, "bf16": torch.bfloat16}
KV = {"e4m3": (co.E4M3, torch.float8_e4m3fn), "i8": (co.I8, torch.int8)}


def h(dtype):
    return torch.finfo(DT[dtype]).eps / 2


def attend_tol(dtype, d, T, ref, weight, reach, v):
    """As derived above."""
    e = (d + 8) * 2.0 ** -24 * reach
    tol = (2 * e + 2.0 ** -21 + (2.0 ** -11 if dtype == "bf16" else 0) + (T / 4 + 16) * 2.0 ** -24)[..., None] * weight + h(dtype) * np.abs(ref)
    return tol + (T * 2.0 ** -29 * np.abs(v).max(initial=0.0) if dtype == "bf16" else 0)


def i32(v):
    return torch.tensor(np.asarray(v), dtype=torch.int32, device="cuda")


def gen(seed):
    return torch.Generator().manual_seed(seed)


# --------------------------------------------------------------------------- rope
def _rope_check(x, got, pos, freq, axis, pairing, inverse, dtype):
    x, got, pos, freq, axis = x.double().cpu().numpy(), got.double().cpu().numpy(), pos.cpu().numpy(), freq.double().cpu().numpy(), axis.cpu().numpy()
    n = len(freq)
    for b in range(x.shape[0]):
        ref = co.rope(x[b], pos[:, b], freq, axis, pairing, inverse)
        mag = np.zeros_like(ref)
        lo, hi = (slice(0, n), slice(n, 2 * n)) if pairing == co.HALVES else (slice(0, 2 * n, 2), slice(1, 2 * n, 2))
        mag[..., lo] = mag[..., hi] = np.abs(x[b][..., lo]) + np.abs(x[b][..., hi])
        err = np.abs(got[b] - ref)
        assert (err <= 5e-7 * mag + h(dtype) * np.abs(ref)).all(), (b, err.max())


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("B,S,hq,hk,d,rot,planes,pairing,far", [
    (3, 1, 28, 4, 128, 128, 3, 0, 500000), (2, 37, 3, 1, 80, 80, 2, 1, 64), (1, 5, 4, 4, 72, 36, 4, 0, 2 ** 31 - 1),
    (2, 9, 2, 2, 24, 14, 1, 1, 100), (1, 3, 1, 1, 8, 2, 1, 0, 9), (1, 3, 1, 1, 8, 2, 2, 1, 9), (5, 700, 7, 1, 64, 32, 3, 0, 30000),
    (1, 2, 2, 1, 512, 512, 16, 1, 1000)])
def test_rope(dtype, B, S, hq, hk, d, rot, planes, pairing, far):
    g = gen(B * S + d)
    qkv = torch.randn((B, S, hq + 2 * hk, d), generator=g).to(DT[dtype]).cuda()
    q, k = qkv[:, :, :hq].transpose(1, 2), qkv[:, :, hq:hq + hk].transpose(1, 2)
    pos = torch.randint(-3, far, (planes, B, S), generator=g, dtype=torch.int32).cuda()
    sizes = [rot // 2 // planes] * planes
    sizes[-1] += rot // 2 - sum(sizes)
    freq, axis = vs.rope_table(rot, sizes, layout="cycled")
    for inverse in (False, True):
        qo, ko = vs.vscan_rope(q, k, pos, freq, axis, pairing=pairing, inverse=inverse)
        _rope_check(q, qo, pos, freq, axis, pairing, inverse, dtype)
        _rope_check(k, ko, pos, freq, axis, pairing, inverse, dtype)
    # one side alone, into another layout; in place within the projection, values behind the keys left alone
    alone = torch.empty((B, hk, S, d), dtype=DT[dtype], device="cuda")
    assert vs.vscan_rope(None, k, pos, freq, axis, pairing=pairing, inverse=True, k_out=alone)[0] is None
    assert torch.equal(alone, ko)
    want_v = qkv[:, :, hq + hk:].clone()
    vs.vscan_rope(q, k, pos, freq, axis, pairing=pairing, inverse=True, q_out=q, k_out=k)
    assert torch.equal(q, qo) and torch.equal(k, ko) and torch.equal(qkv[:, :, hq + hk:], want_v)


def test_rope_axis_out_of_range_is_held_and_empty_calls_do_nothing():
    x = torch.randn((1, 1, 4, 16), generator=gen(1)).cuda()
    pos = torch.arange(8, dtype=torch.int32, device="cuda").view(2, 1, 4)
    freq = torch.ones(8, device="cuda")
    a, _ = vs.vscan_rope(x, None, pos, freq, i32([-5, 0, 1, 99, 1, 0, 7, -1]))
    b, _ = vs.vscan_rope(x, None, pos, freq, i32([0, 0, 1, 1, 1, 0, 1, 0]))
    assert torch.equal(a, b)
    before = vs.kernel_launches()
    vs.vscan_rope(x[:, :, :0], None, pos[:, :, :0].contiguous(), freq, i32([0] * 8))
    assert vs.kernel_launches() == before


def test_rope_gradient_is_the_inverse_call():
    """d(sum w * rope(x)) / dx by central differences in float32; the map is linear, so a difference of step 1 is exact but for
    the roundings of two results of size <= 8: 4 * 2^-24 * 8 + 2 * 5e-7 * 8 < 2e-5."""
    g = gen(3)
    x, w = torch.randn((1, 2, 3, 16), generator=g).cuda(), torch.randn((1, 2, 3, 16), generator=g).cuda()
    pos = torch.randint(0, 1000, (2, 1, 3), generator=g, dtype=torch.int32).cuda()
    freq, axis = vs.rope_table(16, [4, 4], layout="per_axis")
    for pairing in (0, 1):
        grad, _ = vs.vscan_rope(w, None, pos, freq, axis, pairing=pairing, inverse=True)
        for at in [(0, 0, 0, 0), (0, 1, 2, 15), (0, 0, 1, 8), (0, 1, 0, 5)]:
            step = torch.zeros_like(x)
            step[at] = 0.5
            up, down = (vs.vscan_rope(x + s * step, None, pos, freq, axis, pairing=pairing)[0] for s in (1, -1))
            diff = float(((up - down).double() * w.double()).sum())
            assert abs(diff - float(grad[at])) < 2e-5 * float(w.abs().max() + 1)


# --------------------------------------------------------------------------- plan
def _plan_both(past, new, table, ring, state, bs, rows):
    t, r = i32(table).view(len(past), -1), i32(ring)
    slots = torch.full((rows,), -7, dtype=torch.int64, device="cuda")
    places = torch.full((rows,), -7, dtype=torch.int32, device="cuda")
    st = torch.tensor(state, dtype=torch.int64, device="cuda")
    for _ in range(2):        # planned twice from the same state: the same answer
        o = vs.vscan_kv_plan(i32(past), i32(new), t, r, st, bs, out={"slot_map": slots, "row_pos": places})
    ref = co.plan(past, new, table, ring, state, bs, rows)
    n = len(ref["slots"])
    assert o["report"].tolist() == ref["report"]
    assert o["kv_len"].tolist() == ref["kv_len"] and o["row_offset"].tolist() == ref["row_offset"]
    assert o["ring_state_out"].tolist() == ref["state"] and st.tolist() == list(state)
    assert t.tolist() == ref["table"] and r.tolist() == ref["ring"]
    assert slots.tolist() == ref["slots"] + [-7] * (rows - n) and places.tolist() == ref["positions"] + [-7] * (rows - n)
    return ref


@pytest.mark.parametrize("batch,bs,cols,most,seed", [(1, 16, 3, 40, 0), (5, 16, 9, 60, 1), (33, 32, 40, 900, 2), (300, 128, 4, 300, 3), (1000, 16, 12, 40, 4),
                                                     (2, 256, 30, 7000, 5)])
def test_plan_over_many_steps(batch, bs, cols, most, seed):
    rng = np.random.default_rng(seed)
    n = batch * cols * 2 // 3 + 2
    table, ring, state, past = [[-1] * cols for _ in range(batch)], [int(v) for v in rng.permutation(n)], [n - 1, 2 * n - 1], [0] * batch
    codes = set()
    for step in range(6):
        new = []
        for p in past:
            kind = rng.random()
            new.append(1 if kind < 0.4 and p < cols * bs else -p if kind < 0.5 else int(rng.integers(-p, 1)) if kind < 0.6
                       else int(rng.integers(0, min(most, cols * bs - p) + 1)) if kind < 0.95 else 0)
        ref = _plan_both(past, new, table, ring, state, bs, max(sum(max(v, 0) for v in new) + int(rng.integers(0, 5)), 1))
        table, ring, state, past = ref["table"], ref["ring"], ref["state"], ref["kv_len"]
        codes.add(ref["report"][0])
    assert 0 in codes


@pytest.mark.parametrize("change,code", [(dict(ring_free=1), 1), (dict(new=[200, 1]), 2), (dict(rows=5), 4), (dict(new=[-21, 1]), 8), (dict(past=[-1, 3]), 8),
                                         (dict(state=[5, 4]), 16), (dict(state=[0, 11]), 16), (dict(past=[2 ** 31 - 1, 3], new=[2 ** 31 - 1, 1]), 7)])
def test_plan_that_does_not_fit_changes_nothing(change, code):
    past, new = change.get("past", [20, 3]), change.get("new", [30, 5])
    state = change.get("state", [3, 3 + change.get("ring_free", 6)])
    ref = _plan_both(past, new, [[8, 9, -1, -1], [7, -1, -1, -1]], list(range(10)), state, 16, change.get("rows", 40))
    assert ref["report"][0] & code == code and ref["row_offset"] == [0, 0, 0]


def test_plan_of_no_requests_and_without_rows():
    none = i32([])
    o = vs.vscan_kv_plan(none, none, i32([]).view(0, 4), i32([1, 2]), torch.tensor([0, 2], device="cuda"), 16)
    assert o["row_offset"].tolist() == [0] and o["report"].tolist() == [0, 0, 0, 0] and o["ring_state_out"].tolist() == [0, 2]
    t = i32([[-1, -1]])
    o = vs.vscan_kv_plan(i32([0]), i32([20]), t, i32([4, 6]), torch.tensor([1, 3], device="cuda"), 16, rows=20, out={"row_pos": None})
    assert vs.vscan_kv_plan(i32([0]), i32([20]), i32([[-1, -1]]), i32([4, 6]), torch.tensor([1, 3], device="cuda"), 16)["report"].tolist() == [0, 2, 0, 20]
    assert t.tolist() == [[6, 4]] and o["slot_map"].tolist() == [6 * 16 + i for i in range(16)] + [4 * 16 + i for i in range(4)]


# --------------------------------------------------------------------------- write
class Cache:
    """A small cache on the GPU and the oracle's copy of it, filled with bytes that nothing may depend on."""

    def __init__(self, kv, H, bs, d, blocks, seed):
        self.kind, dt = KV[kv]
        self.bs, self.H, self.d, self.blocks = bs, H, d, blocks
        rng = np.random.default_rng(seed)
        self.codes = [rng.integers(0, 127, size=(blocks, H, bs, d)).astype(np.uint8) for _ in range(2)]
        self.scale = [2.0 ** rng.integers(-8, 3, size=(blocks, H)).astype(np.float64) for _ in range(2)]
        self.dev = [torch.from_numpy(c.copy()).cuda().view(dt) for c in self.codes]
        self.dev_scale = [torch.from_numpy(s).float().cuda() for s in self.scale]

    arrays = property(lambda self: (*self.dev, *self.dev_scale))

    def write(self, ks, vs_, kv_len, table):
        for i, rows in enumerate((ks, vs_)):
            co.write(self.codes[i], self.scale[i], [r.double().cpu().numpy() for r in rows], kv_len, table, self.bs, self.kind)

    def same(self):
        for i in range(2):
            np.testing.assert_array_equal(self.dev_scale[i].double().cpu().numpy(), self.scale[i])
            np.testing.assert_array_equal(self.dev[i].view(torch.uint8).cpu().numpy(), self.codes[i])


def _offsets(n):
    return np.concatenate([[0], np.cumsum(n)]).astype(int)


def _tables(lens, bs, cols, blocks, rng):
    ids = list(rng.permutation(blocks))
    return [[int(ids.pop()) if j * bs < n else -1 for j in range(cols)] for n in lens]


@pytest.mark.parametrize("kv", ["e4m3", "i8"])
@pytest.mark.parametrize("dtype,H,bs,d,past,new,padded", [
    ("bf16", 4, 16, 128, [0, 15, 16, 17, 40], [1, 1, 1, 1, 1], False),             # single tokens, each place in a block
    ("bf16", 3, 16, 64, [0, 5, 31, 3, 0], [0, 3, 40, 13, 1], False),               # ragged, a sequence without rows
    ("f32", 2, 32, 80, [7, 0, 63], [1, 100, 34], False), ("bf16", 2, 64, 256, [60, 0], [200, 129], True),
    ("f32", 1, 128, 16, [0], [300], True), ("bf16", 32, 16, 128, [0, 0], [35, 35], True), ("f32", 5, 256, 96, [255, 1], [2, 300], False),
    ("bf16", 1, 16, 240, [9], [5], True), ("f32", 8, 64, 128, [0, 10, 20], [2, 1, 3], True)])
def test_write(kv, dtype, H, bs, d, past, new, padded):
    rng, g = np.random.default_rng(len(past) + d), gen(d + bs)
    B, lens = len(past), [p + n for p, n in zip(past, new)]
    cols = max(-(-n // bs) for n in lens) + 1
    blocks = sum(-(-n // bs) for n in lens) + 3
    c = Cache(kv, H, bs, d, blocks, d)
    table = _tables(lens, bs, cols, blocks, rng)
    off = _offsets(new)
    # sizes over many binades, a few rows much larger, exact qmax edges; one (row, head) of zeros
    rows = [[(torch.randn((n, H, d), generator=g) * torch.exp2(torch.randint(-6, 7, (n, H, 1), generator=g).float())).to(DT[dtype]) for n in new] for _ in range(2)]
    rows[0][-1][0, 0] = 0
    rows[1][-1][-1, -1] = 448.0
    most = max(new) + 2
    sent = []
    for r in rows:
        if padded:
            t = torch.full((B, H, most, d), float("nan"), dtype=DT[dtype])
            for b in range(B):
                t[b, :, :new[b]] = r[b].transpose(0, 1)
            sent.append(t.cuda())
        else:               # rows of a wider buffer, NaN behind the last sequence
            t = torch.full((off[-1] + 3, 2 * H, d), float("nan"), dtype=DT[dtype])
            t[:off[-1], :H] = torch.cat(r)
            sent.append(t.cuda()[:, :H])
    for _ in range(2):      # written twice: the same bytes
        vs.vscan_kv_write(*sent, i32(lens), i32(off), i32(table), *c.arrays)
        if _ == 0:
            c.write(*rows, lens, table)
        c.same()


@pytest.mark.parametrize("kv", ["e4m3", "i8"])
@pytest.mark.parametrize("many", [1, 20])
def test_write_growing_scales_and_what_is_not_finite(kv, many):
    H, bs, d = 2, 32, 32
    c = Cache(kv, H, bs, d, 6, 1)
    table, g, n = [[4, 2, 0]], gen(8), 0
    for step, size in enumerate([1e-20, 1.0, 1.0, 300.0, 1e4, 1e-3, float("inf"), 1.0, 3e30, 2.0]):
        x = torch.randn((many, H, d), generator=g)
        x *= size if np.isfinite(size) else 1.0
        if not np.isfinite(size):
            x[0, 0, 3], x[0, 1, 0] = float("inf"), float("nan")
        n = n + many if n + many <= 3 * bs else many
        y = -x.flip(0)
        vs.vscan_kv_write(x.cuda(), y.cuda(), i32([n]), i32([0, many]), i32(table), *c.arrays)
        c.write([x], [y], [n], table)
        c.same()


def test_write_skips_bad_tables_and_lengths():
    H, bs, d = 1, 16, 16
    x = torch.randn((80, H, d), generator=gen(2))
    for rows in (x, x[:2]):                                     # block form, append form
        n = len(rows) // 2
        for kv_len, off, table in [([n, n], [0, n, 2 * n], [[99, 1, 2, -1], [-1, 3, 2 ** 31 - 1, 4]]), ([n - 1, n + 70], [0, n, 2 * n], [[0, 1, 2, 3], [4, 5, 6, 7]]),
                                   ([n, n], [0, n, 3 * n], [[0, 1, 2, 3], [4, 5, 6, 7]]), ([n, n], [5, 2, -4], [[0, 1, 2, 3], [4, 5, 6, 7]])]:
            c = Cache("i8", H, bs, d, 9, 0)
            before = [t.clone() for t in c.arrays]
            vs.vscan_kv_write(rows.cuda(), rows.cuda(), i32(kv_len), i32(off), i32(table), *c.arrays)
            torch.cuda.synchronize()
            touched = {int(b) for t, u in zip(before[2:], c.arrays[2:]) for b in (t != u).any(1).nonzero()}
            assert touched <= {b for r in table for b in r if 0 <= b < 9}
            untouched = [b for b in range(9) if b not in {b for r in table for b in r}]
            for t, u in zip(before[:2], c.arrays[:2]):
                assert torch.equal(t[untouched], u[untouched])


# --------------------------------------------------------------------------- attention
def _attend_case(kv, dtype, hq, hk, d, bs, past, new, causal, padded, seed, max_q=None, poison=True, q_gain=1.0, missing=()):
    """Runs one call on a random cache and checks it, the rows around it included."""
    rng, g = np.random.default_rng(seed), gen(seed)
    B, lens = len(past), [p + n for p, n in zip(past, new)]
    cols = max(max(-(-n // bs) for n in lens), 1) + 1
    blocks = sum(-(-n // bs) for n in lens) + 2
    kind, dt = KV[kv]
    codes = [rng.integers(0, 256, size=(blocks, hk, bs, d)).astype(np.uint8) for _ in range(2)]
    for c in codes:
        c[(c & 0x7F) == 0x7F] = 0x11 if kind == co.E4M3 else 0x7E
        c[c == 0x80] = 0
    scale = [2.0 ** rng.integers(-9, -6, size=(blocks, hk)) for _ in range(2)]
    table = _tables(lens, bs, cols, blocks, rng)
    for b, j in missing:
        table[b][j] = (-1, blocks, 2 ** 31 - 1, -2 ** 31)[(b + j) % 4]
    dev = [torch.from_numpy(c.copy()) for c in codes]
    dev_scale = [torch.from_numpy(s.copy()).float() for s in scale]
    if poison:              # what lies behind a sequence's end, and in blocks of no sequence, may be anything
        used = {blk: min(bs, lens[b] - j * bs) for b, r in enumerate(table) for j, blk in enumerate(r) if 0 <= blk < blocks}
        for t, s in zip(dev, dev_scale):
            for blk in range(blocks):
                t[blk, :, used.get(blk, 0):] = 0x7F if kind == co.E4M3 else 0x80
                if blk not in used:
                    s[blk] = float("nan")
    dev, dev_scale = [t.cuda().view(dt) for t in dev], [s.cuda() for s in dev_scale]
    top = max_q or max(max(new), 1)
    off, extra = _offsets(new), 3
    qs = [(q_gain * torch.randn((n, hq, d), generator=g)).to(DT[dtype]) for n in new]
    if padded:
        q = torch.full((B, hq, max(new) + 2, d), float("nan"), dtype=DT[dtype])
        for b in range(B):
            q[b, :, :new[b]] = qs[b].transpose(0, 1)
        q = q.cuda()
    else:
        q = torch.full((off[-1] + extra, hq, d), float("nan"), dtype=DT[dtype])
        q[:off[-1]] = torch.cat(qs)
        q = torch.cat([q, q], dim=1).cuda()[:, :hq]                              # rows of a wider buffer
    out, lse = torch.full(q.shape, 7.0, dtype=DT[dtype], device="cuda"), torch.full(q.shape[:-1], 7.0, device="cuda")
    s = d ** -0.5
    ws = vs.vscan_kv_attention_workspace(q, i32(table), dev[0], top)
    ws.buf.fill_(0xEE)
    args = (q, i32(lens), i32(off), i32(table), *dev, *dev_scale, s)
    vs.vscan_kv_attention(*args, max_q_len=top, causal=causal, out=out, lse=lse, workspace=ws)
    assert vs.vscan_check(ws) == (1 if missing else 0)
    again = torch.full(q.shape, 7.0, dtype=DT[dtype], device="cuda")
    vs.vscan_kv_attention(*args, max_q_len=top, causal=causal, out=again, workspace=ws)
    assert torch.equal(out, again), "the same call gives other bits"
    got, stats = out.double().cpu().numpy(), lse.double().cpu().numpy()
    for b in range(B):
        n, T = new[b], lens[b]
        mine, mine_lse = (got[b, :, :n].transpose(1, 0, 2), stats[b, :, :n].T) if padded else (got[off[b]:off[b + 1]], stats[off[b]:off[b + 1]])
        if n == 0:
            continue
        (k, there), (v, _) = (co.gather(codes[i], scale[i], table[b], T, bs, kind) for i in range(2))
        ref, ref_lse, weight, reach = co.attention(qs[b].double().numpy(), k, v, there, s, causal, T - n)
        e = (d + 8) * 2.0 ** -24 * reach
        sums = (T / 4 + 16) * 2.0 ** -24
        tol = attend_tol(dtype, d, T, ref, weight, reach, v[there])
        err = np.abs(mine - ref)
        assert (err <= tol).all(), (b, float((err / np.maximum(tol, 1e-30)).max()), np.argwhere(err > tol)[:4])
        fine = np.isfinite(ref_lse)
        np.testing.assert_array_equal(mine_lse[~fine], ref_lse[~fine])
        err = np.abs(mine_lse[fine] - ref_lse[fine])
        assert (err <= (e + sums + np.abs(np.where(fine, ref_lse, 0)) * 2.0 ** -22)[fine]).all(), float(err.max())
    # rows that no sequence owns are as they were
    if padded:
        for b in range(B):
            assert (got[b, :, new[b]:] == 7).all() and (stats[b, :, new[b]:] == 7).all()
    else:
        assert (got[off[-1]:] == 7).all() and (stats[off[-1]:] == 7).all()


@pytest.mark.parametrize("kv", ["e4m3", "i8"])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("hq,hk,d,bs,past,new", [
    (4, 4, 128, 16, [0, 15, 16, 62, 63, 64], [1, 1, 1, 1, 1, 1]),       # one head a group, ends inside and on tile borders
    (14, 2, 128, 64, [300, 0, 1000], [1, 1, 1]),                        # groups of seven
    (8, 1, 64, 32, [129], [1]), (16, 1, 256, 16, [70, 33], [1, 1]), (2, 1, 80, 128, [200], [1]), (6, 3, 16, 256, [5, 400], [1, 1]),
    (40, 1, 96, 16, [77], [1]), (64, 1, 64, 16, [90], [1]),
    (4, 2, 128, 16, [10, 0, 200], [0, 5, 3]),                           # a sequence without rows, few rows each
    (7, 1, 128, 16, [50, 3, 0], [16, 1, 33]), (2, 2, 64, 16, [0], [70]), (3, 1, 48, 32, [100], [40]),
    # many rows: one and two tiles of 128 rows, several of 256, steps of 128 keys that end inside, whole and short sequences mixed
    (1, 1, 128, 16, [0], [128]), (1, 1, 64, 64, [128], [129]), (7, 1, 128, 64, [300], [75]), (4, 2, 80, 16, [0, 500, 3], [130, 1, 66]),
    (2, 1, 16, 128, [250], [300]), (12, 2, 96, 32, [77, 0], [24, 50]), (2, 1, 256, 16, [40], [30])])
def test_attention(kv, dtype, hq, hk, d, bs, past, new):
    for causal in (True, False):
        _attend_case(kv, dtype, hq, hk, d, bs, past, new, causal, padded=(len(past) % 2 == 0), seed=hq + d)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("hq,hk,past,new", [(4, 1, [5000, 3, 700, 1], [1, 1, 1, 1]), (7, 1, [4000], [2]), (2, 2, [1500], [20]),
                                              (1, 1, [3000], [40]), (5, 1, [2600, 0], [60, 90])])
def test_attention_of_cut_sequences(dtype, hq, hk, past, new):
    _attend_case("e4m3", dtype, hq, hk, 64, 16, past, new, True, padded=False, seed=3)


def test_attention_of_many_pieces_gives_the_same_bits_every_time():
    """Sequences of very different sizes on few CTAs: each runs through pieces with one and with two tiles of rows, whole and
    cut, whose roles hand over to each other in every order that timing allows."""
    past, new = [0, 500, 3, 700, 5, 3, 900], [130, 1, 66, 40, 1, 300, 1]
    lens, off = [p + n for p, n in zip(past, new)], _offsets(new)
    c, g = Cache("e4m3", 2, 16, 80, sum(-(-n // 16) for n in lens) + 2, 12), gen(13)
    table = i32(_tables(lens, 16, 70, c.blocks, np.random.default_rng(0)))
    q = torch.randn((off[-1], 4, 80), generator=g).to(torch.bfloat16).cuda()
    args = (q, i32(lens), i32(off), table, *c.arrays, 0.05)
    ws = vs.vscan_kv_attention_workspace(q, table, c.dev[0], 300)
    first = vs.vscan_kv_attention(*args, max_q_len=300, workspace=ws).clone()
    for _ in range(60):
        assert torch.equal(vs.vscan_kv_attention(*args, max_q_len=300, workspace=ws), first)
        assert vs.vscan_check(ws) == 0


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_attention_rows_that_see_nothing(dtype):
    # no keys at all; more new rows than tokens: the first rows stand before every key
    _attend_case("e4m3", dtype, 4, 2, 64, 16, [0, -3, -30, 0], [0, 5, 40, 2], True, padded=True, seed=5)
    _attend_case("i8", dtype, 4, 2, 64, 16, [-1, -40], [1, 40], True, padded=False, seed=6)
    _attend_case("i8", dtype, 4, 2, 64, 16, [-1, -40, 9], [1, 40, 1], False, padded=False, seed=7)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("new", [[1, 1], [30, 2]])
def test_attention_missing_blocks_are_not_there(dtype, new):
    _attend_case("e4m3", dtype, 4, 2, 64, 16, [100, 50], new, True, padded=False, seed=8, missing=[(0, 0), (0, 3), (1, 1), (1, 3)])
    _attend_case("e4m3", dtype, 4, 2, 64, 16, [10, 50], [1, 1], True, padded=False, seed=9, missing=[(0, 0)])      # all of a sequence


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_attention_max_q_len_larger_and_smaller_than_the_rows(dtype):
    _attend_case("i8", dtype, 2, 1, 64, 16, [10, 40], [2, 3], True, padded=True, seed=10, max_q=100)
    g = gen(4)
    c = Cache("i8", 1, 16, 32, 4, 3)
    q = torch.randn((5, 1, 32), generator=g).to(DT[dtype]).cuda()
    full, part = torch.full_like(q, 7.0), torch.full_like(q, 7.0)
    args = (q, i32([20]), i32([0, 5]), i32([[2, 1]]), *c.arrays, 0.2)
    vs.vscan_kv_attention(*args, max_q_len=5, out=full)
    vs.vscan_kv_attention(*args, max_q_len=3, out=part)
    assert torch.equal(full[:3], part[:3]) and (part[3:] == 7).all()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_attention_one_loud_key_among_many_quiet_ones(dtype):
    """A key with weight 1 and 4000 of weight e^-11 each: the quiet ones carry 6 % of the sum and must not be rounded away."""
    T, d = 4001, 64
    blocks = -(-T // 16)
    k, v = np.zeros((T, 1, d)), np.zeros((T, 1, d))
    k[0, 0, 0], v[0, 0, :32], v[1:, 0, 32:] = 11.0, 1.0, 1.0
    c = Cache("e4m3", 1, 16, d, blocks, 1)
    x = [torch.from_numpy(t).float() for t in (k, v)]
    table = [list(range(blocks))]
    vs.vscan_kv_write(x[0].cuda(), x[1].cuda(), i32([T]), i32([0, T]), i32(table), *c.arrays)
    q = torch.zeros((1, 1, d), dtype=DT[dtype])
    q[..., 0] = 1.0
    out = vs.vscan_kv_attention(q.cuda(), i32([T]), i32([0, 1]), i32(table), *c.arrays, 1.0)[0, 0].double().cpu().numpy()
    quiet = (T - 1) * np.exp(-11.0) / (1 + (T - 1) * np.exp(-11.0))
    tol = 2.0 ** -11 + h(dtype) + 2.0 ** -13 if dtype == "bf16" else (T / 4 + 100) * 2.0 ** -24
    np.testing.assert_allclose(out[:32], 1 - quiet, rtol=tol)
    np.testing.assert_allclose(out[32:], quiet, rtol=tol)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("q_gain", [1e-4, 300.0])
def test_attention_value_scales_far_apart(dtype, q_gain):
    """Values of neighbouring blocks 30 binades apart, scores flat or peaked."""
    H, bs, d, T = 2, 16, 64, 150
    c, g = Cache("i8", H, bs, d, 10, 2), gen(6)
    k = torch.randn((T, H, d), generator=g)
    v = torch.randn((T, H, d), generator=g) * torch.exp2(15.0 * torch.tensor([(t // bs) % 3 - 1 for t in range(T)]).float())[:, None, None]
    table = [list(range(10))]
    vs.vscan_kv_write(k.cuda(), v.cuda(), i32([T]), i32([0, T]), i32(table), *c.arrays)
    c.write([k], [v], [T], table)
    q = (q_gain * torch.randn((1, H, d), generator=g)).to(DT[dtype])
    out = vs.vscan_kv_attention(q.cuda(), i32([T]), i32([0, 1]), i32(table), *c.arrays, 0.125).double().cpu().numpy()
    (kk, there), (vv, _) = (co.gather(c.codes[i], c.scale[i], table[0], T, bs, co.I8) for i in range(2))
    ref, _, weight, reach = co.attention(q.double().numpy(), kk, vv, there, 0.125, True, T - 1)
    assert (np.abs(out - ref) <= attend_tol(dtype, d, T, ref, weight, reach, vv)).all()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_attention_nan_blocks_reach_only_who_sees_them(dtype):
    H, bs, d = 1, 16, 32
    c = Cache("e4m3", H, bs, d, 4, 4)
    x = torch.randn((40, H, d), generator=gen(7))
    x[20] = float("nan")                                         # in the second block
    table = i32([[0, 1, 2]])
    vs.vscan_kv_write(x.cuda(), x.cuda(), i32([40]), i32([0, 40]), table, *c.arrays)
    q = torch.randn((40, 2, d), generator=gen(9)).to(DT[dtype]).cuda()
    out = vs.vscan_kv_attention(q, i32([40]), i32([0, 40]), table, *c.arrays, 0.2, max_q_len=40)
    assert torch.isfinite(out[:16]).all() and torch.isnan(out[16:]).all()


# --------------------------------------------------------------------------- the run of a decode step
@pytest.mark.parametrize("kv", ["e4m3", "i8"])
def test_prune_then_decode_from_the_cache(kv):
    """Stage 2 keeps survivors, the cache takes them, decode steps (eager, then one captured graph replayed) turn, plan, write
    and attend; checked against the oracle's cache step by step."""
    from synth import CONFIGS, stage2_inputs
    cfg = CONFIGS[2].with_(name="cache_run", B=3, C=1, k2=32, Hq=8, Hkv=4, d=64, Dh=256, pos_planes=3)
    d2 = stage2_inputs(cfg, 0, cfg.B)
    red = vs.VScanReducer.from_config(cfg)
    dev = lambda a: torch.from_numpy(np.ascontiguousarray(a)).cuda()  # noqa: E731
    bf = lambda a: dev(a).to(torch.bfloat16)  # noqa: E731
    red.stage2(bf(d2["q_last"]), bf(d2["k"]), bf(d2["v"]), bf(d2["hidden"]), dev(d2["pos_ids"]))
    bs, blocks = 16, 40
    cache = vs.VScanCache(num_blocks=blocks, block_size=bs, kv_heads=cfg.Hkv, head_dim=cfg.d, batch=cfg.B, max_blocks=14, rows=cfg.B * red.S_out, kv_dtype=kv)
    red.cache_survivors(cache)
    kind = KV[kv][0]
    codes = [np.zeros((blocks, cfg.Hkv, bs, cfg.d), np.uint8) for _ in range(2)]
    scale = [np.zeros((blocks, cfg.Hkv)) for _ in range(2)]
    lens = [red.S_out] * cfg.B

    def follow(ks, vv):
        table = cache.block_table.tolist()
        for i, r in enumerate((ks, vv)):
            co.write(codes[i], scale[i], [t.transpose(0, 1).double().cpu().numpy() for t in r], lens, table, bs, kind)
        used = sorted({b for row, n in zip(table, lens) for b in row[:-(-n // bs)]})
        for t, s, c, cs in zip(cache.arrays[:2], cache.arrays[2:], codes, scale):
            np.testing.assert_array_equal(s.double().cpu().numpy()[used], cs[used])
            for row, n in zip(table, lens):
                for j, b in enumerate(row[:-(-n // bs)]):
                    np.testing.assert_array_equal(t.view(torch.uint8).cpu().numpy()[b, :, :n - j * bs], c[b, :, :n - j * bs])
        return table

    follow(red.out2["k"], red.out2["v"])
    rope = vs.rope_table(cfg.d, [8, 12, 12])
    g = gen(11)
    q = torch.empty((cfg.B, cfg.Hq, 1, cfg.d), dtype=torch.bfloat16, device="cuda")
    k, v = (torch.empty((cfg.B, cfg.Hkv, 1, cfg.d), dtype=torch.bfloat16, device="cuda") for _ in range(2))
    pos, one, out = torch.empty((3, cfg.B, 1), dtype=torch.int32, device="cuda"), i32([1] * cfg.B), torch.zeros_like(q)
    sm = cfg.d ** -0.5
    graph = None
    for step in range(7):
        for t in (q, k, v):
            t.copy_(torch.randn(t.shape, generator=g) * (1 + step))
        pos.fill_(4000 + step)
        if step == 3:
            graph = torch.cuda.CUDAGraph()
            with torch.cuda.graph(graph):
                cache.step(q, k, v, pos, rope, one, sm, out=out)
        if graph is not None:
            graph.replay()
        else:
            cache.step(q, k, v, pos, rope, one, sm, out=out)
        assert cache.check() == (0, 0)
        lens = [n + 1 for n in lens]
        assert cache.kv_len.tolist() == lens and cache.row_pos.tolist()[:cfg.B] == [n - 1 for n in lens]
        kr = vs.vscan_rope(None, k, pos, *rope)[1]
        _rope_check(k, kr, pos, *rope, co.HALVES, False, "bf16")
        table = follow(kr, v)
        qr = vs.vscan_rope(q, None, pos, *rope)[0]
        for b in range(cfg.B):
            (kk, there), (vv, _) = (co.gather(codes[i], scale[i], table[b], lens[b], bs, kind) for i in range(2))
            ref, _, weight, reach = co.attention(qr[b].transpose(0, 1).double().cpu().numpy(), kk, vv, there, sm, True, lens[b] - 1)
            tol = attend_tol("bf16", cfg.d, lens[b], ref, weight, reach, vv)
            assert (np.abs(out[b].transpose(0, 1).double().cpu().numpy() - ref) <= tol).all()
    # two sequences end, their blocks come back; a step that does not fit leaves everything as it was
    cache.plan(i32([-lens[0], 0, -lens[2]]))
    assert cache.kv_len.tolist() == [0, lens[1], 0] and cache.report.tolist()[0] == 0 and cache.report.tolist()[2] == 2 * -(-lens[0] // bs)
    cache.plan(i32([10 ** 6, 1, 1]))
    assert cache.report.tolist()[0] & 2 and cache.kv_len.tolist() == [0, lens[1], 0]


def test_two_streams_and_two_graphs_with_workspaces_of_their_own():
    c = Cache("e4m3", 2, 16, 64, 70, 5)
    T = 1000
    table, lens, off = i32([list(range(63))]), i32([T]), i32([0, 1])
    qs = [torch.randn((1, 4, 64), generator=gen(s)).to(torch.bfloat16).cuda() for s in range(2)]
    want = [vs.vscan_kv_attention(q, lens, off, table, *c.arrays, 0.1) for q in qs]
    outs = [torch.zeros_like(q) for q in qs]
    spaces = [vs.vscan_kv_attention_workspace(q, table, c.dev[0], 1) for q in qs]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in qs]
    for _ in range(20):
        for q, o, w, st in zip(qs, outs, spaces, streams):
            with torch.cuda.stream(st):
                vs.vscan_kv_attention(q, lens, off, table, *c.arrays, 0.1, out=o, workspace=w)
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(want, outs))
    graphs = []
    for q, o, w in zip(qs, outs, spaces):
        o.zero_()
        graphs.append(torch.cuda.CUDAGraph())
        with torch.cuda.graph(graphs[-1]):
            vs.vscan_kv_attention(q, lens, off, table, *c.arrays, 0.1, out=o, workspace=w)
    for gr, st in zip(graphs, streams):
        st.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(st):
            gr.replay()
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(want, outs))


@pytest.mark.parametrize("dtype,n", [("bf16", 1), ("bf16", 70), ("f32", 3)])
def test_attention_captured_and_replayed_as_lengths_change(dtype, n):
    """One graph, its lengths read from the GPU at each replay: short, long, none; the same bits as eager calls."""
    H, bs, d, cols = 2, 32, 64, 40
    c, g = Cache("i8", H, bs, d, 90, 7), gen(21)
    table = i32([[int(v) for v in np.random.default_rng(1).permutation(80)[:cols]], list(range(40, 80))])
    lens, off = i32([0, 0]), i32([0, 0, 0])
    q = torch.randn((2 * n, 4, d), generator=g).to(DT[dtype]).cuda()
    out, lse = torch.zeros_like(q), torch.zeros((2 * n, 4), device="cuda")
    ws = vs.vscan_kv_attention_workspace(q, table, c.dev[0], n)
    args = (q, lens, off, table, *c.arrays, 0.1)
    vs.vscan_kv_attention(*args, max_q_len=n, out=out, lse=lse, workspace=ws)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        vs.vscan_kv_attention(*args, max_q_len=n, out=out, lse=lse, workspace=ws)
    for a, b, ra, rb in [(1000, 77, n, n), (n, 1280, n, 1), (0, 5, 0, 1), (1279, 0, n, 0), (640, 641, 1, n)]:
        lens.copy_(i32([a, b]))
        off.copy_(i32([0, ra, ra + rb]))
        out.fill_(7.0)
        lse.fill_(7.0)
        graph.replay()
        got = out.clone(), lse.clone()
        out.fill_(7.0)
        lse.fill_(7.0)
        vs.vscan_kv_attention(*args, max_q_len=n, out=out, lse=lse)
        assert torch.equal(got[0], out) and torch.equal(got[1], lse) and vs.vscan_check(ws) == 0
        out.fill_(-9.0)                      # every row that is owned is written, no other is
        vs.vscan_kv_attention(*args, max_q_len=n, out=out)
        assert torch.equal(out[:ra + rb], got[0][:ra + rb]) and (got[0][ra + rb:] == 7).all() and (out[ra + rb:] == -9).all()


@pytest.mark.parametrize("dtype,n", [("bf16", 1), ("bf16", 40), ("f32", 2)])
def test_offsets_beyond_32_bits(dtype, n):
    """A pool of more than 2^32 codes, its tokens in the last blocks: the same bits as from a small pool."""
    B, hq, hk, bs, d = 2, 8, 4, 128, 128
    lens, big = [300, 150 + n], (1 << 32) // (hk * bs * d) + 100
    g = gen(5)
    k, v = (torch.randn((sum(lens), hk, d), generator=g).to(DT[dtype]).cuda() for _ in range(2))
    q = torch.randn((B * n, hq, d), generator=g).to(DT[dtype]).cuda()
    outs = []
    for blocks in (8, big):
        pools = [torch.empty((blocks, hk, bs, d), dtype=torch.uint8, device="cuda").view(torch.float8_e4m3fn) for _ in range(2)]
        scales = [torch.empty((blocks, hk), device="cuda") for _ in range(2)]
        table = i32([[blocks - 1, blocks - 4, blocks - 2], [blocks - 5, blocks - 3, -1]])
        vs.vscan_kv_write(k, v, i32(lens), i32([0, lens[0], sum(lens)]), table, *pools, *scales)
        out = vs.vscan_kv_attention(q, i32(lens), i32([0, n, 2 * n]), table, *pools, *scales, d ** -0.5, max_q_len=n)
        outs.append((out, pools[0][blocks - 5:].view(torch.uint8).clone(), scales[1][blocks - 5:].clone()))
        del pools
    assert torch.equal(outs[0][0], outs[1][0]) and outs[0][0].abs().max() > 0
    first, second = ({j: t[1][j] for j in range(5)} for t in outs)
    assert all(torch.equal(first[j][:, :20], second[j][:, :20]) for j in range(5))
    assert torch.equal(outs[0][2], outs[1][2])


def test_python_face_refusals():
    c = Cache("e4m3", 2, 16, 32, 4, 0)
    q, lens, off, table = torch.zeros((1, 2, 32), device="cuda"), i32([1]), i32([0, 1]), i32([[0]])
    with pytest.raises(ValueError):
        vs.vscan_kv_attention(q[:, :, :16], lens, off, table, *c.arrays, 1.0)
    with pytest.raises(ValueError):
        vs.vscan_kv_attention(q, lens, off[:1], table, *c.arrays, 1.0)
    with pytest.raises(TypeError):
        vs.vscan_kv_attention(q, lens.long(), off, table, *c.arrays, 1.0)
    with pytest.raises(TypeError):
        vs.vscan_kv_write(q.half(), q.half(), lens, off, table, *c.arrays)
    with pytest.raises(ValueError):
        vs.vscan_kv_write(q, q.cpu(), lens, off, table, *c.arrays)
    with pytest.raises(ValueError):
        vs.vscan_kv_write(q[:, :1], q[:, :1], lens, off, table, *c.arrays)
    with pytest.raises(vs.VScanError):
        vs.vscan_kv_attention(q, lens, off, table, *c.arrays, 1.0, workspace=vs.Workspace(256))
    with pytest.raises(ValueError):
        vs.vscan_kv_attention(q, lens, off, table, *c.arrays, 1.0, lse=torch.zeros(3, device="cuda"))
