"""Pins of the cache oracle, and the host side of vscan_rope and the vscan_kv_* calls: refusals before anything is launched,
struct layout, the frequency tables.  No GPU."""
import ctypes as C
import os
import subprocess
import tempfile

import numpy as np
import pytest
import torch

from oracle import cache_oracle as co
from paper_2505_22654_b200 import _build
from paper_2505_22654_b200 import binding as vb

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


# --------------------------------------------------------------------------- oracle pins
def test_e4m3_codes_are_those_of_the_format():
    v = co.code_values(co.E4M3)
    ref = torch.arange(256, dtype=torch.uint8).view(torch.float8_e4m3fn).double().numpy()
    np.testing.assert_array_equal(v, ref)
    x = np.concatenate([np.random.default_rng(0).normal(size=4000) * 50, v[np.isfinite(v)], (v[:126] + v[1:127]) / 2])
    got = co.encode(x, co.E4M3)
    ref = torch.from_numpy(x).clamp(-448, 448).float().to(torch.float8_e4m3fn).view(torch.uint8).numpy()
    np.testing.assert_array_equal(got, ref)


def test_i8_codes_round_to_even_and_saturate():
    x = np.array([0.5, 1.5, 2.5, -0.5, -1.5, 126.5, 127.4, 500.0, -500.0, np.nan])
    np.testing.assert_array_equal(co.encode(x, co.I8).view(np.int8), [0, 2, 2, 0, -2, 126, 127, 127, -127, 0])


@pytest.mark.parametrize("kind", [co.E4M3, co.I8])
def test_least_scale_is_the_least(kind):
    top = co.Q_MAX[kind]
    for amax in (1.0, top, np.nextafter(top, np.inf), 0.875, 0.0, 1e30, 1e-30):
        s = co.least_scale(amax, kind)
        assert amax <= top * s or s == 2.0 ** co.E_MAX
        assert s == 2.0 ** co.E_MIN or amax > top * s / 2


def test_write_keeps_a_block_in_step_with_its_largest_token():
    codes, scale = np.zeros((2, 1, 16, 16), np.uint8), np.ones((2, 1))
    rng = np.random.default_rng(1)
    x = rng.normal(size=(3, 1, 16))
    x[2] *= 100
    for t in range(3):      # one token at a time, the last one much larger
        co.write(codes, scale, [x[t:t + 1]], [t + 1], [[1]], 16, co.E4M3)
    at_once, s2 = np.zeros_like(codes), np.ones_like(scale)
    co.write(at_once, s2, [x], [3], [[1]], 16, co.E4M3)
    assert scale[1, 0] == s2[1, 0]
    a, b = co.code_values(co.E4M3)[codes[1, 0, :3]] * scale[1, 0], co.code_values(co.E4M3)[at_once[1, 0, :3]] * s2[1, 0]
    np.testing.assert_allclose(a, b, atol=2.0 ** -10 * s2[1, 0])       # half the smallest step: codes below the normal range
    np.testing.assert_allclose(b, x[:, 0], rtol=2.0 ** -4, atol=2.0 ** -10 * s2[1, 0])


def test_rope_turns_by_the_position_difference():
    rng = np.random.default_rng(2)
    q, k = rng.normal(size=(1, 1, 8)), rng.normal(size=(1, 1, 8))
    freq, axis = np.array([1.0, 0.3, 0.7, 0.01]), [0, 1, 1, 2]
    for pairing in (co.HALVES, co.ADJACENT):
        dots = []
        for shift in (0, 5):
            a = co.rope(q, np.array([[3 + shift], [7 + shift], [1 + shift]]), freq, axis, pairing)
            b = co.rope(k, np.array([[1 + shift], [9 + shift], [4 + shift]]), freq, axis, pairing)
            dots.append(float((a * b).sum()))
        assert abs(dots[0] - dots[1]) < 1e-12
        back = co.rope(co.rope(q, np.array([[3], [7], [1]]), freq, axis, pairing), np.array([[3], [7], [1]]), freq, axis, pairing, True)
        np.testing.assert_allclose(back, q, atol=1e-14)


def test_plan_conserves_blocks():
    rng = np.random.default_rng(3)
    bs, cols, n = 16, 6, 40
    table, ring, state = [[-1] * cols for _ in range(5)], list(rng.permutation(n)), [7, 7 + n]
    past = [0] * 5
    for step in range(30):
        new = [int(rng.integers(-p, min(40, cols * bs - p) + 1)) for p in past]
        o = co.plan(past, new, table, ring, state, bs, 10 ** 6)
        if o["report"][0]:
            assert o["kv_len"] == past and o["state"] == state and o["table"] == table
            continue
        table, ring, state, past = o["table"], o["ring"], o["state"], o["kv_len"]
        held = [b for r, p in zip(table, past) for b in r[:-(-p // bs)]]
        free = [ring[i % n] for i in range(state[0], state[1])]
        assert sorted(held + free) == list(range(n))


def test_attention_of_one_key_is_its_value():
    q, k, v = np.ones((2, 2, 4)), np.ones((1, 1, 4)), np.arange(4.0).reshape(1, 1, 4)
    out, lse, _, _ = co.attention(q, k, v, np.array([True]), 0.5, True, -1)
    assert (out[0] == 0).all() and (lse[0] == -np.inf).all()           # the first row stands before every key
    np.testing.assert_array_equal(out[1], np.stack([v[0, 0]] * 2))
    np.testing.assert_allclose(lse[1], 2.0)


# --------------------------------------------------------------------------- host side
@pytest.fixture(scope="module")
def L():
    _build.build()
    return vb.lib()


def test_struct_layout_of_the_new_descriptors():
    fields = {"rope": vb.RopeDesc, "kv_plan": vb.KvPlanDesc, "kv_write": vb.KvWriteDesc, "kv_attention": vb.KvAttentionDesc}
    prog = '#include <stdio.h>\n#include <stddef.h>\n#include "vscan.h"\nint main(void) {\n'
    want = []
    for name, cls in fields.items():
        prog += f'printf("%zu\\n", sizeof(vscan_{name}_desc));\n'
        want.append(C.sizeof(cls))
        for f, _ in cls._fields_:
            prog += f'printf("%zu\\n", offsetof(vscan_{name}_desc, {f}));\n'
            want.append(getattr(cls, f).offset)
    prog += "return 0; }\n"
    with tempfile.TemporaryDirectory() as tmp:
        src, exe = os.path.join(tmp, "a.c"), os.path.join(tmp, "a")
        with open(src, "w") as f:
            f.write(prog)
        subprocess.run(["gcc", "-I", os.path.join(ROOT, "include"), src, "-o", exe], check=True)
        got = subprocess.run([exe], capture_output=True, text=True, check=True).stdout.split()
    assert [int(v) for v in got] == want


BASE = 1 << 40          # host-side checks never read these addresses


def _fill(desc, pointers, spread=1 << 34):
    for i, name in enumerate(pointers):
        setattr(desc, name, BASE + i * spread)
    return desc


def _rope_desc(**kw):
    d = _fill(vb.RopeDesc(vb.BF16, 0, 0, 2, 5, 4, 2, 64, 32, 3), ["pos_ids", "inv_freq", "axis", "q", "q_out", "k", "k_out"])
    for s, heads in (("q_stride", 4), ("q_out_stride", 4), ("k_stride", 2), ("k_out_stride", 2)):
        setattr(d, s, vb._i64x3(heads * 5 * 64, 5 * 64, 64))
    for k, v in kw.items():
        setattr(d, k, v)
    return d


@pytest.mark.parametrize("change,status", [
    (dict(dtype=7), 1), (dict(pairing=2), 1), (dict(head_dim=60), 1), (dict(rot_dim=31), 1), (dict(rot_dim=66), 1), (dict(rot_dim=0), 1),
    (dict(pos_planes=0), 1), (dict(pos_planes=17), 2), (dict(head_dim=520), 2), (dict(q_heads=0), 1), (dict(batch=-1), 1),
    (dict(q_out=None), 1), (dict(q=None), 1), (dict(q=None, q_out=None, k=None, k_out=None), 1), (dict(pos_ids=None), 1), (dict(axis=None), 1),
    (dict(q=BASE + 8), 1), (dict(q_stride=vb._i64x3(1280, 320, 68)), 1),
    (dict(q_out_stride=vb._i64x3(1280, 320, 0)), 1),                                     # rows of the output on top of each other
    (dict(q_out_stride=vb._i64x3(640, 320, 64)), 1),                                     # sequences of the output overlap
    (dict(q_out=BASE + 3 * (1 << 34) + 16), 1),                                          # shifted onto its input
    (dict(q_out=BASE + 3 * (1 << 34), q_out_stride=vb._i64x3(1280, 64, 256)), 1),        # in place, but by other strides
    (dict(k_out=BASE), 1),                                                               # on top of the positions
    (dict(batch=0), 0), (dict(seq_len=0), 0),
])
def test_rope_refusals(L, change, status):
    assert L.vscan_rope(C.byref(_rope_desc(**change)), None) == status


def _plan_desc(**kw):
    d = _fill(vb.KvPlanDesc(4, 16, 100, 8, 50), ["past_len", "new_len", "block_table", "free_ring", "ring_state", "kv_len", "row_offset",
                                                 "slot_map", "row_pos", "ring_state_out", "report"])
    for k, v in kw.items():
        setattr(d, k, v)
    return d


@pytest.mark.parametrize("change,status", [
    (dict(block_size=24), 1), (dict(block_size=8), 1), (dict(batch=-1), 1), (dict(rows=-1), 1), (dict(past_len=None), 1), (dict(kv_len=None), 1),
    (dict(ring_state=None), 1), (dict(report=None), 1), (dict(block_table=None), 1), (dict(free_ring=None), 1), (dict(kv_len=BASE), 1),
    (dict(ring_state_out=BASE + 4 * (1 << 34)), 1), (dict(slot_map=BASE + 4), 1), (dict(batch=8193), 2), (dict(max_blocks=1 << 27), 2)])
def test_plan_refusals(L, change, status):
    assert L.vscan_kv_plan(C.byref(_plan_desc(**change)), None) == status


def _write_desc(**kw):
    d = vb.KvWriteDesc(vb.BF16, vb.KV_E4M3, 4, 2, 64, 16, 100, 8, 50, 0)
    _fill(d, ["k", "v", "kv_len", "row_offset", "block_table", "k_cache", "v_cache", "k_scale", "v_scale"])
    d.k_stride = d.v_stride = vb._i64x3(0, 64, 128)
    for k, v in kw.items():
        setattr(d, k, v)
    return d


@pytest.mark.parametrize("change,status", [
    (dict(dtype=2), 1), (dict(kv_dtype=2), 1), (dict(head_dim=72), 1), (dict(head_dim=0), 1), (dict(block_size=48), 1), (dict(kv_heads=0), 1),
    (dict(k=None), 1), (dict(v_scale=None), 1), (dict(k=BASE + 2), 1), (dict(k_stride=vb._i64x3(0, 64, 129)), 1),
    (dict(k_stride=vb._i64x3(0, -64, 128)), 1), (dict(v_cache=BASE + 5 * (1 << 34)), 1), (dict(k_cache=BASE), 1),
    (dict(head_dim=272), 2), (dict(batch=8193), 2), (dict(batch=0), 0), (dict(rows=0), 0), (dict(num_blocks=0), 0)])
def test_write_refusals(L, change, status):
    assert L.vscan_kv_write(C.byref(_write_desc(**change)), None) == status


def _attend_desc(**kw):
    d = vb.KvAttentionDesc(vb.BF16, vb.KV_E4M3, 4, 8, 2, 64, 16, 100, 8, 50, 0, 1, 1, 0.125)
    _fill(d, ["q", "out", "lse", "kv_len", "row_offset", "block_table", "k_cache", "v_cache", "k_scale", "v_scale"])
    d.q_stride = d.out_stride = vb._i64x3(0, 64, 512)
    d.lse_stride = vb._i64x3(0, 1, 8)
    for k, v in kw.items():
        setattr(d, k, v)
    return d


@pytest.mark.parametrize("change,status", [
    (dict(dtype=2), 1), (dict(kv_dtype=-1), 1), (dict(head_dim=8), 1), (dict(q_heads=7), 1), (dict(block_size=0), 1), (dict(scale=float("nan")), 1),
    (dict(scale=float("inf")), 1), (dict(q=None), 1), (dict(out=None), 1), (dict(kv_len=None), 1), (dict(k_cache=None), 1), (dict(out=BASE), 1),
    (dict(lse=BASE + (1 << 34)), 1), (dict(out=BASE + (1 << 34) + 4), 1), (dict(out_stride=vb._i64x3(0, 60, 512)), 1), (dict(max_q_len=-1), 1),
    (dict(q_heads=130), 2), (dict(head_dim=512), 2), (dict(batch=10000), 2)])
def test_attention_refusals(L, change, status):
    assert L.vscan_kv_attention(C.byref(_attend_desc(**change)), BASE << 1, 1 << 30, None) == status


@pytest.mark.parametrize("change,status", [
    (dict(out_stride=vb._i64x3(0, 64, 0)), 1), (dict(out_stride=vb._i64x3(0, 0, 64)), 1), (dict(out_stride=vb._i64x3(0, 64, 448)), 1),
    (dict(lse_stride=vb._i64x3(0, 1, 0)), 1), (dict(lse_stride=vb._i64x3(0, 1, 7)), 1),
    (dict(padded=1), 1),                                                                 # sequences on top of each other
    (dict(max_blocks=(1 << 27) - 128, num_blocks=1), 2), (dict(rows=(1 << 28) - 1, batch=1), 2)])
def test_attention_outputs_do_not_overlap_themselves_and_fit_32_bits(L, change, status):
    assert L.vscan_kv_attention(C.byref(_attend_desc(**change)), BASE << 1, 1 << 30, None) == status


def test_attention_wants_its_workspace(L):
    d = _attend_desc()
    need = L.vscan_kv_attention_workspace_bytes(C.byref(d))
    assert need > 256
    assert L.vscan_kv_attention(C.byref(d), None, need, None) == vb.ERR_WORKSPACE
    assert L.vscan_kv_attention(C.byref(d), BASE << 1, need - 1, None) == vb.ERR_WORKSPACE
    assert L.vscan_kv_attention(C.byref(d), (BASE << 1) + 128, need, None) == vb.ERR_WORKSPACE
    big = _attend_desc(batch=4096, rows=1 << 20, max_q_len=1 << 20, max_blocks=1 << 20)
    assert L.vscan_kv_attention_workspace_bytes(C.byref(big)) < 256 << 20     # does not grow with the batch or the lengths


def test_rope_table_layouts():
    freq, axis = vb.rope_table(16, [2, 3, 3], base=100.0, device="cpu")
    np.testing.assert_allclose(freq.numpy(), [100.0 ** (-i / 8) for i in range(8)], rtol=1e-6)
    assert axis.tolist() == [0, 0, 1, 1, 1, 2, 2, 2]
    assert vb.rope_table(16, [2, 3, 3], layout="cycled", device="cpu")[1].tolist() == [0, 1, 2, 0, 1, 2, 1, 2]
    freq, axis = vb.rope_table(16, [4, 4], base=100.0, layout="per_axis", device="cpu")
    np.testing.assert_allclose(freq.numpy(), [100.0 ** (-j / 4) for j in range(4)] * 2, rtol=1e-6)
    with pytest.raises(ValueError):
        vb.rope_table(16, [2, 3, 4])
    with pytest.raises(ValueError):
        vb.rope_table(16, [8], layout="spiral")


def test_python_face_refuses_what_is_not_on_a_gpu():
    t = torch.zeros((1, 1, 1, 16))
    with pytest.raises(ValueError):
        vb.vscan_rope(t, None, torch.zeros((1, 1, 1), dtype=torch.int32), torch.zeros(8), torch.zeros(8, dtype=torch.int32))
    with pytest.raises(ValueError):
        vb.vscan_kv_plan(*[torch.zeros(1, dtype=torch.int32)] * 2, torch.zeros((1, 1), dtype=torch.int32), torch.zeros(1, dtype=torch.int32),
                         torch.zeros(2, dtype=torch.int64), 16)


def test_python_face_wants_a_truth_value():
    t = torch.zeros(2)
    with pytest.raises((TypeError, ValueError)):
        vb.vscan_rope(torch.zeros(1, 1, 1, 8), None, torch.zeros(1, 1, 1, dtype=torch.int32), t, t.int(), inverse=torch.zeros(2))
