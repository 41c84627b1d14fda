"""What VScanCache does on the host, on CPU tensors, the library's calls replaced; outputs of vscan_rope on top of each other or of the
other side's input; how many CTAs an attention call plans for; the row limit of a plan; which
stream a status is waited for on.  No GPU."""
import ctypes as C

import pytest
import torch

from paper_2505_22654_b200 import _build
from paper_2505_22654_b200 import binding as vb
from paper_2505_22654_b200.cache import VScanCache


def _cache(**kw):
    return VScanCache(**{**dict(num_blocks=8, block_size=16, kv_heads=2, head_dim=32, batch=2, max_blocks=4, rows=64, device="cpu"), **kw})


@pytest.fixture
def attention(monkeypatch):
    """vscan_kv_attention in which `rows` query rows need 1000 + rows * max_q_len bytes; -> the calls that went through."""
    calls, need = [], lambda q, most: 1000 + q.shape[0] * most

    def run(q, kv_len, row_offset, block_table, k, v, k_scale, v_scale, scale, max_q_len=1, causal=True, out=None, lse=None, workspace=None):
        if workspace.nbytes < need(q, max_q_len):
            raise vb.VScanError(vb.ERR_WORKSPACE, "vscan_kv_attention")
        calls.append((q.shape[0], workspace))
        return out

    monkeypatch.setattr(vb, "vscan_kv_attention", run)
    monkeypatch.setattr(vb, "vscan_kv_attention_workspace", lambda q, table, k, most: vb.Workspace(need(q, most), "cpu"))
    monkeypatch.setattr(vb, "vscan_check", lambda w: int(w.buf[:4].view(torch.int32)))
    return calls


def test_one_workspace_whatever_the_row_counts_are(attention):
    c = _cache()
    for rows in [*range(1, 400), *range(400, 0, -1)]:
        c.attend(torch.zeros((rows, 4, 32)), 1.0, max_q_len=1 + rows % 50)
    held = {id(w): w for _, w in attention}.values()
    assert len(attention) == 799 and len(held) <= 6
    assert sum(w.nbytes for w in held) < 4 * (1000 + 400 * 50)


def test_status_is_that_of_the_last_call_and_of_graphs_on_outgrown_workspaces(attention):
    c = _cache()
    assert c.check() == (0, 0)
    c.attend(torch.zeros((1, 4, 32)), 1.0)
    small = attention[-1][1]
    small.buf[:4].view(torch.int32)[0] = vb.ERR_INVALID_ARG        # what a call with a bad table leaves
    assert c.check() == (vb.ERR_INVALID_ARG, 0)
    c.attend(torch.zeros((500, 4, 32)), 1.0, max_q_len=40)         # a good one, on a larger workspace
    attention[-1][1].buf[:4].zero_()
    assert attention[-1][1] is not small and c.check() == (0, 0)
    small.buf[:4].view(torch.int32)[0] = vb.ERR_TIMEOUT            # a replay of a graph that holds the small one
    assert c.check() == (vb.ERR_TIMEOUT, 0)


def test_other_errors_of_the_attention_are_passed_on(attention, monkeypatch):
    def refuse(*args, **kw):
        raise vb.VScanError(vb.ERR_UNSUPPORTED, "vscan_kv_attention")
    monkeypatch.setattr(vb, "vscan_kv_attention", refuse)
    c = _cache()
    with pytest.raises(vb.VScanError) as e:
        c.attend(torch.zeros((1, 4, 32)), 1.0)
    assert e.value.status == vb.ERR_UNSUPPORTED and c.check() == (0, 0)


# --------------------------------------------------------------------------- vscan_rope
BASE, B, S, D = 1 << 40, 2, 5, 64       # host-side checks never read these addresses
FAR = 1 << 34


def _rope(hq, hk, **sides):
    """Status of a bf16 call whose sides are (address in elements of 2 bytes, strides); any that is not given is far from the rest."""
    _build.build()
    d = vb.RopeDesc(vb.BF16, 0, 0, B, S, hq, hk, D, 32, 3)
    for i, name in enumerate(("pos_ids", "inv_freq", "axis")):
        setattr(d, name, BASE + (20 + i) * FAR)
    for i, (name, heads) in enumerate((("q", hq), ("q_out", hq), ("k", hk), ("k_out", hk))):
        at, strides = sides.get(name, ((4 + i) * FAR, (heads * S * D, S * D, D)))
        setattr(d, name, BASE + 2 * at)
        setattr(d, name + "_stride", vb._i64x3(*strides))
    return vb.lib().vscan_rope(C.byref(d), None)


PLAIN = (4 * S * D, S * D, D)             # [B, 4, S, D]
FUSED = (S * 8 * D, D, 8 * D)             # four heads of [B, S, 8, D]


@pytest.mark.parametrize("sides", [
    dict(q_out=(0, PLAIN), k_out=(0, PLAIN)), dict(q_out=(0, PLAIN), k_out=(8, PLAIN)), dict(q_out=(0, PLAIN), k_out=(S * D, PLAIN)),
    dict(q=(0, PLAIN), q_out=(FAR, PLAIN), k=(FAR, PLAIN), k_out=(0, PLAIN)),                      # each into the other
    dict(k=(0, PLAIN), q_out=(0, PLAIN)), dict(q=(0, PLAIN), k_out=(0, PLAIN)),
    dict(q=(0, PLAIN), q_out=(0, PLAIN), k=(0, PLAIN)),                                            # in place, but the keys read it too
    dict(q_out=(0, FUSED), k_out=(3 * D, FUSED)), dict(q_out=(0, FUSED), k_out=(4 * D + 8, FUSED)), dict(q_out=(0, FUSED), k_out=(5 * D, FUSED)),
    dict(q_out=(0, FUSED), k_out=(8 * D, FUSED)),                                                  # one token on
    dict(q_out=(0, FUSED), k_out=(4 * D, PLAIN)), dict(q_out=(0, FUSED), k_out=(4 * D, (S * 8 * D, D, 4 * D)))])
def test_rope_outputs_on_each_other_or_on_the_other_input_are_refused(sides):
    assert _rope(4, 4, **sides) == vb.ERR_INVALID_ARG


# --------------------------------------------------------------------------- vscan_kv_attention
@pytest.mark.parametrize("max_q_len,rows,per_sm", [(1, 4, 4), (50, 8, 2)])
def test_float32_attention_plans_for_the_ctas_that_fit_at_once(max_q_len, rows, per_sm):
    """The workspace has room for two partial results a CTA, and no launch has more CTAs than the registers of 148 SMs hold: 128
    registers a thread for tiles of 4 rows, up to 254 for tiles of 8."""
    _build.build()
    d = vb.KvAttentionDesc(vb.F32, vb.KV_E4M3, 40, 8, 2, 64, 16, 10000, 200, 2000, 0, max_q_len, 1, 0.125)
    up = lambda n: -(-n // 256) * 256  # noqa: E731
    ctas = 148 * per_sm
    want = 256 + up(4 * ctas) + up(48 * ctas) + up(2 * ctas * rows * (64 + 2) * 4)
    assert vb.lib().vscan_kv_attention_workspace_bytes(C.byref(d)) == want


# --------------------------------------------------------------------------- vscan_kv_plan
@pytest.mark.parametrize("rows,slots,places,limit", [(None, 40, None, 40), (None, 40, 30, 30), (25, 40, 30, 25), (50, 40, 50, 40), (25, None, None, 25),
                                                     (None, None, None, 2 ** 31 - 1)])
def test_plan_keeps_to_the_least_of_its_row_limits(monkeypatch, rows, slots, places, limit):
    given = []

    class Calls:
        @staticmethod
        def kv_plan(*args):
            given.append(args)
            return vb.OK

    monkeypatch.setattr(vb, "_CALLS", Calls)
    i32 = lambda *n: torch.zeros(n, dtype=torch.int32)  # noqa: E731
    out = {name: t for name, t in (("slot_map", slots and torch.zeros(slots, dtype=torch.int64)), ("row_pos", places and i32(places))) if t is not None}
    o = vb.vscan_kv_plan(i32(2), i32(2), i32(2, 4), i32(9), torch.zeros(2, dtype=torch.int64), 16, rows=rows, out=out)
    assert given[0][6] == limit
    for name, size in (("slot_map", slots), ("row_pos", places)):
        assert (o[name] is None) if (rows, slots, places) == (None, None, None) else o[name].shape[0] == (size or limit)


# --------------------------------------------------------------------------- vscan_check
def test_check_waits_for_the_stream_of_the_workspaces_device(monkeypatch):
    """Calls on tensors of another device than the current one run on that device's stream."""
    from types import SimpleNamespace
    asked = []
    monkeypatch.setattr(torch.cuda, "current_stream", lambda device=None: SimpleNamespace(cuda_stream={None: 11, torch.device("cuda", 1): 22}[device]))
    monkeypatch.setattr(vb, "lib", lambda: SimpleNamespace(vscan_check=lambda ptr, stream: asked.append((ptr, stream)) or vb.OK))
    buf = SimpleNamespace(device=torch.device("cuda", 1), data_ptr=lambda: 4096)
    work = vb.Workspace.__new__(vb.Workspace)
    work.buf = buf
    assert vb.vscan_check(work) == vb.OK and asked == [(4096, 22)]
