"""vscan_attention, vscan_kv_weigh and vscan_kv_evict on the host, without a GPU: layouts of their descriptors, what they refuse before a launch,
workspaces; what VScanCache does around them, on CPU tensors, the library's calls replaced."""
import ctypes as C
import os
import subprocess

import pytest
import torch

from paper_2505_22654_b200 import _build
from paper_2505_22654_b200 import binding as vb
from paper_2505_22654_b200.cache import VScanCache

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
STRUCTS = {"vscan_attention_desc": vb.AttentionDesc, "vscan_kv_weigh_desc": vb.KvWeighDesc, "vscan_kv_evict_desc": vb.KvEvictDesc}


@pytest.fixture(scope="module")
def L():
    _build.build()
    return vb.lib()


def test_struct_layouts_match_the_header(tmp_path):
    lines = [f'printf("{s} %zu\\n", sizeof({s}));' for s in STRUCTS]
    lines += [f'printf("{s}.{name} %zu\\n", offsetof({s}, {name}));' for s, t in STRUCTS.items() for name, _ in t._fields_]
    src, exe = tmp_path / "layout.c", tmp_path / "layout"
    src.write_text("#include <stdio.h>\n#include <stddef.h>\n#include \"vscan.h\"\nint main(void) {\n" + "\n".join(lines) + "\nreturn 0;\n}\n")
    subprocess.run(["gcc", "-std=c99", "-I", os.path.join(ROOT, "include"), str(src), "-o", str(exe)], check=True)
    for line in subprocess.run([str(exe)], capture_output=True, text=True, check=True).stdout.strip().splitlines():
        key, value = line.rsplit(" ", 1)
        s, _, field = key.partition(".")
        assert (getattr(STRUCTS[s], field).offset if field else C.sizeof(STRUCTS[s])) == int(value), key


BASE = 1 << 40            # host-side checks never read these addresses
FAR = 1 << 34


def _fill(d, names, **kw):
    for i, n in enumerate(names):
        setattr(d, n, BASE + i * FAR)
    for k, v in kw.items():
        setattr(d, k, vb._i64x3(*v) if isinstance(v, tuple) else v)
    return d


def _attention(**kw):
    d = vb.AttentionDesc(vb.BF16, 2, 4, 2, 64, 10, 12, 0, 10, 1, 0.125)
    st = {"q_stride": (0, 64, 256), "k_stride": (0, 64, 128), "v_stride": (0, 64, 128), "out_stride": (0, 64, 256), "lse_stride": (0, 1, 4)}
    return _fill(d, ("q", "k", "v", "out", "lse", "row_offset", "kv_offset"), **{**st, **kw})


@pytest.mark.parametrize("change,status", [
    ({}, "WORKSPACE"), (dict(kv_offset=None), "WORKSPACE"), (dict(lse=None, lse_stride=(0, 0, 0)), "WORKSPACE"), (dict(scale=-1.0), "WORKSPACE"),
    (dict(kv_rows=0, k=None, v=None), "WORKSPACE"),
    (dict(dtype=2), "INVALID_ARG"), (dict(batch=-1), "INVALID_ARG"), (dict(q_heads=3), "INVALID_ARG"), (dict(kv_heads=0), "INVALID_ARG"),
    (dict(head_dim=60), "INVALID_ARG"), (dict(head_dim=0), "INVALID_ARG"), (dict(rows=-1), "INVALID_ARG"), (dict(max_q_len=-1), "INVALID_ARG"),
    (dict(scale=float("nan")), "INVALID_ARG"), (dict(scale=float("inf")), "INVALID_ARG"), (dict(q=None), "INVALID_ARG"), (dict(k=None), "INVALID_ARG"),
    (dict(row_offset=None), "INVALID_ARG"), (dict(q=BASE + 8), "INVALID_ARG"), (dict(row_offset=BASE + 5 * FAR + 4), "INVALID_ARG"),
    (dict(k_stride=(0, 64, 129)), "INVALID_ARG"), (dict(v_stride=(0, -64, 128)), "INVALID_ARG"), (dict(out_stride=(0, 64, 128)), "INVALID_ARG"),
    (dict(out_stride=(0, 0, 256)), "INVALID_ARG"), (dict(lse_stride=(0, 1, 1)), "INVALID_ARG"), (dict(out=BASE), "INVALID_ARG"),
    (dict(out=BASE + FAR + 64), "INVALID_ARG"), (dict(lse=BASE + 3 * FAR), "INVALID_ARG"), (dict(lse=BASE + 5 * FAR), "INVALID_ARG"),
    (dict(head_dim=264), "UNSUPPORTED"), (dict(q_heads=130), "UNSUPPORTED"), (dict(batch=9000), "UNSUPPORTED"),
    (dict(rows=2 ** 30), "UNSUPPORTED"), (dict(kv_rows=2 ** 31 - 1), "UNSUPPORTED"),
    (dict(batch=0), "OK?"), (dict(rows=0), "OK?"), (dict(max_q_len=0), "OK?")])
def test_attention_refusals(L, change, status):
    d = _attention(**change)
    got = L.vscan_attention(C.byref(d), None, 0, None)         # no workspace: what is legal fails there, before anything is enqueued
    assert got == (vb.ERR_WORKSPACE if status == "OK?" else getattr(vb, "ERR_" + status))
    assert L.vscan_attention_workspace_bytes(C.byref(d)) >= 256


def test_attention_workspace_covers_both_kernels(L):
    """Strides decide between the tensor-core kernel (tiles of whole tokens up to 256 rows) and the other (64 rows), sizes alone the workspace."""
    up = lambda n: -(-n // 256) * 256  # noqa: E731
    for hq, hk, d in ((28, 4, 128), (16, 16, 64), (32, 4, 80)):
        desc = _attention(q_heads=hq, kv_heads=hk, head_dim=d, rows=100000, kv_rows=100000, max_q_len=50000)
        rows, ctas = 2 * (128 // (hq // hk)) * (hq // hk), 148
        tensor = 256 + up(4 * ctas) + up(48 * ctas) + up(2 * ctas * 4 * ((rows * (d + 2) + 3) & ~3))
        flat = 256 + up(4 * 296) + up(48 * 296) + up(2 * 296 * 4 * ((64 * (d + 2) + 3) & ~3))
        assert L.vscan_attention_workspace_bytes(C.byref(desc)) == max(tensor, flat)


def _weigh(**kw):
    d = vb.KvWeighDesc(vb.BF16, vb.KV_E4M3, 2, 4, 2, 64, 16, 40, 9, 10, 0, 5, 100, 1, 0.125, 1.0)
    st = {"q_stride": (0, 64, 256), "lse_stride": (0, 1, 4)}
    return _fill(d, ("q", "lse", "kv_len", "row_offset", "block_table", "k_cache", "k_scale", "weight"), **{**st, **kw})


@pytest.mark.parametrize("change,status", [
    (dict(rows=0), "OK"), (dict(batch=0), "OK"), (dict(max_q_len=0), "OK"), (dict(num_blocks=0), "OK"), (dict(max_blocks=0), "OK"),
    (dict(kv_dtype=2), "ERR_INVALID_ARG"), (dict(dtype=7), "ERR_INVALID_ARG"), (dict(window=0), "ERR_INVALID_ARG"), (dict(q_heads=5), "ERR_INVALID_ARG"),
    (dict(head_dim=24), "ERR_INVALID_ARG"), (dict(block_size=48), "ERR_INVALID_ARG"), (dict(decay=float("nan")), "ERR_INVALID_ARG"),
    (dict(scale=float("inf")), "ERR_INVALID_ARG"), (dict(lse=None), "ERR_INVALID_ARG"), (dict(weight=None), "ERR_INVALID_ARG"),
    (dict(weight=BASE + 5 * FAR), "ERR_INVALID_ARG"), (dict(weight=BASE + FAR), "ERR_INVALID_ARG"), (dict(q_stride=(0, 60, 256)), "ERR_INVALID_ARG"),
    (dict(lse_stride=(0, -1, 4)), "ERR_INVALID_ARG"), (dict(k_cache=BASE + 8), "ERR_INVALID_ARG"), (dict(head_dim=272), "ERR_UNSUPPORTED"),
    (dict(q_heads=130), "ERR_UNSUPPORTED"), (dict(max_blocks=2 ** 28), "ERR_UNSUPPORTED"), (dict(batch=8193), "ERR_UNSUPPORTED")])
def test_weigh_refusals(L, change, status):
    d = _weigh(**change)
    assert L.vscan_kv_weigh(C.byref(d), None) == getattr(vb, status)


def _evict(**kw):
    d = vb.KvEvictDesc(vb.KV_I8, 2, 2, 64, 16, 40, 9, 100, 4, 8, 1)
    return _fill(d, ("kv_len", "budget", "block_table", "weight", "weight_out", "k_cache", "v_cache", "k_scale", "v_scale", "kept", "delta"), **kw)


@pytest.mark.parametrize("change,status", [
    ({}, "WORKSPACE"), (dict(kept=None), "WORKSPACE"), (dict(weight_out=None), "WORKSPACE"), (dict(weight_out=BASE + 3 * FAR), "WORKSPACE"),
    (dict(max_keep=0), "WORKSPACE"), (dict(batch=0), "WORKSPACE"),
    (dict(weight_out=BASE + 3 * FAR + 16), "INVALID_ARG"), (dict(kv_dtype=3), "INVALID_ARG"), (dict(head_dim=40), "INVALID_ARG"),
    (dict(block_size=8), "INVALID_ARG"), (dict(max_keep=-1), "INVALID_ARG"), (dict(keep_first=-1), "INVALID_ARG"), (dict(keep_last=-1), "INVALID_ARG"),
    (dict(budget=None), "INVALID_ARG"), (dict(delta=None), "INVALID_ARG"), (dict(weight=None), "INVALID_ARG"), (dict(k_scale=None), "INVALID_ARG"),
    (dict(delta=BASE), "INVALID_ARG"), (dict(kept=BASE + 5 * FAR), "INVALID_ARG"), (dict(v_cache=BASE + 5 * FAR), "INVALID_ARG"),
    (dict(kv_len=BASE + 4), "INVALID_ARG"), (dict(head_dim=272), "UNSUPPORTED"), (dict(batch=8193), "UNSUPPORTED"),
    (dict(max_blocks=2 ** 28), "UNSUPPORTED"), (dict(kv_heads=60000, batch=8000, max_keep=2 ** 20), "UNSUPPORTED")])
def test_evict_refusals(L, change, status):
    d = _evict(**change)
    assert L.vscan_kv_evict(C.byref(d), None, 0, None) == getattr(vb, "ERR_" + status)
    assert L.vscan_kv_evict_workspace_bytes(C.byref(d)) >= 256


# --------------------------------------------------------------------------- VScanCache
def _cache(**kw):
    return VScanCache(**{**dict(num_blocks=8, block_size=16, kv_heads=2, head_dim=32, batch=2, max_blocks=4, rows=64, device="cpu", weights=True), **kw})


@pytest.fixture
def calls(monkeypatch):
    """The library's calls replaced: each one's name, and whether it is refused."""
    made, refused = [], set()

    def fake(name, result):
        def run(*args, **kw):
            made.append(name)
            if name in refused:
                raise vb.VScanError(vb.ERR_INVALID_ARG, name)
            return result(*args, **kw)
        monkeypatch.setattr(vb, name, run)

    fake("vscan_rope", lambda q, k, *a, **kw: (q, k))
    fake("vscan_kv_plan", lambda past, new, *a, out=None, **kw: out["kv_len"].copy_(past + new))
    fake("vscan_kv_write", lambda *a: None)
    fake("vscan_kv_attention", lambda q, *a, **kw: a[10] if len(a) > 10 else q)
    fake("vscan_kv_attention_workspace", lambda *a: vb.Workspace(1000, "cpu"))
    fake("vscan_attention", lambda q, *a, out=None, **kw: out)
    fake("vscan_attention_workspace", lambda *a: vb.Workspace(2000, "cpu"))
    fake("vscan_kv_weigh", lambda *a, **kw: None)
    fake("vscan_kv_evict_workspace", lambda table, k, max_keep, per_head: vb.Workspace(100 * max_keep, "cpu"))

    def evict(kv_len, budget, *a, max_keep=0, delta=None, workspace=None, **kw):
        if workspace.nbytes < 100 * a[6]:
            raise vb.VScanError(vb.ERR_WORKSPACE, "vscan_kv_evict")
        delta.copy_(torch.minimum(budget, kv_len) - kv_len)
    fake("vscan_kv_evict", evict)
    monkeypatch.setattr(vb, "vscan_check", lambda w: int(w.buf[:4].view(torch.int32)))
    return made, refused


def test_cache_prompts_steps_and_evictions_call_what_they_say(calls):
    made, _ = calls
    c, x, new = _cache(), torch.zeros((2, 2, 5, 32)), torch.tensor([5, 3], dtype=torch.int32)
    c.prompt(x, x, x, None, (None, None), new, 1.0)
    assert [n for n in made if "workspace" not in n] == ["vscan_rope", "vscan_kv_plan", "vscan_attention", "vscan_kv_write", "vscan_kv_weigh"]
    del made[:]
    c.step(x[:, :, :1], x[:, :, :1], x[:, :, :1], None, (None, None), torch.ones(2, dtype=torch.int32), 1.0)
    assert [n for n in made if "workspace" not in n] == ["vscan_rope", "vscan_kv_plan", "vscan_kv_write", "vscan_kv_attention", "vscan_kv_weigh"]
    del made[:]
    assert c.kv_len.tolist() == [6, 4]
    delta = c.evict(torch.tensor([4, 9], dtype=torch.int32), 10)
    assert [n for n in made if "workspace" not in n] == ["vscan_kv_evict", "vscan_kv_plan"] and delta.tolist() == [-2, 0] and c.kv_len.tolist() == [4, 4]
    del made[:]
    plain = _cache(weights=False)
    plain.prompt(x, x, x, None, (None, None), new, 1.0)
    plain.step(x, x, x, None, (None, None), new, 1.0)
    assert "vscan_kv_weigh" not in made and plain.weight is None and c.check() == (0, 0)


@pytest.mark.parametrize("which", ["vscan_attention", "vscan_kv_write", "vscan_kv_weigh"])
def test_cache_a_refused_prompt_leaves_lengths_as_they_were(calls, which):
    made, refused = calls
    c, x = _cache(), torch.zeros((2, 2, 5, 32))
    refused.add(which)
    with pytest.raises(vb.VScanError):
        c.prompt(x, x, x, None, (None, None), torch.tensor([5, 3], dtype=torch.int32), 1.0)
    assert c.kv_len.tolist() == [0, 0]


def test_cache_eviction_workspaces_grow_and_report(calls):
    c, budget = _cache(), torch.zeros(2, dtype=torch.int32)
    for most in (5, 3, 7, 50, 20, 51, 400):
        c.evict(budget, most)
    spaces = [c._spaces["evict"], *c._outgrown]
    assert len(spaces) <= 5 and spaces[0].nbytes >= 40000
    c._outgrown[0].buf[:4].view(torch.int32)[0] = vb.ERR_TIMEOUT
    assert c.check() == (vb.ERR_TIMEOUT, 0)
