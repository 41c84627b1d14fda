"""vscan_attention, vscan_kv_weigh and vscan_kv_evict on the host: sizes that do not fit together."""
import ctypes as C

import pytest
import torch

from paper_2505_22654_b200 import _build
from paper_2505_22654_b200 import binding as vb
from test_prompt_host import _attention, _evict


@pytest.fixture(scope="module")
def L():
    _build.build()
    return vb.lib()


@pytest.mark.parametrize("dtype", [vb.BF16, vb.F32])
@pytest.mark.parametrize("q_heads,kv_heads", [(1, 2), (2, 4), (4, 28), (3, 2), (7, 3), (1, 2 ** 31 - 1)])
def test_attention_of_fewer_or_uneven_query_heads_is_refused(L, dtype, q_heads, kv_heads):
    """Whatever is asked first, the workspace or the call: no division by a group of no heads."""
    d = _attention(dtype=dtype, q_heads=q_heads, kv_heads=kv_heads)
    assert L.vscan_attention_workspace_bytes(C.byref(d)) == 256
    assert L.vscan_attention(C.byref(d), None, 0, None) == vb.ERR_INVALID_ARG


def test_workspace_sizes_of_what_no_call_takes(L):
    """The functions that only say a size take anything."""
    for n in (-(2 ** 31), -1, 0, 1, 2, 2 ** 31 - 1):
        for name, make, size in (("batch rows kv_rows q_heads kv_heads head_dim max_q_len dtype padded", _attention, L.vscan_attention_workspace_bytes),
                                 ("batch kv_heads head_dim block_size num_blocks max_keep per_head kv_dtype", _evict, L.vscan_kv_evict_workspace_bytes)):
            for field in name.split():
                assert size(C.byref(make(**{field: n}))) >= 256
    assert L.vscan_attention_workspace_bytes(None) == 256 and L.vscan_kv_evict_workspace_bytes(None) == 256


def test_python_workspace_of_queries_and_keys_in_each_others_place(L):
    q, k = torch.zeros((5, 4, 64), dtype=torch.bfloat16), torch.zeros((5, 2, 64), dtype=torch.bfloat16)
    off = torch.tensor([0, 5], dtype=torch.int32)
    assert vb.vscan_attention_workspace(k, q, off, 5).nbytes == 256
    assert vb.vscan_attention_workspace(q, k, off, 5).nbytes > 256
