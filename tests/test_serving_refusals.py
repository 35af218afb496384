"""Argument checks of the batched decoding calls, without a GPU: every refused
call returns its status before anything is enqueued or any pointer is read."""
import ctypes as C

import pytest
import torch

from paper_2608_15383_amd import _lib, api
from paper_2608_15383_amd._lib import (EMOE_BF16, EMOE_E4M3, EMOE_EINVAL, EMOE_ESHAPE, EMOE_F16,
                                       EMOE_F32, EMOE_OK)

P = 1 << 20                                    # an aligned pointer that is never read


def kv(**kw):
    f = dict(k_pages=P, v_pages=P, page_stride=16 * 4 * 128, slot_stride=4 * 128, head_stride=128,
             dtype=EMOE_BF16, n_pages=10, page_size=16, n_kv_heads=4, head_dim=128)
    return _lib.PagedKVView(**{**f, **kw})


def append(**kw):
    f = dict(q=P, k=P, v=P, q_out=P, positions=P, seqs=P, page_table=P, inv_freq=P, q_stride=2048,
             k_stride=512, v_stride=512, q_out_stride=2048, table_stride=8, dtype=EMOE_BF16,
             tokens=3, n_heads=16, n_seqs=2, table_width=8, rotary_dim=128, interleaved=0)
    return _lib.PagedAppendArgs(**{**f, **kw})


def attention(**kw):
    f = dict(q=P, out=P, lengths=P, page_table=P, q_stride=2048, out_stride=2048, table_stride=8,
             scale=0.1, dtype=EMOE_BF16, rows=3, n_heads=16, n_seqs=3, table_width=8, max_keys=128)
    return _lib.PagedAttentionArgs(**{**f, **kw})


def logits(**kw):
    f = dict(logits=P, out=P, logits_stride=1000, out_stride=1000, dtype=EMOE_F32, rows=3,
             vocab=1000)
    return _lib.LogitsArgs(**{**f, **kw})


def status(fn, *args):
    st = getattr(_lib.lib(), fn)(*args)
    if st != EMOE_OK:
        assert _lib.lib().emoe_last_error()
    return st


@pytest.mark.parametrize("change,want", [
    (dict(), EMOE_OK),
    (dict(dtype=EMOE_E4M3, k_scale=P, v_scale=P), EMOE_OK),
    (dict(page_stride=4 * 2048, slot_stride=128, head_stride=2048), EMOE_OK),   # heads outside slots
    (dict(n_kv_heads=1, head_stride=7), EMOE_OK),                               # of no meaning
    (dict(n_pages=1, page_stride=3), EMOE_OK),
    (dict(k_pages=None), EMOE_EINVAL),
    (dict(v_pages=P + 8), EMOE_EINVAL),
    (dict(dtype=EMOE_F32), EMOE_EINVAL),
    (dict(dtype=9), EMOE_EINVAL),
    (dict(k_scale=P, v_scale=P), EMOE_EINVAL),                                  # 16-bit cache
    (dict(dtype=EMOE_E4M3, k_scale=P), EMOE_EINVAL),
    (dict(page_size=24), EMOE_ESHAPE),
    (dict(page_size=4), EMOE_ESHAPE),
    (dict(page_size=2048), EMOE_ESHAPE),
    (dict(page_size=-16), EMOE_ESHAPE),
    (dict(head_dim=96), EMOE_ESHAPE),
    (dict(n_pages=0), EMOE_ESHAPE),
    (dict(n_kv_heads=0), EMOE_ESHAPE),
    (dict(slot_stride=4 * 128 + 4), EMOE_EINVAL),
    (dict(slot_stride=3 * 128), EMOE_ESHAPE),                                   # heads overlap slots
    (dict(slot_stride=0), EMOE_ESHAPE),
    (dict(head_stride=-128), EMOE_ESHAPE),
    (dict(page_stride=15 * 512), EMOE_ESHAPE),
    (dict(page_stride=-16 * 512), EMOE_ESHAPE),
    (dict(page_stride=1 << 40, slot_stride=1 << 27), EMOE_ESHAPE),              # a page above 2^30
    (dict(n_kv_heads=1 << 30, slot_stride=1 << 40, page_stride=1 << 45), EMOE_ESHAPE),
])
def test_cache_checks(change, want):
    assert status("emoe_check_paged_kv", C.byref(kv(**change))) == want
    if want != EMOE_OK:
        assert status("emoe_paged_append", C.byref(kv(**change)), C.byref(append()), None) == want
        assert status("emoe_paged_attention", C.byref(kv(**change)), C.byref(attention()), P,
                      1 << 40, None) == want
        assert _lib.lib().emoe_paged_attention_workspace_bytes(C.byref(kv(**change)), 1, 16, 9) == 0


@pytest.mark.parametrize("change,want", [
    (dict(tokens=0, k=None, positions=None), EMOE_OK),
    (dict(tokens=-1), EMOE_EINVAL),
    (dict(dtype=EMOE_F16), EMOE_EINVAL),                # over a bf16 cache
    (dict(dtype=EMOE_F32), EMOE_EINVAL),
    (dict(dtype=EMOE_E4M3), EMOE_EINVAL),
    (dict(k=None), EMOE_EINVAL),
    (dict(v=P + 2), EMOE_EINVAL),
    (dict(q=P + 8), EMOE_EINVAL),
    (dict(q_out=None), EMOE_EINVAL),
    (dict(positions=None), EMOE_EINVAL),
    (dict(inv_freq=None), EMOE_EINVAL),
    (dict(page_table=None), EMOE_EINVAL),
    (dict(n_heads=0), EMOE_ESHAPE),
    (dict(k_stride=511), EMOE_EINVAL),
    (dict(k_stride=504), EMOE_EINVAL),                  # below a token's row
    (dict(v_stride=0), EMOE_EINVAL),
    (dict(q_stride=2047), EMOE_EINVAL),
    (dict(q_out_stride=-2048), EMOE_EINVAL),
    (dict(rotary_dim=130), EMOE_ESHAPE),
    (dict(rotary_dim=256), EMOE_ESHAPE),
    (dict(rotary_dim=8), EMOE_ESHAPE),
    (dict(rotary_dim=-16), EMOE_ESHAPE),
    (dict(interleaved=2), EMOE_EINVAL),
    (dict(table_stride=7), EMOE_EINVAL),
    (dict(n_seqs=-1), EMOE_EINVAL),
    (dict(table_width=-1), EMOE_EINVAL),
])
def test_append_checks(change, want):
    assert status("emoe_paged_append", C.byref(kv()), C.byref(append(**change)), None) == want
    assert status("emoe_paged_append", None, C.byref(append()), None) == EMOE_EINVAL
    assert status("emoe_paged_append", C.byref(kv()), None, None) == EMOE_EINVAL


@pytest.mark.parametrize("heads", [(1 << 20) + 1, 1 << 27, (1 << 31) - 1])
def test_append_bounds_its_heads(heads):
    """A row's items and what a step of the workgroups adds to them stay within 32 bits (2^27
    heads of 128 would have passed them)."""
    for tokens in (0, 1):
        a = append(n_heads=heads, tokens=tokens, q_stride=1 << 40, q_out_stride=1 << 40)
        assert status("emoe_paged_append", C.byref(kv()), C.byref(a), None) == EMOE_ESHAPE


@pytest.mark.parametrize("change,want", [
    (dict(rows=0, q=None), EMOE_OK),
    (dict(rows=-1), EMOE_EINVAL),
    (dict(max_keys=-1), EMOE_EINVAL),
    (dict(window=-1), EMOE_EINVAL),
    (dict(n_heads=0), EMOE_ESHAPE),
    (dict(n_heads=6), EMOE_ESHAPE),
    (dict(scale=float("nan")), EMOE_EINVAL),
    (dict(scale=float("inf")), EMOE_EINVAL),
    (dict(scale=-3e38), EMOE_EINVAL),                   # infinite once it is one of powers of two
    (dict(max_keys=(1 << 30) + 1), EMOE_ESHAPE),
    (dict(max_keys=2 ** 31 - 1), EMOE_ESHAPE),
    (dict(n_heads=1 << 21, q_stride=1 << 28, out_stride=1 << 28), EMOE_ESHAPE),
    (dict(dtype=EMOE_F16), EMOE_EINVAL),
    (dict(dtype=EMOE_F32), EMOE_EINVAL),
    (dict(q=None), EMOE_EINVAL),
    (dict(q=P + 8), EMOE_EINVAL),
    (dict(q_stride=2040), EMOE_EINVAL),
    (dict(out=None), EMOE_EINVAL),
    (dict(out_stride=2050), EMOE_EINVAL),
    (dict(lengths=None), EMOE_EINVAL),
    (dict(page_table=None), EMOE_EINVAL),
    (dict(table_stride=-8), EMOE_EINVAL),
])
def test_attention_checks(change, want):
    args = (C.byref(kv()), C.byref(attention(**change)))
    assert status("emoe_paged_attention", *args, P, 1 << 40, None) == want


def test_attention_needs_its_workspace():
    need = _lib.lib().emoe_paged_attention_workspace_bytes(C.byref(kv()), 3, 16, 128)
    assert need >= _lib.EMOE_SERVING_TICKET_BYTES
    args = (C.byref(kv()), C.byref(attention()))
    assert status("emoe_paged_attention", *args, None, need, None) == EMOE_EINVAL
    assert status("emoe_paged_attention", *args, P, need - 1, None) == EMOE_EINVAL
    for bad in ((-1, 16, 9), (1, 0, 9), (1, 6, 9), (1, 16, -1), (1, 16, 2 ** 31 - 1), (1, 1 << 21, 9)):
        assert _lib.lib().emoe_paged_attention_workspace_bytes(C.byref(kv()), *bad) == 0


@pytest.mark.parametrize("change,want", [
    (dict(rows=0, logits=None), EMOE_OK),
    (dict(rows=-1), EMOE_ESHAPE),
    (dict(vocab=0), EMOE_ESHAPE),
    (dict(vocab=(1 << 30) + 1, logits_stride=1 << 31, out_stride=1 << 31), EMOE_ESHAPE),
    (dict(dtype=EMOE_E4M3), EMOE_EINVAL),
    (dict(logits=None), EMOE_EINVAL),
    (dict(out=None), EMOE_EINVAL),
    (dict(logits=P + 2), EMOE_EINVAL),
    (dict(dtype=EMOE_BF16, out=P + 1), EMOE_EINVAL),
    (dict(logits_stride=999), EMOE_EINVAL),
    (dict(out_stride=999), EMOE_EINVAL),
    (dict(repetition=P), EMOE_EINVAL),                                # without a history
    (dict(history=P, history_width=5, history_stride=4), EMOE_EINVAL),
    (dict(history=P, history_width=-5), EMOE_EINVAL),
    (dict(bias_ids=P, bias_width=3, bias_stride=3), EMOE_EINVAL),     # no values
    (dict(bias_values=P, bias_width=3, bias_stride=3), EMOE_EINVAL),
    (dict(bias_ids=P, bias_values=P, bias_width=3, bias_stride=2), EMOE_EINVAL),
    (dict(mask=P, n_masks=2, mask_stride=32), EMOE_EINVAL),           # fewer masks than rows
    (dict(mask=P, n_masks=3, mask_stride=31), EMOE_EINVAL),
    (dict(mask_rows=P), EMOE_EINVAL),
    (dict(next_token=P), EMOE_EINVAL),                                # no workspace
])
def test_logits_checks(change, want):
    assert status("emoe_process_logits", C.byref(logits(**change)), None, 0, None) == want


def test_logits_need_their_workspace():
    need = _lib.lib().emoe_process_logits_workspace_bytes(3, 1000)
    assert need > 0
    a = C.byref(logits(next_token=P))
    assert status("emoe_process_logits", a, P, need - 1, None) == EMOE_EINVAL
    assert status("emoe_process_logits", a, P + 4, need, None) == EMOE_EINVAL
    assert status("emoe_process_logits", None, P, need, None) == EMOE_EINVAL
    assert _lib.lib().emoe_process_logits_workspace_bytes(-1, 1000) == 0
    assert _lib.lib().emoe_process_logits_workspace_bytes(3, 0) == 0


def test_binding_refuses_what_the_library_cannot_see():
    for make in (lambda: api.PagedKV(torch.zeros(2, 16, 1, 64, dtype=torch.bfloat16),
                                     torch.zeros(2, 16, 1, 64, dtype=torch.bfloat16)),
                 lambda: api.process_logits(torch.zeros(2, 100))):       # host tensors
        with pytest.raises(_lib.ExactMoEError) as e:
            make()
        assert e.value.status == EMOE_EINVAL
