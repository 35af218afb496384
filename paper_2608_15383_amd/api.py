"""Thin Python binding of libexactmoe.so with the C ABI's names.

PyTorch only supplies device memory, pinned host memory and streams; every
step of the layer runs in the HIP library.  Tensors holding bf16 data may be
torch.bfloat16 or int16/uint16 bit patterns; they are passed by data_ptr().
"""
from __future__ import annotations

import ctypes as C

import numpy as np

from . import _lib
from ._lib import (DecoderDims, DecoderWeights, Dims, PagedKVView, Stats, WsLayout, binding, check,
                   lib, EMOE_BF16, EMOE_E4M3, EMOE_EINVAL, EMOE_F16, EMOE_PATH_AUTO, EMOE_PATH_GEMV, EMOE_PATH_MFMA, EMOE_PATH_MIXED,
                   EMOE_MIXED_MFMA_ROWS, ExactMoEError)


def _ptr(t) -> int | None:
    if t is None:
        return None
    if isinstance(t, np.ndarray):
        return t.ctypes.data
    return t.data_ptr()


def _stream(stream) -> int | None:
    if stream is None:
        import torch
        return torch.cuda.current_stream().cuda_stream
    if isinstance(stream, int):
        return stream
    return stream.cuda_stream


def dims(d_model: int, d_ff: int, n_experts: int, top_k: int) -> Dims:
    return Dims(d_model, d_ff, n_experts, top_k)


def check_dims(dm: Dims) -> None:
    check(lib().emoe_check_dims(C.byref(dm)))


def expert_record_bytes(dm: Dims) -> int:
    return int(lib().emoe_expert_record_bytes(C.byref(dm)))


def workspace_layout(dm: Dims, max_tokens: int) -> WsLayout:
    out = WsLayout()
    check(lib().emoe_workspace_layout(C.byref(dm), max_tokens, C.byref(out)))
    return out


def workspace_bytes(dm: Dims, max_tokens: int) -> int:
    return int(lib().emoe_workspace_bytes(C.byref(dm), max_tokens))


def quantize_experts(dm: Dims, w_gate, w_up, w_down, records, stream=None) -> None:
    """emoe_quantize_experts: device bf16 weights -> device packed records."""
    n = w_gate.shape[0]
    check(lib().emoe_quantize_experts(C.byref(dm), n, _ptr(w_gate), _ptr(w_up), _ptr(w_down),
                                      _ptr(records), _stream(stream)))


def unpack_expert(dm: Dims, record: np.ndarray) -> dict:
    """emoe_unpack_expert on a host copy of one record (numpy uint8)."""
    d, f = dm.d_model, dm.d_ff
    out = dict(q_gate=np.empty((f, d), np.int8), s_gate=np.empty((f, d // 128), np.uint16),
               q_up=np.empty((f, d), np.int8), s_up=np.empty((f, d // 128), np.uint16),
               q_down=np.empty((d, f), np.int8), s_down=np.empty((d, f // 128), np.uint16))
    rec = np.ascontiguousarray(record, dtype=np.uint8)
    check(lib().emoe_unpack_expert(C.byref(dm), rec.ctypes.data, *[out[k].ctypes.data for k in
                                   ("q_gate", "s_gate", "q_up", "s_up", "q_down", "s_down")]))
    return out


def pack_expert(dm: Dims, q_gate, s_gate, q_up, s_up, q_down, s_down) -> np.ndarray:
    """emoe_pack_expert: plain codes/scales (host) -> one packed record (numpy uint8)."""
    rec = np.zeros(expert_record_bytes(dm), np.uint8)
    arrs = [np.ascontiguousarray(a) for a in (q_gate, s_gate, q_up, s_up, q_down, s_down)]
    check(lib().emoe_pack_expert(C.byref(dm), *[a.ctypes.data for a in arrs], rec.ctypes.data))
    return rec


def route(dm: Dims, tokens: int, h, w_router, logits_override, renormalize: bool, logits,
          topk_ids, topk_w, counts, offsets, sorted_pairs, active, n_active, stream=None) -> None:
    """emoe_route: Eq. 1 logits, top-k, mixture weights and grouping on the device."""
    check(lib().emoe_route(C.byref(dm), tokens, _ptr(h), _ptr(w_router), _ptr(logits_override),
                           int(bool(renormalize)), _ptr(logits), _ptr(topk_ids), _ptr(topk_w),
                           _ptr(counts), _ptr(offsets), _ptr(sorted_pairs), _ptr(active),
                           _ptr(n_active), _stream(stream)))


class Cache:
    """emoe_cache_*: one layer's slot cache (Sec. 3.3)."""

    def __init__(self, dm: Dims, capacity: int, slot_bank=None, host_bank=None):
        self.dims = dm
        self.capacity = capacity
        self._keep = (slot_bank, host_bank)
        handle = C.c_void_p()
        check(lib().emoe_cache_create(C.byref(dm), capacity, _ptr(slot_bank), _ptr(host_bank),
                                      C.byref(handle)))
        self.handle = handle

    def close(self) -> None:
        if self.handle:
            lib().emoe_cache_destroy(self.handle)
            self.handle = C.c_void_p()

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    def preload_all(self, stream=None) -> None:
        check(lib().emoe_cache_preload_all(self.handle, _stream(stream)))

    def state(self):
        e, c = self.dims.n_experts, self.capacity
        so, eo, st = np.empty(e, np.int32), np.empty(c, np.int32), np.empty(c, np.int64)
        check(lib().emoe_cache_state(self.handle, so.ctypes.data, eo.ctypes.data, st.ctypes.data))
        return so, eo, st

    def sync_timeouts(self) -> int:
        """emoe_cache_sync_timeouts: bounded device waits that gave up (0 when healthy)."""
        n = C.c_int64()
        check(lib().emoe_cache_sync_timeouts(self.handle, C.byref(n)))
        return n.value

    def set_wave_overlap(self, enable: bool) -> None:
        """emoe_cache_set_wave_overlap: waves of C/2 when the active set does not fit,
        so each wave's fills proceed while the previous wave computes."""
        check(lib().emoe_cache_set_wave_overlap(self.handle, int(bool(enable))))

    def set_wave_delay(self, microseconds: int) -> None:
        """emoe_test_set_wave_delay: spin before each wave's projections (test hook)."""
        check(lib().emoe_test_set_wave_delay(self.handle, int(microseconds)))

    def set_decode_waits(self, spin_limit: int = 1 << 20, unmatched: bool = False) -> None:
        """emoe_test_set_decode_waits: the fused decode launch's waits give up after
        `spin_limit` polls; with `unmatched` they wait for a tag no writer uses (test hook)."""
        check(lib().emoe_test_set_decode_waits(self.handle, int(spin_limit), int(bool(unmatched))))

    def plan_waves(self, counts) -> list[list[int]]:
        e = self.dims.n_experts
        cnt = np.ascontiguousarray(counts, np.int32)
        we, wo, nw = np.empty(e, np.int32), np.empty(e + 1, np.int32), C.c_int32()
        check(lib().emoe_plan_waves(self.handle, cnt.ctypes.data, we.ctypes.data, wo.ctypes.data,
                                    C.byref(nw)))
        return [we[wo[i]:wo[i + 1]].tolist() for i in range(nw.value)]

    def build_slot_map(self, wave, stats: Stats | None = None):
        e = self.dims.n_experts
        w = np.ascontiguousarray(wave, np.int32)
        sm = np.empty(e, np.int32)
        fe, fs = np.empty(max(len(w), 1), np.int32), np.empty(max(len(w), 1), np.int32)
        nf = C.c_int32()
        check(lib().emoe_build_slot_map(self.handle, w.ctypes.data, len(w), sm.ctypes.data,
                                        fe.ctypes.data, fs.ctypes.data, C.byref(nf),
                                        C.byref(stats) if stats is not None else None))
        return sm, list(zip(fe[:nf.value].tolist(), fs[:nf.value].tolist()))

    def fill_slots(self, fills, stream=None) -> None:
        fe = np.array([a for a, _ in fills], np.int32)
        fs = np.array([b for _, b in fills], np.int32)
        check(lib().emoe_fill_slots(self.handle, fe.ctypes.data, fs.ctypes.data, len(fills),
                                    _stream(stream)))


def moe_forward(cache: Cache, h, w_router, y, workspace, logits_override=None,
                renormalize: bool = True, path: int = EMOE_PATH_AUTO, stats: Stats | None = None,
                stream=None, sequential: bool = False) -> None:
    """emoe_moe_forward (or emoe_moe_forward_sequential): y = the MoE layer of Eq. 2."""
    fn = lib().emoe_moe_forward_sequential if sequential else lib().emoe_moe_forward
    tokens = h.shape[0]
    nbytes = workspace.numel() * workspace.element_size()
    check(fn(cache.handle, tokens, _ptr(h), _ptr(w_router), _ptr(logits_override),
             int(bool(renormalize)), path, _ptr(y), _ptr(workspace), nbytes, _stream(stream),
             C.byref(stats) if stats is not None else None))


def moe_forward_noalloc(cache: Cache, h, w_router, y, logits_override=None,
                        renormalize: bool = True, path: int = EMOE_PATH_AUTO,
                        stats: Stats | None = None, stream=None) -> None:
    """emoe_moe_forward_noalloc: the layer call with the library's own scratch workspace."""
    check(lib().emoe_moe_forward_noalloc(cache.handle, h.shape[0], _ptr(h), _ptr(w_router),
                                         _ptr(logits_override), int(bool(renormalize)), path,
                                         _ptr(y), _stream(stream),
                                         C.byref(stats) if stats is not None else None))


def moe_forward_sequential(cache: Cache, h, w_router, y, workspace, **kw) -> None:
    moe_forward(cache, h, w_router, y, workspace, sequential=True, **kw)


def test_fail_copy_after(copies: int) -> None:
    """emoe_test_fail_copy_after: make the slot copy after `copies` more fail (-1 disarms)."""
    check(lib().emoe_test_fail_copy_after(int(copies)))


def decoder_dims(n_layers: int, n_heads: int, head_dim: int, vocab: int, max_positions: int,
                 moe: Dims, rope_base: float = 10000.0, rms_eps: float = 1e-5,
                 renormalize: bool = True) -> DecoderDims:
    return DecoderDims(n_layers, n_heads, head_dim, vocab, max_positions, rope_base, rms_eps,
                       int(bool(renormalize)), moe)


def decoder_kv_bytes(dd: DecoderDims) -> int:
    return int(lib().emoe_decoder_kv_bytes(C.byref(dd)))


def decoder_workspace_bytes(dd: DecoderDims, max_tokens: int) -> int:
    return int(lib().emoe_decoder_workspace_bytes(C.byref(dd), max_tokens))


class Decoder:
    """emoe_decoder_*: the synthetic decoder around one slot cache per layer.

    weights: dict of device bf16 tensors: embed [V][d], lm_head [V][d],
    final_norm [d], and per-layer lists attn_norm, wqkv [3d][d], wo [d][d],
    moe_norm, w_router [E][d].  caches: list of Cache (one per layer).
    kv: device buffer of decoder_kv_bytes(dd) bytes, or None for forward_paged only."""

    def __init__(self, dd: DecoderDims, weights: dict, caches, kv=None):
        n = dd.n_layers
        arr = lambda name: (C.c_void_p * n)(*[_ptr(t) for t in weights[name]])
        self._arrays = {k: arr(k) for k in ("attn_norm", "wqkv", "wo", "moe_norm", "w_router")}
        cast = lambda a: C.cast(a, C.POINTER(C.c_void_p))
        w = DecoderWeights(_ptr(weights["embed"]), _ptr(weights["lm_head"]),
                           _ptr(weights["final_norm"]), cast(self._arrays["attn_norm"]),
                           cast(self._arrays["wqkv"]), cast(self._arrays["wo"]),
                           cast(self._arrays["moe_norm"]), cast(self._arrays["w_router"]))
        handles = (C.c_void_p * n)(*[c.handle.value for c in caches])
        self.dims = dd
        self.device = weights["embed"].device
        self._keep = (weights, caches, kv, handles)
        h = C.c_void_p()
        check(lib().emoe_decoder_create(C.byref(dd), C.byref(w), C.cast(handles, C.POINTER(C.c_void_p)),
                                        _ptr(kv), C.byref(h)))
        self.handle = h

    def close(self) -> None:
        if self.handle:
            lib().emoe_decoder_destroy(self.handle)
            self.handle = C.c_void_p()

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    def set_step_keys(self, keys: int = -1) -> None:
        """emoe_test_set_step_keys: positions up to which a decode step runs rotation and
        attention in one launch (test hook; -1 restores the default)."""
        check(lib().emoe_test_set_step_keys(self.handle, int(keys)))

    def forward(self, tokens, pos0: int, logits, next_token, workspace, stream=None,
                stats: Stats | None = None) -> None:
        """emoe_decoder_forward: tokens (device int32 [T]) at positions pos0 .. pos0+T-1."""
        nbytes = workspace.numel() * workspace.element_size()
        check(lib().emoe_decoder_forward(self.handle, _ptr(tokens), tokens.shape[0], pos0,
                                         _ptr(logits), _ptr(next_token), _ptr(workspace), nbytes,
                                         _stream(stream),
                                         C.byref(stats) if stats is not None else None))

    def forward_paged(self, kvs, tokens, positions, page_table, logits, workspace, max_keys: int,
                      seqs=None, out_rows=None, next_token=None, stream=None,
                      stats: Stats | None = None, history=None, history_lengths=None,
                      prompt_lengths=None, repetition=None, presence=None, frequency=None,
                      bias_ids=None, bias_values=None, bias_counts=None, mask=None,
                      mask_rows=None) -> None:
        """emoe_decoder_forward_paged: tokens, positions (device int32 [n], of sequences seqs [n] or
        0 .. n-1) over one PagedKV per layer; logits f32 [n or len(out_rows)][V], processed as by
        process_logits with the last eleven arguments (of the logits' rows)."""
        if len(kvs) != self.dims.n_layers or any(kv.device != self.device for kv in kvs):
            _refuse(f"need {self.dims.n_layers} caches on the decoder's device, {self.device}")
        views = (PagedKVView * len(kvs))(*[kv.view for kv in kvs])
        device = kvs[0].index
        binding().decoder_forward_paged(
            self.handle.value, C.addressof(views), self.dims.vocab, device, tokens, positions,
            page_table, logits, workspace, max_keys, seqs, out_rows, next_token,
            0 if stats is None else C.addressof(stats), history, history_lengths, prompt_lengths,
            repetition, presence, frequency, bias_ids, bias_values, bias_counts, mask, mask_rows,
            _stream_on(device, stream))


# ---------------------------------------------------------------- many sequences at once
# The calls of exactmoe_serving.h.  A pointer says nothing about its tensor: what
# the library cannot see (types, shapes, strides, devices) is checked in
# csrc/binding.cpp, and here for a new cache.
def _refuse(message: str):
    raise ExactMoEError(EMOE_EINVAL, message)


def _stream_on(device: int, stream) -> int:
    """Handle of a stream, by default of that device's current one."""
    if stream is None:
        import torch
        return torch._C._cuda_getCurrentRawStream(device)  # 1.8 us less than by a Stream object
    if isinstance(stream, int):
        return stream
    if stream.device.index != device:
        _refuse(f"stream of {stream.device} for tensors on cuda:{device}")
    return stream.cuda_stream


def _cache_types() -> dict:
    import torch
    return {torch.bfloat16: EMOE_BF16, torch.int16: EMOE_BF16, torch.uint16: EMOE_BF16,
            torch.float16: EMOE_F16, torch.float8_e4m3fn: EMOE_E4M3}


class PagedKV:
    """emoe_paged_kv: one layer's paged cache.  k_pages, v_pages: [pages][page_size][kv heads]
    [head_dim] of bf16, fp16 or float8_e4m3fn, of equal strides (a permuted view of pages that
    hold their heads outside their slots does too).  k_scale, v_scale: f32 [kv heads], E4M3 only."""

    def __init__(self, k_pages, v_pages, k_scale=None, v_scale=None):
        import torch
        if k_pages.device.type != "cuda":
            _refuse(f"k_pages is on {k_pages.device}")
        if k_pages.dim() != 4 or k_pages.dtype not in _cache_types() or k_pages.stride(3) != 1:
            _refuse(f"k_pages: shape {tuple(k_pages.shape)}, type {k_pages.dtype}: need 4 axes of "
                    "bf16, fp16 or e4m3, the last one dense")
        for what in ("device", "dtype", "shape"):
            if getattr(v_pages, what) != getattr(k_pages, what):
                _refuse(f"v_pages: another {what} than k_pages")
        if v_pages.stride() != k_pages.stride():
            _refuse("v_pages: other strides than k_pages")
        for name, s in (("k_scale", k_scale), ("v_scale", v_scale)):
            if s is not None and (s.device != k_pages.device or s.dtype != torch.float32
                                  or tuple(s.shape) != (k_pages.shape[2],) or not s.is_contiguous()):
                _refuse(f"{name}: need f32 [{k_pages.shape[2]}] on {k_pages.device}")
        self.device, self.index = k_pages.device, k_pages.device.index
        self._keep = (k_pages, v_pages, k_scale, v_scale)
        self.view = PagedKVView(*[_ptr(t) for t in self._keep], *k_pages.stride()[:3],
                                _cache_types()[k_pages.dtype], *k_pages.shape)
        self.address = C.addressof(self.view)
        check(lib().emoe_check_paged_kv(C.byref(self.view)))


def rope_frequencies(rotary_dim: int, base: float = 10000.0, device="cuda"):
    """f64 [rotary_dim / 2]: base^(-2i / rotary_dim), the angles' frequencies of paged_append."""
    import torch
    return torch.tensor([base ** (-2.0 * i / rotary_dim) for i in range(rotary_dim // 2)],
                        dtype=torch.float64, device=device)


def paged_append(kv: PagedKV, q, k, v, positions, page_table, inv_freq, seqs=None, q_out=None,
                 interleaved: bool = False, stream=None) -> None:
    """emoe_paged_append: q_out (q itself when None) = the rotated q; the rotated k and v go to the
    pages of each token's position.  q [n][heads][dim] or None, k, v [n][kv heads][dim]; positions,
    seqs i32 [n]; page_table i32 [sequences][pages]; inv_freq f64 [rotary_dim / 2] or None."""
    binding().paged_append(kv.address, kv.index, q, k, v, positions, page_table, inv_freq, seqs, q_out,
                           interleaved, _stream_on(kv.index, stream))


def paged_attention_workspace_bytes(kv: PagedKV, rows: int, n_heads: int, max_keys: int) -> int:
    return int(lib().emoe_paged_attention_workspace_bytes(C.byref(kv.view), rows, n_heads,
                                                          max_keys))


def paged_attention(kv: PagedKV, q, page_table, lengths, out, workspace, max_keys: int, seqs=None,
                    scale: float | None = None, window: int = 0, lse=None, stream=None) -> None:
    """emoe_paged_attention: out[r] = attention of the token q[r] over the first lengths[r] keys of
    its sequence.  q, out [rows][heads][dim]; lengths, seqs i32 [rows]; page_table i32 [sequences]
    [pages]; lse f32 [rows][heads] or None; scale 1 / sqrt(dim) when None.  workspace: zeroed once
    (paged_attention_workspace_bytes)."""
    if scale is None:
        scale = kv.view.head_dim ** -0.5
    binding().paged_attention(kv.address, kv.index, q, page_table, lengths, out, workspace, max_keys,
                              seqs, scale, window, lse, _stream_on(kv.index, stream))


def process_logits_workspace_bytes(rows: int, vocab: int) -> int:
    return int(lib().emoe_process_logits_workspace_bytes(rows, vocab))


def process_logits(logits, out=None, workspace=None, history=None, history_lengths=None,
                   prompt_lengths=None, repetition=None, presence=None, frequency=None,
                   bias_ids=None, bias_values=None, bias_counts=None, mask=None, mask_rows=None,
                   next_token=None, stream=None) -> None:
    """emoe_process_logits: out (logits itself when None) = the logits [rows][vocab] after
    penalties, biases and mask; next_token i32 [rows] = the greedy choice.  history i32 [rows]
    [width], lengths i32 [rows]; repetition, presence, frequency f32 [rows]; bias_ids i32 and
    bias_values f32 [rows][width]; mask i32 words [masks][>= vocab / 32], mask_rows i32 [rows].
    workspace: zeroed once (process_logits_workspace_bytes), needed with next_token."""
    if not logits.is_cuda:
        _refuse(f"logits is on {logits.device}")
    binding().process_logits(logits, out, workspace, next_token, history, history_lengths,
                             prompt_lengths, repetition, presence, frequency, bias_ids, bias_values,
                             bias_counts, mask, mask_rows,
                             _stream_on(logits.device.index, stream))


def decoder_paged_workspace_bytes(dd: DecoderDims, n_tokens: int, n_out: int, max_keys: int) -> int:
    return int(lib().emoe_decoder_paged_workspace_bytes(C.byref(dd), n_tokens, n_out, max_keys))


# ---------------------------------------------------------------- drafted tokens
# The calls of exactmoe_drafts.h.
def _check_cache(kv) -> None:
    if not isinstance(kv, PagedKV):
        _refuse("kv: need a PagedKV")


def paged_append_axes(kv: PagedKV, q, k, v, positions, angles, axes, page_table, inv_freq, seqs=None,
                      q_out=None, interleaved: bool = False, stream=None) -> None:
    """emoe_paged_append_axes: paged_append with angles[t][axes[i]] * inv_freq[i] in place of
    positions[t] * inv_freq[i].  angles i32 [n][axes]; axes i32 [rotary_dim / 2], the axis of each
    pair, or None: the first one.  A drafted node of depth d behind n keys: angles [[n + d]]."""
    _check_cache(kv)
    binding().paged_append_axes(kv.address, kv.index, q, k, v, positions, page_table, inv_freq, seqs,
                                q_out, interleaved, angles, axes, _stream_on(kv.index, stream))


def paged_tree_attention_workspace_bytes(kv: PagedKV, trees: int, n_heads: int, max_keys: int,
                                         max_nodes: int) -> int:
    _check_cache(kv)
    return int(lib().emoe_paged_tree_attention_workspace_bytes(C.byref(kv.view), trees, n_heads,
                                                               max_keys, max_nodes))


def paged_tree_attention(kv: PagedKV, q, page_table, lengths, out, workspace, max_keys: int,
                         max_nodes: int, tree=None, starts=None, seqs=None,
                         scale: float | None = None, cap: float = 0.0, slopes=None, window: int = 0,
                         lse=None, stream=None) -> None:
    """emoe_paged_tree_attention: out[r] = attention of node r of the trees behind the first
    lengths[g] keys of their sequences, over those keys and the nodes of its mask.  q, out [rows]
    [heads][dim]; lengths, seqs i32 [trees]; starts i32 [trees + 1], the trees' first rows (None:
    max_nodes rows each); tree i64 [rows], bit j: sees node j (None: chains); page_table i32
    [sequences][pages]; slopes f32 [heads]; lse f32 [rows][heads]; scale 1 / sqrt(dim) when None.
    max_keys bounds lengths and nodes together, max_nodes a tree's nodes (the nearer, the faster).
    workspace: paged_tree_attention_workspace_bytes, of any content."""
    _check_cache(kv)
    if scale is None:
        scale = kv.view.head_dim ** -0.5
    binding().paged_tree_attention(kv.address, kv.index, q, page_table, lengths, out, workspace,
                                   max_keys, max_nodes, tree, starts, seqs, scale, cap, slopes,
                                   window, lse, _stream_on(kv.index, stream))


def accept_drafts(tokens, chosen, lengths, path, accepted, new_tokens=None, new_lengths=None,
                  tree=None, starts=None, stream=None) -> None:
    """emoe_accept_drafts: from each tree's first node down, as long as a child's token is the one
    chosen after its parent.  tokens, chosen i32 [rows]; tree, starts as in paged_tree_attention;
    path, new_tokens i32 [trees][most nodes], accepted i32 [trees]; new_lengths = lengths +
    accepted, i32 [trees]."""
    if not getattr(tokens, "is_cuda", False):
        _refuse("tokens: need a tensor on a GPU")
    binding().accept_drafts(tokens, chosen, lengths, path, accepted, new_tokens, new_lengths, tree,
                            starts, _stream_on(tokens.device.index, stream))


def _device_of(kvs) -> int:
    if not isinstance(kvs, (list, tuple)) or not kvs or not isinstance(kvs[0], PagedKV):
        _refuse("kvs: need a list of PagedKV")
    return kvs[0].index


def paged_compact(kvs, page_table, lengths, path, accepted, seqs=None, stream=None) -> None:
    """emoe_paged_compact: in every cache of the list kvs, position lengths[g] + i of a sequence
    takes what lengths[g] + path[g][i] held, for i < accepted[g].  path i32 [trees][most nodes];
    lengths (those before the acceptance), accepted, seqs i32 [trees]."""
    device = _device_of(kvs)
    binding().paged_compact(kvs, PagedKV, device, page_table, lengths, path, accepted, seqs,
                            _stream_on(device, stream))


def paged_fork(kvs, page_table, parents, lengths, fresh, new_table, stream=None) -> None:
    """emoe_paged_fork: new_table[f] = the pages of the first lengths[f] positions of sequence
    parents[f]; a page in use only in part is copied to page fresh[f] of every cache of the list kvs
    (fresh None or outside the pool: shared).  parents, lengths, fresh i32 [forks]; new_table i32
    [forks][the width of page_table]."""
    device = _device_of(kvs)
    binding().paged_fork(kvs, PagedKV, device, page_table, parents, lengths, fresh, new_table,
                         _stream_on(device, stream))


def profile_begin(max_kernels: int) -> None:
    """emoe_profile_begin: time each kernel the layer calls launch from this thread."""
    check(lib().emoe_profile_begin(max_kernels))


def profile_end(max_out: int = 1 << 16) -> list[tuple[str, float]]:
    """emoe_profile_end: [(kernel name, milliseconds)] in launch order."""
    kinds = np.empty(max_out, np.int32)
    ms = np.empty(max_out, np.float32)
    n = C.c_int32()
    check(lib().emoe_profile_end(kinds.ctypes.data, ms.ctypes.data, max_out, C.byref(n)))
    m = min(n.value, max_out)
    return [(_lib.KERNEL_NAMES[k], float(t)) for k, t in zip(kinds[:m], ms[:m])]


__all__ = ["Dims", "Stats", "WsLayout", "ExactMoEError", "EMOE_PATH_AUTO", "EMOE_PATH_GEMV",
           "EMOE_PATH_MFMA", "EMOE_PATH_MIXED", "EMOE_MIXED_MFMA_ROWS", "dims", "check_dims", "expert_record_bytes", "workspace_layout",
           "workspace_bytes", "quantize_experts", "unpack_expert", "pack_expert", "route", "Cache",
           "moe_forward", "moe_forward_noalloc", "decoder_dims", "decoder_kv_bytes",
           "decoder_workspace_bytes", "Decoder", "moe_forward_sequential", "test_fail_copy_after", "profile_begin", "profile_end",
           "PagedKV", "rope_frequencies", "paged_append", "paged_attention",
           "paged_attention_workspace_bytes", "decoder_paged_workspace_bytes", "process_logits", "process_logits_workspace_bytes",
           "paged_append_axes", "paged_tree_attention", "paged_tree_attention_workspace_bytes",
           "accept_drafts", "paged_compact", "paged_fork", "lib"]
