"""MI355X-native hot path of one DualDiffusion draft-then-verify step.

Thin binding over the C ABI in ``include/dd.h`` (``libdd.so``, hand-written
gfx950 HIP kernels).  The functions here have the C entry points' names and only
marshal arguments: torch tensors supply device memory and the current stream, every
step of the computation runs in the library's kernels.  The marshalling itself is native
(``csrc/binding.cpp``); the C ABI is also reachable through ``lib()`` (ctypes).  There is no CPU
fallback: if a library cannot be loaded, the first call raises.
"""
from __future__ import annotations

import ctypes as C
import os
from typing import Optional

F32, BF16, FP8_E4M3 = 0, 1, 2
TRUST, KL_THRESH, CONF_THRESH, KL_PROB, CONF_PROB, KL_TOPK, CONF_TOPK = 0, 1, 2, 3, 4, 5, 6
UNMASK_THRESH, UNMASK_TOPK = 0, 1

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libdd.so")
BINDING_PATH = os.path.join(_HERE, "_binding.so")
_lib = None
_native = None


class DDError(RuntimeError):
    def __init__(self, status: int, where: str):
        self.status = status
        super().__init__(f"{where}: {lib().dd_strerror(status).decode()} (status {status})")


def lib():
    """The loaded C-ABI library (built on first use only when no built library exists)."""
    global _lib
    if _lib is not None:
        return _lib
    if not os.path.exists(LIB_PATH):
        from .build import build_library
        build_library(force=True)
    # torch ships its own copy of the HIP runtime (same soname).  It has to be mapped first so
    # that this library binds to that copy: streams and device pointers handed over by torch
    # are only valid inside the runtime instance that created them.
    import torch  # noqa: F401
    L = C.CDLL(LIB_PATH)
    vp, i, sz = C.c_void_p, C.c_int, C.c_size_t
    L.dd_strerror.restype = C.c_char_p
    L.dd_strerror.argtypes = [i]
    L.dd_version.restype = i
    L.dd_bidir_attention.restype = i
    L.dd_bidir_attention.argtypes = [vp, vp, vp, vp, i, i, i, i, i, i, i, vp, vp, vp, sz, vp]
    L.dd_bidir_attention_workspace_bytes.restype = sz
    L.dd_bidir_attention_workspace_bytes.argtypes = [i, i, i, i, i, i, i]
    L.dd_block_attention_cached.restype = i
    L.dd_block_attention_cached.argtypes = [vp, vp, vp, vp, i, i, vp, vp, i, i, i, i, i, i, i, vp, vp, vp, sz, vp]
    L.dd_block_attention_cached_workspace_bytes.restype = sz
    L.dd_block_attention_cached_workspace_bytes.argtypes = [i, i, i, i, i, i, i, i]
    L.dd_bidir_attention_fp8v.restype = i
    L.dd_bidir_attention_fp8v.argtypes = [vp, vp, vp, vp, i, i, i, i, i, vp, vp, vp, vp]
    L.dd_bidir_attention_mx.restype = i
    L.dd_bidir_attention_mx.argtypes = [vp, vp, vp, vp, vp, vp, vp, i, i, i, i, i, vp]
    L.dd_block_attention_cached_fp8v.restype = i
    L.dd_block_attention_cached_fp8v.argtypes = [vp, vp, vp, vp, i, i, vp, vp, i, i, i, i, i, vp, vp, vp, vp, sz, vp]
    L.dd_block_attention_cached_fp8v_workspace_bytes.restype = sz
    L.dd_block_attention_cached_fp8v_workspace_bytes.argtypes = [i, i, i, i, i, i]
    L.dd_verify_remask.restype = i
    L.dd_verify_remask.argtypes = [vp, vp, vp, i, C.c_float, C.c_uint64, vp, vp, vp, i, i, i, i, vp, sz, vp]
    L.dd_verify_remask_workspace_bytes.restype = sz
    L.dd_verify_remask_workspace_bytes.argtypes = [i, i, i, i]
    L.dd_verify_remask_static.restype = i
    L.dd_verify_remask_static.argtypes = [vp, vp, vp, i, C.c_float, C.c_uint64, vp, vp, vp, i, i, i, i, vp]
    L.dd_unmask.restype = i
    L.dd_unmask.argtypes = [vp, vp, i, C.c_float, vp, vp, vp, vp, i, i, i, i, vp, sz, vp]
    L.dd_unmask_workspace_bytes.restype = sz
    L.dd_unmask_workspace_bytes.argtypes = [i, i, i, i]
    L.dd_block_attention_refresh.restype = i
    L.dd_block_attention_refresh.argtypes = [vp, vp, vp, vp, i, i, vp, vp, i, i, i, i, i, i, i, vp, vp, vp, sz, vp]
    L.dd_block_attention_refresh_workspace_bytes.restype = sz
    L.dd_block_attention_refresh_workspace_bytes.argtypes = [i, i, i, i, i, i, i, i]
    L.dd_block_attention_window.restype = i
    L.dd_block_attention_window.argtypes = [vp, vp, vp, vp, i, i, i, i, vp, vp, i, i, i, i, i, i, i, vp, vp, vp, sz, vp]
    L.dd_block_attention_window_workspace_bytes.restype = sz
    L.dd_block_attention_window_workspace_bytes.argtypes = [i, i, i, i, i, i, i, i, i]
    L.dd_block_attention_batched.restype = i
    L.dd_block_attention_batched.argtypes = [vp, vp, vp, vp, vp, i, vp, vp, i, i, i, i, i, i, i, vp, vp, vp, sz, vp]
    L.dd_block_attention_batched_workspace_bytes.restype = sz
    L.dd_block_attention_batched_workspace_bytes.argtypes = [i, i, i, i, i, i, i, i]
    L.dd_cache_insert_rows.restype = i
    L.dd_cache_insert_rows.argtypes = [vp, vp, vp, vp, vp, i, i, i, i, i, i, i, vp]
    L.dd_verify_scores.restype = i
    L.dd_verify_scores.argtypes = [vp, vp, vp, vp, vp, vp, vp, i, i, i, vp, sz, vp]
    L.dd_verify_scores_workspace_bytes.restype = sz
    L.dd_verify_scores_workspace_bytes.argtypes = [i, i, i]
    i64, f = C.c_int64, C.c_float
    L.dd_qk_norm_rope.restype = i
    L.dd_qk_norm_rope.argtypes = [vp, i64, i64, i64, vp, i64, i64, i64, vp, vp, f, vp, i, i, vp, vp, vp, i, i, i, i, i, i, vp]
    L.dd_paged_cache_append.restype = i
    L.dd_paged_cache_append.argtypes = [vp, vp, vp, vp, vp, i64, i64, i64, vp, i64, i64, i64, vp, vp, vp, vp, vp, f, vp, i, i,
                                        i, i, i, i, i, i, i, i, i, vp]
    L.dd_paged_attention.restype = i
    L.dd_paged_attention.argtypes = [vp, vp, vp, vp, vp, vp, vp, vp, i, i, i, i, i, i, i, i, i, vp, sz, vp]
    L.dd_paged_attention_workspace_bytes.restype = sz
    L.dd_paged_attention_workspace_bytes.argtypes = [i, i, i, i, i, i, i, i]
    L.dd_paged_resize.restype = i
    L.dd_paged_resize.argtypes = [vp, vp, vp, vp, vp, vp, vp, vp, i, i, i, i, i, vp, sz, vp]
    L.dd_paged_resize_workspace_bytes.restype = sz
    L.dd_paged_resize_workspace_bytes.argtypes = [i, i, i, i]
    L.dd_paged_attention_shared.restype = i
    L.dd_paged_attention_shared.argtypes = [vp, vp, vp, vp, vp, vp, vp, vp, vp, vp, vp, i, i, i, i, i, i, i, i, i, i, i, vp, sz, vp]
    L.dd_paged_attention_shared_workspace_bytes.restype = sz
    L.dd_paged_attention_shared_workspace_bytes.argtypes = [i, i, i, i, i, i, i, i, i, i]
    L.dd_verify_draft.restype = i
    L.dd_verify_draft.argtypes = [vp, vp, vp, vp, vp, vp, vp, vp, vp, i, i, i, i, i, vp, sz, vp]
    L.dd_verify_draft_workspace_bytes.restype = sz
    L.dd_verify_draft_workspace_bytes.argtypes = [i, i, i, i, i, i]
    _lib = L
    return L


EXPORTS = ("dd_strerror", "dd_version", "dd_bidir_attention", "dd_bidir_attention_workspace_bytes",
           "dd_block_attention_cached", "dd_block_attention_cached_workspace_bytes",
           "dd_verify_remask", "dd_verify_remask_workspace_bytes", "dd_verify_remask_static", "dd_unmask", "dd_unmask_workspace_bytes",
           "dd_verify_scores", "dd_verify_scores_workspace_bytes",
           "dd_block_attention_refresh", "dd_block_attention_refresh_workspace_bytes",
           "dd_block_attention_window", "dd_block_attention_window_workspace_bytes", "dd_cache_insert_rows",
           "dd_block_attention_batched", "dd_block_attention_batched_workspace_bytes",
           "dd_bidir_attention_fp8v", "dd_block_attention_cached_fp8v", "dd_block_attention_cached_fp8v_workspace_bytes",
           "dd_bidir_attention_mx", "dd_qk_norm_rope", "dd_paged_cache_append", "dd_paged_attention",
           "dd_paged_attention_workspace_bytes", "dd_verify_draft", "dd_verify_draft_workspace_bytes",
           "dd_paged_attention_shared", "dd_paged_attention_shared_workspace_bytes",
           "dd_paged_resize", "dd_paged_resize_workspace_bytes")


# ---------------------------------------------------------------- marshalling (csrc/binding.cpp)
def native():
    """The binding's native module (built on first use only when no built one exists)."""
    global _native
    if _native is not None:
        return _native
    lib()                                         # first: it brings torch's HIP runtime with it
    if not os.path.exists(BINDING_PATH):
        from .build import build_binding
        build_binding()
    from importlib.machinery import ExtensionFileLoader
    from importlib.util import module_from_spec, spec_from_file_location
    name = __name__ + "._binding"
    spec = spec_from_file_location(name, BINDING_PATH, loader=ExtensionFileLoader(name, BINDING_PATH))
    mod = module_from_spec(spec)
    spec.loader.exec_module(mod)
    mod.set_error_class(DDError)
    _native = mod
    return mod


def reset_workspace_peak() -> None:
    native().reset_workspace_peak()


def workspace_peak() -> int:
    """The largest scratch size any call of this thread has asked for since its reset_workspace_peak()."""
    return native().workspace_peak()


class fixed_workspace:
    """Context manager: calls of the binding that its thread makes inside it use `tensor` (uint8, on the GPU) as their scratch
    memory instead of the per-stream cached one; they must all be ordered on one stream.  For graph capture: the
    tensor is allocated before the capture and kept alive by whoever keeps the graph."""

    def __init__(self, tensor):
        self.tensor = tensor

    def __enter__(self):
        self.prev = native().set_fixed_workspace(self.tensor)
        return self.tensor

    def __exit__(self, *exc):
        native().set_fixed_workspace(self.prev)
        return False


# ---------------------------------------------------------------- entry points
def dd_bidir_attention_workspace_bytes(B, H, Hkv, N, d, qk_dtype, v_dtype) -> int:
    return lib().dd_bidir_attention_workspace_bytes(B, H, Hkv, N, d, qk_dtype, v_dtype)


def dd_bidir_attention(Q, K, V, O=None, q_scale=None, k_scale=None, qk_dtype: Optional[int] = None,
                       v_dtype: Optional[int] = None):
    """Verifier attention over all positions.  Q [B,H,N,d], K,V [B,Hkv,N,d] -> O [B,H,N,d] (V's type)."""
    return native().bidir(Q, K, V, O, q_scale, k_scale, qk_dtype, v_dtype)


def dd_block_attention_cached_workspace_bytes(block_len, B, H, Hkv, N, d, qk_dtype, v_dtype) -> int:
    return lib().dd_block_attention_cached_workspace_bytes(block_len, B, H, Hkv, N, d, qk_dtype, v_dtype)


def dd_block_attention_cached(Qblk, Kc, Vc, block_start: int, O=None, Kblk=None, Vblk=None, q_scale=None,
                              k_scale=None, qk_dtype: Optional[int] = None, v_dtype: Optional[int] = None,
                              _refresh: bool = False):
    """Drafter attention: the active block's queries over cached K/V.
    Qblk [B,H,bl,d], Kc,Vc [B,Hkv,N,d], optional Kblk,Vblk [B,Hkv,bl,d] -> O [B,H,bl,d]."""
    return native().block(1 if _refresh else 0, Qblk, Kc, Vc, block_start, 0, 0, O, Kblk, Vblk, q_scale, k_scale,
                          qk_dtype, v_dtype)


def dd_bidir_attention_fp8v(Q, K, V, q_scale, k_scale, v_scale, O=None):
    """Verifier attention with Q, K and V all stored as e4m3 codes (uint8) and per-head fp32 scales -> O bf16
    (as int16 bit patterns unless O is given)."""
    return native().bidir_fp8v(Q, K, V, q_scale, k_scale, v_scale, O)


def dd_bidir_attention_mx(Q, Qs, K, Ks, V, Vs, O=None):
    """Verifier attention on block-scaled inputs: Q [B,H,N,d], K [B,Hkv,N,d] e4m3 codes, V [B,Hkv,N,d/2] packed e2m1
    codes, each with E8M0 scales [..., d/32] (all uint8) -> O bf16 (as int16 bit patterns unless O is given)."""
    return native().bidir_mx(Q, Qs, K, Ks, V, Vs, O)


def dd_block_attention_cached_fp8v(Qblk, Kc, Vc, block_start: int, q_scale, k_scale, v_scale, O=None, Kblk=None, Vblk=None):
    """Drafter attention with every operand stored as e4m3 codes; shapes as for dd_block_attention_cached -> O bf16."""
    return native().block_fp8v(Qblk, Kc, Vc, block_start, q_scale, k_scale, v_scale, O, Kblk, Vblk)


def dd_block_attention_refresh_workspace_bytes(block_len, B, H, Hkv, N, d, qk_dtype, v_dtype) -> int:
    return lib().dd_block_attention_refresh_workspace_bytes(block_len, B, H, Hkv, N, d, qk_dtype, v_dtype)


def dd_block_attention_refresh(Qblk, Kc, Vc, block_start: int, Kblk, Vblk, O=None, q_scale=None, k_scale=None,
                               qk_dtype: Optional[int] = None, v_dtype: Optional[int] = None):
    """Drafter attention of a completed block: as dd_block_attention_cached with Kblk/Vblk, and rows
    [block_start, block_start + bl) of Kc / Vc are overwritten with Kblk / Vblk in the same call."""
    return dd_block_attention_cached(Qblk, Kc, Vc, block_start, O=O, Kblk=Kblk, Vblk=Vblk, q_scale=q_scale,
                                     k_scale=k_scale, qk_dtype=qk_dtype, v_dtype=v_dtype, _refresh=True)


def dd_block_attention_window_workspace_bytes(block_len, win_len, B, H, Hkv, N, d, qk_dtype, v_dtype) -> int:
    return lib().dd_block_attention_window_workspace_bytes(block_len, win_len, B, H, Hkv, N, d, qk_dtype, v_dtype)


def dd_block_attention_window(Qblk, Kc, Vc, block_start: int, win_start: int, win_len: int, O=None, Kblk=None,
                              Vblk=None, q_scale=None, k_scale=None, qk_dtype: Optional[int] = None,
                              v_dtype: Optional[int] = None):
    """Drafter attention over the key rows [win_start, win_start + win_len) of the cache only.
    Shapes as for dd_block_attention_cached (Kc, Vc are the whole cache)."""
    return native().block(2, Qblk, Kc, Vc, block_start, win_start, win_len, O, Kblk, Vblk, q_scale, k_scale,
                          qk_dtype, v_dtype)


def dd_block_attention_batched(Qblk, Kc, Vc, block_starts, Kblk, Vblk, O=None, q_scale=None, k_scale=None,
                               qk_dtype: Optional[int] = None, v_dtype: Optional[int] = None):
    """Drafter attention with one block position per batch entry: block_starts [B] i32 on the device."""
    return native().block(3, Qblk, Kc, Vc, block_starts, 0, 0, O, Kblk, Vblk, q_scale, k_scale, qk_dtype, v_dtype)


def dd_cache_insert_rows(Kc, Vc, Krows, Vrows, positions, qk_dtype: Optional[int] = None, v_dtype: Optional[int] = None):
    """Kc/Vc [B,Hkv,N,d] <- rows of Krows/Vrows [B,Hkv,n,d] at positions [B,n] (i32, on the device; entries outside
    [0, N) skip their row).  In place; returns None."""
    native().cache_insert(Kc, Vc, Krows, Vrows, positions, qk_dtype, v_dtype)


def dd_qk_norm_rope(Q, K=None, q_weight=None, k_weight=None, eps: float = 1e-6, inv_freq=None, positions=None,
                    interleaved: bool = False, Qo=None, Ko=None, dtype: Optional[int] = None):
    """Head norms and the rotation by position, from a projection's rows to dense queries and keys.  Q [B,H,n,d],
    K [B,Hkv,n,d] (optional): any strides, the last dimension contiguous (q.view(B,n,H,d).transpose(1,2) of a fused
    projection); weights [d] of the same type; inv_freq [rot_dim/2] f32; positions [B,n] i32 (default 0..n-1).
    Returns (Qo, Ko), contiguous; Ko is None without K."""
    return native().qk_norm_rope(Q, K, q_weight, k_weight, eps, inv_freq, positions, interleaved, Qo, Ko, dtype)


def dd_paged_cache_append(Kc, Vc, K, V, block_table, starts, kv_lens=None, n_rows=None, k_scale=None, v_scale=None, k_weight=None,
                          eps: float = 1e-6, inv_freq=None, interleaved: bool = False, row_dtype: Optional[int] = None,
                          cache_dtype: Optional[int] = None):
    """Rows K, V [B,Hkv,n,d] (any strides) into the pages Kc [pages,Hkv,page_size,d], Vc [pages,Hkv,d,page_size] of their
    sequences: row r of sequence b to position starts[b] + r, keys normed (k_weight) and rotated (inv_freq) on the way.  bf16
    pages, or e4m3 pages with k_scale, v_scale [pages,Hkv] f32.  block_table [B,max_pages], starts, kv_lens (lengths before the
    call; default: starts), n_rows (default: n) [B]: i32, on the device.  In place; returns None."""
    native().paged_append(Kc, Vc, K, V, block_table, starts, kv_lens, n_rows, k_scale, v_scale, k_weight, eps, inv_freq, interleaved,
                          row_dtype, cache_dtype)


def dd_paged_resize_workspace_bytes(n, B, page_size, max_pages) -> int:
    return lib().dd_paged_resize_workspace_bytes(n, B, page_size, max_pages)


def dd_paged_resize(block_table, free_pages, num_free, lens, new_lens, page_size: int, n: int = 0, out_lens=None, positions=None, slots=None):
    """Sequences of lens [B] positions grow or shrink to new_lens [B]: pages that are over go back from block_table [B,max_pages] to
    the stack free_pages [pages] (its first num_free [1] entries are free), what is missing is taken from there, in place; a
    sequence whose pages are not there stays as it is, and so do those behind it that ask for any.  All int32 on the device.  Returns (out_lens [B]: the lengths now; positions
    [B,n] and slots [B,n] of the n rows behind lens: page * page_size + offset, -1 where the sequence has none; None each for n == 0)."""
    return native().paged_resize(block_table, free_pages, num_free, lens, new_lens, page_size, n, out_lens, positions, slots)


def dd_paged_attention_workspace_bytes(n, B, H, Hkv, d, page_size, max_pages, cache_dtype) -> int:
    return lib().dd_paged_attention_workspace_bytes(n, B, H, Hkv, d, page_size, max_pages, cache_dtype)


def dd_paged_attention(Q, Kc, Vc, block_table, kv_lens, k_scale=None, v_scale=None, O=None, cache_dtype: Optional[int] = None):
    """Attention of Q [B,H,n,d] (bf16) over the kv_lens[b] positions that each sequence holds in a paged cache (shapes as for
    dd_paged_cache_append) -> O [B,H,n,d] bf16; a sequence that holds none gets zeros."""
    return native().paged_attention(Q, Kc, Vc, block_table, kv_lens, k_scale, v_scale, O, cache_dtype)


def dd_paged_attention_shared_workspace_bytes(n, B, H, Hkv, d, page_size, G, max_prefix_pages, max_pages, cache_dtype) -> int:
    return lib().dd_paged_attention_shared_workspace_bytes(n, B, H, Hkv, d, page_size, G, max_prefix_pages, max_pages, cache_dtype)


def dd_paged_attention_shared(Q, Kc, Vc, prefix_table, prefix_lens, group_starts, block_table, kv_lens, k_scale=None, v_scale=None, O=None,
                              cache_dtype: Optional[int] = None):
    """dd_paged_attention for sequences that share prefixes: sequences group_starts[g] .. group_starts[g+1] - 1 attend the
    prefix_lens[g] positions on the pages prefix_table[g] and then their own kv_lens[b] on block_table[b]; a prefix is read once for all
    of them where that pays by sizes and capacities, else by each sequence in one go with its own.  prefix_table [G,max_prefix_pages], prefix_lens [G], group_starts [G+1], not descending: i32, on the device."""
    return native().paged_attention_shared(Q, Kc, Vc, prefix_table, prefix_lens, group_starts, block_table, kv_lens, k_scale, v_scale, O, cache_dtype)


def dd_verify_remask_workspace_bytes(B, G, V, logit_dtype) -> int:
    return lib().dd_verify_remask_workspace_bytes(B, G, V, logit_dtype)


def dd_verify_remask(logits_d, logits_v, mask, mode: int, threshold: float, seed: int, B: int, G: int,
                     out_mask=None, out_tokens=None, out_scores=None, logit_dtype: Optional[int] = None):
    """Verification rule over the vocabulary.  logits [B*G, V]; mask [B*G] u8 (1 = still masked).
    Returns (out_mask u8, out_tokens i32, out_scores f32)."""
    return native().verify_remask(0, logits_d, logits_v, mask, mode, threshold, seed, B, G, out_mask, out_tokens, out_scores,
                                  logit_dtype)


def dd_verify_remask_static(logits_d, logits_v, mask, mode: int, threshold: float, seed: int, B: int, G: int,
                            out_mask, out_tokens, out_scores, logit_dtype: Optional[int] = None):
    """dd_verify_remask without a workspace: the library's static device array holds the partial states.  The
    three output tensors are the caller's (nothing is allocated here either).  Returns them."""
    return native().verify_remask(1, logits_d, logits_v, mask, mode, threshold, seed, B, G, out_mask, out_tokens, out_scores,
                                  logit_dtype)


def dd_unmask_workspace_bytes(B, G, V, logit_dtype) -> int:
    return lib().dd_unmask_workspace_bytes(B, G, V, logit_dtype)


def dd_unmask(logits_d, mask, mode: int, threshold: float, B: int, G: int, x_tokens=None, out_mask=None,
              out_tokens=None, out_conf=None, logit_dtype: Optional[int] = None):
    """One drafter unmasking step.  logits_d [B*G, V]; mask [B*G] u8 (1 = still masked); x_tokens [B*G] i32
    (optional, updated in place where a position is revealed).  Returns (out_mask u8, out_tokens i32, out_conf f32)."""
    return native().unmask(logits_d, mask, mode, threshold, B, G, x_tokens, out_mask, out_tokens, out_conf, logit_dtype)


def dd_verify_scores_workspace_bytes(P, V, logit_dtype) -> int:
    return lib().dd_verify_scores_workspace_bytes(P, V, logit_dtype)


def dd_verify_scores(logits_d, logits_v, drafter: bool = True, logit_dtype: Optional[int] = None):
    """Divergence, both confidences and both argmax tokens of every row in one pass.  logits_d, logits_v [P, V].
    Returns (kl f32, conf_v f32, tok_v i32, conf_d f32 | None, tok_d i32 | None)."""
    return native().verify_scores(logits_d, logits_v, drafter, logit_dtype)


def dd_verify_draft_workspace_bytes(B, n, bonus, V, with_drafter, logit_dtype) -> int:
    return lib().dd_verify_draft_workspace_bytes(B, n, bonus, V, with_drafter, logit_dtype)


def dd_verify_draft(logits_v, logits_d, tokens, uniforms, temperature=None, n_draft=None, out_tokens=None, out_accepted=None,
                    out_chances=None, logit_dtype: Optional[int] = None):
    """Drafted tokens [B,n] i32 against the verifier's probabilities, by given random numbers: uniforms [B,n+1] f32 (the last one
    draws the token behind the drafts that stand).  logits_v [B,n+1,V], or [B,n,V] for no token behind a draft that stands whole;
    logits_d [B,n,V], or None where the drafter was sure of its tokens; temperature [B] f32 (0: the largest logit; default 1);
    n_draft [B] i32 (default n).  Returns (tokens [B,n+1] i32: kept drafts, the drawn token, then -1; accepted [B] i32; chances
    [B,n] f32: the probability with which each draft stands)."""
    return native().verify_draft(logits_v, logits_d, tokens, uniforms, temperature, n_draft, out_tokens, out_accepted, out_chances, logit_dtype)
