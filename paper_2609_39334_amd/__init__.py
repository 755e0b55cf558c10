"""Python binding of libtreekv.so: tree-shared paged attention for speculative search on MI355X.

Argument marshalling only -- every step of the path (block manager, coalescing, planning and the
attention kernels) runs in the C/HIP library; PyTorch provides device memory and streams.  The
functions carry the names of the C entry points in include/treekv.h; failures raise TkvError
with the library's message.  The library must be built first (``python -m
paper_2609_39334_amd.build``); any entry point raises if it is missing -- there is no fallback.
"""
from __future__ import annotations

import ctypes
import os
import struct
from typing import Optional, Sequence

import numpy as np
import torch  # imported before the library so that both share torch's HIP runtime

HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(HERE, "libtreekv.so")

TKV_OK, TKV_EINVAL, TKV_ENOMEM, TKV_ENOSEQ, TKV_ECAP, TKV_EHIP = 0, -1, -2, -3, -4, -5
TKV_NOALLOC_MAX_BYTES = 64 << 20   # the static workspace of tkv_verify_noalloc (treekv.h)


class TkvError(RuntimeError):
    def __init__(self, code: int, msg: str):
        super().__init__(f"[{code}] {msg}")
        self.code = code


class tkv_shape(ctypes.Structure):
    _fields_ = [("hq", ctypes.c_int32), ("hkv", ctypes.c_int32), ("d", ctypes.c_int32),
                ("block_size", ctypes.c_int32), ("num_blocks", ctypes.c_int32)]


class tkv_plan_options(ctypes.Structure):
    _fields_ = [(n, ctypes.c_int32) for n in ("wave_max_rows", "tile_min_items", "waves", "tile8_max_items",
                                              "wide_chunk_blocks", "fold_blocks")]


class tkv_plan_stats(ctypes.Structure):
    _fields_ = [(n, ctypes.c_int32) for n in ("n_rows", "n_qtok", "n_items", "n_items_shared", "n_items_row",
                                              "n_slots", "n_merge", "n_segments", "n_shared_segments",
                                              "n_items_wave", "n_waves", "n_idle_waves")] + \
               [(n, ctypes.c_int64) for n in ("logical_qtok", "uniq_kv_tokens", "path_kv_tokens", "flops")]


class tkv_plan_layout(ctypes.Structure):
    _fields_ = [(n, ctypes.c_size_t) for n in ("items", "toks", "blks", "merges", "merge_slots", "wave_records",
                                               "wave_off", "wave_tiles", "end")]


class tkv_plan_view(ctypes.Structure):
    _fields_ = [(n, ctypes.POINTER(ctypes.c_int32)) for n in ("items", "toks", "blks", "merges", "merge_slots")] + \
               [(n, ctypes.c_int32) for n in ("n_items", "n_toks", "n_blks", "n_merge", "n_merge_slots", "n_slots")]


class tkv_draft_batch(ctypes.Structure):
    _fields_ = [(n, ctypes.c_int32) for n in ("n_rows", "n_qtok", "max_q", "n_kv_blocks", "max_blocks", "mask_words")] + \
               [(n, ctypes.c_void_p) for n in ("q_indptr", "kv_indptr", "kv_blocks", "block_len", "mask")]


class tkv_evict_batch(ctypes.Structure):
    _fields_ = [(n, ctypes.c_int32) for n in ("n_rows", "n_kv_blocks", "max_blocks", "n_new_blocks", "max_budget", "sink",
                                              "recent")] + \
               [(n, ctypes.c_void_p) for n in ("kv_indptr", "kv_blocks", "block_len", "new_indptr", "new_blocks", "budget")]


class tkv_logit_rules(ctypes.Structure):
    _fields_ = [(n, ctypes.c_void_p) for n in ("prompt_len", "repetition", "presence", "frequency", "bias_indptr", "bias_token",
                                               "bias_value", "grammar", "allowed")] + \
               [(n, ctypes.c_int32) for n in ("n_bias", "n_grammars", "allowed_words")]


_P = ctypes.c_void_p
_I32 = ctypes.c_int32
_PI32 = ctypes.POINTER(ctypes.c_int32)
_PU8 = ctypes.POINTER(ctypes.c_uint8)
_SIG = {
    "tkv_last_error": (ctypes.c_char_p, []),
    "tkv_bm_create": (ctypes.c_int, [_I32, _I32, _I32, ctypes.POINTER(_P)]),
    "tkv_bm_destroy": (None, [_P]),
    "tkv_bm_extend": (ctypes.c_int, [_P, _I32, _PI32, _I32, _I32, _PI32, _PI32, _PU8, _I32, _PI32]),
    "tkv_prune": (ctypes.c_int, [_P, _I32, _PI32, _I32, _PI32]),
    "tkv_bm_append": (ctypes.c_int, [_P, _I32, _PI32, _I32, _PI32, _I32]),
    "tkv_bm_seal": (ctypes.c_int, [_P, _I32, _PI32, _I32, _PI32]),
    "tkv_bm_fork": (ctypes.c_int, [_P, _I32, _PI32, _I32, _PI32, _I32]),
    "tkv_extend_slots": (ctypes.c_int, [_PI32, _PU8, _I32, _I32, _I32, _PI32]),
    "tkv_bm_table": (ctypes.c_int, [_P, _I32, _PI32, _I32, _PI32, _PI32]),
    "tkv_bm_refcount": (ctypes.c_int, [_P, _I32, _PI32]),
    "tkv_bm_block_len": (ctypes.c_int, [_P, _PI32]),
    "tkv_bm_snapshot": (ctypes.c_int, [_P, _P, ctypes.c_size_t, ctypes.POINTER(ctypes.c_size_t)]),
    "tkv_bm_coalesce": (ctypes.c_int, [_P, _I32, _PI32, _PI32, _PI32, _PI32, _PI32, _PI32]),
    "tkv_plan_create": (ctypes.c_int, [ctypes.POINTER(tkv_shape), _I32, _PI32, _PI32, _PI32, _PI32, _PI32,
                                       ctypes.POINTER(_P)]),
    "tkv_plan_create_ex": (ctypes.c_int, [ctypes.POINTER(tkv_shape), _I32, _PI32, _PI32, _PI32, _PI32, _PI32,
                                          ctypes.POINTER(tkv_plan_options), ctypes.POINTER(_P)]),
    "tkv_plan_workspace_bytes": (ctypes.c_size_t, [_P]),
    "tkv_plan_upload": (ctypes.c_int, [_P, _P, ctypes.c_size_t, _P]),
    "tkv_plan_update": (ctypes.c_int, [_P, _P, _P, _P, ctypes.POINTER(ctypes.c_int32)]),
    "tkv_plan_image": (ctypes.c_int, [_P, ctypes.POINTER(_P), ctypes.POINTER(tkv_plan_layout)]),
    "tkv_plan_dirty": (ctypes.c_int, [_P, ctypes.POINTER(_PI32), ctypes.POINTER(ctypes.c_int32),
                                      ctypes.POINTER(ctypes.c_int32)]),
    "tkv_plan_destroy": (None, [_P]),
    "tkv_plan_get_stats": (ctypes.c_int, [_P, ctypes.POINTER(tkv_plan_stats)]),
    "tkv_plan_get_view": (ctypes.c_int, [_P, ctypes.POINTER(tkv_plan_view)]),
    "tkv_decode": (ctypes.c_int, [_P, _P, _P, _P, _P, _P, _P]),
    "tkv_verify": (ctypes.c_int, [_P, _P, _P, _P, _P, _P, _P]),
    "tkv_verify_noalloc": (ctypes.c_int, [_P, _P, _P, _P, _P, _P, _P]),
    "tkv_kv_append": (ctypes.c_int, [ctypes.POINTER(tkv_shape), _P, _I32, _P, _P, _P, _P, _P]),
    "tkv_draft_mask": (ctypes.c_int, [_I32, _PI32, _I32, _P, _PI32]),
    "tkv_draft_workspace_bytes": (ctypes.c_int, [ctypes.POINTER(tkv_shape), ctypes.POINTER(tkv_draft_batch),
                                                 ctypes.POINTER(ctypes.c_size_t)]),
    "tkv_draft_verify": (ctypes.c_int, [ctypes.POINTER(tkv_shape), ctypes.POINTER(tkv_draft_batch), _P, _P, _P, _P, _P, _P,
                                        ctypes.c_size_t, _P]),
    # (shape, batch and rules of these three go as packed bytes: 0.4 us a structure instead of 1.2)
    "tkv_key_weights": (ctypes.c_int, [_P, _P, _P, _P, _P, _P, ctypes.c_float, _P, _P, ctypes.c_int64, _P]),
    "tkv_evict_keys": (ctypes.c_int, [_P, _P, _P, _P, ctypes.c_int64, _P, _P, _P, _P, _P]),
    "tkv_add_rmsnorm": (ctypes.c_int, [_I32, _I32, ctypes.c_float, _P, _P, _P, _P, _P]),
    "tkv_rope_append": (ctypes.c_int, [ctypes.POINTER(tkv_shape), _I32, _P, _P, _P, _P, _P, _P, _P, _P]),
    "tkv_norm_rope_append": (ctypes.c_int, [ctypes.POINTER(tkv_shape), _I32, _P, ctypes.c_int64, _P, _P, ctypes.c_float, _P, _P,
                                            _I32, _P, _P, _P, _P, _P]),
    "tkv_swiglu": (ctypes.c_int, [_I32, _I32, _P, _P, _P]),
    "tkv_cd_sample": (ctypes.c_int, [_I32, _I32, ctypes.c_float, _I32, _P, _P, _P, _I32, _P, _P, _P, _P]),
    "tkv_filter_sample_workspace_bytes": (ctypes.c_size_t, [_I32, _I32]),
    "tkv_filter_sample": (ctypes.c_int, [_I32, _I32, _I32, _P, ctypes.c_int64, _P, _P, _P, _P, _I32, _P, _P, _I32, _P, _P, _P, _P,
                                         ctypes.c_size_t, _P]),
    "tkv_adjust_logits": (ctypes.c_int, [_I32, _P, _P, _P, _I32, _I32, _P, ctypes.c_int64, _I32, _P, ctypes.c_int64, _P]),
    "tkv_search_create": (ctypes.c_int, [_I32, _I32, _I32, _I32, ctypes.POINTER(_P)]),
    "tkv_search_destroy": (None, [_P]),
    "tkv_search_expand": (ctypes.c_int, [_P, _I32, _I32, _PI32]),
    "tkv_search_complete": (ctypes.c_int, [_P, _I32, _I32, _PI32]),
    "tkv_search_tick": (ctypes.c_int, [_P, _PI32]),
    "tkv_search_flush": (ctypes.c_int, [_P, _PI32, _I32, _PI32]),
    "tkv_search_score": (ctypes.c_int, [_P, _I32, _PI32, ctypes.POINTER(ctypes.c_float)]),
    "tkv_search_pruned": (ctypes.c_int, [_P, _PI32, _I32, _PI32]),
    "tkv_search_node": (ctypes.c_int, [_P, _I32, _PI32, _PI32, _PI32, ctypes.POINTER(ctypes.c_float)]),
    "tkv_search_round": (ctypes.c_int, [_P, _I32, _PI32, _I32, _PI32, _PI32]),
    "tkv_search_snapshot": (ctypes.c_int, [_P, _P, ctypes.c_size_t, ctypes.POINTER(ctypes.c_size_t)]),
    "tkv_plan_profile": (ctypes.c_int, [_P, _I32]),
    "tkv_plan_profile_read": (ctypes.c_int, [_P, _PI32, ctypes.POINTER(ctypes.c_float), ctypes.POINTER(ctypes.c_float)]),
}
EXPORTED = tuple(_SIG)
_pack_shape, _pack_draft = struct.Struct("@5i").pack, struct.Struct("@6i5P").pack          # tkv_shape, tkv_draft_batch
_pack_evict, _pack_rules = struct.Struct("@7i6P0P").pack, struct.Struct("@9P3i0P").pack    # tkv_evict_batch, tkv_logit_rules

_lib = None


def lib() -> ctypes.CDLL:
    """The loaded libtreekv.so (raises if it has not been built)."""
    global _lib
    if _lib is None:
        if not os.path.exists(LIB_PATH):
            raise RuntimeError(f"{LIB_PATH} is not built: run `python -m paper_2609_39334_amd.build` "
                               "(or __graft_entry__.build()) first")
        L = ctypes.CDLL(LIB_PATH)
        for name, (res, args) in _SIG.items():
            f = getattr(L, name)
            f.restype = res
            f.argtypes = args
        _lib = L
    return _lib


def _check(rc: int) -> None:
    if rc != TKV_OK:
        raise TkvError(rc, lib().tkv_last_error().decode())


def _i32(a) -> np.ndarray:
    return np.ascontiguousarray(np.asarray(a, dtype=np.int32).reshape(-1))


def _ptr(a: np.ndarray):
    return a.ctypes.data_as(_PI32)


def _stream(stream) -> Optional[int]:
    if stream is None:
        return torch.cuda.current_stream().cuda_stream
    return getattr(stream, "cuda_stream", stream)


# ------------------------------------------------------------------------- C entry points

def tkv_last_error() -> str:
    return lib().tkv_last_error().decode()


def tkv_bm_create(num_blocks: int, block_size: int, max_seqs: int) -> int:
    h = _P()
    _check(lib().tkv_bm_create(num_blocks, block_size, max_seqs, ctypes.byref(h)))
    return h.value


def tkv_bm_destroy(bm: int) -> None:
    lib().tkv_bm_destroy(bm)


def tkv_bm_extend(bm: int, parent: int, tokens, seal: bool, block_size: int = 16):
    """Returns (seq, block ids, hit flags) of the new sequence's step."""
    t = _i32(tokens)
    cap = max(1, -(-len(t) // block_size))
    blk = np.zeros(cap, dtype=np.int32)
    hit = np.zeros(cap, dtype=np.uint8)
    child, n = _I32(), _I32()
    _check(lib().tkv_bm_extend(bm, parent, _ptr(t), len(t), int(bool(seal)), ctypes.byref(child), _ptr(blk),
                               hit.ctypes.data_as(_PU8), cap, ctypes.byref(n)))
    return child.value, blk[:n.value].copy(), hit[:n.value].copy()


def tkv_prune(bm: int, seq: int, cap: int = None) -> np.ndarray:
    """Releases a sequence; returns the freed block ids in table order."""
    if cap is None:
        n, _ = _table_len(bm, seq)
        cap = max(1, n)
    out = np.zeros(cap, dtype=np.int32)
    n = _I32()
    _check(lib().tkv_prune(bm, seq, _ptr(out), cap, ctypes.byref(n)))
    return out[:n.value].copy()


def tkv_bm_append(bm: int, seq: int, tokens) -> np.ndarray:
    """Grows a sequence in place; returns each token's pool slot (block * block_size + slot)."""
    t = _i32(tokens)
    dst = np.zeros(max(1, len(t)), dtype=np.int32)
    _check(lib().tkv_bm_append(bm, seq, _ptr(t), len(t), _ptr(dst), len(t)))
    return dst[:len(t)].copy()


def tkv_bm_seal(bm: int, seq: int):
    """Completes the open step of a sequence; returns the (own block, sealed block) replacements."""
    n = _I32()
    rc = lib().tkv_bm_seal(bm, seq, None, 0, ctypes.byref(n))
    if rc == TKV_OK:
        return []
    if rc != TKV_ECAP:
        _check(rc)
    out = np.zeros(2 * n.value, dtype=np.int32)
    _check(lib().tkv_bm_seal(bm, seq, _ptr(out), n.value, ctypes.byref(n)))
    return [(int(out[2 * i]), int(out[2 * i + 1])) for i in range(n.value)]


def tkv_bm_fork(bm: int, seq: int, tokens) -> list:
    """Branches a sequence: seals its open step, then one open child per token; returns the children."""
    t = _i32(tokens)
    out = np.zeros(max(1, len(t)), dtype=np.int32)
    _check(lib().tkv_bm_fork(bm, seq, _ptr(t), len(t), _ptr(out), len(t)))
    return [int(x) for x in out[:len(t)]]


def tkv_extend_slots(blk, hit, n_tok: int, block_size: int = 16) -> np.ndarray:
    """Pool slots of a new step's tokens (-1 where the block was a deduplication hit)."""
    b = _i32(blk)
    h = np.ascontiguousarray(np.asarray(hit, dtype=np.uint8).reshape(-1))
    dst = np.zeros(max(1, n_tok), dtype=np.int32)
    _check(lib().tkv_extend_slots(_ptr(b), h.ctypes.data_as(_PU8), len(b), n_tok, block_size, _ptr(dst)))
    return dst[:n_tok].copy()


def _table_len(bm: int, seq: int):
    n, kv = _I32(), _I32()
    rc = lib().tkv_bm_table(bm, seq, None, 0, ctypes.byref(n), ctypes.byref(kv))
    if rc not in (TKV_OK, TKV_ECAP):
        _check(rc)
    return n.value, kv.value


def tkv_bm_table(bm: int, seq: int):
    """Returns (block table, kv_len)."""
    n, _ = _table_len(bm, seq)
    out = np.zeros(max(1, n), dtype=np.int32)
    nn, kv = _I32(), _I32()
    _check(lib().tkv_bm_table(bm, seq, _ptr(out), len(out), ctypes.byref(nn), ctypes.byref(kv)))
    return out[:nn.value].copy(), kv.value


def tkv_bm_refcount(bm: int, blk: int) -> int:
    rc = _I32()
    _check(lib().tkv_bm_refcount(bm, blk, ctypes.byref(rc)))
    return rc.value


def tkv_bm_block_len(bm: int, num_blocks: int) -> np.ndarray:
    out = np.zeros(num_blocks, dtype=np.int32)
    _check(lib().tkv_bm_block_len(bm, _ptr(out)))
    return out


def tkv_bm_snapshot(bm: int, seqs: bool = True) -> dict:
    """Parsed state; seqs=False skips decoding the per-sequence tables."""
    used = ctypes.c_size_t()
    lib().tkv_bm_snapshot(bm, None, 0, ctypes.byref(used))
    buf = np.zeros(used.value // 4, dtype=np.int32)
    _check(lib().tkv_bm_snapshot(bm, buf.ctypes.data_as(_P), used.value, ctypes.byref(used)))
    nb, bs, ms, nlive = (int(x) for x in buf[:4])
    w = 4
    snap = {"refcount": buf[w:w + nb].copy(), "block_len": buf[w + nb:w + 2 * nb].copy(),
            "indexed": buf[w + 2 * nb:w + 3 * nb].copy(), "seqs": {}}
    w += 3 * nb
    for _ in range(nlive if seqs else 0):
        s, sealed, n_open, n = (int(x) for x in buf[w:w + 4])
        snap["seqs"][s] = (tuple(int(b) for b in buf[w + 4:w + 4 + n]), sealed, n_open)
        w += 4 + n
    return snap


def tkv_bm_coalesce(bm: int, seqs: Sequence[int], q_lens: Sequence[int]):
    """Returns (row of each candidate, first candidate of each row, multiplicity of each row)."""
    s, q = _i32(seqs), _i32(q_lens)
    n = len(s)
    row_of = np.zeros(max(1, n), dtype=np.int32)
    first = np.zeros(max(1, n), dtype=np.int32)
    mult = np.zeros(max(1, n), dtype=np.int32)
    nr = _I32()
    _check(lib().tkv_bm_coalesce(bm, n, _ptr(s), _ptr(q), _ptr(row_of), _ptr(first), _ptr(mult), ctypes.byref(nr)))
    return row_of[:n].copy(), first[:nr.value].copy(), mult[:nr.value].copy()


def tkv_plan_create(shape, q_indptr, kv_indptr, kv_blocks, block_len, multiplicity=None) -> int:
    """shape = (hq, hkv, d, block_size, num_blocks)."""
    sh = tkv_shape(*[int(x) for x in shape])
    qi, ki, kb, bl = _i32(q_indptr), _i32(kv_indptr), _i32(kv_blocks), _i32(block_len)
    mu = None if multiplicity is None else _i32(multiplicity)
    h = _P()
    _check(lib().tkv_plan_create(ctypes.byref(sh), len(qi) - 1, _ptr(qi), _ptr(ki), _ptr(kb) if len(kb) else None,
                                 _ptr(bl), None if mu is None else _ptr(mu), ctypes.byref(h)))
    return h.value


def tkv_plan_create_ex(shape, q_indptr, kv_indptr, kv_blocks, block_len, multiplicity=None, options=None) -> int:
    """tkv_plan_create with placement options: a dict over the tkv_plan_options fields (missing
    fields, or None, keep the defaults)."""
    sh = tkv_shape(*[int(x) for x in shape])
    qi, ki, kb, bl = _i32(q_indptr), _i32(kv_indptr), _i32(kv_blocks), _i32(block_len)
    mu = None if multiplicity is None else _i32(multiplicity)
    opts = None
    if options is not None:
        unknown = set(options) - {f for f, _ in tkv_plan_options._fields_}
        if unknown:
            raise ValueError(f"unknown plan options {sorted(unknown)}")
        opts = tkv_plan_options(*[int(options.get(f, -1)) for f, _ in tkv_plan_options._fields_])
    h = _P()
    _check(lib().tkv_plan_create_ex(ctypes.byref(sh), len(qi) - 1, _ptr(qi), _ptr(ki), _ptr(kb) if len(kb) else None,
                                    _ptr(bl), None if mu is None else _ptr(mu),
                                    None if opts is None else ctypes.byref(opts), ctypes.byref(h)))
    return h.value


def tkv_plan_workspace_bytes(plan: int) -> int:
    return int(lib().tkv_plan_workspace_bytes(plan))


def tkv_plan_upload(plan: int, workspace: torch.Tensor, stream=None) -> None:
    _check(lib().tkv_plan_upload(plan, workspace.data_ptr(), workspace.numel() * workspace.element_size(),
                                 _stream(stream)))


def tkv_plan_destroy(plan: int) -> None:
    lib().tkv_plan_destroy(plan)


def tkv_plan_update(plan: int, kv_indptr, kv_blocks, block_len) -> bool:
    """Bring the plan to new tables for the same rows; True if it was patched in place, False if
    it was planned again.  It must be uploaded again either way."""
    ki, kb, bl = _i32(kv_indptr), _i32(kv_blocks), _i32(block_len)
    flag = ctypes.c_int32(0)
    _check(lib().tkv_plan_update(plan, _ptr(ki), _ptr(kb) if len(kb) else None, _ptr(bl), ctypes.byref(flag)))
    return bool(flag.value)


def tkv_plan_dirty(plan: int):
    """(word indices the plan's in-place updates changed since its last upload, complete?)."""
    words, n, complete = _PI32(), ctypes.c_int32(0), ctypes.c_int32(0)
    _check(lib().tkv_plan_dirty(plan, ctypes.byref(words), ctypes.byref(n), ctypes.byref(complete)))
    idx = np.ctypeslib.as_array(words, shape=(n.value,)).copy() if n.value else np.zeros(0, dtype=np.int32)
    return idx, bool(complete.value)


def tkv_plan_image(plan: int):
    """A copy of the plan's host descriptor image (what tkv_plan_upload copies) and the byte
    offsets of its sections: (bytes, dict)."""
    data, lay = _P(), tkv_plan_layout()
    _check(lib().tkv_plan_image(plan, ctypes.byref(data), ctypes.byref(lay)))
    layout = {f: int(getattr(lay, f)) for f, _ in tkv_plan_layout._fields_}
    return (ctypes.string_at(data.value, layout["end"]) if layout["end"] else b""), layout


def tkv_plan_get_stats(plan: int) -> dict:
    st = tkv_plan_stats()
    _check(lib().tkv_plan_get_stats(plan, ctypes.byref(st)))
    return {n: int(getattr(st, n)) for n, _ in tkv_plan_stats._fields_}


def tkv_plan_get_view(plan: int) -> dict:
    v = tkv_plan_view()
    _check(lib().tkv_plan_get_view(plan, ctypes.byref(v)))

    def arr(p, n, w):
        if n == 0:
            return np.zeros((0, w), dtype=np.int32)
        return np.ctypeslib.as_array(p, shape=(n * w,)).reshape(n, w).copy()
    return {"items": arr(v.items, v.n_items, 8), "toks": arr(v.toks, v.n_toks, 4), "blks": arr(v.blks, v.n_blks, 2),
            "merges": arr(v.merges, v.n_merge, 4),
            "merge_slots": arr(v.merge_slots, v.n_merge_slots, 1).reshape(-1), "n_slots": int(v.n_slots)}


def _attn(fn, plan, q, k, v, o, lse, stream):
    for name, t in (("q", q), ("k", k), ("v", v), ("o", o)):
        if not (t.is_cuda and t.dtype == torch.bfloat16 and t.is_contiguous()):
            raise TkvError(TKV_EINVAL, f"{name} must be a contiguous bfloat16 device tensor")
    if lse is not None and not (lse.is_cuda and lse.dtype == torch.float32 and lse.is_contiguous()):
        raise TkvError(TKV_EINVAL, "lse must be a contiguous float32 device tensor")
    _check(fn(plan, q.data_ptr(), k.data_ptr(), v.data_ptr(), o.data_ptr(),
              None if lse is None else lse.data_ptr(), _stream(stream)))


def tkv_decode(plan: int, q, k, v, o, lse=None, stream=None) -> None:
    _attn(lib().tkv_decode, plan, q, k, v, o, lse, stream)


def tkv_verify(plan: int, q, k, v, o, lse=None, stream=None) -> None:
    _attn(lib().tkv_verify, plan, q, k, v, o, lse, stream)


def tkv_verify_noalloc(plan: int, q, k, v, o, lse=None, stream=None) -> None:
    """tkv_verify on the library's static workspace (the plan need not be uploaded)."""
    _attn(lib().tkv_verify_noalloc, plan, q, k, v, o, lse, stream)


def tkv_kv_append(dst: torch.Tensor, k_new: torch.Tensor, v_new: torch.Tensor, k: torch.Tensor, v: torch.Tensor,
                  stream=None) -> None:
    """Writes new tokens' K/V rows into the paged pool at their slots (dst int32, -1 = skip).
    k_new, v_new: [n_tok, hkv, d] bf16; k, v: [num_blocks, hkv, block_size, d] bf16 (all on the GPU)."""
    nb, hkv, bs, d = k.shape
    n = int(dst.numel())
    for t, shp in ((k_new, (n, hkv, d)), (v_new, (n, hkv, d)), (v, tuple(k.shape))):
        if tuple(t.shape) != shp or t.dtype != torch.bfloat16 or not t.is_contiguous() or not t.is_cuda:
            raise ValueError(f"tkv_kv_append: expected a contiguous bf16 GPU tensor of shape {shp}, got {tuple(t.shape)}")
    if k.dtype != torch.bfloat16 or not k.is_contiguous() or not k.is_cuda:
        raise ValueError("tkv_kv_append: the pool must be a contiguous bf16 GPU tensor")
    if dst.dtype != torch.int32 or not dst.is_cuda or not dst.is_contiguous():
        raise ValueError("tkv_kv_append: dst must be a contiguous int32 GPU tensor")
    shape = tkv_shape(0, hkv, d, bs, nb)
    _check(lib().tkv_kv_append(ctypes.byref(shape), dst.data_ptr(), n, k_new.data_ptr(), v_new.data_ptr(),
                               k.data_ptr(), v.data_ptr(), _stream(stream)))


def _expect(fn: str, name: str, t: torch.Tensor, dtype, shape) -> None:
    if t.dtype != dtype or tuple(t.shape) != tuple(shape) or not t.is_contiguous() or not t.is_cuda:
        raise ValueError(f"{fn}: {name} must be a contiguous {dtype} GPU tensor of shape {tuple(shape)}, got {t.dtype} "
                         f"{tuple(t.shape)}")


def tkv_add_rmsnorm(x: torch.Tensor, delta: Optional[torch.Tensor], weight: torch.Tensor, eps: float,
                    stream=None) -> torch.Tensor:
    """x [rows, hidden] fp32 += delta (bf16, or None) in place; returns RMSNorm(x) * weight in bf16."""
    rows, hidden = x.shape
    _expect("tkv_add_rmsnorm", "x", x, torch.float32, (rows, hidden))
    _expect("tkv_add_rmsnorm", "weight", weight, torch.float32, (hidden,))
    if delta is not None:
        _expect("tkv_add_rmsnorm", "delta", delta, torch.bfloat16, (rows, hidden))
    h = torch.empty((rows, hidden), dtype=torch.bfloat16, device=x.device)
    _check(lib().tkv_add_rmsnorm(rows, hidden, float(eps), x.data_ptr(), None if delta is None else delta.data_ptr(),
                                 weight.data_ptr(), h.data_ptr(), _stream(stream)))
    return h


def tkv_rope_append(qkv: torch.Tensor, cos: torch.Tensor, sin: torch.Tensor, dst: torch.Tensor, hq: int,
                    k: torch.Tensor, v: torch.Tensor, stream=None) -> torch.Tensor:
    """RoPE of qkv [n, (hq + 2 hkv) * d] bf16; writes k and v rows to the pool slots dst (int32, -1 = skip) and
    returns the rotated queries [n, hq, d].  cos, sin: [n, d / 2] fp32; k, v: the pools."""
    fn = "tkv_rope_append"
    nb, hkv, bs, d = k.shape
    n = int(dst.numel())
    _expect(fn, "qkv", qkv, torch.bfloat16, (n, (hq + 2 * hkv) * d))
    _expect(fn, "cos", cos, torch.float32, (n, d // 2))
    _expect(fn, "sin", sin, torch.float32, (n, d // 2))
    _expect(fn, "k", k, torch.bfloat16, k.shape)
    _expect(fn, "v", v, torch.bfloat16, k.shape)
    _expect(fn, "dst", dst, torch.int32, dst.shape)
    q = torch.empty((n, hq, d), dtype=torch.bfloat16, device=qkv.device)
    shape = tkv_shape(hq, hkv, d, bs, nb)
    _check(lib().tkv_rope_append(ctypes.byref(shape), n, qkv.data_ptr(), cos.data_ptr(), sin.data_ptr(), dst.data_ptr(),
                                 q.data_ptr(), k.data_ptr(), v.data_ptr(), _stream(stream)))
    return q


# A device's current stream as a raw handle, without the stream object around it (0.1 us instead of 1.7).
_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None) or (lambda index: torch.cuda.current_stream(index).cuda_stream)


class _Call:
    """The device and stream of a call: its outputs and workspaces are allocated for that stream, and its work is enqueued
    there (the current stream of the tensors' device without a stream; never the current device's, if that is
    another)."""
    __slots__ = ("index", "device", "side", "handle")

    def __init__(self, fn: str, pool: torch.Tensor, stream):
        self.index, self.device = pool.get_device(), pool.device
        self.handle = _raw_stream(self.index)
        self.side = None  # another stream than the current one
        if stream is None:
            return
        if hasattr(stream, "cuda_stream"):
            if stream.device != self.device:
                raise ValueError(f"{fn}: the stream is {stream.device}'s, the tensors are on {self.device}")
        else:
            stream = torch.cuda.ExternalStream(stream, device=self.device) if stream else torch.cuda.default_stream(self.device)
        if stream.cuda_stream != self.handle:
            self.side, self.handle = stream, stream.cuda_stream

    def empty(self, shape, dtype) -> torch.Tensor:
        if self.side is None:
            return torch.empty(shape, dtype=dtype, device=self.device)
        with torch.cuda.stream(self.side):
            t = torch.empty(shape, dtype=dtype, device=self.device)
        # not handed out again before the current stream's work so far, and its later reads
        t.record_stream(torch.cuda.current_stream(self.device))
        return t

    def uses(self, *tensors) -> None:
        """The call's tensors (None: not given): dropped after it, they are not handed out again before another stream's
        work."""
        if self.side is not None:
            for t in tensors:
                if t is not None:
                    t.record_stream(self.side)

    def run(self, entry, *args) -> None:
        if torch.cuda.current_device() == self.index:
            _check(entry(*args, self.handle))
        else:
            with torch.cuda.device(self.device):
                _check(entry(*args, self.handle))


def _past_32_bits(fn: str) -> ValueError:
    return ValueError(f"{fn}: a size or a number is no whole number of 32 bits")


def _tensors(fn: str, index: int, *specs) -> None:
    """Checks (name, tensor, dtype, shape): contiguous, of that type and shape, on GPU `index`."""
    for name, t, dtype, shape in specs:
        if t.dtype is not dtype or t.shape != shape or t.get_device() != index or index < 0 or not t.is_contiguous():
            raise ValueError(f"{fn}: {name} must be a contiguous {dtype} tensor of shape {tuple(shape)} on GPU {max(index, 0)}, got "
                             f"{t.dtype} {tuple(t.shape)}, strides {t.stride()}, on {t.device}")


def tkv_norm_rope_append(qkv: torch.Tensor, q_weight: torch.Tensor, k_weight: torch.Tensor, eps: float,
                         cos: torch.Tensor, sin: torch.Tensor, dst: torch.Tensor, hq: int, k: torch.Tensor,
                         v: torch.Tensor, stream=None) -> torch.Tensor:
    """tkv_rope_append with a norm of every query and key head (weights [d] fp32) before the rotation.  qkv's rows may
    be a slice of wider ones (row stride a multiple of 8); cos, sin: [n, rot / 2] fp32, of the first rot <= d elements
    of a head (rot a multiple of 16; 0: none)."""
    fn = "tkv_norm_rope_append"
    if k.dim() != 4 or cos.dim() != 2:
        raise ValueError(f"{fn}: k must be a pool [num_blocks, hkv, block_size, d], cos [n, rot / 2]")
    nb, hkv, bs, d = k.shape
    n, half = int(dst.numel()), int(cos.shape[1])
    width = (hq + 2 * hkv) * d
    if (qkv.dtype is not torch.bfloat16 or qkv.shape != (n, width) or qkv.get_device() != k.get_device()
            or (n and (qkv.stride(1) != 1 or (n > 1 and qkv.stride(0) < width)))):
        raise ValueError(f"{fn}: qkv must be a bfloat16 tensor of shape {(n, width)} with contiguous rows on the pools' GPU, got "
                         f"{qkv.dtype} {tuple(qkv.shape)}, strides {qkv.stride()}, on {qkv.device}")
    index = k.get_device()
    pool = k.shape
    _tensors(fn, index, ("k", k, torch.bfloat16, pool), ("v", v, torch.bfloat16, pool), ("q_weight", q_weight, torch.float32, (d,)),
             ("k_weight", k_weight, torch.float32, (d,)), ("cos", cos, torch.float32, (n, half)),
             ("sin", sin, torch.float32, (n, half)), ("dst", dst, torch.int32, dst.shape))
    call = _Call(fn, k, stream)
    call.uses(qkv, q_weight, k_weight, cos, sin, dst, k, v)
    q = call.empty((n, hq, d), torch.bfloat16)
    shape = tkv_shape(hq, hkv, d, bs, nb)
    call.run(lib().tkv_norm_rope_append, ctypes.byref(shape), n, qkv.data_ptr(), qkv.stride(0) if n > 1 else width,
             q_weight.data_ptr(), k_weight.data_ptr(), float(eps), cos.data_ptr(), sin.data_ptr(), 2 * half, dst.data_ptr(),
             q.data_ptr(), k.data_ptr(), v.data_ptr())
    return q


def tkv_draft_mask(parents, words: Optional[int] = None):
    """Who sees whom in one row's drafted tree: (mask [n, words] uint64, depth [n] int32) of parents[i] < i (-1: the
    context).  words defaults to what n tokens need; a batch uses one number for all its rows."""
    p = _i32(parents)
    n = len(p)
    words = -(-n // 64) if words is None else int(words)
    mask = np.zeros((n, max(0, words)), dtype=np.uint64)
    depth = np.zeros(n, dtype=np.int32)
    _check(lib().tkv_draft_mask(n, _ptr(p), words, mask.ctypes.data_as(_P), _ptr(depth)))
    return mask, depth


def tkv_draft_workspace_bytes(shape, n_rows: int, n_qtok: int, max_q: int, n_kv_blocks: int, max_blocks: int,
                              mask_words: int) -> int:
    """Workspace of tkv_draft_verify for these numbers; shape = (hq, hkv, d, block_size, num_blocks)."""
    sh, n = tkv_shape(*[int(x) for x in shape]), ctypes.c_size_t()
    batch = tkv_draft_batch(n_rows, n_qtok, max_q, n_kv_blocks, max_blocks, mask_words)
    _check(lib().tkv_draft_workspace_bytes(ctypes.byref(sh), ctypes.byref(batch), ctypes.byref(n)))
    return n.value


def tkv_draft_verify(q_indptr: torch.Tensor, kv_indptr: torch.Tensor, kv_blocks: torch.Tensor, block_len: torch.Tensor,
                     mask: torch.Tensor, max_q: int, max_blocks: int, q: torch.Tensor, k: torch.Tensor, v: torch.Tensor,
                     o: torch.Tensor, lse: Optional[torch.Tensor] = None, workspace: Optional[torch.Tensor] = None,
                     stream=None) -> None:
    """Attention of drafted trees: row r's tokens [q_indptr[r], q_indptr[r + 1]) over its block table
    kv_blocks[kv_indptr[r] : kv_indptr[r + 1]], whose last keys are the tokens themselves.  mask [n_qtok, words] int64:
    bit j of token i's words is set where it sees the row's drafted token j (tkv_draft_mask).  All on the GPU; max_q and
    max_blocks bound a row's tokens and blocks.  A workspace (uint8, tkv_draft_workspace_bytes) is made for the call
    if none is given."""
    fn = "tkv_draft_verify"
    if k.dim() != 4 or q.dim() != 3 or mask.dim() != 2:
        raise ValueError(f"{fn}: k must be a pool [num_blocks, hkv, block_size, d], q [n, hq, d], mask [n, words]")
    nb, hkv, bs, d = k.shape
    n, hq, words = q.shape[0], q.shape[1], mask.shape[1]
    n_rows, n_kv = q_indptr.numel() - 1, kv_blocks.numel()
    index, pool, head = k.get_device(), k.shape, q.shape
    _tensors(fn, index, ("k", k, torch.bfloat16, pool), ("v", v, torch.bfloat16, pool), ("q", q, torch.bfloat16, head),
             ("o", o, torch.bfloat16, head), ("q_indptr", q_indptr, torch.int32, (max(0, n_rows) + 1,)),
             ("kv_indptr", kv_indptr, torch.int32, (n_rows + 1,)), ("kv_blocks", kv_blocks, torch.int32, (n_kv,)),
             ("block_len", block_len, torch.int32, (nb,)), ("mask", mask, torch.int64, (n, words)))
    if lse is not None:
        _tensors(fn, index, ("lse", lse, torch.float32, (n, hq)))
    if workspace is not None and (workspace.get_device() != index or not workspace.is_contiguous()):
        raise ValueError(f"{fn}: workspace must be contiguous, on GPU {index}")
    call = _Call(fn, k, stream)
    call.uses(q_indptr, kv_indptr, kv_blocks, block_len, mask, q, k, v, o, lse, workspace)
    sh = tkv_shape(hq, hkv, d, bs, nb)
    batch = tkv_draft_batch(n_rows, n, int(max_q), n_kv, int(max_blocks), words, q_indptr.data_ptr(), kv_indptr.data_ptr(),
                            kv_blocks.data_ptr(), block_len.data_ptr(), mask.data_ptr())
    need = ctypes.c_size_t()
    _check(lib().tkv_draft_workspace_bytes(ctypes.byref(sh), ctypes.byref(batch), ctypes.byref(need)))
    if workspace is None and need.value:
        workspace = call.empty((need.value,), torch.uint8)
    call.run(lib().tkv_draft_verify, ctypes.byref(sh), ctypes.byref(batch), q.data_ptr(), k.data_ptr(), v.data_ptr(),
             o.data_ptr(), None if lse is None else lse.data_ptr(), None if workspace is None else workspace.data_ptr(),
             0 if workspace is None else workspace.numel() * workspace.element_size())


def tkv_key_weights(q_indptr: torch.Tensor, kv_indptr: torch.Tensor, kv_blocks: torch.Tensor, block_len: torch.Tensor,
                    mask: torch.Tensor, max_q: int, max_blocks: int, q: torch.Tensor, k: torch.Tensor, lse: torch.Tensor,
                    out: torch.Tensor, before: Optional[torch.Tensor] = None, decay: float = 1.0,
                    coef: Optional[torch.Tensor] = None, stream=None) -> None:
    """Adds the attention weight of a batch's queries to its rows' keys: out [n_rows, hkv, keys] fp32 (keys >= 16 max_blocks)
    gets, at 16 e + s for the key in slot s of a row's entry e, decay * before (None: 0; may be out; not for the row's last
    keys, which enter) + the sum of coef (None: 1) times the queries' weights.  lse [n, hq] is the attention's; the other
    arguments are tkv_draft_verify's.  A row without tokens is left out, its weights not decayed and its part of out not
    written: where rows pause, out has to be before."""
    fn = "tkv_key_weights"
    if k.dim() != 4 or q.dim() != 3 or mask.dim() != 2 or out.dim() != 3:
        raise ValueError(f"{fn}: k must be a pool [num_blocks, hkv, block_size, d], q [n, hq, d], mask [n, words], out [n_rows, "
                         f"hkv, keys]")
    pool = k.shape
    nb, hkv, bs, d = pool
    n, hq = q.shape[:2]
    words, n_rows, n_kv, keys = mask.shape[1], q_indptr.numel() - 1, kv_blocks.numel(), out.shape[2]
    index, sums = k.get_device(), (n_rows, hkv, keys)
    specs = [("k", k, torch.bfloat16, pool), ("q", q, torch.bfloat16, (n, hq, d)), ("lse", lse, torch.float32, (n, hq)),
             ("q_indptr", q_indptr, torch.int32, (max(0, n_rows) + 1,)), ("kv_indptr", kv_indptr, torch.int32, (n_rows + 1,)),
             ("kv_blocks", kv_blocks, torch.int32, (n_kv,)), ("block_len", block_len, torch.int32, (nb,)),
             ("mask", mask, torch.int64, (n, words)), ("out", out, torch.float32, sums)]
    if before is not None:
        specs.append(("before", before, torch.float32, sums))
    if coef is not None:
        specs.append(("coef", coef, torch.float32, (n,)))
    _tensors(fn, index, *specs)
    call = _Call(fn, k, stream)
    call.uses(q_indptr, kv_indptr, kv_blocks, block_len, mask, q, k, lse, out, before, coef)
    try:
        shape = _pack_shape(hq, hkv, d, bs, nb)
        batch = _pack_draft(n_rows, n, max_q, n_kv, max_blocks, words, q_indptr.data_ptr(), kv_indptr.data_ptr(),
                            kv_blocks.data_ptr(), block_len.data_ptr(), mask.data_ptr())
    except struct.error:
        raise _past_32_bits(fn) from None
    call.run(lib().tkv_key_weights, shape, batch, q.data_ptr(), k.data_ptr(), lse.data_ptr(),
             None if coef is None else coef.data_ptr(), decay, None if before is None else before.data_ptr(), out.data_ptr(), keys)


def tkv_evict_keys(kv_indptr: torch.Tensor, kv_blocks: torch.Tensor, block_len: torch.Tensor, max_blocks: int,
                   new_indptr: torch.Tensor, new_blocks: torch.Tensor, budget: torch.Tensor, sink: int, recent: int,
                   weights: torch.Tensor, k: torch.Tensor, v: torch.Tensor, out: torch.Tensor, kept: torch.Tensor,
                   n_kept: torch.Tensor, stream=None) -> None:
    """Moves the keys that stay to new tables: of each row, and each KV head for itself, the first `sink`, the last `recent` and
    the heaviest of those between, min(budget[r], keys) in all, to the slots of new_blocks[new_indptr[r] : new_indptr[r + 1]]
    (blocks in no table of the call).  weights, out [n_rows, hkv, keys] fp32 as in tkv_key_weights: the kept keys' go to their
    new places in out.  kept [n_rows, hkv, most] int32: their old places, then -1; n_kept [n_rows]: how many (-1: the row's
    arrays do not fit, nothing was moved)."""
    fn = "tkv_evict_keys"
    if k.dim() != 4 or weights.dim() != 3 or kept.dim() != 3:
        raise ValueError(f"{fn}: k must be a pool [num_blocks, hkv, block_size, d], weights [n_rows, hkv, keys], kept [n_rows, "
                         f"hkv, most]")
    nb, hkv, bs, d = k.shape
    n_rows, n_kv, n_new = kv_indptr.numel() - 1, kv_blocks.numel(), new_blocks.numel()
    keys, most, index = weights.shape[2], kept.shape[2], k.get_device()
    rows = max(0, n_rows)
    _tensors(fn, index, ("k", k, torch.bfloat16, k.shape), ("v", v, torch.bfloat16, k.shape),
             ("kv_indptr", kv_indptr, torch.int32, (rows + 1,)), ("kv_blocks", kv_blocks, torch.int32, (n_kv,)),
             ("block_len", block_len, torch.int32, (nb,)), ("new_indptr", new_indptr, torch.int32, (rows + 1,)),
             ("new_blocks", new_blocks, torch.int32, (n_new,)), ("budget", budget, torch.int32, (rows,)),
             ("weights", weights, torch.float32, (rows, hkv, keys)), ("out", out, torch.float32, (rows, hkv, keys)),
             ("kept", kept, torch.int32, (rows, hkv, most)), ("n_kept", n_kept, torch.int32, (rows,)))
    call = _Call(fn, k, stream)
    call.uses(kv_indptr, kv_blocks, block_len, new_indptr, new_blocks, budget, weights, k, v, out, kept, n_kept)
    try:
        shape = _pack_shape(hkv, hkv, d, bs, nb)
        batch = _pack_evict(n_rows, n_kv, max_blocks, n_new, most, sink, recent, kv_indptr.data_ptr(), kv_blocks.data_ptr(),
                            block_len.data_ptr(), new_indptr.data_ptr(), new_blocks.data_ptr(), budget.data_ptr())
    except struct.error:
        raise _past_32_bits(fn) from None
    call.run(lib().tkv_evict_keys, shape, batch, weights.data_ptr(), out.data_ptr(), keys, k.data_ptr(), v.data_ptr(),
             kept.data_ptr(), n_kept.data_ptr())


def tkv_swiglu(gu: torch.Tensor, stream=None) -> torch.Tensor:
    """SiLU(gate) * up of gu [rows, 2 * inter] bf16 (gate first), in bf16."""
    rows, two = gu.shape
    _expect("tkv_swiglu", "gu", gu, torch.bfloat16, (rows, two - two % 2))
    out = torch.empty((rows, two // 2), dtype=torch.bfloat16, device=gu.device)
    _check(lib().tkv_swiglu(rows, two // 2, gu.data_ptr(), out.data_ptr(), _stream(stream)))
    return out


def tkv_cd_sample(logits: torch.Tensor, temperature: float, draw_off: torch.Tensor, uniform: torch.Tensor,
                  max_potential: int, stream=None):
    """Draws each row's potential-many tokens and groups them; returns device tensors
    (tokens, counts, n_groups): row r's groups at [draw_off[r], draw_off[r] + n_groups[r]).  A row
    whose draws fall outside `uniform` gets n_groups -1."""
    if logits.dim() != 2 or logits.dtype != torch.float32 or not logits.is_cuda or not logits.is_contiguous():
        raise ValueError("tkv_cd_sample: logits must be a contiguous float32 GPU tensor [n_rows, vocab]")
    n_rows, vocab = logits.shape
    if draw_off.dtype != torch.int32 or draw_off.numel() != n_rows + 1 or not draw_off.is_cuda:
        raise ValueError("tkv_cd_sample: draw_off must be an int32 GPU tensor of n_rows + 1 entries")
    if uniform.dtype != torch.float32 or not uniform.is_cuda or not uniform.is_contiguous():
        raise ValueError("tkv_cd_sample: uniform must be a contiguous float32 GPU tensor")
    n = max(1, int(uniform.numel()))
    tok = torch.empty(n, dtype=torch.int32, device=logits.device)
    cnt = torch.empty(n, dtype=torch.int32, device=logits.device)
    ng = torch.empty(max(1, n_rows), dtype=torch.int32, device=logits.device)
    _check(lib().tkv_cd_sample(n_rows, vocab, float(temperature), int(max_potential), logits.data_ptr(),
                               uniform.data_ptr(), draw_off.data_ptr(), int(uniform.numel()), tok.data_ptr(),
                               cnt.data_ptr(), ng.data_ptr(), _stream(stream)))
    return tok, cnt, ng[:n_rows]


def tkv_filter_sample_workspace_bytes(n_rows: int, vocab: int) -> int:
    return int(lib().tkv_filter_sample_workspace_bytes(n_rows, vocab))


def tkv_filter_sample(logits: torch.Tensor, temperature: torch.Tensor, draw_off: torch.Tensor, uniform: torch.Tensor,
                      max_potential: int, top_k: Optional[torch.Tensor] = None, top_p: Optional[torch.Tensor] = None,
                      min_p: Optional[torch.Tensor] = None, workspace: Optional[torch.Tensor] = None, stream=None):
    """tkv_cd_sample's draws from each row's distribution truncated by top-k, top-p and min-p (in this order), with settings
    for each row: temperature, top_p, min_p [n_rows] fp32, top_k [n_rows] int32 (None: off).  logits [n_rows, vocab] fp32
    or bf16, rows may be slices of longer ones.  Returns (tokens, counts, n_groups); the entries of a row's range past
    its groups are -1 and 0.  A workspace (uint8, tkv_filter_sample_workspace_bytes) is made if none is given."""
    fn = "tkv_filter_sample"
    if (logits.dim() != 2 or logits.dtype not in (torch.float32, torch.bfloat16) or not logits.is_cuda
            or (logits.numel() and logits.shape[1] > 1 and logits.stride(1) != 1)
            or (logits.shape[0] > 1 and logits.stride(0) < logits.shape[1])):
        raise ValueError(f"{fn}: logits must be a float32 or bfloat16 GPU tensor [n_rows, vocab] with contiguous rows")
    n_rows, vocab = logits.shape
    index, n = logits.get_device(), uniform.numel()
    _tensors(fn, index, ("temperature", temperature, torch.float32, (n_rows,)), ("draw_off", draw_off, torch.int32, (n_rows + 1,)),
             ("uniform", uniform, torch.float32, (n,)))
    for name, t, dtype in (("top_k", top_k, torch.int32), ("top_p", top_p, torch.float32), ("min_p", min_p, torch.float32)):
        if t is not None:
            _tensors(fn, index, (name, t, dtype, (n_rows,)))
    if workspace is not None and (workspace.get_device() != index or not workspace.is_contiguous()):
        raise ValueError(f"{fn}: workspace must be contiguous, on GPU {index}")
    call = _Call(fn, logits, stream)
    call.uses(logits, temperature, draw_off, uniform, top_k, top_p, min_p, workspace)
    need = tkv_filter_sample_workspace_bytes(n_rows, vocab)
    if workspace is None and need:
        workspace = call.empty((need,), torch.uint8)
    tok, cnt, ng = call.empty((2 * n + n_rows,), torch.int32).split((n, n, n_rows))  # (one allocation: 1.4 us each)

    def ptr(t):
        return None if t is None else t.data_ptr()
    call.run(lib().tkv_filter_sample, n_rows, vocab, int(logits.dtype == torch.bfloat16), logits.data_ptr(),
             logits.stride(0) if n_rows > 1 else vocab, temperature.data_ptr(), ptr(top_k), ptr(top_p), ptr(min_p),
             int(max_potential), uniform.data_ptr(), draw_off.data_ptr(), n, tok.data_ptr(), cnt.data_ptr(), ng.data_ptr(),
             ptr(workspace), 0 if workspace is None else workspace.numel() * workspace.element_size())
    return tok, cnt, ng


def _logit_rows(fn: str, name: str, t: torch.Tensor, rows: int, vocab: int, index: int) -> int:
    """Checks logits [rows, vocab], fp32 or bf16, with contiguous rows on GPU `index`; returns the rows' stride."""
    if t.shape == (rows, vocab) and (t.dtype is torch.float32 or t.dtype is torch.bfloat16) and t.get_device() == index >= 0:
        step, one = t.stride()
        if (one == 1 or vocab <= 1) and (step >= vocab or rows <= 1) or not rows:
            return step if rows > 1 else vocab
    raise ValueError(f"{fn}: {name} must be a float32 or bfloat16 tensor of shape {(rows, vocab)} with contiguous rows on GPU "
                     f"{max(index, 0)}, got {t.dtype} {tuple(t.shape)}, strides {t.stride()}, on {t.device}")


def tkv_adjust_logits(q_indptr: torch.Tensor, kv_indptr: torch.Tensor, kv_blocks: torch.Tensor, block_len: torch.Tensor,
                      mask: torch.Tensor, max_q: int, max_blocks: int, tokens: torch.Tensor, logits: torch.Tensor,
                      prompt_len: Optional[torch.Tensor] = None, repetition: Optional[torch.Tensor] = None,
                      presence: Optional[torch.Tensor] = None, frequency: Optional[torch.Tensor] = None,
                      bias_indptr: Optional[torch.Tensor] = None, bias_token: Optional[torch.Tensor] = None,
                      bias_value: Optional[torch.Tensor] = None, grammar: Optional[torch.Tensor] = None,
                      allowed: Optional[torch.Tensor] = None, out: Optional[torch.Tensor] = None, stream=None) -> torch.Tensor:
    """Logits [n_qtok, vocab] (fp32 or bf16) of a batch's query tokens under their rows' rules; each follows the tokens that it
    sees of its row's path, which lie in the pool tokens [num_blocks, 16] int32 under the batch's tables.
    repetition, presence, frequency [n_rows] fp32: penalties for tokens of the path, the last two for those past its first
    prompt_len [n_rows] int32; bias_token int32, bias_value fp32: row r's biases at [bias_indptr[r], bias_indptr[r + 1]);
    grammar [n_qtok] int32: each token's row of the masks allowed [masks, words] int32 (bit j % 32 of word j / 32: j is
    allowed; negative: no mask).  None: off.  out: fp32 or bf16, made as logits are if not given, or logits itself."""
    fn = "tkv_adjust_logits"
    if tokens.dim() != 2 or mask.dim() != 2 or logits.dim() != 2:
        raise ValueError(f"{fn}: tokens must be a pool [num_blocks, 16], mask [n, words], logits [n, vocab]")
    if (bias_indptr is None) != (bias_token is None) or (bias_token is None) != (bias_value is None):
        raise ValueError(f"{fn}: bias_indptr, bias_token and bias_value go together")
    if grammar is not None and allowed is None:
        raise ValueError(f"{fn}: a grammar needs the masks it names")
    nb, vocab, index = tokens.shape[0], logits.shape[1], tokens.get_device()
    n, words = mask.shape
    n_rows, n_kv = q_indptr.numel() - 1, kv_blocks.numel()
    i32, f32, rows = torch.int32, torch.float32, (max(0, n_rows),)
    ends = (rows[0] + 1,)
    specs = [("tokens", tokens, i32, (nb, 16)), ("q_indptr", q_indptr, i32, ends), ("kv_indptr", kv_indptr, i32, ends),
             ("kv_blocks", kv_blocks, i32, (n_kv,)), ("block_len", block_len, i32, (nb,)), ("mask", mask, torch.int64, (n, words))]
    p0 = p1 = p2 = p3 = p4 = p5 = p6 = p7 = p8 = n_bias = n_masks = mask_words = 0
    if prompt_len is not None:
        specs.append(("prompt_len", prompt_len, i32, rows))
        p0 = prompt_len.data_ptr()
    if repetition is not None:
        specs.append(("repetition", repetition, f32, rows))
        p1 = repetition.data_ptr()
    if presence is not None:
        specs.append(("presence", presence, f32, rows))
        p2 = presence.data_ptr()
    if frequency is not None:
        specs.append(("frequency", frequency, f32, rows))
        p3 = frequency.data_ptr()
    if bias_token is not None:
        n_bias = bias_token.numel()
        specs += (("bias_indptr", bias_indptr, i32, ends), ("bias_token", bias_token, i32, (n_bias,)),
                  ("bias_value", bias_value, f32, (n_bias,)))
        p4, p5, p6 = bias_indptr.data_ptr(), bias_token.data_ptr(), bias_value.data_ptr()
    if grammar is not None:
        specs.append(("grammar", grammar, i32, (n,)))
        p7 = grammar.data_ptr()
    if allowed is not None:
        if allowed.dim() != 2:
            raise ValueError(f"{fn}: allowed must be [masks, words]")
        n_masks, mask_words = allowed.shape
        specs.append(("allowed", allowed, i32, (n_masks, mask_words)))
        p8 = allowed.data_ptr()
    _tensors(fn, index, *specs)
    stride = _logit_rows(fn, "logits", logits, n, vocab, index)
    if vocab >> 31:  # (an int32 argument of a call would be cut to 32 bits without a word)
        raise _past_32_bits(fn)
    call = _Call(fn, tokens, stream)
    if out is None:
        out = call.empty((n, vocab), logits.dtype)
    out_stride = _logit_rows(fn, "out", out, n, vocab, index)
    call.uses(q_indptr, kv_indptr, kv_blocks, block_len, mask, tokens, logits, prompt_len, repetition, presence, frequency,
              bias_indptr, bias_token, bias_value, grammar, allowed, out)
    try:
        rules = _pack_rules(p0, p1, p2, p3, p4, p5, p6, p7, p8, n_bias, n_masks, mask_words)
        batch = _pack_draft(n_rows, n, max_q, n_kv, max_blocks, words, q_indptr.data_ptr(), kv_indptr.data_ptr(),
                            kv_blocks.data_ptr(), block_len.data_ptr(), mask.data_ptr())
    except struct.error:
        raise _past_32_bits(fn) from None
    call.run(lib().tkv_adjust_logits, nb, tokens.data_ptr(), batch, rules, vocab, logits.dtype is torch.bfloat16, logits.data_ptr(),
             stride, out.dtype is torch.bfloat16, out.data_ptr(), out_stride)
    return out


def tkv_plan_profile(plan: int, max_calls: int) -> None:
    _check(lib().tkv_plan_profile(plan, max_calls))


def tkv_plan_profile_read(plan: int):
    """Returns (recorded calls, summed main-kernel ms, summed merge-kernel ms)."""
    n, a, b = _I32(), ctypes.c_float(), ctypes.c_float()
    _check(lib().tkv_plan_profile_read(plan, ctypes.byref(n), ctypes.byref(a), ctypes.byref(b)))
    return n.value, a.value, b.value


CAND_GENERATING, CAND_QUEUED, CAND_VERIFYING, CAND_VERIFIED, CAND_SELECTED, CAND_PRUNED = range(6)


def tkv_search_create(k: int, max_nodes: int, token_threshold: int, max_deferrals: int) -> int:
    h = _P()
    _check(lib().tkv_search_create(k, max_nodes, token_threshold, max_deferrals, ctypes.byref(h)))
    return h.value


def tkv_search_destroy(s: int) -> None:
    lib().tkv_search_destroy(s)


def tkv_search_expand(s: int, parent: int, n: int) -> int:
    first = _I32()
    _check(lib().tkv_search_expand(s, parent, n, ctypes.byref(first)))
    return first.value


def tkv_search_complete(s: int, node: int, n_tokens: int) -> bool:
    f = _I32()
    _check(lib().tkv_search_complete(s, node, n_tokens, ctypes.byref(f)))
    return bool(f.value)


def tkv_search_tick(s: int) -> bool:
    f = _I32()
    _check(lib().tkv_search_tick(s, ctypes.byref(f)))
    return bool(f.value)


def _take(fn, s: int) -> list:
    n = _I32()
    rc = fn(s, None, 0, ctypes.byref(n))
    if rc not in (TKV_OK, TKV_ECAP):
        _check(rc)
    out = np.zeros(max(1, n.value), dtype=np.int32)
    _check(fn(s, _ptr(out), len(out), ctypes.byref(n)))
    return [int(x) for x in out[:n.value]]


def tkv_search_flush(s: int) -> list:
    return _take(lib().tkv_search_flush, s)


def tkv_search_score(s: int, nodes, scores) -> None:
    nd = _i32(nodes)
    sc = np.ascontiguousarray(np.asarray(scores, dtype=np.float32).reshape(-1))
    if len(sc) != len(nd):
        raise ValueError("one score per node")
    _check(lib().tkv_search_score(s, len(nd), _ptr(nd), sc.ctypes.data_as(ctypes.POINTER(ctypes.c_float))))


def tkv_search_pruned(s: int) -> list:
    return _take(lib().tkv_search_pruned, s)


def tkv_search_node(s: int, node: int):
    """Returns (state, parent, depth, score or None)."""
    st, pa, de, sc = _I32(), _I32(), _I32(), ctypes.c_float()
    _check(lib().tkv_search_node(s, node, ctypes.byref(st), ctypes.byref(pa), ctypes.byref(de), ctypes.byref(sc)))
    return st.value, pa.value, de.value, (None if sc.value < 0 else sc.value)


def tkv_search_round(s: int, depth: int):
    """Returns (decided, selected ids ascending)."""
    n, dec = _I32(), _I32()
    rc = lib().tkv_search_round(s, depth, None, 0, ctypes.byref(n), ctypes.byref(dec))
    if rc not in (TKV_OK, TKV_ECAP):
        _check(rc)
    out = np.zeros(max(1, n.value), dtype=np.int32)
    _check(lib().tkv_search_round(s, depth, _ptr(out), len(out), ctypes.byref(n), ctypes.byref(dec)))
    return bool(dec.value), [int(x) for x in out[:n.value]]


def tkv_search_snapshot(s: int) -> dict:
    """Parsed state: nodes as (parent, depth, state, n_children, tokens, deferrals, arrival, score bits)."""
    used = ctypes.c_size_t()
    lib().tkv_search_snapshot(s, None, 0, ctypes.byref(used))
    buf = np.zeros(used.value // 4, dtype=np.int32)
    _check(lib().tkv_search_snapshot(s, buf.ctypes.data_as(_P), used.value, ctypes.byref(used)))
    w = [int(x) for x in buf]
    k, thr, md, n_roots, qtok, n = w[:6]
    i = 6
    nodes = [tuple(w[i + 8 * j:i + 8 * j + 8]) for j in range(n)]
    i += 8 * n
    nq = w[i]
    queue = w[i + 1:i + 1 + nq]
    i += 1 + nq
    rounds = []
    for _ in range(w[i]):
        i += 1
        dec, ns = w[i], w[i + 1]
        rounds.append((dec, tuple(w[i + 2:i + 2 + ns])))
        i += 1 + ns
    return {"k": k, "token_threshold": thr, "max_deferrals": md, "n_roots": n_roots, "queued_tokens": qtok,
            "nodes": nodes, "queue": queue, "rounds": rounds}


# ------------------------------------------------------------------------- owning wrappers

class BlockManager:
    """Owns a tkv_bm handle; methods forward to the C entry points."""

    def __init__(self, num_blocks: int, block_size: int = 16, max_seqs: int = 1024):
        self.num_blocks, self.block_size = num_blocks, block_size
        self.h = tkv_bm_create(num_blocks, block_size, max_seqs)

    def __del__(self):
        if getattr(self, "h", None) and _lib is not None:
            tkv_bm_destroy(self.h)
            self.h = None

    def extend(self, parent, tokens, seal):
        return tkv_bm_extend(self.h, parent, tokens, seal, self.block_size)

    def prune(self, seq):
        return tkv_prune(self.h, seq)

    def append(self, seq, tokens):
        return tkv_bm_append(self.h, seq, tokens)

    def seal(self, seq):
        return tkv_bm_seal(self.h, seq)

    def fork(self, seq, tokens):
        return tkv_bm_fork(self.h, seq, tokens)

    def table(self, seq):
        return tkv_bm_table(self.h, seq)[0]

    def block_len(self):
        return tkv_bm_block_len(self.h, self.num_blocks)

    def snapshot(self, seqs=True):
        return tkv_bm_snapshot(self.h, seqs)

    def coalesce(self, seqs, q_lens):
        return tkv_bm_coalesce(self.h, seqs, q_lens)


class Plan:
    """Owns a tkv_plan handle and the device workspace it was uploaded to."""

    def __init__(self, shape, q_indptr, kv_indptr, kv_blocks, block_len, multiplicity=None,
                 device="cuda", stream=None, upload=True, options=None):
        self.h = tkv_plan_create_ex(shape, q_indptr, kv_indptr, kv_blocks, block_len, multiplicity, options)
        self.workspace = None
        if upload:
            nbytes = tkv_plan_workspace_bytes(self.h)
            self.workspace = torch.empty(nbytes, dtype=torch.uint8, device=device)
            tkv_plan_upload(self.h, self.workspace, stream)

    def __del__(self):
        if getattr(self, "h", None) and _lib is not None:
            tkv_plan_destroy(self.h)
            self.h = None

    @property
    def stats(self):
        return tkv_plan_get_stats(self.h)

    def update(self, kv_indptr, kv_blocks, block_len, stream=None) -> bool:
        """tkv_plan_update, then (for an uploaded plan) the upload again, into a larger workspace
        if the plan now needs one.  Returns whether the plan was patched in place."""
        in_place = tkv_plan_update(self.h, kv_indptr, kv_blocks, block_len)
        if self.workspace is not None:
            nbytes = tkv_plan_workspace_bytes(self.h)
            if nbytes > self.workspace.numel():
                self.workspace = torch.empty(nbytes, dtype=torch.uint8, device=self.workspace.device)
            tkv_plan_upload(self.h, self.workspace, stream)
        return in_place

    def image(self) -> bytes:
        return tkv_plan_image(self.h)

    def view(self):
        return tkv_plan_get_view(self.h)

    def decode(self, q, k, v, o, lse=None, stream=None):
        tkv_decode(self.h, q, k, v, o, lse, stream)

    def verify(self, q, k, v, o, lse=None, stream=None):
        tkv_verify(self.h, q, k, v, o, lse, stream)


class DraftBatch:
    """The device arrays of a drafted batch for tkv_draft_verify, in one upload: row r's block table (its last keys are the
    drafted tokens), the parents of its drafted tokens (earlier ones, or -1 for the context), and every block's length.
    A batch serves every layer.  positions, depth: each token's position in its path (int64, device) and its
    number of drafted ancestors (host).  evicted: how many keys each row's path has lost (tkv_evict_keys), which its tokens'
    positions still count (None: none)."""

    def __init__(self, tables, parents, block_len, device="cuda", evicted=None):
        if len(tables) != len(parents):
            raise ValueError("DraftBatch: a table and a tree for every row")
        lens, n_blk = [len(p) for p in parents], [len(t) for t in tables]
        bl = _i32(block_len)
        self.max_q, self.max_blocks = max(lens, default=1), max(n_blk, default=1)
        if any(n < 1 for n in lens):
            raise ValueError("DraftBatch: every row needs a drafted token")
        words = -(-self.max_q // 64)
        trees = [tkv_draft_mask(p, words) for p in parents]
        self.depth = np.concatenate([d for _, d in trees]) if trees else np.zeros(0, np.int32)
        kv = np.concatenate([_i32(t) for t in tables]) if tables else np.zeros(0, np.int32)
        if len(kv) and (kv.min() < 0 or kv.max() >= len(bl)):
            raise ValueError("DraftBatch: a table names a block outside block_len")
        if len(kv) and (bl[kv].min() < 0 or bl[kv].max() > 16):
            raise ValueError("DraftBatch: a table's block has a length outside [0, 16]")
        context = [int(bl[_i32(t)].sum()) - n for t, n in zip(tables, lens)]
        if any(c < 0 for c in context):
            raise ValueError("DraftBatch: a row's path is shorter than its draft")
        if evicted is not None:
            if len(evicted) != len(tables) or any(int(e) < 0 for e in evicted):
                raise ValueError("DraftBatch: a number of evicted keys, 0 or more, for every row")
            context = [c + int(e) for c, e in zip(context, evicted)]
        positions = np.repeat(np.asarray(context, np.int64), lens) + self.depth
        mask = np.concatenate([m for m, _ in trees]) if trees else np.zeros((0, words), np.uint64)
        parts = [positions.astype(np.int64).view(np.int32), mask.view(np.int32).reshape(-1),
                 np.cumsum([0] + lens).astype(np.int32), np.cumsum([0] + n_blk).astype(np.int32), kv, bl]
        flat = torch.from_numpy(np.concatenate(parts)).to(device)
        at = np.cumsum([0] + [len(p) for p in parts])
        cut = [flat[a:b] for a, b in zip(at[:-1], at[1:])]
        n = len(positions)
        self.positions = cut[0].view(torch.int64) if n else torch.zeros(0, dtype=torch.int64, device=device)
        self.mask = cut[1].view(torch.int64).view(n, words) if n else torch.zeros((0, words), dtype=torch.int64, device=device)
        self.q_indptr, self.kv_indptr, self.kv_blocks, self.block_len = cut[2:]

    def verify(self, q, k, v, o, lse=None, workspace=None, stream=None):
        tkv_draft_verify(self.q_indptr, self.kv_indptr, self.kv_blocks, self.block_len, self.mask, self.max_q, self.max_blocks,
                         q, k, v, o, lse, workspace, stream)

    def key_weights(self, q, k, lse, out, before=None, decay=1.0, coef=None, stream=None):
        """tkv_key_weights of this batch, after its attention wrote lse; out may be before."""
        tkv_key_weights(self.q_indptr, self.kv_indptr, self.kv_blocks, self.block_len, self.mask, self.max_q, self.max_blocks,
                        q, k, lse, out, before, decay, coef, stream)

    def adjust_logits(self, tokens, logits, **rules):
        """tkv_adjust_logits with this batch's tables (those of the tokens' pool); its rules, out and stream by name."""
        return tkv_adjust_logits(self.q_indptr, self.kv_indptr, self.kv_blocks, self.block_len, self.mask, self.max_q,
                                 self.max_blocks, tokens, logits, **rules)


class EvictBatch:
    """The device arrays of an eviction (tkv_evict_keys), in one upload: row r's path in tables[r] keeps at most budget[r]
    keys a KV head, in the blocks new_tables[r] (as many as they need, in no other table of the batch: e.g. of a sequence that
    BlockManager.extend made without a parent and with seal=False).  Rows that share blocks each keep copies of their own: a
    shared prefix is worth evicting where it and the rest are more than what all rows keep.  A batch serves every layer.
    n_kept: how many each row keeps, evicted: how many it loses (host)."""

    def __init__(self, tables, new_tables, budget, block_len, device="cuda"):
        if not len(tables) == len(new_tables) == len(budget):
            raise ValueError("EvictBatch: a table, a new table and a budget for every row")
        bl, budget = _i32(block_len), [int(b) for b in budget]
        old, new = [_i32(t) for t in tables], [_i32(t) for t in new_tables]
        if any(b < 0 for b in budget):
            raise ValueError("EvictBatch: a budget below 0")
        every = np.concatenate(old + new) if tables else np.zeros(0, np.int32)
        if len(every) and (every.min() < 0 or every.max() >= len(bl)):
            raise ValueError("EvictBatch: a table names a block outside block_len")
        if any(len(t) and (bl[t].min() < 0 or bl[t].max() > 16) for t in old):
            raise ValueError("EvictBatch: a table's block has a length outside [0, 16]")
        fresh = np.concatenate(new) if new else np.zeros(0, np.int32)
        if len(np.unique(fresh)) < len(fresh) or (len(fresh) and np.isin(fresh, np.concatenate(old)).any()):
            raise ValueError("EvictBatch: a block of a new table is in another table too, or twice in its own")
        lens = [int(bl[t].sum()) for t in old]
        self.n_kept = [min(n, b) for n, b in zip(lens, budget)]
        self.evicted = [n - m for n, m in zip(lens, self.n_kept)]
        for t, m in zip(new, self.n_kept):
            if 16 * len(t) < m:
                raise ValueError(f"EvictBatch: {len(t)} blocks do not hold {m} keys")
        self.max_blocks, self.most = max([len(t) for t in old], default=1) or 1, max(self.n_kept, default=0)
        parts = [np.cumsum([0] + [len(t) for t in old]).astype(np.int32), np.cumsum([0] + [len(t) for t in new]).astype(np.int32),
                 np.asarray(self.n_kept, np.int32), np.concatenate(old) if old else fresh, fresh, bl]
        flat = torch.from_numpy(np.concatenate(parts)).to(device)
        at = np.cumsum([0] + [len(p) for p in parts])
        self.kv_indptr, self.new_indptr, self.budget, self.kv_blocks, self.new_blocks, self.block_len = \
            [flat[a:b] for a, b in zip(at[:-1], at[1:])]

    def evict(self, weights, k, v, sink=0, recent=0, out=None, kept=None, n_kept=None, stream=None):
        """One layer's eviction; returns (weights at their new places, kept, n_kept), made if not given (weights past a row's kept
        ones are not written)."""
        call = _Call("EvictBatch.evict", k, stream)
        rows, hkv = self.budget.numel(), k.shape[1]
        out = call.empty(weights.shape, torch.float32) if out is None else out
        kept = call.empty((rows, hkv, self.most), torch.int32) if kept is None else kept
        n_kept = call.empty((rows,), torch.int32) if n_kept is None else n_kept
        tkv_evict_keys(self.kv_indptr, self.kv_blocks, self.block_len, self.max_blocks, self.new_indptr, self.new_blocks, self.budget,
                       sink, recent, weights, k, v, out, kept, n_kept, stream)
        return out, kept, n_kept


class Search:
    """Owns a tkv_search handle (speculative beam-search controller); methods forward to the C
    entry points."""

    def __init__(self, k: int, max_nodes: int = 4096, token_threshold: int = 2048, max_deferrals: int = 6):
        self.h = tkv_search_create(k, max_nodes, token_threshold, max_deferrals)

    def __del__(self):
        if getattr(self, "h", None) and _lib is not None:
            tkv_search_destroy(self.h)
            self.h = None

    def expand(self, parent, n):
        return tkv_search_expand(self.h, parent, n)

    def complete(self, node, n_tokens):
        return tkv_search_complete(self.h, node, n_tokens)

    def tick(self):
        return tkv_search_tick(self.h)

    def flush(self):
        return tkv_search_flush(self.h)

    def score(self, nodes, scores):
        tkv_search_score(self.h, nodes, scores)

    def pruned(self):
        return tkv_search_pruned(self.h)

    def node(self, node):
        return tkv_search_node(self.h, node)

    def round(self, depth):
        return tkv_search_round(self.h, depth)

    def snapshot(self):
        return tkv_search_snapshot(self.h)
