"""Binding of include/efim.h.  Argument marshalling only (the per-step calls through the
extension csrc/calls.c, everything else through ctypes): every step of the path runs inside
libefim.so.  There is no fallback: if the library is missing or cannot be loaded,
load_library() raises."""
import ctypes
import importlib.machinery
import importlib.util
import os
from ctypes import c_int32, c_int64, c_void_p, c_float, c_double, c_size_t, c_char_p, POINTER, Structure

import numpy as np

_LIB = None
_HERE = os.path.dirname(os.path.abspath(__file__))


class EfimError(RuntimeError):
    def __init__(self, code, where):
        self.code = int(code)
        detail = f" [{load_library().efim_last_cuda_error().decode()}]" if int(code) == 5 else ""
        super().__init__(f"{where}: {efim_strerror(code)} (status {int(code)}){detail}")


class _CacheDesc(Structure):
    _fields_ = [("d_k_pool", c_void_p), ("d_v_pool", c_void_p), ("num_pages", c_int32),
                ("page_size", c_int32), ("num_q_heads", c_int32), ("num_kv_heads", c_int32),
                ("head_dim", c_int32)]


class _BatchDesc(Structure):
    _fields_ = [("batch", c_int32), ("max_pages_per_seq", c_int32), ("total_new_tokens", c_int32),
                ("d_cached_len", c_void_p), ("d_new_len", c_void_p), ("d_q_indptr", c_void_p),
                ("d_block_table", c_void_p), ("h_cached_len", c_void_p), ("h_new_len", c_void_p)]


class _RopeDesc(Structure):
    _fields_ = [("d_cos_sin", c_void_p), ("max_position", c_int32), ("interleaved", c_int32)]


class _QkNormDesc(Structure):
    _fields_ = [("d_q_weight", c_void_p), ("d_k_weight", c_void_p), ("weight_f32", c_int32), ("eps", c_float),
                ("weight_offset", c_float)]


class _Cache4Desc(Structure):
    _fields_ = [("d_k_codes", c_void_p), ("d_v_codes", c_void_p), ("d_k_scales", c_void_p), ("d_v_scales", c_void_p),
                ("num_pages", c_int32), ("page_size", c_int32), ("num_q_heads", c_int32), ("num_kv_heads", c_int32),
                ("head_dim", c_int32), ("k_scale", c_float), ("v_scale", c_float)]


class _AdjustDesc(Structure):
    _fields_ = [("batch", c_int32), ("total_rows", c_int32), ("vocab", c_int32), ("logits_f32", c_int32), ("d_row_indptr", c_void_p),
                ("d_logits", c_void_p), ("logits_stride", c_int64), ("d_tokens", c_void_p), ("d_history", c_void_p),
                ("history_stride", c_int64), ("max_len", c_int32), ("bias_entries", c_int32), ("d_len", c_void_p),
                ("d_prompt_len", c_void_p), ("d_repetition", c_void_p), ("d_presence", c_void_p), ("d_frequency", c_void_p),
                ("d_bias_indptr", c_void_p), ("d_bias_tokens", c_void_p), ("d_bias", c_void_p), ("d_mask", c_void_p),
                ("mask_stride", c_int64)]


class _VerifyDesc(Structure):
    _fields_ = [("batch", c_int32), ("total_rows", c_int32), ("vocab", c_int32), ("target_kind", c_int32),
                ("d_row_indptr", c_void_p), ("d_tokens", c_void_p), ("d_target", c_void_p), ("target_stride", c_int64),
                ("d_draft_probs", c_void_p), ("draft_stride", c_int64), ("d_uniform", c_void_p), ("d_noise", c_void_p),
                ("noise_stride", c_int64), ("d_temperature", c_void_p)]


EXPORTS = ("efim_last_cuda_error", "efim_strerror", "efim_version", "efim_rope_table_build", "efim_kv_append",
           "efim_prefill_workspace_bytes", "efim_append_prefill_attn",
           "efim_decode_workspace_bytes", "efim_decode_attn",
           "efim_decode_static_scratch_bytes", "efim_decode_attn_static",
           "efim_prefill_launch_count", "efim_decode_launch_count",
           "efim_prefill_plan_bytes", "efim_prefill_plan", "efim_append_prefill_attn_planned", "efim_decode_step",
           "efim_append_prefill_step", "efim_selftest_bounded_wait",
           "efim_qk_norm_append", "efim_draft_lookup", "efim_verify_workspace_bytes", "efim_verify_drafts",
           "efim_kv4_append", "efim_kv4_unpack", "efim_kv4_decode_workspace_bytes", "efim_kv4_decode_attn",
           "efim_kv4_prefill_workspace_bytes", "efim_kv4_append_prefill_attn",
           "efim_step_tables_workspace_bytes", "efim_step_tables", "efim_release_pages", "efim_adjust_logits",
           "efim_fragment_cuts", "efim_fim_split", "efim_fim_fragment_spans",
           "efim_frontend_create", "efim_frontend_destroy", "efim_frontend_transform", "efim_frontend_admit",
           "efim_frontend_finish", "efim_frontend_stats")


def library_path() -> str:
    return os.path.join(_HERE, "libefim.so")


def load_library():
    """dlopen libefim.so (built in-tree by paper_2505_21889_b200.build). Raises if absent."""
    global _LIB
    if _LIB is not None:
        return _LIB
    path = library_path()
    if not os.path.exists(path):
        raise RuntimeError(f"{path} not found: build it first (python -m paper_2505_21889_b200.build); "
                           "there is no CPU fallback")
    lib = ctypes.CDLL(path)
    lib.efim_strerror.restype = c_char_p
    lib.efim_strerror.argtypes = [ctypes.c_int]
    lib.efim_last_cuda_error.restype = c_char_p
    lib.efim_version.restype = ctypes.c_int
    lib.efim_rope_table_build.restype = ctypes.c_int
    lib.efim_rope_table_build.argtypes = [c_double, c_int32, c_int32, c_void_p]
    lib.efim_kv_append.restype = ctypes.c_int
    lib.efim_kv_append.argtypes = [POINTER(_CacheDesc), POINTER(_BatchDesc), POINTER(_RopeDesc),
                                   c_void_p, c_void_p, c_void_p, c_void_p, c_void_p]
    lib.efim_prefill_workspace_bytes.restype = c_size_t
    lib.efim_prefill_workspace_bytes.argtypes = [POINTER(_CacheDesc), POINTER(_BatchDesc)]
    lib.efim_append_prefill_attn.restype = ctypes.c_int
    lib.efim_append_prefill_attn.argtypes = [POINTER(_CacheDesc), POINTER(_BatchDesc), c_void_p, c_void_p,
                                             c_void_p, c_float, c_void_p, c_size_t, c_void_p, c_void_p]
    lib.efim_prefill_plan_bytes.restype = c_size_t
    lib.efim_prefill_plan_bytes.argtypes = [POINTER(_CacheDesc), POINTER(_BatchDesc)]
    lib.efim_prefill_plan.restype = ctypes.c_int
    lib.efim_prefill_plan.argtypes = [POINTER(_CacheDesc), POINTER(_BatchDesc), c_void_p, c_size_t]
    lib.efim_append_prefill_attn_planned.restype = ctypes.c_int
    lib.efim_append_prefill_attn_planned.argtypes = [POINTER(_CacheDesc), POINTER(_BatchDesc), c_void_p, c_size_t,
                                                     c_int32, c_void_p, c_void_p, c_void_p, c_float, c_void_p, c_size_t,
                                                     c_void_p, c_void_p]
    lib.efim_append_prefill_step.restype = ctypes.c_int
    lib.efim_append_prefill_step.argtypes = [POINTER(_CacheDesc), POINTER(_BatchDesc), POINTER(_RopeDesc), c_void_p,
                                             c_void_p, c_void_p, c_void_p, c_void_p, c_float, c_void_p, c_size_t,
                                             c_int32, c_void_p, c_size_t, c_void_p, c_void_p]
    lib.efim_qk_norm_append.restype = ctypes.c_int
    lib.efim_qk_norm_append.argtypes = [POINTER(_CacheDesc), POINTER(_BatchDesc), POINTER(_QkNormDesc), POINTER(_RopeDesc),
                                        c_void_p, c_int64, c_void_p, c_int64, c_void_p, c_int64, c_void_p, c_void_p, c_void_p]
    lib.efim_draft_lookup.restype = ctypes.c_int
    lib.efim_draft_lookup.argtypes = [c_int32, c_void_p, c_int64, c_int32, c_void_p, c_int32, c_int32, c_int32, c_void_p,
                                      c_void_p, c_void_p, c_void_p]
    lib.efim_verify_drafts.restype = ctypes.c_int
    lib.efim_verify_drafts.argtypes = [POINTER(_VerifyDesc), c_void_p, c_void_p, c_void_p, c_void_p, c_int32, c_void_p,
                                       c_size_t, c_void_p, c_void_p]
    lib.efim_verify_workspace_bytes.restype = c_size_t
    lib.efim_verify_workspace_bytes.argtypes = [c_int32, c_int32, c_int32, c_int32]
    lib.efim_kv4_append.restype = ctypes.c_int
    lib.efim_kv4_append.argtypes = [POINTER(_Cache4Desc), POINTER(_BatchDesc), POINTER(_QkNormDesc), POINTER(_RopeDesc),
                                    c_void_p, c_int64, c_void_p, c_int64, c_void_p, c_int64, c_void_p, c_void_p, c_void_p]
    lib.efim_kv4_unpack.restype = ctypes.c_int
    lib.efim_kv4_unpack.argtypes = [POINTER(_Cache4Desc), c_void_p, c_int32, c_void_p, c_void_p, c_void_p, c_void_p]
    lib.efim_kv4_decode_workspace_bytes.restype = c_size_t
    lib.efim_kv4_decode_workspace_bytes.argtypes = [POINTER(_Cache4Desc), c_int32, c_int32, c_int32]
    lib.efim_kv4_decode_attn.restype = ctypes.c_int
    lib.efim_kv4_decode_attn.argtypes = [POINTER(_Cache4Desc), c_int32, c_void_p, c_int32, c_void_p, c_int32, c_void_p, c_int32,
                                         c_int32, c_void_p, c_void_p, c_void_p, c_float, c_void_p, c_size_t, c_void_p, c_void_p]
    lib.efim_kv4_prefill_workspace_bytes.restype = c_size_t
    lib.efim_kv4_prefill_workspace_bytes.argtypes = [POINTER(_Cache4Desc), POINTER(_BatchDesc)]
    lib.efim_kv4_append_prefill_attn.restype = ctypes.c_int
    lib.efim_kv4_append_prefill_attn.argtypes = [POINTER(_Cache4Desc), POINTER(_BatchDesc), c_void_p, c_void_p, c_void_p, c_float,
                                                 c_void_p, c_size_t, c_void_p, c_void_p]
    lib.efim_step_tables_workspace_bytes.restype = c_size_t
    lib.efim_step_tables_workspace_bytes.argtypes = [c_int32]
    lib.efim_step_tables.restype = ctypes.c_int
    lib.efim_step_tables.argtypes = [c_int32, c_void_p, c_void_p, c_void_p, c_int32, c_void_p, c_int32, c_void_p, c_void_p, c_void_p,
                                     c_void_p, c_int32, c_void_p, c_void_p, c_void_p, c_void_p, c_size_t, c_void_p, c_void_p]
    lib.efim_release_pages.restype = ctypes.c_int
    lib.efim_release_pages.argtypes = [c_int32, c_void_p, c_void_p, c_int32, c_void_p, c_int32, c_void_p, c_void_p, c_size_t, c_void_p,
                                       c_void_p]
    lib.efim_adjust_logits.restype = ctypes.c_int
    lib.efim_adjust_logits.argtypes = [POINTER(_AdjustDesc), c_void_p, c_int64, c_void_p, c_void_p]
    lib.efim_selftest_bounded_wait.restype = ctypes.c_int
    lib.efim_selftest_bounded_wait.argtypes = [ctypes.c_uint64, c_void_p, c_void_p, c_void_p]
    lib.efim_decode_workspace_bytes.restype = c_size_t
    lib.efim_decode_workspace_bytes.argtypes = [POINTER(_CacheDesc), c_int32, c_int32]
    lib.efim_decode_attn.restype = ctypes.c_int
    lib.efim_decode_attn.argtypes = [POINTER(_CacheDesc), c_int32, c_void_p, c_int32, c_void_p, c_int32,
                                     c_void_p, c_void_p, c_void_p, c_float, c_void_p, c_size_t,
                                     c_void_p, c_void_p]
    lib.efim_decode_step.restype = ctypes.c_int
    lib.efim_decode_step.argtypes = [POINTER(_CacheDesc), c_int32, c_void_p, c_int32, c_void_p, c_int32,
                                     POINTER(_RopeDesc), c_void_p, c_void_p, c_void_p, c_void_p, c_void_p, c_float,
                                     c_void_p, c_size_t, c_void_p, c_void_p]
    lib.efim_prefill_launch_count.restype = c_int32
    lib.efim_prefill_launch_count.argtypes = [POINTER(_CacheDesc), POINTER(_BatchDesc)]
    lib.efim_decode_launch_count.restype = c_int32
    lib.efim_decode_launch_count.argtypes = [POINTER(_CacheDesc), c_int32, c_int32]
    lib.efim_decode_static_scratch_bytes.restype = c_size_t
    lib.efim_decode_static_scratch_bytes.argtypes = []
    lib.efim_decode_attn_static.restype = ctypes.c_int
    lib.efim_decode_attn_static.argtypes = [POINTER(_CacheDesc), c_int32, c_void_p, c_int32, c_void_p, c_int32,
                                            c_void_p, c_void_p, c_void_p, c_float, c_void_p, c_void_p]
    lib.efim_frontend_create.restype = c_void_p
    lib.efim_frontend_create.argtypes = [c_int32, c_int32, c_int32, c_int32, c_int32, c_int32]
    lib.efim_frontend_destroy.restype = None
    lib.efim_frontend_destroy.argtypes = [c_void_p]
    lib.efim_frontend_transform.restype = ctypes.c_int
    lib.efim_frontend_transform.argtypes = [c_void_p, ctypes.c_int64, c_void_p, c_int32, c_void_p, c_int32, c_void_p,
                                            c_int32, c_void_p, c_void_p, c_void_p]
    lib.efim_frontend_admit.restype = ctypes.c_int
    lib.efim_frontend_admit.argtypes = [c_void_p, c_void_p, c_int32, c_int32, c_void_p, c_int32, c_void_p, c_void_p,
                                        c_void_p]
    lib.efim_frontend_finish.restype = ctypes.c_int
    lib.efim_frontend_finish.argtypes = [c_void_p, ctypes.c_int64, c_void_p, c_int32]
    lib.efim_frontend_stats.restype = None
    lib.efim_frontend_stats.argtypes = [c_void_p, c_void_p]
    _LIB = lib
    return lib


class _Calls:
    """The extension module with the per-step calls, loaded (with the library) on first use."""

    def __getattr__(self, name):
        load_library()
        path = os.path.join(_HERE, "_calls.so")
        if not os.path.exists(path):
            raise RuntimeError(f"{path} not found: build it first (python -m paper_2505_21889_b200.build)")
        loader = importlib.machinery.ExtensionFileLoader("_calls", path)
        module = importlib.util.module_from_spec(importlib.util.spec_from_loader("_calls", loader))
        loader.exec_module(module)
        for m in ("kv_append", "append_prefill_attn", "append_prefill_step", "decode_attn", "decode_step",
                  "qk_norm_append", "draft_lookup", "verify_workspace_bytes", "verify_drafts",
                  "kv4_append", "kv4_unpack", "kv4_decode_attn", "kv4_append_prefill_attn", "step_tables", "release_pages", "adjust_logits"):
            setattr(self, m, getattr(module, m))          # found directly from now on
        return self.__dict__[name]


_calls = _Calls()
_addr = ctypes.addressof


def exported_symbols():
    """Names declared in include/efim.h that the loaded library exports."""
    lib = load_library()
    return [n for n in EXPORTS if hasattr(lib, n)]


def efim_strerror(code) -> str:
    return load_library().efim_strerror(int(code)).decode()


def efim_version() -> int:
    return load_library().efim_version()


def _ptr(t):
    """Device/host address of a torch tensor, numpy array, int or None."""
    if t is None:
        return None
    if isinstance(t, int):
        return t
    if isinstance(t, np.ndarray):
        return t.ctypes.data
    return t.data_ptr()


def _current_stream():
    """The raw handle of torch's current stream (building a Stream object costs 3 us more).  torch is looked up
    on the first call: the host-only parts of the package work without it."""
    global _current_stream
    from torch import _C
    raw_stream, device = _C._cuda_getCurrentRawStream, _C._cuda_getDevice

    def _current_stream():
        return raw_stream(device())
    return _current_stream()


def _stream_ptr(stream):
    if stream is None:
        return _current_stream()
    if isinstance(stream, int):
        return stream
    return stream.cuda_stream


def _current_stream_of(index):
    """torch's current stream, if its device is number `index`."""
    global _current_stream_of
    from torch import _C
    raw_stream, device = _C._cuda_getCurrentRawStream, _C._cuda_getDevice

    def _current_stream_of(index):
        now = device()
        if now != index:
            raise ValueError(f"the tensors are on device {index}, the current one is {now}: torch.cuda.device(...) first")
        return raw_stream(now)
    return _current_stream_of(index)


def _stream_beside(stream, index):
    """The stream of a call on tensors of device `index`; without one given, torch's current stream, which has to be of that device."""
    return _current_stream_of(index) if stream is None else _stream_ptr(stream)


def _torch():
    import torch
    return torch


def _check(ok, what):
    if not ok:
        raise ValueError(what)


class Cache:
    """Paged KV cache of one layer: two torch.bfloat16 CUDA tensors
    [num_pages, num_kv_heads, page_size, head_dim] owned by the caller."""

    def __init__(self, k_pool, v_pool, num_q_heads):
        assert k_pool.shape == v_pool.shape and k_pool.is_contiguous() and v_pool.is_contiguous()
        self.k_pool, self.v_pool = k_pool, v_pool
        n, hkv, p, d = k_pool.shape
        self.head_dim = d
        self.desc = _CacheDesc(k_pool.data_ptr(), v_pool.data_ptr(), n, p, num_q_heads, hkv, d)


class Batch:
    """Ragged batch descriptor.  `cached_len`, `new_len` are host int32 arrays (kept
    as the host mirrors); the device copies and q_indptr are made here with torch."""

    def __init__(self, cached_len, new_len, block_table, device="cuda"):
        import torch
        self.h_cached_len = np.ascontiguousarray(cached_len, dtype=np.int32)
        self.h_new_len = np.ascontiguousarray(new_len, dtype=np.int32)
        indptr = np.zeros(len(self.h_new_len) + 1, dtype=np.int32)
        np.cumsum(self.h_new_len, out=indptr[1:])
        self.h_q_indptr = indptr
        self.d_cached_len = torch.from_numpy(self.h_cached_len).to(device)
        self.d_new_len = torch.from_numpy(self.h_new_len).to(device)
        self.d_q_indptr = torch.from_numpy(indptr).to(device)
        if isinstance(block_table, np.ndarray):
            block_table = torch.from_numpy(np.ascontiguousarray(block_table, dtype=np.int32)).to(device)
        self.d_block_table = block_table
        self.desc = _BatchDesc(len(self.h_new_len), self.d_block_table.shape[1], int(indptr[-1]),
                               self.d_cached_len.data_ptr(), self.d_new_len.data_ptr(),
                               self.d_q_indptr.data_ptr(), self.d_block_table.data_ptr(),
                               self.h_cached_len.ctypes.data, self.h_new_len.ctypes.data)


    @classmethod
    def from_device(cls, cached_len, new_len, q_indptr, block_table, rows):
        """A batch whose lengths only the device knows (what efim_step_tables leaves): int32 CUDA tensors, `rows` rows of q, k and v, of which
        those behind q_indptr's last are not used.  For calls that read no lengths on the host: efim_kv4_append."""
        torch = _torch()
        given = (cached_len, new_len, q_indptr, block_table)
        _check(all(x.dtype == torch.int32 and x.is_contiguous() for x in given) and block_table.dim() == 2,
               "lengths, row offsets and the block table are packed int32 tensors")
        n = block_table.shape[0]
        _check(cached_len.numel() >= n and new_len.numel() >= n and q_indptr.numel() >= n + 1, "a length per sequence, and one more row offset")
        batch = cls.__new__(cls)
        batch.d_cached_len, batch.d_new_len, batch.d_q_indptr, batch.d_block_table = given
        batch.h_cached_len = batch.h_new_len = batch.h_q_indptr = None
        batch.desc = _BatchDesc(n, block_table.shape[1], rows, *(x.data_ptr() for x in given), None, None)
        return batch


class Rope:
    """Rotary table on the device (built on the host by the library in double)."""

    def __init__(self, base, head_dim, max_position, interleaved=False, device="cuda"):
        import torch
        host = efim_rope_table_build(base, head_dim, max_position)
        self.table = torch.from_numpy(host).to(device)
        self.head_dim = head_dim
        self.desc = _RopeDesc(self.table.data_ptr(), max_position, 1 if interleaved else 0)

    @classmethod
    def from_table(cls, table, interleaved=False):
        """A table that is on the device already: fp32 [max_position, head_dim], cos then sin (with any scaling).  Its width has to be
        the head_dim of the caches that it is used with."""
        _check(table.dtype == _torch().float32 and table.dim() == 2 and table.is_contiguous(),
               "the rotary table is a contiguous fp32 matrix")
        rope = cls.__new__(cls)
        rope.table, rope.head_dim = table, table.shape[1]
        rope.desc = _RopeDesc(table.data_ptr(), table.shape[0], 1 if interleaved else 0)
        return rope


def _rope_addr(cache, rope):
    """The kernels know a table's rows but not its width."""
    if rope is None:
        return None
    if rope.head_dim != cache.head_dim:
        raise ValueError(f"the rotary table is for heads of {rope.head_dim}, the cache's have {cache.head_dim}")
    return _addr(rope.desc)


class QkNorm:
    """Norms of query and key heads: weights [head_dim] in bf16 or fp32 on the device, or None for weights of one."""

    def __init__(self, q_weight, k_weight, eps=1e-6, weight_offset=0.0):
        torch = _torch()
        given = [w for w in (q_weight, k_weight) if w is not None]
        _check(all(w.dtype in (torch.bfloat16, torch.float32) and w.dim() == 1 and w.numel() > 0 and w.is_contiguous() for w in given)
               and len({(w.dtype, w.shape) for w in given}) <= 1, "the norms' weights are two bf16 or two fp32 vectors of one length")
        self.q_weight, self.k_weight = q_weight, k_weight
        self.head_dim = given[0].shape[0] if given else 0         # 0: of any
        self.desc = _QkNormDesc(_ptr(q_weight), _ptr(k_weight), 1 if given and given[0].dtype == torch.float32 else 0, eps,
                                weight_offset)


def efim_rope_table_build(base, head_dim, max_position) -> np.ndarray:
    out = np.empty((max_position, head_dim), dtype=np.float32)
    st = load_library().efim_rope_table_build(float(base), head_dim, max_position, out.ctypes.data)
    if st != 0:
        raise EfimError(st, "efim_rope_table_build")
    return out


def _exact(batch):
    """Calls that take every row for a new token have no use for rows behind the last sequence."""
    if batch.h_new_len is None:
        raise ValueError("a batch whose lengths only the device knows goes to the calls over a 4-bit cache")


def efim_kv_append(cache: Cache, batch: Batch, rope, q, k_new, v_new, status=None, stream=None):
    _exact(batch)
    st = _calls.kv_append(_addr(cache.desc), _addr(batch.desc), _rope_addr(cache, rope),
                          q, k_new, v_new, status, _stream_ptr(stream))
    if st != 0:
        raise EfimError(st, "efim_kv_append")


def efim_qk_norm_append(cache: Cache, batch: Batch, norm: QkNorm, rope, q, k, v, q_out, status=None, stream=None):
    """efim_kv_append with a norm of every q and k head before the rotation.  q, k and v: bf16, one row per new token (of any rank
    past the first, packed), views of one buffer allowed; q_out: packed.  q and q_out may both be None."""
    _exact(batch)
    st = _calls.qk_norm_append(_addr(cache.desc), _addr(batch.desc), _addr(norm.desc), norm.head_dim,
                               _rope_addr(cache, rope), q, k, v, q_out, status, _stream_ptr(stream))
    if st != 0:
        raise EfimError(st, "efim_qk_norm_append")


def efim_draft_lookup(history, lengths, min_ngram, max_ngram, drafts, draft_len, status=None, stream=None):
    """Drafts for each row of `history` (int32 [batch, max_len], rows may be further apart) from what followed its last tokens
    earlier on; drafts: int32 [batch, num_drafts]."""
    st = _calls.draft_lookup(history, lengths, min_ngram, max_ngram, drafts, draft_len, status, _stream_ptr(stream))
    if st != 0:
        raise EfimError(st, "efim_draft_lookup")


def efim_verify_workspace_bytes(batch: int, target, target_is_probs=False) -> int:
    """Bytes of workspace for target rows of this shape and type (0: none is needed)."""
    return _calls.verify_workspace_bytes(batch, target, target_is_probs)


def efim_verify_drafts(row_indptr, tokens, target, accepted, next_token, uniform=None, noise=None, draft_probs=None,
                       temperature=None, target_is_probs=False, out_tokens=None, out_logprobs=None, workspace=None, status=None,
                       stream=None):
    """Accepted drafts and next token of every sequence of a step.  target: [rows, vocab] logits in bf16 or fp32, or with
    `target_is_probs` probabilities in fp32; draft_probs fp32 [rows, vocab]; noise fp32 [batch, vocab] (none: greedy); dimensions of
    size 1 between the two are allowed, others are not ([batch, drafts, vocab] is not [rows, vocab]).
    out_tokens and out_logprobs: packed [batch, n] of the same n.  Without a workspace one is taken from torch's allocator, on
    torch's current stream, which the call then has to run on."""
    if workspace is None and stream is not None and _calls.verify_workspace_bytes(accepted.shape[0], target, target_is_probs) and \
            _stream_ptr(stream) != _current_stream():
        raise ValueError("a call on another stream than torch's current one brings its workspace along")
    st = _calls.verify_drafts(accepted.shape[0], row_indptr, tokens, target, target_is_probs, draft_probs, uniform, noise, temperature,
                              accepted, next_token, out_tokens, out_logprobs, workspace, status, _stream_ptr(stream))
    if st != 0:
        raise EfimError(st, "efim_verify_drafts")


class Cache4:
    """KV cache of one layer in 4 bits: torch.uint8 CUDA tensors owned by the caller, codes [num_pages, num_kv_heads, 16, head_dim / 2] and
    scales [num_pages, num_kv_heads, 16, head_dim / 16] of keys and of values; k_scale and v_scale, powers of two, say how large they
    are: about the largest values over 2,688, or a little less where few are that large."""

    def __init__(self, k_codes, v_codes, k_scales, v_scales, num_q_heads, k_scale=1.0, v_scale=1.0):
        torch = _torch()
        pools = (k_codes, v_codes, k_scales, v_scales)
        _check(all(x.dtype == torch.uint8 and x.dim() == 4 and x.is_contiguous() for x in pools), "codes and scales are packed uint8 tensors")
        n, hkv, page, half = k_codes.shape
        _check(v_codes.shape == k_codes.shape and k_scales.shape == v_scales.shape == (n, hkv, page, half // 8),
               "codes are [pages, kv heads, 16, head_dim / 2], scales [pages, kv heads, 16, head_dim / 16]")
        _check(len({x.device for x in pools}) == 1, "codes and scales are on one device")
        self.k_codes, self.v_codes, self.k_scales, self.v_scales = pools
        self.head_dim, self.device_index = 2 * half, k_codes.get_device()
        self.desc = _Cache4Desc(*(x.data_ptr() for x in pools), n, page, num_q_heads, hkv, 2 * half, k_scale, v_scale)

    @classmethod
    def empty(cls, num_pages, num_kv_heads, head_dim, num_q_heads, k_scale=1.0, v_scale=1.0, device="cuda"):
        """A cache with pools of its own, all zeros."""
        torch = _torch()
        codes, scales = ((num_pages, num_kv_heads, 16, head_dim // n) for n in (2, 16))
        return cls(*(torch.zeros(s, dtype=torch.uint8, device=device) for s in (codes, codes, scales, scales)), num_q_heads, k_scale, v_scale)


def efim_kv4_append(cache: Cache4, batch: Batch, norm, rope, q, k, v, q_out, status=None, stream=None):
    """Norm (a QkNorm, or None), rotation (a Rope, or None) and append to a 4-bit cache; operands as for efim_qk_norm_append."""
    st = _calls.kv4_append(_addr(cache.desc), _addr(batch.desc), None if norm is None else _addr(norm.desc), 0 if norm is None else norm.head_dim,
                           _rope_addr(cache, rope), q, k, v, q_out, status, _stream_beside(stream, cache.device_index))
    if st != 0:
        raise EfimError(st, "efim_kv4_append")


def efim_kv4_unpack(cache: Cache4, pages, k_out, v_out, status=None, stream=None):
    """The int32 `pages` of a 4-bit cache as bf16 pages [n, num_kv_heads, 16, head_dim]; k_out or v_out may be None."""
    st = _calls.kv4_unpack(_addr(cache.desc), pages, k_out, v_out, status, _stream_beside(stream, cache.device_index))
    if st != 0:
        raise EfimError(st, "efim_kv4_unpack")


def efim_kv4_decode_workspace_bytes(cache: Cache4, batch: int, max_new_len: int, max_ctx_len: int) -> int:
    return int(load_library().efim_kv4_decode_workspace_bytes(ctypes.byref(cache.desc), batch, max_new_len, max_ctx_len))


def efim_kv4_decode_attn(cache: Cache4, batch: int, d_ctx_len, max_ctx_len, d_block_table, q, out, lse=None, sm_scale=0.0, q_indptr=None,
                         max_new_len=1, workspace=None, status=None, stream=None):
    """Attention of the new tokens (one a sequence; with q_indptr up to max_new_len) over a 4-bit cache that holds them already.  ctx_len
    counts all of a sequence's keys.  q and out: packed [rows, num_q_heads, head_dim]."""
    st = _calls.kv4_decode_attn(_addr(cache.desc), batch, d_ctx_len, int(max_ctx_len), d_block_table, q_indptr, max_new_len, q, out, lse,
                                sm_scale, workspace, status, _stream_beside(stream, cache.device_index))
    if st != 0:
        raise EfimError(st, "efim_kv4_decode_attn")


def efim_kv4_prefill_workspace_bytes(cache: Cache4, batch: Batch) -> int:
    return int(load_library().efim_kv4_prefill_workspace_bytes(ctypes.byref(cache.desc), ctypes.byref(batch.desc)))


def efim_kv4_append_prefill_attn(cache: Cache4, batch: Batch, q, out, lse=None, sm_scale=0.0, workspace=None, status=None, stream=None):
    """Attention of a turn's new tokens, appended already, over a 4-bit cache."""
    st = _calls.kv4_append_prefill_attn(_addr(cache.desc), _addr(batch.desc), q, out, lse, sm_scale, workspace, status, _stream_beside(stream, cache.device_index))
    if st != 0:
        raise EfimError(st, "efim_kv4_append_prefill_attn")


def efim_step_tables_workspace_bytes(batch: int) -> int:
    return int(load_library().efim_step_tables_workspace_bytes(batch))


def _own_workspace(workspace, stream):
    """A workspace that the call takes itself comes from torch's allocator on torch's current stream."""
    if workspace is None and stream is not None and _stream_ptr(stream) != _current_stream():
        raise ValueError("a call on another stream than torch's current one brings its workspace along")


def efim_step_tables(cached_len, new_len, block_table, free_pages, num_free, q_indptr, positions=None, slots=None, sequences=None,
                     block_table_out=None, num_free_out=None, workspace=None, status=None, stream=None):
    """Row offsets, positions, slots and sequences of a step's new tokens, and pages for them from a stack of free ones, all from
    lengths on the device.  Without block_table_out and num_free_out those are changed in place; slots are int64, all else int32."""
    _own_workspace(workspace, stream)
    st = _calls.step_tables(cached_len, new_len, block_table, free_pages, num_free, q_indptr, positions, slots, sequences, block_table_out,
                            num_free_out, workspace, status, _stream_beside(stream, cached_len.get_device()))
    if st != 0:
        raise EfimError(st, "efim_step_tables")


def efim_release_pages(keep_len, block_table, free_pages, num_free, workspace=None, status=None, stream=None):
    """Pages behind each row's first keep_len tokens back to the stack of free ones."""
    _own_workspace(workspace, stream)
    st = _calls.release_pages(keep_len, block_table, free_pages, num_free, workspace, status, _stream_beside(stream, keep_len.get_device()))
    if st != 0:
        raise EfimError(st, "efim_release_pages")


def efim_adjust_logits(row_indptr, logits, out=None, history=None, lengths=None, prompt_len=None, tokens=None, repetition=None,
                       presence=None, frequency=None, bias=None, mask=None, status=None, stream=None):
    """Penalties, biases and grammar masks on a step's rows of logits (bf16 or fp32 [rows, vocab]), in place without `out`.  history: int32
    [batch, max_len] of `lengths` tokens, the first `prompt_len` of them the prompt; tokens: the step's, whose drafts count for the rows
    behind them; bias: (entries' offsets by sequence, tokens, values); mask: int32 [rows, ceil(vocab / 32)], a bit per allowed token."""
    bias_indptr, bias_tokens, bias_values = bias if bias is not None else (None, None, None)
    _check(bias is None or (bias_tokens.numel() == bias_values.numel()), "the bias has as many tokens as values")
    st = _calls.adjust_logits(row_indptr, logits, out, row_indptr.shape[0] - 1, history, lengths, prompt_len, tokens, repetition, presence,
                              frequency, bias_indptr, bias_tokens, bias_values, mask, status, _stream_beside(stream, logits.get_device()))
    if st != 0:
        raise EfimError(st, "efim_adjust_logits")


def efim_prefill_workspace_bytes(cache: Cache, batch: Batch) -> int:
    return int(load_library().efim_prefill_workspace_bytes(ctypes.byref(cache.desc), ctypes.byref(batch.desc)))


def efim_prefill_plan(cache: Cache, batch: Batch) -> np.ndarray:
    """The work list of efim_append_prefill_attn for this batch as a host blob (uint8 array);
    pass it as `plan=` to run without planning, e.g. once per layer."""
    lib = load_library()
    n = int(lib.efim_prefill_plan_bytes(ctypes.byref(cache.desc), ctypes.byref(batch.desc)))
    if n == 0:
        raise EfimError(1, "efim_prefill_plan_bytes")
    blob = np.zeros(n, np.uint8)
    st = lib.efim_prefill_plan(ctypes.byref(cache.desc), ctypes.byref(batch.desc), blob.ctypes.data, n)
    if st != 0:
        raise EfimError(st, "efim_prefill_plan")
    return blob


def efim_append_prefill_attn(cache: Cache, batch: Batch, q, out, lse=None, sm_scale=0.0,
                             workspace=None, status=None, stream=None, plan=None, lists_resident=False):
    st = _calls.append_prefill_attn(_addr(cache.desc), _addr(batch.desc), q, out, lse, sm_scale, workspace, status,
                                    _stream_ptr(stream), plan, 1 if lists_resident else 0)
    if st != 0:
        raise EfimError(st, "efim_append_prefill_attn")


def efim_append_prefill_step(cache: Cache, batch: Batch, rope, q, k_new, v_new, out, lse=None, sm_scale=0.0,
                             workspace=None, status=None, stream=None, plan=None, lists_resident=False):
    """kv_append of the new tokens' k/v, then append-prefill attention of q rotated by its positions.  q is not modified, unless
    out is q (which is allowed): the append may leave the rotated queries in out, where their outputs go afterwards.  A call that
    is refused has changed nothing."""
    st = _calls.append_prefill_step(_addr(cache.desc), _addr(batch.desc), _rope_addr(cache, rope),
                                    q, k_new, v_new, out, lse, sm_scale, plan, 1 if lists_resident else 0, workspace,
                                    status, _stream_ptr(stream))
    if st != 0:
        raise EfimError(st, "efim_append_prefill_step")


def efim_selftest_bounded_wait(limit_ns: int, status, waited_ns=None, stream=None):
    st = load_library().efim_selftest_bounded_wait(int(limit_ns), _ptr(status), _ptr(waited_ns), _stream_ptr(stream))
    if st != 0:
        raise EfimError(st, "efim_selftest_bounded_wait")


def efim_decode_workspace_bytes(cache: Cache, batch: int, max_ctx_len: int) -> int:
    return int(load_library().efim_decode_workspace_bytes(ctypes.byref(cache.desc), batch, max_ctx_len))


def efim_decode_attn(cache: Cache, batch: int, d_ctx_len, max_ctx_len, d_block_table, q, out, lse=None,
                     sm_scale=0.0, workspace=None, status=None, stream=None):
    st = _calls.decode_attn(_addr(cache.desc), batch, d_ctx_len, int(max_ctx_len), d_block_table, d_block_table.shape[1],
                            q, out, lse, sm_scale, workspace, status, _stream_ptr(stream))
    if st != 0:
        raise EfimError(st, "efim_decode_attn")


def efim_decode_static_scratch_bytes() -> int:
    return int(load_library().efim_decode_static_scratch_bytes())


def efim_decode_attn_static(cache: Cache, batch: int, d_ctx_len, max_ctx_len, d_block_table, q, out, lse=None,
                            sm_scale=0.0, status=None, stream=None):
    """efim_decode_attn for callers that cannot allocate a workspace: the chunk
    partials use the library's fixed 8 MiB array (shared by all calls on the device)."""
    st = load_library().efim_decode_attn_static(ctypes.byref(cache.desc), batch, _ptr(d_ctx_len), int(max_ctx_len),
                                                _ptr(d_block_table), int(d_block_table.shape[1]), _ptr(q),
                                                _ptr(out), _ptr(lse), float(sm_scale), _ptr(status),
                                                _stream_ptr(stream))
    if st != 0:
        raise EfimError(st, "efim_decode_attn_static")


def efim_prefill_launch_count(cache: Cache, batch: Batch) -> int:
    return int(load_library().efim_prefill_launch_count(ctypes.byref(cache.desc), ctypes.byref(batch.desc)))


def efim_decode_launch_count(cache: Cache, batch: int, max_ctx_len: int) -> int:
    return int(load_library().efim_decode_launch_count(ctypes.byref(cache.desc), batch, max_ctx_len))


class Frontend:
    """The host-side front end of include/efim.h (prompt transformation of Sec. 3.1 and
    page-granular cross-request KV reuse); every method is one C call on numpy arrays."""

    def __init__(self, tok_p, tok_s, tok_m, num_pages, page_size=16, rebase_inc_tokens=0):
        self._lib = load_library()
        self._fe = self._lib.efim_frontend_create(tok_p, tok_s, tok_m, rebase_inc_tokens, num_pages, page_size)
        if not self._fe:
            raise EfimError(1, "efim_frontend_create")
        self.page_size = page_size

    def close(self):
        if self._fe:
            self._lib.efim_frontend_destroy(self._fe)
            self._fe = None

    def __del__(self):
        self.close()

    def transform(self, user, prefix, suffix):
        """-> (prompt int32 array, format, inc_len)."""
        prefix = np.ascontiguousarray(prefix, np.int32)
        suffix = np.ascontiguousarray(suffix, np.int32)
        out = np.empty(len(prefix) + len(suffix) + 3, np.int32)
        n, fmt, inc = c_int32(), c_int32(), c_int32()
        st = self._lib.efim_frontend_transform(self._fe, int(user), prefix.ctypes.data, len(prefix),
                                               suffix.ctypes.data, len(suffix), out.ctypes.data, len(out),
                                               ctypes.addressof(n), ctypes.addressof(fmt), ctypes.addressof(inc))
        if st != 0:
            raise EfimError(st, "efim_frontend_transform")
        return out[:n.value], fmt.value, inc.value

    def admit(self, prompt, reserve_tokens, block_table_row):
        """Fills `block_table_row` (int32 numpy row) -> (handle, cached_len, pages used)."""
        prompt = np.ascontiguousarray(prompt, np.int32)
        assert block_table_row.dtype == np.int32 and block_table_row.flags.c_contiguous
        cached, npages, handle = c_int32(), c_int32(), ctypes.c_int64()
        st = self._lib.efim_frontend_admit(self._fe, prompt.ctypes.data, len(prompt), int(reserve_tokens),
                                           block_table_row.ctypes.data, len(block_table_row),
                                           ctypes.addressof(cached), ctypes.addressof(npages),
                                           ctypes.addressof(handle))
        if st != 0:
            raise EfimError(st, "efim_frontend_admit")
        return handle.value, cached.value, npages.value

    def finish(self, handle, tokens):
        tokens = np.ascontiguousarray(tokens, np.int32)
        st = self._lib.efim_frontend_finish(self._fe, int(handle), tokens.ctypes.data, len(tokens))
        if st != 0:
            raise EfimError(st, "efim_frontend_finish")

    def stats(self):
        out = np.zeros(4, np.int64)
        self._lib.efim_frontend_stats(self._fe, out.ctypes.data)
        return dict(prompt_tokens=int(out[0]), hit_tokens=int(out[1]), evictions=int(out[2]), free_pages=int(out[3]))


def efim_decode_step(cache: Cache, batch: int, d_ctx_len, max_ctx_len, d_block_table, rope, q, k_new, v_new, out,
                     lse=None, sm_scale=0.0, workspace=None, status=None, stream=None):
    """kv_append of one token per row and decode attention in one launch (q is not modified)."""
    st = _calls.decode_step(_addr(cache.desc), batch, d_ctx_len, int(max_ctx_len), d_block_table, d_block_table.shape[1],
                            _rope_addr(cache, rope), q, k_new, v_new, out, lse, sm_scale,
                            workspace, status, _stream_ptr(stream))
    if st != 0:
        raise EfimError(st, "efim_decode_step")
