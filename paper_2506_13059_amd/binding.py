"""Thin ctypes binding of libmp.so: argument marshalling only.

Every step of the path runs inside the library's HIP kernels; torch supplies device memory
(``tensor.data_ptr()``) and the current stream.  There is no CPU fallback: if the library is
missing, importing or calling fails loudly.
"""
from __future__ import annotations

import ctypes as C
import os

import torch

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libmp.so")

MP_OK, MP_EINVAL, MP_ENOMEM, MP_ESTATE, MP_ECAPACITY, MP_EHIP = range(6)
MP_DECODE_NO_MULTIPOLE = 1

EXPORTS = [
    "mp_create", "mp_destroy", "mp_last_error", "mp_device_bytes", "mp_plan_blocks", "mp_cluster_kv",
    "mp_set_clustering", "mp_update_clusters", "mp_decode_attention", "mp_get_sizes", "mp_get_assignments",
    "mp_get_centroids", "mp_get_selection", "mp_get_counters", "mp_get_layout", "mp_dense_workspace_bytes",
    "mp_dense_attention", "mp_version", "mp_enable_stage_timing", "mp_get_stage_timing", "mp_update_seed_counts", "mp_local_buffer_init", "mp_local_buffer_size", "mp_decode_step",
    "mp_dense_static_scratch_bytes", "mp_dense_attention_static", "mp_get_kv_codes", "mp_rotary_frequencies", "mp_rotary",
    "mp_paged_append", "mp_paged_attention", "mp_paged_gather", "mp_paged_workspace_bytes", "mp_norm_rotary", "mp_paged_append_norm", "mp_paged_reserve",
    "mp_paged_tree_plan", "mp_paged_tree_attention", "mp_paged_tree_keep",
]

MP_KV_BF16, MP_KV_E4M3 = 0, 1
MP_ROTARY_HALF, MP_ROTARY_INTERLEAVED = 0, 1
MP_ROTARY_PLAIN, MP_ROTARY_LINEAR, MP_ROTARY_BASE, MP_ROTARY_BY_PARTS = range(4)
MP_TREE_EVERY_ROW = 256


class MpError(RuntimeError):
    def __init__(self, status, msg):
        super().__init__(f"mp status {status}: {msg}")
        self.status = status


class MpConfig(C.Structure):
    _fields_ = [(n, C.c_int32) for n in (
        "batch", "n_q_heads", "n_kv_heads", "head_dim", "max_tokens", "levels", "max_fine", "max_coarse",
        "block_w", "block_alpha", "max_tail", "lookup_keys")] + [("softmax_scale", C.c_float), ("kv_format", C.c_int32)]


class MpRotarySpec(C.Structure):
    _fields_ = [("freqs", C.c_void_p), ("rot_dim", C.c_int32), ("layout", C.c_int32), ("amplitude", C.c_float)]


class MpHeadNormSpec(C.Structure):
    _fields_ = [("weight", C.c_void_p), ("n_heads", C.c_int32), ("offset", C.c_float), ("eps", C.c_float)]


class MpPagePoolArgs(C.Structure):
    _fields_ = [(n, C.c_void_p) for n in ("page_table", "kv_len", "q_start", "free_pages", "n_free")] + \
               [(n, C.c_int32) for n in ("n_pages", "page_size", "n_seqs", "table_stride")]


class MpPagedKvArgs(C.Structure):
    _fields_ = [(n, C.c_void_p) for n in ("k_pages", "v_pages", "page_table", "kv_len", "q_start")] + \
               [(n, C.c_int32) for n in ("n_pages", "page_size", "n_kv_heads", "head_dim", "n_seqs", "table_stride")]


_lib = None


def lib():
    """Load libmp.so (built beforehand by paper_2506_13059_amd.build); raises if it is missing."""
    global _lib
    if _lib is None:
        if not os.path.exists(LIB_PATH):
            raise FileNotFoundError(
                f"{LIB_PATH} is missing: build it first with `python -m paper_2506_13059_amd.build`")
        L = C.CDLL(LIB_PATH)
        vp, i32, u64, u32, f32, sz = C.c_void_p, C.c_int32, C.c_uint64, C.c_uint32, C.c_float, C.c_size_t
        L.mp_version.restype = C.c_char_p
        L.mp_last_error.restype = C.c_char_p
        L.mp_last_error.argtypes = [vp]
        L.mp_create.argtypes = [C.POINTER(MpConfig), C.POINTER(vp)]
        L.mp_destroy.argtypes = [vp]
        L.mp_destroy.restype = None
        L.mp_device_bytes.argtypes = [vp]
        L.mp_device_bytes.restype = sz
        L.mp_plan_blocks.argtypes = [i32, i32, i32, i32, i32, vp, i32]
        L.mp_plan_blocks.restype = i32
        L.mp_cluster_kv.argtypes = [vp, vp, vp, vp, i32, i32, i32, i32, u64, vp, vp, vp]
        L.mp_set_clustering.argtypes = [vp, vp, vp, vp, i32, vp, i32, vp, i32, vp]
        L.mp_update_clusters.argtypes = [vp, vp, vp, vp, i32, i32, i32, i32, i32, u64, vp, vp]
        L.mp_decode_attention.argtypes = [vp, vp, vp, vp, vp, i32, i32, i32, i32, u32, vp, vp, vp]
        L.mp_update_seed_counts.argtypes = [vp, i32, i32, i32, vp]
        L.mp_local_buffer_init.argtypes = [vp, i32, vp, vp, i32, vp, vp, vp, i32, vp]
        L.mp_local_buffer_size.argtypes = [vp, vp, vp, vp]
        L.mp_decode_step.argtypes = [vp, vp, vp, vp, vp, vp, i32, i32, u32, i32, i32, i32, i32, u64, vp, vp, vp, vp]
        L.mp_update_seed_counts.restype = i32
        L.mp_enable_stage_timing.argtypes = [vp, i32]
        L.mp_get_stage_timing.argtypes = [vp, vp]
        L.mp_get_sizes.argtypes = [vp, vp, vp, vp, vp]
        L.mp_get_assignments.argtypes = [vp, vp, vp, vp]
        L.mp_get_centroids.argtypes = [vp, i32, vp, vp, vp, vp]
        L.mp_get_selection.argtypes = [vp, vp, vp, vp, vp, vp]
        L.mp_get_counters.argtypes = [vp, vp, vp]
        L.mp_get_layout.argtypes = [vp, vp, vp, vp, vp, vp]
        L.mp_get_kv_codes.argtypes = [vp, vp, vp, vp, vp]
        L.mp_dense_workspace_bytes.argtypes = [i32, i32, i32, i32]
        L.mp_dense_workspace_bytes.restype = sz
        L.mp_dense_attention.argtypes = [vp, vp, vp, i32, i32, i32, i32, f32, vp, vp, vp, sz, vp]
        L.mp_dense_static_scratch_bytes.argtypes = []
        L.mp_dense_static_scratch_bytes.restype = sz
        L.mp_dense_attention_static.argtypes = [vp, vp, vp, i32, i32, i32, i32, f32, vp, vp, vp]
        i64, f64 = C.c_int64, C.c_double
        L.mp_rotary_frequencies.argtypes = [i32, f64, i32, f64, f64, f64, f64, vp]
        L.mp_rotary.argtypes = [vp, vp, i64, vp, i32, i32, vp, i64, vp, i32, vp]
        L.mp_paged_append.argtypes = [vp, vp, vp, i64, i32, vp, vp, i64, vp, i64, i32, vp]
        L.mp_paged_attention.argtypes = [vp, vp, i64, i32, i32, i32, i32, f32, vp, vp, vp, sz, vp]
        L.mp_paged_gather.argtypes = [vp, vp, i32, i32, i32, vp, vp, vp, vp]
        L.mp_norm_rotary.argtypes = [vp, vp, vp, i64, vp, i32, i32, vp, i64, vp, i32, vp]
        L.mp_paged_append_norm.argtypes = [vp, vp, vp, vp, vp, vp, i64, i32, vp, vp, i64, vp, i64, i32, vp]
        L.mp_paged_reserve.argtypes = [vp, vp, vp, vp, vp, vp, vp, i32, vp]
        L.mp_paged_tree_plan.argtypes = [vp, vp, i32, i32, vp, vp, vp]
        L.mp_paged_tree_attention.argtypes = [vp, vp, i64, vp, i32, i32, i32, i32, i32, f32, vp, vp, vp, sz, vp]
        L.mp_paged_tree_keep.argtypes = [vp, vp, i32, i32, vp, vp, vp]
        L.mp_paged_workspace_bytes.argtypes = [i32, i32, i32, i32, i32]
        L.mp_paged_workspace_bytes.restype = sz
        _lib = L
    return _lib


# (a short decode or dense call is over in 11 to 15 us on the device and cost as much here: addresses go as plain integers, which the
# declared argument types take, and the stream's handle is asked for without an object around it -- enqueueing a dense call
# 11.6 -> 8 us, a decode step 14 -> 11)
def _ptr(t):
    if t is None:
        return None
    assert t.is_contiguous(), "tensors passed to the library must be contiguous"
    return t.data_ptr()


def _stream():
    return torch._C._cuda_getCurrentRawStream(torch.cuda.current_device())


_stream_of = torch._C._cuda_getCurrentRawStream


def _check(status, ctx=None):
    if status != MP_OK:
        msg = lib().mp_last_error(ctx).decode()
        raise MpError(status, msg)


def _host_i32(t):
    """Host int32 array argument: accepts a CPU int32 tensor (or None)."""
    if t is None:
        return None, None
    t = t.to(dtype=torch.int32, device="cpu").contiguous()
    return t, C.c_void_p(t.data_ptr())


def mp_plan_blocks(n_tokens, block_w, block_alpha, n_fine, n_coarse):
    n = lib().mp_plan_blocks(n_tokens, block_w, block_alpha, n_fine, n_coarse, None, 0)
    if n < 0:
        raise MpError(MP_EINVAL, "mp_plan_blocks: invalid arguments")
    buf = (C.c_int32 * (6 * n))()
    lib().mp_plan_blocks(n_tokens, block_w, block_alpha, n_fine, n_coarse, C.cast(buf, C.c_void_p), n)
    keys = ("t0", "t1", "f0", "f1", "c0", "c1")
    return [dict(zip(keys, buf[6 * i:6 * i + 6])) for i in range(n)]


def mp_dense_workspace_bytes(batch, n_q_heads, n_kv_heads, n):
    return int(lib().mp_dense_workspace_bytes(batch, n_q_heads, n_kv_heads, n))


def mp_dense_attention(q, k, v, out=None, lse=None, workspace=None, softmax_scale=0.0):
    """q [B,Hq,128], k/v [B,Hkv,n,128] bf16 CUDA tensors -> out [B,Hq,128] bf16 (and lse fp32 [B,Hq])."""
    B, Hq, _ = q.shape
    Hkv, n = k.shape[1], k.shape[2]
    if workspace is None:
        workspace = torch.empty(max(mp_dense_workspace_bytes(B, Hq, Hkv, n), 16), dtype=torch.uint8, device=q.device)
    if out is None:
        out = torch.empty_like(q)
    st = lib().mp_dense_attention(_ptr(q), _ptr(k), _ptr(v), B, Hq, Hkv, n, softmax_scale, _ptr(out), _ptr(lse),
                                  _ptr(workspace), workspace.numel() * workspace.element_size(), _stream())
    _check(st)
    return out


def mp_dense_static_scratch_bytes():
    return int(lib().mp_dense_static_scratch_bytes())


def mp_dense_attention_static(q, k, v, out, lse=None, softmax_scale=0.0):
    """mp_dense_attention without a workspace: `out` (and lse) are the caller's, nothing is allocated."""
    B, Hq, _ = q.shape
    Hkv, n = k.shape[1], k.shape[2]
    st = lib().mp_dense_attention_static(_ptr(q), _ptr(k), _ptr(v), B, Hq, Hkv, n, softmax_scale, _ptr(out), _ptr(lse),
                                         _stream())
    _check(st)
    return out


def _reject(msg):
    raise MpError(MP_EINVAL, msg)


# (a call for a few tokens is over in 5 us on the device: the checks look at each tensor once and ask for the current device once a call)
def _dense(t, name, dtype, shape, device):
    """A contiguous tensor on the current device, of the type and shape that the kernels take it to have."""
    if t.dtype is not dtype or t.get_device() != device or t.shape != shape or not t.is_contiguous():
        _reject(f"{name}: a contiguous tensor {tuple(shape)} of {dtype} on the current device expected, got {tuple(t.shape)} with strides {t.stride()} of {t.dtype} "
                f"on {t.device}")
    return t


def _token_rows(t, name, device):
    """(tokens, heads, token stride) of a bf16 tensor [tokens, heads, 128] whose tokens may be apart, as in the rows of a fused projection."""
    if t.dtype is torch.bfloat16 and t.get_device() == device and t.dim() == 3:
        n, h, d = t.shape
        s0, s1, s2 = t.stride()
        if d == 128 and s2 == 1 and (s1 == 128 or h <= 1) and (n <= 1 or s0 >= h * 128):      # (a broadcast token's stride of 0 would mean densely packed)
            return n, h, s0 if n > 1 else 0
    _reject(f"{name}: bf16 [tokens, heads, 128] on the current device, each token's rows behind one another, expected, got {tuple(t.shape)} with strides {t.stride()} of "
            f"{t.dtype} on {t.device}")


_here = torch.cuda.current_device


def mp_rotary_frequencies(rot_dim=128, base=10000.0, scaling=MP_ROTARY_PLAIN, factor=1.0, original_len=0.0, low=1.0, high=32.0):
    """fp64 CPU tensor [rot_dim / 2]: radians a position of every pair."""
    out = torch.empty(max(rot_dim // 2, 1), dtype=torch.float64)
    _check(lib().mp_rotary_frequencies(rot_dim, base, scaling, factor, original_len, low, high, out.data_ptr()))
    return out


class MpHeadNorm:
    """Norm of a head's rows, x / sqrt(mean(x^2) + eps) * (weight + offset): weight bf16 [128], the same for all heads, or [heads, 128], on the current device."""

    def __init__(self, weight, offset=0.0, eps=1e-6):
        heads = weight.shape[0] if weight.dim() == 2 else 1
        self.weight = _dense(weight, "weight", torch.bfloat16, (heads, 128) if weight.dim() == 2 else (128,), _here())
        self.device = self.weight.get_device()
        self.spec = MpHeadNormSpec(self.weight.data_ptr(), heads, offset, eps)
        self.at = C.addressof(self.spec)

    def _on(self, device):
        if self.device != device:
            _reject(f"the weights lie on device {self.device}, the tensors on device {device}")
        return self.at


class MpRotary:
    """Rotary positions: frequencies on the current device (given, or worked out by mp_rotary_frequencies), layout and amplitude."""

    def __init__(self, rot_dim=128, layout=MP_ROTARY_HALF, base=10000.0, scaling=MP_ROTARY_PLAIN, factor=1.0, original_len=0.0, low=1.0, high=32.0,
                 amplitude=1.0, freqs=None):
        if freqs is None:
            freqs = mp_rotary_frequencies(rot_dim, base, scaling, factor, original_len, low, high).cuda()
        self.freqs = _dense(freqs, "freqs", torch.float64, (rot_dim // 2,), _here())
        self.device = self.freqs.get_device()
        self.spec = MpRotarySpec(self.freqs.data_ptr(), rot_dim, layout, amplitude)
        self.at = C.addressof(self.spec)

    def _on(self, device):
        if self.device != device:
            _reject(f"the frequencies lie on device {self.device}, the tensors on device {device}")
        return self.at

    def mp_rotary(self, x, positions=None, out=None, lookup_position=None, out_lookup=None):
        """x bf16 [tokens, heads, 128] at positions int32 [tokens] -> out (like x, densely packed; `out` may be x).  With a lookup_position:
        (out, out_lookup), out_lookup turned to that one position; positions may then be None for the second alone."""
        return self._turn(None, x, positions, out, lookup_position, out_lookup)

    def mp_norm_rotary(self, norm, x, positions=None, out=None, lookup_position=None, out_lookup=None):
        """mp_rotary of rows that are normed first (norm: MpHeadNorm), in the same pass."""
        if norm is None:
            _reject("the norm is missing")
        return self._turn(norm, x, positions, out, lookup_position, out_lookup)

    def _turn(self, norm, x, positions, out, lookup_position, out_lookup):
        device = _here()
        n, h, stride = _token_rows(x, "x", device)
        to_stride = to = look = at = 0
        if positions is not None:
            at = _dense(positions, "positions", torch.int32, (n,), device).data_ptr()
            if out is None:
                out = x.new_empty(n, h, 128)
            else:
                no, ho, to_stride = _token_rows(out, "out", device)
                if no != n or ho != h:
                    _reject(f"out: [{n}, {h}, 128] expected, got {tuple(out.shape)}")
            to = out.data_ptr()
        elif out is not None or lookup_position is None:
            _reject("positions are missing")
        if lookup_position is not None:
            if out_lookup is None:
                out_lookup = x.new_empty(n, h, 128)
            else:
                _dense(out_lookup, "out_lookup", torch.bfloat16, (n, h, 128), device)
            look = out_lookup.data_ptr()
        elif out_lookup is not None:
            _reject("out_lookup needs a lookup_position")
        args = (self._on(device), x.data_ptr(), stride, at, n, h, to, to_stride, look, lookup_position or 0, _stream_of(device))
        st = lib().mp_rotary(*args) if norm is None else lib().mp_norm_rotary(norm._on(device), *args)
        if st:
            _check(st)
        return out if lookup_position is None else (out, out_lookup)


def mp_paged_workspace_bytes(n_tokens, n_q_heads, n_kv_heads, n_seqs, max_new):
    return int(lib().mp_paged_workspace_bytes(n_tokens, n_q_heads, n_kv_heads, n_seqs, max_new))


class MpPagedKv:
    """A batch of sequences over a paged cache: k_pages, v_pages bf16 [n_pages, Hkv, page_size, 128], page_table int32 [n_seqs, pages],
    kv_len int32 [n_seqs], q_start int32 [n_seqs + 1].  The tensors are kept, not copied: change them in place between calls."""

    def __init__(self, k_pages, v_pages, page_table, kv_len, q_start):
        device = self.device = _here()
        if k_pages.dim() != 4 or page_table.dim() != 2:
            _reject(f"k_pages [n_pages, Hkv, page_size, 128] and page_table [n_seqs, pages] expected, got {tuple(k_pages.shape)} and {tuple(page_table.shape)}")
        n_pages, self.n_kv_heads, page_size, d = k_pages.shape
        self.n_seqs = page_table.shape[0]
        _dense(k_pages, "k_pages", torch.bfloat16, k_pages.shape, device)
        _dense(v_pages, "v_pages", torch.bfloat16, k_pages.shape, device)
        _dense(page_table, "page_table", torch.int32, page_table.shape, device)
        _dense(kv_len, "kv_len", torch.int32, (self.n_seqs,), device)
        _dense(q_start, "q_start", torch.int32, (self.n_seqs + 1,), device)
        self.tensors = (k_pages, v_pages, page_table, kv_len, q_start)
        self.args = MpPagedKvArgs(*(t.data_ptr() for t in self.tensors), n_pages, page_size, self.n_kv_heads, d, self.n_seqs, page_table.shape[1])
        self.at = C.addressof(self.args)

    def _current(self):
        device = _here()
        if self.device != device:
            _reject(f"the cache lies on device {self.device}, not on the current device {device}")
        return device

    def mp_paged_append(self, k, v, rotary=None, q=None, q_out=None):
        """k, v bf16 [tokens, Hkv, 128] join the cache; returns the turned queries q_out [tokens, Hq, 128], or None without q."""
        return self._append(k, v, rotary, q, q_out, False)

    def mp_paged_append_norm(self, k, v, rotary=None, q=None, q_out=None, q_norm=None, k_norm=None, positions=None):
        """mp_paged_append of queries and keys that are normed first (q_norm, k_norm: MpHeadNorm, or None for rows that are not), turned to positions int32
        [tokens], or None: to where they stand in their sequences."""
        return self._append(k, v, rotary, q, q_out, True, q_norm, k_norm, positions)

    def _append(self, k, v, rotary, q, q_out, norms, q_norm=None, k_norm=None, positions=None):
        device = self._current()
        n, h, ks = _token_rows(k, "k", device)
        nv, hv, vs = _token_rows(v, "v", device)
        if h != self.n_kv_heads or hv != h or nv != n:
            _reject(f"k, v: [tokens, {self.n_kv_heads}, 128] expected, got {tuple(k.shape)} and {tuple(v.shape)}")
        hq = qs = from_ = to = 0
        if q is not None:
            nq, hq, qs = _token_rows(q, "q", device)
            if nq != n:
                _reject(f"q: {n} tokens expected, got {nq}")
            if q_out is None:
                q_out = q.new_empty(n, hq, 128)
            else:
                _dense(q_out, "q_out", torch.bfloat16, (n, hq, 128), device)
            from_, to = q.data_ptr(), q_out.data_ptr()
        elif q_out is not None:
            _reject("q_out needs q")
        turn = None if rotary is None else rotary._on(device)
        rows = (from_, qs, hq, to, k.data_ptr(), ks, v.data_ptr(), vs, n, _stream_of(device))
        if norms:
            at = 0 if positions is None else _dense(positions, "positions", torch.int32, (n,), device).data_ptr()
            st = lib().mp_paged_append_norm(self.at, turn, None if q_norm is None else q_norm._on(device), None if k_norm is None else k_norm._on(device), at, *rows)
        else:
            st = lib().mp_paged_append(self.at, turn, *rows)
        if st:
            _check(st)
        return q_out

    def mp_paged_attention(self, q, max_new=0, window=0, softmax_scale=0.0, out=None, lse=None, workspace=None):
        """q bf16 [tokens, Hq, 128] -> out bf16 [tokens, Hq, 128] (and lse fp32 [tokens, Hq]); max_new: as many new tokens a sequence at most.  0 stands for
        as many as q has: a decode step passes 1, which takes the kernel for it, probabilities in two bf16 parts and 4 MiB of workspace.  Without a workspace one is
        allocated (up to 69 MiB)."""
        return self._attend(q, None, max_new, window, softmax_scale, out, lse, workspace)

    def mp_paged_tree_attention(self, q, mask, max_new=0, window=0, softmax_scale=0.0, out=None, lse=None, workspace=None):
        """mp_paged_attention of a tree's tokens: each attends its sequence's older keys and the new ones that its mask (int64 [tokens, words]) marks."""
        if mask is None:
            _reject("the mask is missing")
        return self._attend(q, mask, max_new, window, softmax_scale, out, lse, workspace)

    def _attend(self, q, mask, max_new, window, softmax_scale, out, lse, workspace):
        device = self._current()
        n, hq, qs = _token_rows(q, "q", device)
        if out is None:
            out = q.new_empty(n, hq, 128)
        else:
            _dense(out, "out", torch.bfloat16, (n, hq, 128), device)
        if lse is not None:
            _dense(lse, "lse", torch.float32, (n, hq), device)
        if workspace is None:
            workspace = torch.empty(mp_paged_workspace_bytes(n, hq, self.n_kv_heads, self.n_seqs, max_new), dtype=torch.uint8, device=q.device)
        elif workspace.get_device() != device or not workspace.is_contiguous():
            _reject(f"workspace: a contiguous tensor on the current device expected, got one on {workspace.device}")
        rest = (n, hq, max_new, window, softmax_scale, out.data_ptr(), None if lse is None else lse.data_ptr(), workspace.data_ptr(), workspace.nbytes, _stream_of(device))
        if mask is None:
            st = lib().mp_paged_attention(self.at, q.data_ptr(), qs, *rest)
        else:
            at, words = self._mask(mask, n, device)
            st = lib().mp_paged_tree_attention(self.at, q.data_ptr(), qs, at, words, *rest)
        if st:
            _check(st)
        return out

    def _mask(self, mask, n, device):
        if mask.dim() != 2:
            _reject(f"mask: int64 [{n}, words] expected, got {tuple(mask.shape)}")
        return _dense(mask, "mask", torch.int64, (n, mask.shape[1]), device).data_ptr(), mask.shape[1]

    def mp_paged_tree_plan(self, parents, mask_words=1, mask=None, positions=None):
        """parents int32 [tokens], numbers within a sequence's new tokens (no token before it: none) -> (mask int64 [tokens, mask_words] of each token and its
        ancestors, positions int32 [tokens]).  Tokens of a sequence from 64 * mask_words on, and rows of no sequence, have no result: a mask of zeros and position -1
        in tensors that are made here; in tensors that are passed, such rows are left as they were."""
        device = self._current()
        n = parents.shape[0] if parents.dim() == 1 else -1
        _dense(parents, "parents", torch.int32, (n,), device)
        if not 1 <= mask_words <= 16:
            _reject(f"mask_words = {mask_words} is not 1 .. 16")
        words = mask_words
        if mask is None and positions is None:
            words |= MP_TREE_EVERY_ROW
            mask, positions = parents.new_empty(n, mask_words, dtype=torch.int64), torch.empty_like(parents)
        else:
            mask = parents.new_zeros((n, mask_words), dtype=torch.int64) if mask is None else _dense(mask, "mask", torch.int64, (n, mask_words), device)
            positions = torch.full_like(parents, -1) if positions is None else _dense(positions, "positions", torch.int32, (n,), device)
        st = lib().mp_paged_tree_plan(self.at, parents.data_ptr(), n, words, mask.data_ptr(), positions.data_ptr(), _stream_of(device))
        if st:
            _check(st)
        return mask, positions

    def mp_paged_tree_keep(self, mask, leaf, keep=None):
        """The rows of the path that ends in new token leaf[b] (int32 [n_seqs]; anything else: none) moved together behind the older ones -> keep int32 [n_seqs], the
        keys that stay of each sequence."""
        device = self._current()
        n = mask.shape[0]
        at, words = self._mask(mask, n, device)
        _dense(leaf, "leaf", torch.int32, (self.n_seqs,), device)
        keep = torch.empty_like(leaf) if keep is None else _dense(keep, "keep", torch.int32, (self.n_seqs,), device)
        st = lib().mp_paged_tree_keep(self.at, at, words, n, leaf.data_ptr(), keep.data_ptr(), _stream_of(device))
        if st:
            _check(st)
        return keep

    def mp_paged_gather(self, n, first=0, rotary=None, lookup_position=None, k=None, v=None, k_lookup=None):
        """Keys and values [first, first + n) of every sequence: (k, v) bf16 [n_seqs, Hkv, n, 128], with a lookup_position (k, v, k_lookup).  Rows that a
        sequence does not hold are zero, and would be keys to mp_cluster_kv: gather sequences of other lengths through an MpPagedKv of their own (page_table[b:b + 1], ...)."""
        device = self._current()
        if n < 0:
            _reject(f"n = {n} < 0")
        shape, pages = (self.n_seqs, self.n_kv_heads, n, 128), self.tensors[0]
        k, v = (pages.new_empty(shape) if t is None else _dense(t, "k, v", torch.bfloat16, shape, device) for t in (k, v))
        look = 0
        if lookup_position is not None:
            if rotary is None:
                _reject("a lookup_position needs the rotary that the keys were stored with")
            k_lookup = pages.new_empty(shape) if k_lookup is None else _dense(k_lookup, "k_lookup", torch.bfloat16, shape, device)
            look = k_lookup.data_ptr()
        elif k_lookup is not None:
            _reject("k_lookup needs a lookup_position")
        if n > 0 and self.n_seqs > 0:
            _check(lib().mp_paged_gather(self.at, None if rotary is None else rotary._on(device), first, n, lookup_position or 0, k.data_ptr(), look, v.data_ptr(),
                                         _stream_of(device)))
        return (k, v) if lookup_position is None else (k, v, k_lookup)


class MpPagePool:
    """Pages in no use beside the tensors of an MpPagedKv (the same page_table, kv_len and q_start): free_pages int32 [n_pages], a stack of which the first n_free
    (int32 [1]) entries count.  The tensors are kept, not copied, and changed in place."""

    def __init__(self, page_table, kv_len, q_start, free_pages, n_free, page_size):
        device = self.device = _here()
        if page_table.dim() != 2 or free_pages.dim() != 1:
            _reject(f"page_table [n_seqs, pages] and free_pages [n_pages] expected, got {tuple(page_table.shape)} and {tuple(free_pages.shape)}")
        self.n_seqs, columns = page_table.shape
        _dense(page_table, "page_table", torch.int32, page_table.shape, device)
        _dense(kv_len, "kv_len", torch.int32, (self.n_seqs,), device)
        _dense(q_start, "q_start", torch.int32, (self.n_seqs + 1,), device)
        _dense(free_pages, "free_pages", torch.int32, free_pages.shape, device)
        _dense(n_free, "n_free", torch.int32, (1,), device)
        self.tensors = (page_table, kv_len, q_start, free_pages, n_free)
        self.args = MpPagePoolArgs(*(t.data_ptr() for t in self.tensors), free_pages.shape[0], page_size, self.n_seqs, columns)
        self.at = C.addressof(self.args)

    def mp_paged_reserve(self, n_new, keep=None, granted=None, sequence=None, positions=None, slots=None):
        """Pages of keys past keep (int32 [n_seqs]; None: all stay) go back, n_new (int32 [n_seqs]) tokens get theirs; kv_len and q_start follow.  granted int32 [n_seqs],
        and of the step's rows sequence, positions int32 [rows], slots int64 [rows] are written where they are passed (as many rows in each)."""
        device = _here()
        if self.device != device:
            _reject(f"the pool lies on device {self.device}, not on the current device {device}")
        _dense(n_new, "n_new", torch.int32, (self.n_seqs,), device)
        if keep is not None:
            _dense(keep, "keep", torch.int32, (self.n_seqs,), device)
        if granted is not None:
            _dense(granted, "granted", torch.int32, (self.n_seqs,), device)
        rows = None
        for t, name, dtype in ((sequence, "sequence", torch.int32), (positions, "positions", torch.int32), (slots, "slots", torch.int64)):
            if t is not None:
                rows = (t.shape[0] if t.dim() == 1 else -1) if rows is None else rows
                _dense(t, name, dtype, (rows,), device)
        st = lib().mp_paged_reserve(self.at, n_new.data_ptr(), *(None if t is None else t.data_ptr() for t in (keep, granted, sequence, positions, slots)), rows or 0,
                                    _stream_of(device))
        if st:
            _check(st)


class MpContext:
    """Owns an mp_ctx handle.  Method names and arguments mirror the C entry points."""

    def __init__(self, batch, n_q_heads, n_kv_heads, max_tokens, levels, max_fine, max_coarse=0, block_w=0,
                 block_alpha=0, max_tail=0, softmax_scale=0.0, head_dim=128, lookup_keys=False, kv_format=MP_KV_BF16):
        self.cfg = MpConfig(batch, n_q_heads, n_kv_heads, head_dim, max_tokens, levels, max_fine, max_coarse,
                            block_w, block_alpha, max_tail, 1 if lookup_keys else 0, softmax_scale, kv_format)
        self.kv_format = kv_format
        self.h = C.c_void_p()
        st = lib().mp_create(C.byref(self.cfg), C.byref(self.h))
        _check(st)
        self.U = batch * n_kv_heads
        self.G = n_q_heads // n_kv_heads

    def close(self):
        if getattr(self, "h", None) is not None and self.h.value:
            lib().mp_destroy(self.h)
            self.h = C.c_void_p()

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    def device_bytes(self):
        return int(lib().mp_device_bytes(self.h))

    def mp_cluster_kv(self, k, v, n_fine, n_coarse=0, iters=10, seed=0, init_fine=None, init_coarse=None,
                      k_lookup=None):
        n_tokens = k.shape[2]
        f_keep, f_ptr = _host_i32(init_fine)
        c_keep, c_ptr = _host_i32(init_coarse)
        st = lib().mp_cluster_kv(self.h, _ptr(k), _ptr(k_lookup), _ptr(v), n_tokens, n_fine, n_coarse, iters, seed,
                                 f_ptr, c_ptr, _stream())
        _check(st, self.h)

    def mp_set_clustering(self, k, v, fine_of_token, n_fine, coarse_of_fine=None, n_coarse=0, k_lookup=None):
        n_tokens = k.shape[2]
        st = lib().mp_set_clustering(self.h, _ptr(k), _ptr(k_lookup), _ptr(v), n_tokens, _ptr(fine_of_token), n_fine,
                                     _ptr(coarse_of_fine), n_coarse, _stream())
        _check(st, self.h)

    def mp_update_clusters(self, k_new, v_new, n_new_fine, n_new_coarse=0, refine_iters=3, split_iters=10, seed=0,
                           seeds=None, k_new_lookup=None):
        n_new = k_new.shape[2]
        s_keep, s_ptr = _host_i32(seeds)
        st = lib().mp_update_clusters(self.h, _ptr(k_new), _ptr(k_new_lookup), _ptr(v_new), n_new, n_new_fine, n_new_coarse,
                                      refine_iters, split_iters, seed, s_ptr, _stream())
        _check(st, self.h)

    def mp_local_buffer_init(self, window, k_sink=None, v_sink=None, k_recent=None, v_recent=None,
                             k_recent_lookup=None):
        n_sink = 0 if k_sink is None else k_sink.shape[2]
        n_recent = 0 if k_recent is None else k_recent.shape[2]
        st = lib().mp_local_buffer_init(self.h, window, _ptr(k_sink), _ptr(v_sink), n_sink, _ptr(k_recent),
                                        _ptr(k_recent_lookup), _ptr(v_recent), n_recent, _stream())
        _check(st, self.h)

    def mp_local_buffer_size(self):
        buf = (C.c_int32 * 3)()
        base = C.addressof(buf)
        st = lib().mp_local_buffer_size(self.h, C.c_void_p(base), C.c_void_p(base + 4), C.c_void_p(base + 8))
        _check(st, self.h)
        return dict(window=buf[0], n_sink=buf[1], n_recent=buf[2])

    def mp_decode_step(self, q, k_new, v_new, key_budget, coarse_budget=0, n_new_fine=0, n_new_coarse=0,
                       refine_iters=3, split_iters=10, seed=0, seeds=None, out=None, lse=None, flags=0,
                       q_lookup=None, k_new_lookup=None):
        if out is None:
            out = torch.empty_like(q)
        s_keep, s_ptr = _host_i32(seeds)
        st = lib().mp_decode_step(self.h, _ptr(q), _ptr(q_lookup), _ptr(k_new), _ptr(k_new_lookup), _ptr(v_new),
                                  key_budget, coarse_budget, flags,
                                  n_new_fine, n_new_coarse, refine_iters, split_iters, seed, s_ptr, _ptr(out),
                                  _ptr(lse), _stream())
        _check(st, self.h)
        return out

    def mp_update_seed_counts(self, n_new, n_new_fine, n_new_coarse=0):
        buf = (C.c_int32 * 6)()
        t = lib().mp_update_seed_counts(self.h, n_new, n_new_fine, n_new_coarse, C.cast(buf, C.c_void_p))
        if t < 0:
            raise MpError(MP_EINVAL, "mp_update_seed_counts: invalid arguments or no index yet")
        return list(buf)

    def mp_decode_attention(self, q, key_budget, coarse_budget=0, k_tail=None, v_tail=None, out=None, lse=None,
                            flags=0, n_tail=None, q_lookup=None):
        """k_tail / v_tail [B, Hkv, rows, 128]; n_tail (default: all rows) = rows of every unit in use."""
        tail_stride = 0 if k_tail is None else k_tail.shape[2]
        if n_tail is None:
            n_tail = tail_stride
        if out is None:
            out = torch.empty_like(q)
        st = lib().mp_decode_attention(self.h, _ptr(q), _ptr(q_lookup), _ptr(k_tail), _ptr(v_tail), n_tail, tail_stride, key_budget,
                                       coarse_budget, flags, _ptr(out), _ptr(lse), _stream())
        _check(st, self.h)
        return out

    def mp_enable_stage_timing(self, enable=True):
        _check(lib().mp_enable_stage_timing(self.h, 1 if enable else 0), self.h)

    def mp_get_stage_timing(self):
        buf = (C.c_float * 4)()
        _check(lib().mp_get_stage_timing(self.h, C.cast(buf, C.c_void_p)), self.h)
        return dict(coarse_ms=buf[0], fine_ms=buf[1], value_ms=buf[2], merge_ms=buf[3])

    def mp_get_sizes(self):
        v = [C.c_int32() for _ in range(4)]
        st = lib().mp_get_sizes(self.h, *[C.cast(C.byref(x), C.c_void_p) for x in v])
        _check(st, self.h)
        return dict(n_tokens=v[0].value, n_fine=v[1].value, n_coarse=v[2].value, n_blocks=v[3].value)

    def mp_get_assignments(self):
        s = self.mp_get_sizes()
        dev = torch.device("cuda")
        fot = torch.empty(self.U, s["n_tokens"], dtype=torch.int32, device=dev)
        cof = torch.empty(self.U, max(s["n_fine"], 1), dtype=torch.int32, device=dev) if self.cfg.levels == 2 else None
        st = lib().mp_get_assignments(self.h, _ptr(fot), _ptr(cof), _stream())
        _check(st, self.h)
        return fot, (cof[:, :s["n_fine"]] if cof is not None else None)

    def mp_get_centroids(self, level):
        s = self.mp_get_sizes()
        n = s["n_fine"] if level == 0 else s["n_coarse"]
        dev = torch.device("cuda")
        kc = torch.empty(self.U, n, 128, dtype=torch.bfloat16, device=dev)
        vc = torch.empty(self.U, n, 128, dtype=torch.bfloat16, device=dev)
        nm = torch.empty(self.U, n, dtype=torch.int32, device=dev)
        st = lib().mp_get_centroids(self.h, level, _ptr(kc), _ptr(vc), _ptr(nm), _stream())
        _check(st, self.h)
        return kc, vc, nm

    def mp_get_selection(self):
        s = self.mp_get_sizes()
        dev = torch.device("cuda")
        nf, nc = s["n_fine"], max(s["n_coarse"], 1)
        fs = torch.empty(self.U, nf, dtype=torch.uint8, device=dev)
        cp = torch.empty(self.U, nc, dtype=torch.uint8, device=dev)
        rf = torch.empty(self.U, nf, dtype=torch.float64, device=dev)
        rc = torch.empty(self.U, nc, dtype=torch.float64, device=dev)
        two = self.cfg.levels == 2
        st = lib().mp_get_selection(self.h, _ptr(fs), _ptr(cp) if two else None, _ptr(rf), _ptr(rc) if two else None,
                                    _stream())
        _check(st, self.h)
        return dict(fine_selected=fs, coarse_promising=cp[:, :s["n_coarse"]] if two else None, r_fine=rf,
                    r_coarse=rc[:, :s["n_coarse"]] if two else None)

    def mp_get_counters(self):
        c = torch.empty(self.U, 4, dtype=torch.int32, device="cuda")
        st = lib().mp_get_counters(self.h, _ptr(c), _stream())
        _check(st, self.h)
        return c

    def mp_get_layout(self):
        """(k_perm, v_perm, perm, fine_start); k_perm and v_perm are None for a context with 8-bit rows."""
        s = self.mp_get_sizes()
        dev = torch.device("cuda")
        kp = vp = None
        if self.kv_format == MP_KV_BF16:
            kp = torch.empty(self.U, s["n_tokens"], 128, dtype=torch.bfloat16, device=dev)
            vp = torch.empty_like(kp)
        perm = torch.empty(self.U, s["n_tokens"], dtype=torch.int32, device=dev)
        fs = torch.empty(self.U, s["n_fine"] + 1, dtype=torch.int32, device=dev)
        st = lib().mp_get_layout(self.h, _ptr(kp), _ptr(vp), _ptr(perm), _ptr(fs), _stream())
        _check(st, self.h)
        return kp, vp, perm, fs

    def mp_get_kv_codes(self):
        """(k_codes uint8 [U, n, 128], v_codes, scales fp32 [U, n, 2]) of a context with 8-bit rows."""
        s = self.mp_get_sizes()
        dev = torch.device("cuda")
        kc = torch.empty(self.U, s["n_tokens"], 128, dtype=torch.uint8, device=dev)
        vc = torch.empty_like(kc)
        sc = torch.empty(self.U, s["n_tokens"], 2, dtype=torch.float32, device=dev)
        st = lib().mp_get_kv_codes(self.h, _ptr(kc), _ptr(vc), _ptr(sc), _stream())
        _check(st, self.h)
        return kc, vc, sc
