"""ctypes binding of libfc.so: argument marshalling only (pointers, sizes, strides, the stream)."""
from __future__ import annotations

import ctypes as C
import os
import re
import struct
from array import array

import numpy as np
import torch

_PKG = os.path.dirname(os.path.abspath(__file__))
_ROOT = os.path.dirname(_PKG)
# FC_LIB=debug selects the bounds-checking build (libfc_debug.so, see build.py); anything else the normal library
_LIB_PATH = os.path.join(_PKG, "libfc_debug.so" if os.environ.get("FC_LIB") == "debug" else "libfc.so")
_HEADER = os.path.join(_ROOT, "include", "fc.h")

BF16, F32 = 0, 1
POLICY_CHUNKWISE, POLICY_UNIFORM = 0, 1
RED_MEANKEY, RED_TILED, RED_TILED_MAX = 0, 1, 2
NORM_NONE, NORM_RMS = 0, 1
ROPE_PAIRS, ROPE_HALVES = 0, 1
KV4_GROUP = 32  # elements of a packed row that share a scale
STATUS_BITS = {"timeout": 1, "nan_score": 2, "bad_index": 4, "nonfinite": 8}


class FcError(RuntimeError):
    pass


class _AttnDesc(C.Structure):
    _fields_ = [("H_q", C.c_int32), ("H_kv", C.c_int32), ("d", C.c_int32), ("W", C.c_int32),
                ("q_hs", C.c_int64), ("q_rs", C.c_int64), ("k_hs", C.c_int64), ("k_rs", C.c_int64),
                ("v_hs", C.c_int64), ("v_rs", C.c_int64), ("o_hs", C.c_int64), ("o_rs", C.c_int64),
                ("kv_rows", C.c_int64), ("scale", C.c_float), ("impl", C.c_int32)]


class _ScoreDesc(C.Structure):
    _fields_ = [("H_q", C.c_int32), ("H_kv", C.c_int32), ("d", C.c_int32), ("L_q", C.c_int32),
                ("L_k", C.c_int32), ("q_hs", C.c_int64), ("q_rs", C.c_int64), ("k_hs", C.c_int64),
                ("k_rs", C.c_int64), ("scale", C.c_float), ("lambda_", C.c_float),
                ("pool_k", C.c_int32), ("impl", C.c_int32), ("red_mode", C.c_int32)]


class _SelectOpts(C.Structure):
    _fields_ = [("unit", C.c_int32), ("n_protect", C.c_int32)]


class _RopeDesc(C.Structure):
    _fields_ = [("H_q", C.c_int32), ("H_kv", C.c_int32), ("d", C.c_int32), ("T", C.c_int32),
                ("q_hs", C.c_int64), ("q_rs", C.c_int64), ("k_hs", C.c_int64), ("k_rs", C.c_int64),
                ("qo_hs", C.c_int64), ("qo_rs", C.c_int64), ("ko_hs", C.c_int64), ("ko_rs", C.c_int64),
                ("axis_dim", C.c_int32 * 3), ("pairing", C.c_int32), ("norm", C.c_int32), ("eps", C.c_float),
                ("theta", C.c_double), ("grid_t0", C.c_int32), ("grid_h", C.c_int32), ("grid_w", C.c_int32)]


class _Kv4Cache(C.Structure):
    _fields_ = [("k_codes", C.c_void_p), ("k_scales", C.c_void_p), ("v_codes", C.c_void_p), ("v_scales", C.c_void_p),
                ("code_hs", C.c_int64), ("code_rs", C.c_int64), ("scale_hs", C.c_int64), ("scale_rs", C.c_int64),
                ("rows", C.c_int64)]


class _Kv4PackDesc(C.Structure):
    _fields_ = [("H", C.c_int32), ("d", C.c_int32), ("n_old", C.c_int32), ("n_new", C.c_int32), ("n_out", C.c_int32),
                ("dst_row", C.c_int64), ("k_hs", C.c_int64), ("k_rs", C.c_int64), ("v_hs", C.c_int64), ("v_rs", C.c_int64)]


class _Kv4UnpackDesc(C.Structure):
    _fields_ = [("H", C.c_int32), ("d", C.c_int32), ("n", C.c_int32), ("src_row", C.c_int64), ("k_hs", C.c_int64),
                ("k_rs", C.c_int64), ("v_hs", C.c_int64), ("v_rs", C.c_int64)]


class _CompactStrides(C.Structure):
    _fields_ = [("src_hs", C.c_int64), ("src_rs", C.c_int64), ("dst_hs", C.c_int64), ("dst_rs", C.c_int64)]


_lib = None


def lib_path() -> str:
    return _LIB_PATH


def lib():
    """Load libfc.so.  There is no fallback: a missing library is an error."""
    global _lib
    if _lib is None:
        if not os.path.exists(_LIB_PATH):
            raise FcError(f"{_LIB_PATH} is missing: build it with `python -m paper_2602_10825_b200.build` "
                          "(or __graft_entry__.build()); this package has no CPU or PyTorch fallback")
        L = C.CDLL(_LIB_PATH)
        L.fc_status_string.restype = C.c_char_p
        L.fc_last_cuda_error.restype = C.c_char_p
        for name in ("fc_chunk_decide_static_max_bytes", "fc_chunk_decide_workspace_bytes", "fc_chunk_attention_workspace_bytes",
                     "fc_kv_score_workspace_bytes", "fc_kv_select_compact_workspace_bytes",
                     "fc_kv_select_compact_ex_workspace_bytes", "fc_chunk_attention_kv4_workspace_bytes"):
            getattr(L, name).restype = C.c_size_t
        L.fc_chunk_decide_workspace_bytes.argtypes = [C.c_int64, C.c_int]
        p, i32, i64 = C.c_void_p, C.c_int, C.c_int64
        L.fc_qk_norm_rope.argtypes = [p, p, p, p, p, i32, p, p, p, p, p, p]
        L.fc_kv4_pack.argtypes = [p, p, p, p, p, i32, p, p, i64, p, p]
        L.fc_kv4_unpack.argtypes = [p, p, p, p, p, p, i32]
        L.fc_chunk_attention_kv4_workspace_bytes.argtypes = [p, p, i32, p, p, i32]
        L.fc_chunk_attention_kv4.argtypes = [p, p, p, p, p, i32, p, p, i32, p, p, p, p, i32, p, p, p, p, i64, p, p, C.c_size_t]
        _lib = L
    return _lib


def declared_symbols():
    """Names of the functions include/fc.h declares."""
    text = open(_HEADER).read()
    text = re.sub(r"/\*.*?\*/", "", text, flags=re.S)
    return sorted(set(re.findall(r"\b(fc_[a-z_0-9]+)\s*\(", text)))


def exported_symbols():
    """Subset of the declared names that libfc.so actually exports."""
    L = lib()
    return sorted(n for n in declared_symbols() if hasattr(L, n))


def _dt(t: torch.Tensor) -> int:
    if t.dtype == torch.bfloat16:
        return BF16
    if t.dtype == torch.float32:
        return F32
    raise FcError(f"unsupported tensor dtype {t.dtype}")


def _dev(t, name, dtype=None):
    if t is None:
        return None
    if not (isinstance(t, torch.Tensor) and t.is_cuda):
        raise FcError(f"{name} must be a CUDA tensor")
    if dtype is not None and t.dtype != dtype:
        raise FcError(f"{name} must have dtype {dtype}, got {t.dtype}")
    return C.c_void_p(t.data_ptr())


def _hsr(t, name):
    """(head stride, row stride) in elements of a [heads, rows, d] tensor with contiguous d."""
    if t.dim() != 3 or t.stride(2) != 1:
        raise FcError(f"{name} must be [heads, rows, d] with a contiguous last dimension")
    return int(t.stride(0)), int(t.stride(1))


def _host_i32(x):
    a = np.ascontiguousarray(np.asarray(x, dtype=np.int32))
    return a, a.ctypes.data_as(C.c_void_p)


def _packer(cls):
    """Packs the fields of a structure, in their order, into its bytes: a third of the time of filling a ctypes structure."""
    kinds = {C.c_int32: "i", C.c_int64: "q", C.c_float: "f", C.c_double: "d", C.c_void_p: "P"}
    parts = [f"{t._length_}{kinds[t._type_]}" if issubclass(t, C.Array) else kinds[t] for _, t in cls._fields_]
    return struct.Struct("@" + "".join(parts) + "0q")  # padded at the end as the structure is


# The descriptors of the calls around the 4-bit store.
_ROPE_FIELDS, _PACK_FIELDS, _UNPACK_FIELDS = _packer(_RopeDesc), _packer(_Kv4PackDesc), _packer(_Kv4UnpackDesc)
_ATTN_FIELDS, _CACHE_FIELDS = _packer(_AttnDesc), _packer(_Kv4Cache)


def _int32(x):
    """int32 values as bytes that a call can take the address of."""
    return array("i", x).tobytes()


class Kv4Cache:
    """A 4-bit store of K and V rows (fc_kv4_cache): codes uint8 [H, rows, d/2] and scales bf16 [H, rows, d/32].

    Strided views (a slice of a larger store) are fine as long as K and V share strides and the last dimensions are
    contiguous; the format is described in include/fc.h.  The four tensors are fixed, and so is their memory (their contents are
    not): build another store, which costs a microsecond or two, to use others."""

    k_codes, k_scales, v_codes, v_scales = (property(lambda self, i=i: self._tensors[i]) for i in range(4))

    def __init__(self, k_codes, k_scales, v_codes, v_scales):
        self._tensors = k_codes, k_scales, v_codes, v_scales
        shape, s_shape, strides, s_strides = k_codes.shape, k_scales.shape, k_codes.stride(), k_scales.stride()
        if len(shape) != 3 or len(s_shape) != 3:
            raise FcError("codes and scales must be [heads, rows, ...]")
        H, rows, half = shape
        if not (k_codes.dtype is v_codes.dtype is torch.uint8 and k_scales.dtype is v_scales.dtype is torch.bfloat16):
            raise FcError("codes must be uint8 and scales bfloat16")
        if v_codes.shape != shape or v_scales.shape != s_shape or s_shape != (H, rows, half // 16):
            raise FcError(f"codes must be [heads, rows, d/2] and scales [heads, rows, d/32], got {list(shape)}, {list(s_shape)}, "
                          f"{list(v_codes.shape)}, {list(v_scales.shape)}")
        device = k_codes.get_device()
        if not (device == v_codes.get_device() == k_scales.get_device() == v_scales.get_device()):
            raise FcError("codes and scales must be on one device")
        ch, cr, c1 = strides
        sh, sr, s1 = s_strides
        if v_codes.stride() != strides or v_scales.stride() != s_strides or c1 != 1 or s1 != 1:
            raise FcError("K and V must share strides, with a contiguous last dimension")
        self.H, self.rows, self.d, self._device = H, rows, 2 * half, device
        self._c = _CACHE_FIELDS.pack(k_codes.data_ptr(), k_scales.data_ptr(), v_codes.data_ptr(), v_scales.data_ptr(), ch, cr, sh, sr, rows)

    @property
    def device(self):
        return self.k_codes.device

    @staticmethod
    def empty(H, rows, d, device="cuda"):
        """An uninitialised store of H heads x rows rows of d elements."""
        if d % KV4_GROUP:
            raise FcError(f"d must be a multiple of {KV4_GROUP}")
        codes = [torch.empty((H, rows, d // 2), dtype=torch.uint8, device=device) for _ in range(2)]
        scales = [torch.empty((H, rows, d // KV4_GROUP), dtype=torch.bfloat16, device=device) for _ in range(2)]
        return Kv4Cache(codes[0], scales[0], codes[1], scales[1])


class Context:
    """A libfc context on one CUDA device (fc_create / fc_destroy)."""

    def __init__(self, device: int = 0):
        self._h = C.c_void_p()
        self._L = lib()
        self.device = int(device)
        self._dev = torch.device("cuda", self.device)
        rc = self._L.fc_create(C.byref(self._h), self.device)
        self._check(rc, "fc_create")
        self._ws = {}

    def close(self):
        if getattr(self, "_h", None) is not None and self._h:
            self._L.fc_destroy(self._h)
            self._h = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    @property
    def sm_count(self) -> int:
        return int(self._L.fc_sm_count(self._h))

    def _check(self, rc, what):
        if rc != 0:
            msg = self._L.fc_status_string(rc).decode()
            if rc == -6:
                msg += ": " + self._L.fc_last_cuda_error().decode()
            raise FcError(f"{what} failed ({rc}): {msg}")

    def _stream(self):
        return C.c_void_p(torch.cuda.current_stream(self.device).cuda_stream)

    def workspace(self, key, n_bytes):
        """A cached device scratch buffer (the binding's convenience; the C call never allocates)."""
        n_bytes = max(int(n_bytes), 256)
        buf = self._ws.get(key)
        if buf is None or buf.numel() < n_bytes:
            buf = torch.empty(n_bytes, dtype=torch.uint8, device=f"cuda:{self.device}")
            self._ws[key] = buf
        return buf

    # ------------------------------------------------------------------ fc_selftest_bounded_wait
    def selftest_bounded_wait(self, limit_ns, status, waited_ns=None):
        rc = self._L.fc_selftest_bounded_wait(self._h, self._stream(), C.c_uint64(int(limit_ns)),
                                              _dev(status, "status", torch.int32), _dev(waited_ns, "waited_ns", torch.int32))
        self._check(rc, "fc_selftest_bounded_wait")

    # ------------------------------------------------------------------ fc_chunk_decide
    def chunk_decide(self, cur, prev, chunk_elem_off, chunk_step, warmup_m, eps, acc, *, force=None,
                     policy=POLICY_CHUNKWISE, l1rel=None, recompute=None, active_ids=None, n_active=None, status=None, ws=None):
        off = np.ascontiguousarray(np.asarray(chunk_elem_off, dtype=np.int64))
        n = len(off) - 1
        dev = cur.device
        l1rel = torch.empty(n, dtype=torch.float32, device=dev) if l1rel is None else l1rel
        recompute = torch.empty(n, dtype=torch.uint8, device=dev) if recompute is None else recompute
        active_ids = torch.empty(n, dtype=torch.int32, device=dev) if active_ids is None else active_ids
        n_active = torch.empty(1, dtype=torch.int32, device=dev) if n_active is None else n_active
        need = self._L.fc_chunk_decide_workspace_bytes(C.c_int64(int(off[-1])), n)
        ws = self.workspace("decide", need) if ws is None else ws
        rc = self._L.fc_chunk_decide(
            self._h, self._stream(), _dev(cur, "cur"), _dev(prev, "prev"), _dt(cur),
            off.ctypes.data_as(C.c_void_p), n, _dev(chunk_step, "chunk_step", torch.int32), int(warmup_m),
            C.c_float(eps), _dev(force, "force", torch.uint8), int(policy), _dev(acc, "acc", torch.float32),
            _dev(l1rel, "l1rel", torch.float32), _dev(recompute, "recompute", torch.uint8),
            _dev(active_ids, "active_ids", torch.int32), _dev(n_active, "n_active", torch.int32),
            _dev(status, "status", torch.int32), _dev(ws, "ws"), C.c_size_t(ws.numel()))
        self._check(rc, "fc_chunk_decide")
        return dict(l1rel=l1rel, recompute=recompute, active_ids=active_ids, n_active=n_active, acc=acc)

    def chunk_decide_static(self, cur, prev, chunk_elem_off, chunk_step, warmup_m, eps, acc, *, l1rel, recompute,
                            active_ids, n_active, force=None, policy=POLICY_CHUNKWISE, status=None):
        """fc_chunk_decide_static: the decision without a workspace, for callers that cannot allocate device
        memory (the scratch is a fixed 1 MiB array inside the library).  Every output tensor is passed in, so
        this wrapper allocates nothing on the device either."""
        off = np.ascontiguousarray(np.asarray(chunk_elem_off, dtype=np.int64))
        n = len(off) - 1
        rc = self._L.fc_chunk_decide_static(
            self._h, self._stream(), _dev(cur, "cur"), _dev(prev, "prev"), _dt(cur),
            off.ctypes.data_as(C.c_void_p), n, _dev(chunk_step, "chunk_step", torch.int32), int(warmup_m),
            C.c_float(eps), _dev(force, "force", torch.uint8), int(policy), _dev(acc, "acc", torch.float32),
            _dev(l1rel, "l1rel", torch.float32), _dev(recompute, "recompute", torch.uint8),
            _dev(active_ids, "active_ids", torch.int32), _dev(n_active, "n_active", torch.int32),
            _dev(status, "status", torch.int32))
        self._check(rc, "fc_chunk_decide_static")
        return dict(l1rel=l1rel, recompute=recompute, active_ids=active_ids, n_active=n_active, acc=acc)

    # ------------------------------------------------------------------ fc_chunk_cache_apply
    def chunk_cache_apply(self, x_in, y_io, cache, chunk_elem_off, recompute, *, status=None):
        off = np.ascontiguousarray(np.asarray(chunk_elem_off, dtype=np.int64))
        if not (x_in.dtype == y_io.dtype == cache.dtype):
            raise FcError("x_in, y_io and cache must share one dtype")
        for name, t in (("x_in", x_in), ("y_io", y_io), ("cache", cache)):
            if not t.is_contiguous() or t.numel() < int(off[-1]):
                raise FcError(f"{name} must be contiguous and hold every chunk's elements")
        rc = self._L.fc_chunk_cache_apply(
            self._h, self._stream(), _dev(x_in, "x_in"), _dev(y_io, "y_io"), _dev(cache, "cache"), _dt(x_in),
            off.ctypes.data_as(C.c_void_p), len(off) - 1, _dev(recompute, "recompute", torch.uint8),
            _dev(status, "status", torch.int32))
        self._check(rc, "fc_chunk_cache_apply")
        return y_io, cache

    # ------------------------------------------------------------------ fc_chunk_attention
    def chunk_attention(self, Q, K, V, q_chunk_row_off, kv_visible_len, seg_logical_off, seg_phys_off,
                        active_ids, n_active, O, *, lse=None, kv_token_index=None, scale=0.0, impl=0,
                        status=None, ws=None):
        q_hs, q_rs = _hsr(Q, "Q")
        k_hs, k_rs = _hsr(K, "K")
        v_hs, v_rs = _hsr(V, "V")
        o_hs, o_rs = _hsr(O, "O")
        W = len(q_chunk_row_off) - 1
        desc = _AttnDesc(Q.shape[0], K.shape[0], Q.shape[2], W, q_hs, q_rs, k_hs, k_rs, v_hs, v_rs, o_hs, o_rs,
                         K.shape[1], scale, impl)
        qo, qo_p = _host_i32(q_chunk_row_off)
        vis, vis_p = _host_i32(kv_visible_len)
        if seg_phys_off is not None:
            sl, sl_p = _host_i32(seg_logical_off)
            sp, sp_p = _host_i32(seg_phys_off)
            n_seg = len(sp)
        else:
            sl_p = sp_p = None
            n_seg = 0
        tok_hs = 0
        if kv_token_index is not None:
            if kv_token_index.dim() != 2 or kv_token_index.stride(1) != 1:
                raise FcError("kv_token_index must be [H_kv, L_logical] with contiguous rows")
            tok_hs = int(kv_token_index.stride(0))
        lse_hs = 0 if lse is None else int(lse.stride(0))
        need = self._L.fc_chunk_attention_workspace_bytes(C.byref(desc))
        ws = self.workspace("attention", need) if ws is None else ws
        if O.dtype != Q.dtype or K.dtype != Q.dtype or V.dtype != Q.dtype:
            raise FcError("Q, K, V, O must share one dtype")
        rc = self._L.fc_chunk_attention(
            self._h, self._stream(), C.byref(desc), _dev(Q, "Q"), _dev(K, "K"), _dev(V, "V"), _dt(Q), qo_p,
            vis_p, sl_p, sp_p, n_seg, _dev(kv_token_index, "kv_token_index", torch.int32), C.c_int64(tok_hs),
            _dev(active_ids, "active_ids", torch.int32), _dev(n_active, "n_active", torch.int32), _dev(O, "O"),
            _dev(lse, "lse", torch.float32), C.c_int64(lse_hs), _dev(status, "status", torch.int32),
            _dev(ws, "ws"), C.c_size_t(ws.numel()))
        self._check(rc, "fc_chunk_attention")
        return O

    # ------------------------------------------------------------------ fc_kv_score
    def kv_score(self, Q_obs, K_cand, *, lambda_=0.07, pool_k=7, scale=0.0, imp_accum=None, accum_phase=0,
                 n_steps=1, imp=None, red=None, score=None, impl=0, red_mode=RED_MEANKEY, status=None, ws=None):
        q_hs, q_rs = _hsr(Q_obs, "Q_obs")
        k_hs, k_rs = _hsr(K_cand, "K_cand")
        H_kv, L_k, d = K_cand.shape
        desc = _ScoreDesc(Q_obs.shape[0], H_kv, d, Q_obs.shape[1], L_k, q_hs, q_rs, k_hs, k_rs, scale, lambda_,
                          pool_k, impl, red_mode)
        if score is None and accum_phase != 1:
            score = torch.empty((H_kv, L_k), dtype=torch.float32, device=K_cand.device)
        for name, t in (("imp", imp), ("red", red), ("score", score), ("imp_accum", imp_accum)):
            if t is not None and not (t.is_contiguous() and tuple(t.shape) == (H_kv, L_k)):
                raise FcError(f"{name} must be a contiguous [H_kv, L_k] tensor")
        need = self._L.fc_kv_score_workspace_bytes(C.byref(desc))
        ws = self.workspace("score", need) if ws is None else ws
        rc = self._L.fc_kv_score(
            self._h, self._stream(), C.byref(desc), _dev(Q_obs, "Q_obs"), _dev(K_cand, "K_cand"), _dt(K_cand),
            _dev(imp_accum, "imp_accum", torch.float32), int(accum_phase), int(n_steps),
            _dev(imp, "imp", torch.float32), _dev(red, "red", torch.float32), _dev(score, "score", torch.float32),
            _dev(status, "status", torch.int32), _dev(ws, "ws"), C.c_size_t(ws.numel()))
        self._check(rc, "fc_kv_score")
        return dict(imp=imp, red=red, score=score)

    # ------------------------------------------------------------------ fc_kv_select_compact
    def kv_select_compact(self, score, B, K_src=None, V_src=None, K_dst=None, V_dst=None, *, kept_idx=None,
                          n_kept=None, status=None, ws=None, unit=1, n_protect=0):
        """fc_kv_select_compact, or fc_kv_select_compact_ex when a selection unit or a protected tail is given."""
        H, L_k = score.shape
        if not score.is_contiguous():
            raise FcError("score must be contiguous [n_heads, L_k]")
        n_keep = min(int(B), L_k)
        dev = score.device
        kept_idx = torch.empty((H, n_keep), dtype=torch.int32, device=dev) if kept_idx is None else kept_idx
        n_kept = torch.empty(1, dtype=torch.int32, device=dev) if n_kept is None else n_kept
        strides, dtype, d = None, BF16, 0
        if K_src is not None:
            s_hs, s_rs = _hsr(K_src, "K_src")
            if _hsr(V_src, "V_src") != (s_hs, s_rs):
                raise FcError("K_src and V_src must share strides")
            if K_dst is None:
                K_dst = torch.empty((H, n_keep, K_src.shape[2]), dtype=K_src.dtype, device=dev)
                V_dst = torch.empty_like(K_dst)
            d_hs, d_rs = _hsr(K_dst, "K_dst")
            if _hsr(V_dst, "V_dst") != (d_hs, d_rs):
                raise FcError("K_dst and V_dst must share strides")
            strides = _CompactStrides(s_hs, s_rs, d_hs, d_rs)
            dtype, d = _dt(K_src), K_src.shape[2]
        if unit != 1 or n_protect != 0:
            need = self._L.fc_kv_select_compact_ex_workspace_bytes(H, L_k, int(unit))
            ws = self.workspace("select", need) if ws is None else ws
            opts = _SelectOpts(int(unit), int(n_protect))
            rc = self._L.fc_kv_select_compact_ex(
                self._h, self._stream(), _dev(score, "score", torch.float32), H, L_k, int(B), C.byref(opts),
                _dev(K_src, "K_src"), _dev(V_src, "V_src"), _dev(K_dst, "K_dst"), _dev(V_dst, "V_dst"), dtype, d,
                None if strides is None else C.byref(strides), _dev(kept_idx, "kept_idx", torch.int32),
                _dev(n_kept, "n_kept", torch.int32), _dev(status, "status", torch.int32), _dev(ws, "ws"),
                C.c_size_t(ws.numel()))
            self._check(rc, "fc_kv_select_compact_ex")
            return dict(kept_idx=kept_idx, n_kept=n_kept, K_dst=K_dst, V_dst=V_dst)
        need = self._L.fc_kv_select_compact_workspace_bytes(H, L_k)
        ws = self.workspace("select", need) if ws is None else ws
        rc = self._L.fc_kv_select_compact(
            self._h, self._stream(), _dev(score, "score", torch.float32), H, L_k, int(B), _dev(K_src, "K_src"),
            _dev(V_src, "V_src"), _dev(K_dst, "K_dst"), _dev(V_dst, "V_dst"), dtype, d,
            None if strides is None else C.byref(strides), _dev(kept_idx, "kept_idx", torch.int32),
            _dev(n_kept, "n_kept", torch.int32), _dev(status, "status", torch.int32), _dev(ws, "ws"),
            C.c_size_t(ws.numel()))
        self._check(rc, "fc_kv_select_compact")
        return dict(kept_idx=kept_idx, n_kept=n_kept, K_dst=K_dst, V_dst=V_dst)

    # ------------------------------------------------------------------ the calls around the 4-bit store
    # These calls take a few microseconds on the device where there is one token; the checks below are written for a
    # host that should not take longer: one pass over each tensor's attributes, no temporaries.
    def _ptr(self, t, name, dtype=None):
        """Device pointer of a tensor on this context's device (None for None)."""
        if t is None:
            return None
        if t.get_device() != self.device:
            raise FcError(f"{name} must be on cuda:{self.device}, got {t.device}")
        if dtype is not None and t.dtype is not dtype:
            raise FcError(f"{name} must have dtype {dtype}, got {t.dtype}")
        return t.data_ptr()

    def _rows(self, t, name, shape, dtype):
        """Pointer and (head, row) strides of a [heads, rows, d] tensor."""
        if t.shape != shape or t.dtype is not dtype:
            raise FcError(f"{name} must be {list(shape)} of {dtype}, got {list(t.shape)} of {t.dtype}")
        if t.get_device() != self.device:
            raise FcError(f"{name} must be on cuda:{self.device}, got {t.device}")
        hs, rs, one = t.stride()
        if one != 1:
            raise FcError(f"{name} must be [heads, rows, d] with a contiguous last dimension")
        return t.data_ptr(), hs, rs

    def _raw_stream(self):
        """Handle of the current stream, without building a Stream object (several microseconds)."""
        return torch._C._cuda_getCurrentRawStream(self.device)

    def _scratch(self, key, n_bytes, stream):
        """Workspace of a call on `stream`: one buffer per stream, since calls on different streams may overlap; during a
        capture the graph gets its own, which lives in the graph's memory pool."""
        if torch.cuda.current_device() == self.device:
            capturing = torch.cuda.is_current_stream_capturing()
        else:
            with torch.cuda.device(self._dev):
                capturing = torch.cuda.is_current_stream_capturing()
        if capturing:
            return torch.empty(n_bytes, dtype=torch.uint8, device=self._dev)
        return self.workspace((key, stream), n_bytes)

    # ------------------------------------------------------------------ fc_qk_norm_rope
    def qk_norm_rope(self, Q, K, *, axes, norm=True, q_weight=None, k_weight=None, eps=1e-6, theta=10000.0, grid=None,
                     pos=None, pairing=ROPE_PAIRS, inv_freq=None, Q_out=None, K_out=None):
        """RMS norm per head and rotation over (time, height, width) of Q [H_q, T, d] and K [H_kv, T, d]; either may be None.

        axes: elements of a head that turn with each axis.  grid = (t0, height, width) places the tokens of a chunk in
        order; pos [T, 3] int32 gives each its own place.  Q_out / K_out may be the inputs themselves."""
        like = K if Q is None else Q
        if like is None:
            raise FcError("Q and K are both None")
        if like.dim() != 3:
            raise FcError("Q and K must be [heads, rows, d]")
        dtype = like.dtype
        hq, hk, (_, T, d) = 0, 0, like.shape
        qp = qop = qw = kp = kop = kw = None
        qh = qr = qoh = qor = kh = kr = koh = kor = 0
        if Q is not None:
            hq = Q.shape[0]
            shape = (hq, T, d)
            if Q_out is None:
                Q_out = torch.empty(shape, dtype=dtype, device=self._dev)
            qp, qh, qr = self._rows(Q, "Q", shape, dtype)
            qop, qoh, qor = self._rows(Q_out, "Q_out", shape, dtype)
            if q_weight is not None:
                qw = self._weight(q_weight, d)
        if K is not None:
            hk = K.shape[0]
            shape = (hk, T, d)
            if K_out is None:
                K_out = torch.empty(shape, dtype=dtype, device=self._dev)
            kp, kh, kr = self._rows(K, "K", shape, dtype)
            kop, koh, kor = self._rows(K_out, "K_out", shape, dtype)
            if k_weight is not None:
                kw = self._weight(k_weight, d)
        if pos is not None and (pos.shape != (T, 3) or not pos.is_contiguous()):
            raise FcError(f"pos must be contiguous [{T}, 3]")
        if grid is None:
            if pos is None and any(axes):
                raise FcError("give the tokens' places: grid or pos")
            grid = (0, 0, 0)
        freq = None
        if inv_freq is not None:
            freq = np.ascontiguousarray(np.asarray(inv_freq, dtype=np.float64))
            if freq.shape != (sum(axes) // 2,):
                raise FcError(f"inv_freq must have {sum(axes) // 2} entries")
        a, b, c = axes
        t0, gh, gw = grid
        desc = _ROPE_FIELDS.pack(hq, hk, d, T, qh, qr, kh, kr, qoh, qor, koh, kor, a, b, c, pairing, NORM_RMS if norm else NORM_NONE,
                                 eps, theta, t0, gh, gw)
        rc = self._L.fc_qk_norm_rope(self._h, self._raw_stream(), desc, qp, kp, _dt(like), qw, kw,
                                     self._ptr(pos, "pos", torch.int32), None if freq is None else freq.ctypes.data, qop, kop)
        if rc:
            self._check(rc, "fc_qk_norm_rope")
        return Q_out, K_out

    def _weight(self, w, d):
        if w.shape != (d,) or w.stride(0) != 1:
            raise FcError(f"a norm's weight must be contiguous [{d}]")
        return self._ptr(w, "a norm's weight", torch.float32)

    # ------------------------------------------------------------------ fc_kv4_pack / fc_kv4_unpack
    def _store(self, s, name):
        """A store's C struct, as bytes that a call can take the address of."""
        if s is None:
            return None
        if s._device != self.device:
            raise FcError(f"{name} must be on cuda:{self.device}, got {s.device}")
        return s._c

    def kv4_pack(self, K, V, dst, *, old=None, n_old=None, kept_idx=None, dst_row=0, status=None):
        """Quantises rows of K, V [H, n_new, d] into the store `dst`, from row dst_row on; returns dst.

        With kept_idx [H, n_out] the rows are picked from [the first n_old rows of the store `old` | the new rows], the
        old ones copied as they are.  K and V may be None if only old rows are picked."""
        H, d = dst.H, dst.d
        n_old = 0 if old is None else old.rows if n_old is None else int(n_old)
        n_new, dt, kp, vp, kh, kr, vh, vr = 0, BF16, None, None, 0, 0, 0, 0
        if K is not None and V is not None:
            n_new, dt = K.shape[1], _dt(K)
            shape = (H, n_new, d)
            kp, kh, kr = self._rows(K, "K", shape, K.dtype)
            vp, vh, vr = self._rows(V, "V", shape, K.dtype)
        elif K is not None or V is not None:
            raise FcError("K and V: give both or neither")
        if old is not None and (old.H != H or old.d != d):
            raise FcError("old and dst must share heads and head size")
        n_out, kept_hs = n_old + n_new, 0
        if kept_idx is not None:
            if kept_idx.dim() != 2 or kept_idx.shape[0] != H or kept_idx.stride(1) != 1:
                raise FcError(f"kept_idx must be [{H}, rows] with contiguous rows")
            n_out = kept_idx.shape[1]
            kept_hs = kept_idx.stride(0) if H > 1 else n_out
        desc = _PACK_FIELDS.pack(H, d, n_old, n_new, n_out, dst_row, kh, kr, vh, vr)
        rc = self._L.fc_kv4_pack(self._h, self._raw_stream(), desc, kp, vp, dt, self._store(old, "old"),
                                 self._ptr(kept_idx, "kept_idx", torch.int32), kept_hs, self._store(dst, "dst"),
                                 self._ptr(status, "status", torch.int32))
        if rc:
            self._check(rc, "fc_kv4_pack")
        return dst

    def kv4_unpack(self, src, *, row=0, n=None, K_dst=None, V_dst=None, dtype=torch.bfloat16, keys_only=False):
        """Values of rows row .. row + n - 1 of a store as plain [H, n, d] tensors (K, V); V is None with keys_only."""
        given = K_dst if K_dst is not None else V_dst
        if given is not None:
            dtype = given.dtype
        n = (src.rows - row if given is None else given.shape[1]) if n is None else int(n)
        shape = (src.H, n, src.d)
        if K_dst is None:
            K_dst = torch.empty(shape, dtype=dtype, device=self._dev)
        kp, kh, kr = self._rows(K_dst, "K_dst", shape, dtype)
        vp, vh, vr = None, 0, 0
        if keys_only:
            V_dst = None
        else:
            if V_dst is None:
                V_dst = torch.empty(shape, dtype=dtype, device=self._dev)
            vp, vh, vr = self._rows(V_dst, "V_dst", shape, dtype)
        desc = _UNPACK_FIELDS.pack(src.H, src.d, n, row, kh, kr, vh, vr)
        rc = self._L.fc_kv4_unpack(self._h, self._raw_stream(), desc, self._store(src, "src"), kp, vp, _dt(K_dst))
        if rc:
            self._check(rc, "fc_kv4_unpack")
        return K_dst, V_dst

    # ------------------------------------------------------------------ fc_chunk_attention_kv4
    def chunk_attention_kv4(self, Q, cache, K, V, q_chunk_row_off, kv_visible_len, active_ids, n_active, O, *,
                            seg_logical_off=None, seg_phys_off=None, n_cache=None, lse=None, scale=0.0, impl=0, status=None,
                            ws=None):
        """fc_chunk_attention over [the first n_cache rows of the 4-bit store | the window K, V].

        cache may be None (no clean region), K and V too (no window).  Without a segment table the window is the rows of
        K and V in order; with one, its logical offsets count from the window's start."""
        if cache is None and K is None:
            raise FcError("give a store, a window, or both")
        if Q.dim() != 3:
            raise FcError("Q must be [heads, rows, d]")
        H_q, rows, d = shape = Q.shape
        dtype, dt = Q.dtype, _dt(Q)
        qp, qh, qr = self._rows(Q, "Q", shape, dtype)
        op, oh, orow = self._rows(O, "O", shape, dtype)
        H_kv = cache.H if cache is not None else K.shape[0]
        if cache is not None and cache.d != d:
            raise FcError("Q and the store must share the head size")
        n_cache = (0 if cache is None else cache.rows) if n_cache is None else int(n_cache)
        W = len(kv_visible_len)
        if not active_ids.is_contiguous():
            raise FcError("active_ids must be contiguous")
        if len(q_chunk_row_off) != W + 1 or q_chunk_row_off[W] > rows or active_ids.numel() > W:
            raise FcError("q_chunk_row_off must have one entry more than kv_visible_len and stay inside Q; active_ids at most as many")
        kp = vp = sl = sp = None
        kh = kr = vh = vr = n_window = n_seg = 0
        if K is not None and V is not None:
            n_window = K.shape[1]
            kp, kh, kr = self._rows(K, "K", (H_kv, n_window, d), dtype)
            vp, vh, vr = self._rows(V, "V", (H_kv, n_window, d), dtype)
            if seg_phys_off is None:
                if n_window:
                    n_seg, sl, sp = 1, _int32((0, n_window)), _int32((0,))
            else:
                n_seg = len(seg_phys_off)
                if len(seg_logical_off) != n_seg + 1:
                    raise FcError("seg_logical_off must have one entry more than seg_phys_off")
                sl, sp = _int32(seg_logical_off), _int32(seg_phys_off)
        elif K is not None or V is not None:
            raise FcError("K and V: give both or neither")
        dp = _ATTN_FIELDS.pack(H_q, H_kv, d, W, qh, qr, kh, kr, vh, vr, oh, orow, n_window, scale, impl)
        off, vis, stream = _int32(q_chunk_row_off), _int32(kv_visible_len), self._raw_stream()
        lse_hs = 0
        if lse is not None:
            if lse.dim() != 2 or lse.shape[0] != H_q or lse.shape[1] < q_chunk_row_off[W] or lse.stride(1) != 1:
                raise FcError("lse must be [H_q, rows] with contiguous rows")
            lse_hs = max(lse.stride(0), 1)
        if ws is None:
            need = self._L.fc_chunk_attention_kv4_workspace_bytes(self._h, dp, dt, off, vis, n_cache)
            if need:
                ws = self._scratch("attention_kv4", need, stream)
        rc = self._L.fc_chunk_attention_kv4(
            self._h, stream, dp, qp, self._store(cache, "cache"), n_cache, kp, vp, dt, off, vis, sl, sp, n_seg,
            self._ptr(active_ids, "active_ids", torch.int32), self._ptr(n_active, "n_active", torch.int32), op,
            self._ptr(lse, "lse", torch.float32), lse_hs, self._ptr(status, "status", torch.int32), self._ptr(ws, "ws"),
            0 if ws is None else ws.numel())
        if rc:
            self._check(rc, "fc_chunk_attention_kv4")
        return O
