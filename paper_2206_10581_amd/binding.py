"""ctypes binding of libtt_emb.so: same names as the C ABI, argument marshalling only.

There is no fallback: if the shared library has not been built, loading raises.
"""
from __future__ import annotations

import ctypes
import math
import os
import warnings
from ctypes import POINTER, byref, c_char_p, c_double, c_float, c_int, c_int32, c_int64, c_size_t, \
    c_uint32, c_void_p
from typing import Any, NamedTuple

_HERE = os.path.dirname(os.path.abspath(__file__))
_LIB_PATH = os.path.join(_HERE, "libtt_emb.so")

TT_EMB_OK, TT_EMB_EINVAL, TT_EMB_ENOSPC, TT_EMB_ESTATE, TT_EMB_EHIP, TT_EMB_ERANGE, \
    TT_EMB_EINTERNAL = 0, -1, -2, -3, -4, -5, -6
TT_EMB_FLAG_CHECK_RANGE = 1
TT_EMB_FLAG_GENERIC_KERNELS = 2
TT_EMB_FLAG_IDS_READY = 4
TT_EMB_FLAG_INDEXED_KERNELS = 8


class TTEmbConfig(ctypes.Structure):
    _fields_ = [("n", c_int64 * 3), ("d", c_int32 * 3), ("r", c_int32 * 2), ("max_batch", c_int64),
                ("device", c_int32), ("flags", c_uint32)]


TT_EMB_FP32, TT_EMB_BF16, TT_EMB_FP16 = 0, 1, 2
_TYPE_BYTES = (4, 2, 2)


class TTEmbMatrix(ctypes.Structure):
    _fields_ = [("data", c_void_p), ("rows", c_int64), ("ld", c_int64), ("cols", c_int32), ("type", c_int32)]


class TTEmbValues(ctypes.Structure):
    _fields_ = [("data", c_void_p), ("count", c_int64), ("type", c_int32), ("unused", c_int32)]


class TTEmbTokenOut(ctypes.Structure):
    _fields_ = [("logprob", c_void_p), ("entropy", c_void_p), ("state", c_void_p), ("top_ids", c_void_p),
                ("top_logprob", c_void_p), ("top", c_int32), ("unused", c_int32)]


class TTEmbPairs(ctypes.Structure):
    _fields_ = [("data", c_void_p), ("batch_ld", c_int64), ("head_ld", c_int64), ("query_ld", c_int64),
                ("queries", c_int64), ("keys", c_int64), ("batch", c_int32), ("heads", c_int32), ("type", c_int32),
                ("unused", c_int32)]


class TTEmbDistances(ctypes.Structure):
    _fields_ = [("bucket_of", c_void_p), ("offsets", c_void_p), ("offset", c_int64), ("span", c_int32), ("unused", c_int32)]


class TTEmbError(RuntimeError):
    def __init__(self, code: int, where: str):
        self.code = code
        super().__init__(f"{where}: {tt_emb_strerror(code)} (code {code})")


_lib = None


def load_library():
    """Loads libtt_emb.so from the package directory; raises if it has not been built."""
    global _lib
    if _lib is not None:
        return _lib
    if not os.path.exists(_LIB_PATH):
        raise ImportError(f"{_LIB_PATH} is missing: run `python -m paper_2206_10581_amd.build` "
                          "(there is no CPU fallback)")
    # PyTorch carries its own copy of the HIP runtime; importing it first makes this library bind
    # to that same copy (one runtime per process), whatever order the caller imports things in.
    import torch  # noqa: F401
    lib = ctypes.CDLL(_LIB_PATH)
    cfgp = POINTER(TTEmbConfig)
    lib.tt_emb_workspace_bytes.argtypes = [cfgp, POINTER(c_size_t)]
    lib.tt_emb_create.argtypes = [POINTER(c_void_p), cfgp, c_void_p, c_void_p, c_void_p, c_void_p,
                                  c_size_t]
    lib.tt_emb_forward.argtypes = [c_void_p, c_void_p, c_int64, c_void_p, c_void_p]
    lib.tt_emb_backward_update.argtypes = [c_void_p, c_void_p, c_float, c_void_p]
    lib.tt_emb_forward_eval.argtypes = [c_void_p, c_void_p, c_int64, c_void_p, c_void_p]
    lib.tt_emb_materialize.argtypes = [c_void_p, c_int64, c_int64, c_void_p, c_void_p]
    lib.tt_emb_lookup_static.argtypes = [cfgp, c_void_p, c_void_p, c_void_p, c_void_p, c_int64,
                                         c_void_p, c_void_p]
    lib.tt_emb_set_reindex.argtypes = [c_void_p, c_void_p, c_int64]
    lib.tt_emb_set_adagrad.argtypes = [c_void_p, c_void_p, c_void_p, c_void_p, c_float]
    lib.tt_emb_wait_backward.argtypes = [c_void_p, c_int]
    lib.tt_emb_set_adam.argtypes = [c_void_p] + [c_void_p] * 6 + [c_float, c_float, c_float, c_int64]
    lib.tt_emb_prepare.argtypes = [c_void_p, c_void_p, c_int64, c_void_p]
    lib.tt_emb_get_stats.argtypes = [c_void_p, POINTER(c_int64), POINTER(c_int64), POINTER(c_int64)]
    matp, valp = POINTER(TTEmbMatrix), POINTER(TTEmbValues)
    lib.tt_emb_dense_forward.argtypes = [matp, c_void_p, c_float, matp, c_void_p]
    lib.tt_emb_dense_workspace_bytes.argtypes = [c_int32, c_int64, POINTER(c_size_t)]
    lib.tt_emb_dense_backward.argtypes = [c_void_p, matp, c_float, c_int64, matp, c_int, c_void_p, c_size_t,
                                          c_void_p]
    lib.tt_emb_norm_workspace_bytes.argtypes = [c_int32, POINTER(c_size_t)]
    lib.tt_emb_grad_norm.argtypes = [valp, c_int32, c_float, c_void_p, c_void_p, c_size_t, c_void_p]
    lib.tt_emb_grad_clip.argtypes = [valp, valp, c_int32, c_float, c_float, c_float, c_void_p, c_void_p, c_size_t,
                                     c_void_p]
    tokp, pairp, distp = POINTER(TTEmbTokenOut), POINTER(TTEmbPairs), POINTER(TTEmbDistances)
    lib.tt_emb_token_workspace_bytes.argtypes = [POINTER(c_size_t)]
    lib.tt_emb_token_scores.argtypes = [matp, c_void_p, c_float, tokp, c_void_p, c_size_t, c_void_p]
    lib.tt_emb_token_backward.argtypes = [matp, c_void_p, c_float, c_void_p, c_void_p, c_void_p, c_void_p, matp, c_void_p]
    lib.tt_emb_token_loss.argtypes = [matp, c_void_p, c_float, c_void_p, c_float, c_void_p, matp, c_void_p, c_size_t,
                                      c_void_p]
    lib.tt_emb_bias_forward.argtypes = [matp, distp, c_float, pairp, pairp, c_void_p]
    lib.tt_emb_bias_workspace_bytes.argtypes = [pairp, c_int32, POINTER(c_size_t)]
    lib.tt_emb_bias_backward.argtypes = [pairp, distp, matp, c_int, c_void_p, c_size_t, c_void_p]
    lib.tt_emb_profile_enable.argtypes = [c_void_p, c_int]
    lib.tt_emb_profile_slots.argtypes = []
    lib.tt_emb_profile_read.argtypes = [c_void_p, c_int, POINTER(c_char_p), POINTER(c_int64),
                                        POINTER(c_double)]
    lib.tt_emb_profile_peaks.argtypes = [c_void_p, c_size_t, c_void_p, POINTER(c_double),
                                         POINTER(c_double), POINTER(c_double), POINTER(c_double)]
    lib.tt_emb_destroy.argtypes = [c_void_p]
    lib.tt_emb_strerror.argtypes = [c_int]
    lib.tt_emb_strerror.restype = c_char_p
    for name in ("tt_emb_workspace_bytes", "tt_emb_create", "tt_emb_forward", "tt_emb_prepare",
                 "tt_emb_backward_update", "tt_emb_forward_eval", "tt_emb_materialize", "tt_emb_lookup_static",
                 "tt_emb_set_reindex", "tt_emb_set_adagrad", "tt_emb_set_adam", "tt_emb_wait_backward", "tt_emb_get_stats", "tt_emb_profile_enable",
                 "tt_emb_dense_forward", "tt_emb_dense_workspace_bytes", "tt_emb_dense_backward",
                 "tt_emb_norm_workspace_bytes", "tt_emb_grad_norm", "tt_emb_grad_clip",
                 "tt_emb_token_workspace_bytes", "tt_emb_token_scores", "tt_emb_token_backward", "tt_emb_token_loss",
                 "tt_emb_bias_forward", "tt_emb_bias_workspace_bytes", "tt_emb_bias_backward",
                 "tt_emb_profile_slots", "tt_emb_profile_read", "tt_emb_profile_peaks", "tt_emb_destroy"):
        getattr(lib, name).restype = c_int
    _lib = lib
    return lib


def make_config(n, d, r, max_batch: int, device: int = 0, flags: int = 0) -> TTEmbConfig:
    c = TTEmbConfig()
    for k in range(3):
        c.n[k] = int(n[k])
        c.d[k] = int(d[k])
    c.r[0], c.r[1] = int(r[0]), int(r[1])
    c.max_batch, c.device, c.flags = int(max_batch), int(device), int(flags)
    return c


# ---- the C entry points, one to one (integers are raw pointers: tensor.data_ptr(), stream handles)

def tt_emb_strerror(code: int) -> str:
    return load_library().tt_emb_strerror(int(code)).decode()


def tt_emb_workspace_bytes(cfg: TTEmbConfig):
    out = c_size_t(0)
    rc = load_library().tt_emb_workspace_bytes(byref(cfg), byref(out))
    return rc, int(out.value)


def tt_emb_create(cfg: TTEmbConfig, g1_ptr: int, g2_ptr: int, g3_ptr: int, ws_ptr: int, ws_bytes: int):
    h = c_void_p(None)
    rc = load_library().tt_emb_create(byref(h), byref(cfg), c_void_p(g1_ptr), c_void_p(g2_ptr),
                                      c_void_p(g3_ptr), c_void_p(ws_ptr), c_size_t(ws_bytes))
    return rc, h


def tt_emb_forward(h, ids_ptr: int, B: int, out_ptr: int, stream: int) -> int:
    return load_library().tt_emb_forward(h, c_void_p(ids_ptr), c_int64(B), c_void_p(out_ptr),
                                         c_void_p(stream))


def tt_emb_forward_eval(h, ids_ptr: int, B: int, out_ptr: int, stream: int) -> int:
    return load_library().tt_emb_forward_eval(h, c_void_p(ids_ptr), c_int64(B), c_void_p(out_ptr),
                                              c_void_p(stream))


def tt_emb_materialize(h, first_row: int, count: int, out_ptr: int, stream: int) -> int:
    return load_library().tt_emb_materialize(h, c_int64(first_row), c_int64(count),
                                             c_void_p(out_ptr), c_void_p(stream))


def tt_emb_lookup_static(cfg: TTEmbConfig, g1_ptr: int, g2_ptr: int, g3_ptr: int, ids_ptr: int, B: int,
                         out_ptr: int, stream: int) -> int:
    return load_library().tt_emb_lookup_static(byref(cfg), c_void_p(g1_ptr), c_void_p(g2_ptr),
                                               c_void_p(g3_ptr), c_void_p(ids_ptr), c_int64(B),
                                               c_void_p(out_ptr), c_void_p(stream))


def tt_emb_set_reindex(h, table_ptr: int, n_ids: int) -> int:
    return load_library().tt_emb_set_reindex(h, c_void_p(table_ptr), c_int64(n_ids))


def tt_emb_wait_backward(h, age: int) -> int:
    return load_library().tt_emb_wait_backward(h, c_int(age))


def tt_emb_set_adam(h, m_ptrs, v_ptrs, beta1: float, beta2: float, eps: float, steps_done: int = 0) -> int:
    ptrs = [c_void_p(p) for p in (*m_ptrs, *v_ptrs)]
    return load_library().tt_emb_set_adam(h, *ptrs, c_float(beta1), c_float(beta2), c_float(eps),
                                          c_int64(steps_done))


def tt_emb_set_adagrad(h, s1_ptr: int, s2_ptr: int, s3_ptr: int, eps: float) -> int:
    return load_library().tt_emb_set_adagrad(h, c_void_p(s1_ptr), c_void_p(s2_ptr), c_void_p(s3_ptr),
                                             c_float(eps))


def tt_emb_prepare(h, ids_ptr: int, B: int, stream: int) -> int:
    return load_library().tt_emb_prepare(h, c_void_p(ids_ptr), c_int64(B), c_void_p(stream))


def tt_emb_backward_update(h, grad_ptr: int, lr: float, stream: int) -> int:
    return load_library().tt_emb_backward_update(h, c_void_p(grad_ptr), c_float(lr), c_void_p(stream))


def tt_emb_get_stats(h):
    U, Q, oob = c_int64(0), c_int64(0), c_int64(0)
    rc = load_library().tt_emb_get_stats(h, byref(U), byref(Q), byref(oob))
    return rc, int(U.value), int(Q.value), int(oob.value)


def tt_emb_profile_enable(h, enable: bool) -> int:
    return load_library().tt_emb_profile_enable(h, c_int(1 if enable else 0))


def tt_emb_profile_slots() -> int:
    return load_library().tt_emb_profile_slots()


def tt_emb_profile_read(h, slot: int):
    name, n, ms = c_char_p(None), c_int64(0), c_double(0.0)
    rc = load_library().tt_emb_profile_read(h, c_int(slot), byref(name), byref(n), byref(ms))
    return rc, (name.value or b"").decode(), int(n.value), float(ms.value)


def tt_emb_profile_peaks(buf_ptr: int, nbytes: int, stream: int):
    copy, mfma, gather, far = c_double(0.0), c_double(0.0), c_double(0.0), c_double(0.0)
    rc = load_library().tt_emb_profile_peaks(c_void_p(buf_ptr), c_size_t(nbytes), c_void_p(stream),
                                             byref(copy), byref(mfma), byref(gather), byref(far))
    return rc, float(copy.value), float(mfma.value), float(gather.value), float(far.value)


def tt_emb_destroy(h) -> int:
    return load_library().tt_emb_destroy(h)


def tt_emb_dense_forward(table: TTEmbMatrix, ids_ptr: int, scale: float, out: TTEmbMatrix, stream: int) -> int:
    return load_library().tt_emb_dense_forward(byref(table), ids_ptr, scale, byref(out), stream)


def tt_emb_dense_workspace_bytes(cols: int, max_batch: int):
    out = c_size_t(0)
    rc = load_library().tt_emb_dense_workspace_bytes(cols, max_batch, byref(out))
    return rc, int(out.value)


def tt_emb_dense_backward(ids_ptr: int, grad: TTEmbMatrix, scale: float, padding_id: int, dtable: TTEmbMatrix,
                          add: bool, ws_ptr: int, ws_bytes: int, stream: int) -> int:
    return load_library().tt_emb_dense_backward(ids_ptr, byref(grad), scale, padding_id, byref(dtable),
                                                1 if add else 0, ws_ptr, ws_bytes, stream)


def tt_emb_norm_workspace_bytes(n: int):
    out = c_size_t(0)
    rc = load_library().tt_emb_norm_workspace_bytes(n, byref(out))
    return rc, int(out.value)


def tt_emb_grad_norm(values, n: int, scale: float, norm_ptr: int, ws_ptr: int, ws_bytes: int, stream: int) -> int:
    """values: a ctypes array of n TTEmbValues (or None for n = 0), as in tt_emb_grad_clip."""
    return load_library().tt_emb_grad_norm(values, n, scale, norm_ptr, ws_ptr, ws_bytes, stream)


def tt_emb_grad_clip(values, out, n: int, scale: float, max_norm: float, eps: float, norm_ptr: int, ws_ptr: int,
                     ws_bytes: int, stream: int) -> int:
    return load_library().tt_emb_grad_clip(values, out, n, scale, max_norm, eps, norm_ptr, ws_ptr, ws_bytes, stream)


def _ref(structure):
    return None if structure is None else byref(structure)


def tt_emb_token_workspace_bytes():
    out = c_size_t(0)
    rc = load_library().tt_emb_token_workspace_bytes(byref(out))
    return rc, int(out.value)


def tt_emb_token_scores(logits: TTEmbMatrix, tokens_ptr: int, scale: float, out: TTEmbTokenOut, ws_ptr: int, ws_bytes: int,
                        stream: int) -> int:
    return load_library().tt_emb_token_scores(_ref(logits), tokens_ptr, scale, _ref(out), ws_ptr, ws_bytes, stream)


def tt_emb_token_backward(logits: TTEmbMatrix, tokens_ptr: int, scale: float, state_ptr: int, entropy_ptr: int,
                          d_logprob_ptr: int, d_entropy_ptr: int, dlogits: TTEmbMatrix, stream: int) -> int:
    return load_library().tt_emb_token_backward(_ref(logits), tokens_ptr, scale, state_ptr, entropy_ptr, d_logprob_ptr,
                                                d_entropy_ptr, _ref(dlogits), stream)


def tt_emb_token_loss(logits: TTEmbMatrix, tokens_ptr: int, scale: float, weights_ptr: int, weight: float,
                      logprob_ptr: int, dlogits: TTEmbMatrix, ws_ptr: int, ws_bytes: int, stream: int) -> int:
    return load_library().tt_emb_token_loss(_ref(logits), tokens_ptr, scale, weights_ptr, weight, logprob_ptr,
                                            _ref(dlogits), ws_ptr, ws_bytes, stream)


def tt_emb_bias_forward(table: TTEmbMatrix, distances: TTEmbDistances, fill: float, scores, out: TTEmbPairs,
                        stream: int) -> int:
    """scores: a TTEmbPairs, or None for the bias alone."""
    return load_library().tt_emb_bias_forward(_ref(table), _ref(distances), fill, _ref(scores), _ref(out), stream)


def tt_emb_bias_workspace_bytes(grad: TTEmbPairs, span: int):
    out = c_size_t(0)
    rc = load_library().tt_emb_bias_workspace_bytes(_ref(grad), span, byref(out))
    return rc, int(out.value)


def tt_emb_bias_backward(grad: TTEmbPairs, distances: TTEmbDistances, dtable: TTEmbMatrix, add: bool, ws_ptr: int,
                         ws_bytes: int, stream: int) -> int:
    return load_library().tt_emb_bias_backward(_ref(grad), _ref(distances), _ref(dtable), 1 if add else 0, ws_ptr, ws_bytes,
                                               stream)


# ---- convenience wrappers over torch tensors (memory and streams only)

class TTEmbedding:
    """Owns the device tensors the library borrows: three cores and the workspace."""

    def __init__(self, n, d, r, max_batch: int, cores, device="cuda:0", flags: int = 0):
        import torch
        self.torch = torch
        self.device = torch.device(device)
        self.n, self.d, self.r = tuple(n), tuple(d), tuple(r)
        self.D = self.d[0] * self.d[1] * self.d[2]
        shapes = ((n[0], d[0], r[0]), (n[1], r[0], d[1], r[1]), (n[2], r[1], d[2]))
        self.cores = []
        for c, s in zip(cores, shapes):
            if (isinstance(c, torch.Tensor) and c.device == self.device and c.dtype == torch.float32
                    and c.is_contiguous()):
                t = c                      # caller-owned device tensor: borrowed, updated in place
            else:
                t = torch.as_tensor(c).to(device=self.device, dtype=torch.float32).contiguous().clone()
            if tuple(t.shape) != tuple(s):
                raise ValueError(f"core shape {tuple(t.shape)} != {s}")
            self.cores.append(t)
        index = self.device.index if self.device.index is not None else 0
        self.cfg = make_config(n, d, r, max_batch, index, flags)
        rc, nbytes = tt_emb_workspace_bytes(self.cfg)
        if rc:
            raise TTEmbError(rc, "tt_emb_workspace_bytes")
        self.workspace = torch.empty(nbytes + 256, dtype=torch.uint8, device=self.device)
        base = self.workspace.data_ptr()
        self._ws_ptr = (base + 255) & ~255
        self.workspace_bytes = nbytes
        rc, self.handle = tt_emb_create(self.cfg, *(t.data_ptr() for t in self.cores), self._ws_ptr,
                                        nbytes)
        if rc:
            raise TTEmbError(rc, "tt_emb_create")

    def _stream(self) -> int:
        return int(self.torch.cuda.current_stream(self.device).cuda_stream)

    def forward(self, ids, out=None):
        torch = self.torch
        assert ids.dtype == torch.int64 and ids.is_contiguous() and ids.device == self.device
        B = ids.numel()
        if out is None:
            out = torch.empty((B, self.D), dtype=torch.float32, device=self.device)
        assert out.is_contiguous() and out.shape == (B, self.D) and out.dtype == torch.float32
        rc = tt_emb_forward(self.handle, ids.data_ptr() if B else 0, B, out.data_ptr() if B else 0,
                            self._stream())
        if rc:
            raise TTEmbError(rc, "tt_emb_forward")
        return out

    def forward_eval(self, ids, out=None):
        """Lookup without keeping anything for a backward pass."""
        torch = self.torch
        assert ids.dtype == torch.int64 and ids.is_contiguous() and ids.device == self.device
        B = ids.numel()
        if out is None:
            out = torch.empty((B, self.D), dtype=torch.float32, device=self.device)
        assert out.is_contiguous() and out.shape == (B, self.D) and out.dtype == torch.float32
        rc = tt_emb_forward_eval(self.handle, ids.data_ptr() if B else 0, B,
                                 out.data_ptr() if B else 0, self._stream())
        if rc:
            raise TTEmbError(rc, "tt_emb_forward_eval")
        return out

    def materialize(self, first_row: int = 0, count: int | None = None, out=None):
        """Rows first_row .. first_row+count-1 of the dense table the cores define."""
        torch = self.torch
        N = self.n[0] * self.n[1] * self.n[2]
        count = N - first_row if count is None else count
        if out is None:
            out = torch.empty((count, self.D), dtype=torch.float32, device=self.device)
        assert out.is_contiguous() and out.shape == (count, self.D) and out.dtype == torch.float32
        rc = tt_emb_materialize(self.handle, first_row, count, out.data_ptr() if count else 0,
                                self._stream())
        if rc:
            raise TTEmbError(rc, "tt_emb_materialize")
        return out

    def set_reindex(self, new_id_of):
        """Installs (or, with None, removes) an old-id -> table-row table: device int32 tensor."""
        torch = self.torch
        if new_id_of is None:
            self._reindex = None
            rc = tt_emb_set_reindex(self.handle, 0, 0)
        else:
            assert new_id_of.dtype == torch.int32 and new_id_of.is_contiguous()
            assert new_id_of.device == self.device
            self._reindex = new_id_of          # keeps the borrowed table alive
            rc = tt_emb_set_reindex(self.handle, new_id_of.data_ptr(), new_id_of.numel())
        if rc:
            raise TTEmbError(rc, "tt_emb_set_reindex")

    def set_adagrad(self, eps: float = 1e-10, enable: bool = True):
        """Switches backward_update to row-sparse Adagrad (state tensors are created here, zeroed)
        or back to SGD."""
        torch = self.torch
        if not enable:
            self.adagrad_state = None
            rc = tt_emb_set_adagrad(self.handle, 0, 0, 0, 0.0)
        else:
            self.adagrad_state = [torch.zeros_like(c) for c in self.cores]
            rc = tt_emb_set_adagrad(self.handle, *(t.data_ptr() for t in self.adagrad_state), eps)
        if rc:
            raise TTEmbError(rc, "tt_emb_set_adagrad")

    def set_adam(self, beta1: float = 0.9, beta2: float = 0.999, eps: float = 1e-8,
                 enable: bool = True):
        """Switches backward_update to row-sparse Adam (moment tensors are created here, zeroed) or
        back to SGD."""
        torch = self.torch
        self.adagrad_state = None
        if not enable:
            self.adam_state = None
            rc = tt_emb_set_adam(self.handle, (0, 0, 0), (0, 0, 0), 0.0, 0.0, 0.0)
        else:
            self.adam_state = ([torch.zeros_like(c) for c in self.cores],
                               [torch.zeros_like(c) for c in self.cores])
            rc = tt_emb_set_adam(self.handle, [t.data_ptr() for t in self.adam_state[0]],
                                 [t.data_ptr() for t in self.adam_state[1]], beta1, beta2, eps)
        if rc:
            raise TTEmbError(rc, "tt_emb_set_adam")

    def wait_backward(self, age: int = 1):
        """Host-side flow control: returns once the backward_update made `age` calls before the
        latest one has finished on the device."""
        rc = tt_emb_wait_backward(self.handle, age)
        if rc:
            raise TTEmbError(rc, "tt_emb_wait_backward")

    def prepare(self, ids):
        """Index work of the next batch, overlapped with whatever follows on the current stream."""
        torch = self.torch
        assert ids.dtype == torch.int64 and ids.is_contiguous() and ids.device == self.device
        rc = tt_emb_prepare(self.handle, ids.data_ptr() if ids.numel() else 0, ids.numel(),
                            self._stream())
        if rc:
            raise TTEmbError(rc, "tt_emb_prepare")

    def backward_update(self, grad_out, lr: float):
        torch = self.torch
        assert grad_out.dtype == torch.float32 and grad_out.is_contiguous()
        assert grad_out.device == self.device
        rc = tt_emb_backward_update(self.handle, grad_out.data_ptr() if grad_out.numel() else 0,
                                    float(lr), self._stream())
        if rc:
            raise TTEmbError(rc, "tt_emb_backward_update")

    def stats(self, check: bool = True):
        rc, U, Q, oob = tt_emb_get_stats(self.handle)
        if rc and (check or rc not in (TT_EMB_ERANGE,)):
            raise TTEmbError(rc, "tt_emb_get_stats")
        return {"U": U, "Q": Q, "out_of_range": oob}

    def profile(self, enable: bool):
        rc = tt_emb_profile_enable(self.handle, enable)
        if rc:
            raise TTEmbError(rc, "tt_emb_profile_enable")

    def profile_read(self):
        res = {}
        for k in range(tt_emb_profile_slots()):
            rc, name, n, ms = tt_emb_profile_read(self.handle, k)
            if rc:
                raise TTEmbError(rc, "tt_emb_profile_read")
            res[name] = {"launches": n, "ms": ms}
        return res

    def close(self):
        if getattr(self, "handle", None) is not None:
            tt_emb_destroy(self.handle)
            self.handle = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass


class _OnDevice:
    """Device, stream and workspace of the wrappers below."""

    def __init__(self, device):
        import torch
        if device.type != "cuda":
            raise ValueError(f"tensors on {device}: a GPU needed")
        self.torch, self.device, self.index = torch, device, device.index
        self.lib = load_library()
        # the handle alone where torch gives it: making a stream object takes 1 us of a call's 7
        self._stream = getattr(torch._C, "_cuda_getCurrentRawStream", None) or (
            lambda index: torch.cuda.current_stream(index).cuda_stream)

    def _call(self, function, *args):
        """The C function with the current stream of this object's device as its last argument."""
        cuda, stream = self.torch.cuda, self._stream(self.index)
        if stream != self._home:  # its memory is not given to others before this stream is done with it
            self.workspace.record_stream(cuda.current_stream(self.index))
        if cuda.current_device() == self.index:
            rc = function(*args, stream)
        else:
            with cuda.device(self.index):
                rc = function(*args, stream)
        if rc:
            raise TTEmbError(rc, function.__name__)

    def _type(self, t):
        torch = self.torch
        kind = t.dtype
        if kind is torch.float32:
            return TT_EMB_FP32
        if kind is torch.bfloat16:
            return TT_EMB_BF16
        if kind is torch.float16:
            return TT_EMB_FP16
        raise ValueError(f"type {kind}: float32, bfloat16 or float16 needed")

    def _matrix(self, t):
        if t.dim() != 2 or t.device != self.device:
            raise ValueError(f"matrix on {self.device} needed: shape {tuple(t.shape)} on {t.device}")
        rows, cols = t.shape
        step, side = t.stride()
        if cols > 1 and side != 1 or rows > 1 and step < cols:
            raise ValueError(f"strides {t.stride()}: values of a row side by side, rows that do not overlap needed")
        return TTEmbMatrix(t.data_ptr(), rows, step if rows > 1 else cols, cols, self._type(t))

    def _capturing(self):
        cuda = self.torch.cuda
        if cuda.current_device() == self.index:
            return cuda.is_current_stream_capturing()
        with cuda.device(self.index):
            return cuda.is_current_stream_capturing()

    def _make_workspace(self, nbytes):
        self._home = self._stream(self.index)  # the workspace belongs to this stream
        self.workspace = self.torch.empty(nbytes + 256, dtype=self.torch.uint8, device=self.device)
        self._ws_ptr = (self.workspace.data_ptr() + 255) & ~255
        self.workspace_bytes = nbytes


class DenseEmbedding(_OnDevice):
    """A table kept as a plain matrix, beside tensor-train ones: lookup times a scale, and gradient.

    weight: [rows, dim] on the GPU, float32, bfloat16 or float16, values of a row side by side (rows may lie further
    apart); borrowed, and taken with the memory, shape, strides and type that it has at the time of a call.  Ids outside
    the table give zero rows and no gradient; padding_id is an id that has a row but no gradient.  Outputs must not
    overlap what a call reads.  Must not be used from two threads or streams at once (the workspace of backward)."""

    def __init__(self, weight, max_batch: int, scale: float = 1.0, padding_id: int | None = None):
        super().__init__(weight.device)
        self.weight, self.max_batch, self.scale = weight, int(max_batch), float(scale)
        self.padding_id = -1 if padding_id is None else int(padding_id)
        self._described, self._table, self._spaces, self.workspace_bytes = None, None, [], 0
        self._weight()

    def _ids(self, ids):
        if ids.dtype != self.torch.int64 or ids.device != self.device or ids.dim() != 1 or not ids.is_contiguous():
            raise ValueError("ids: contiguous int64 vector on the table's device needed")
        if ids.numel() > self.max_batch:
            raise TTEmbError(TT_EMB_ENOSPC, "DenseEmbedding")
        return ids.data_ptr()

    @property
    def rows(self):
        return self.weight.shape[0]

    @property
    def dim(self):
        return self.weight.shape[1]

    def _weight(self):
        """The weight as it is now.  Its address alone does not tell: a view of the same memory may have other rows,
        and a freed address may be given to a smaller tensor of another type."""
        w = self.weight
        now = (w.data_ptr(), w.dtype, w.shape, w.stride())
        if now != self._described:
            table = self._matrix(w)
            if table.cols < 1:
                raise ValueError("rows without values")
            rc, nbytes = tt_emb_dense_workspace_bytes(table.cols, self.max_batch)
            if rc:
                raise TTEmbError(rc, "tt_emb_dense_workspace_bytes")
            if nbytes > self.workspace_bytes:
                self._make_workspace(nbytes)
                self._spaces.append(self.workspace)  # a captured graph may go on using a smaller one
            self._table, self._described = table, now
        return self._table

    def forward(self, ids, out=None, dtype=None):
        """scale * weight[ids], in the weight's type unless out or dtype says otherwise."""
        table, ptr = self._weight(), self._ids(ids)
        if out is None:
            out = self.torch.empty((ids.numel(), table.cols), dtype=dtype or self.weight.dtype, device=self.device)
        elif out.shape != (ids.numel(), table.cols) or dtype not in (None, out.dtype):
            raise ValueError(f"out: {(ids.numel(), table.cols)} of {dtype or out.dtype} needed, not {tuple(out.shape)}")
        self._call(self.lib.tt_emb_dense_forward, byref(table), ptr, self.scale, byref(self._matrix(out)))
        return out

    def backward(self, ids, grad_out, out=None, dtype=None, add: bool = False):
        """Gradient of forward(ids) with respect to the weight, [rows, dim], for the upstream gradient grad_out.
        With add, it is added to out, whose other rows are left alone."""
        table = self._weight()
        shape = (table.rows, table.cols)
        if out is None:
            if add:
                raise ValueError("add needs out")
            out = self.torch.empty(shape, dtype=dtype or self.weight.dtype, device=self.device)
        elif out.shape != shape or dtype not in (None, out.dtype):
            raise ValueError(f"out: {shape} of {dtype or out.dtype} needed, not {tuple(out.shape)}")
        self._backward(ids, grad_out, self.scale, self._matrix(out), add)
        return out

    def backward_update(self, ids, grad_out, lr: float):
        """SGD step of the weight's rows that ids name: weight -= lr * gradient, rounded to the weight's type."""
        self._backward(ids, grad_out, -float(lr) * self.scale, self._weight(), True)

    def _backward(self, ids, grad_out, scale, target, add):
        ptr = self._ids(ids)
        if grad_out.shape != (ids.numel(), target.cols):
            raise ValueError(f"grad_out: {(ids.numel(), target.cols)} needed, not {tuple(grad_out.shape)}")
        self._call(self.lib.tt_emb_dense_backward, ptr, byref(self._matrix(grad_out)), scale, self.padding_id, byref(target),
                   1 if add else 0, self._ws_ptr, self.workspace_bytes)


class GradientClip(_OnDevice):
    """The 2-norm over all values of many tensors, and the tensors scaled to a largest norm.

    tensors: on one GPU, float32, bfloat16 or float16, each without gaps (any order of dimensions); borrowed, with the
    memory that they have now: make a new object for gradients that are not kept from step to step (set to None) and for
    tensors whose .data is replaced.  A call warns where it finds one replaced that shares its storage with no other, and
    raises where the memory was freed.  out: tensors of the same sizes, in any of the types, that receive the scaled
    values; None: in place.  What clip writes may overlap nothing but its own input.  Must not be used from two threads
    or streams at once."""

    def __init__(self, tensors, out=None):
        self.tensors = list(tensors)
        if not self.tensors:
            raise ValueError("no tensors")
        super().__init__(self.tensors[0].device)
        self._in, read = self._values(self.tensors)
        written = read
        self.out, self._out = None, None
        if out is not None:
            self.out = list(out)
            if [t.shape for t in self.out] != [t.shape for t in self.tensors]:
                raise ValueError("out: tensors of the same shapes needed")
            if any(a.stride() != b.stride() and self._order(a) != self._order(b) for a, b in zip(self.tensors, self.out)
                   if a.numel() > 1):
                raise ValueError("out: tensors of the same strides needed")
            self._out, written = self._values(self.out)
        self._apart = self._written_apart(read, written)
        if out is not None and not self._apart:
            raise ValueError("out: tensors that overlap nothing but each its own input needed")
        self._watch()
        rc, nbytes = tt_emb_norm_workspace_bytes(len(self.tensors))
        if rc:
            raise TTEmbError(rc, "tt_emb_norm_workspace_bytes")
        self._make_workspace(nbytes)

    def _values(self, tensors):
        """The tensors as the library takes them, and the (start, end, type) of each in memory."""
        values, spans = (TTEmbValues * len(tensors))(), []
        for v, t in zip(values, tensors):
            if t.device != self.device:
                raise ValueError(f"tensor on {t.device}, not {self.device}")
            if not (t.is_contiguous() or self._dense(t)):
                raise ValueError(f"tensor of shape {tuple(t.shape)} and strides {t.stride()} has gaps or overlaps")
            at, count, kind = t.data_ptr(), t.numel(), self._type(t)
            v.data, v.count, v.type = at, count, kind
            spans.append((at, at + count * _TYPE_BYTES[kind], kind))
        return values, spans

    @staticmethod
    def _written_apart(read, written):
        """Whether clip writes every value's place once and reads none that it writes elsewhere."""
        spans = [(start, end, True) for start, end, _ in written if start < end]
        if read is not written:
            spans += [(start, end, False) for (start, end, kind), to in zip(read, written)
                      if start < end and (start, end, kind) != to]
        read_to = written_to = 0
        for start, end, writes in sorted(spans):
            if start < written_to or writes and start < read_to:
                return False
            if writes:
                written_to = end
            elif end > read_to:
                read_to = end
        return True

    @staticmethod
    def _order(t):
        return [s for s, n in zip(t.stride(), t.shape) if n > 1]  # the others say nothing

    @staticmethod
    def _dense(t):
        size = 1
        for step, n in sorted((s, n) for s, n in zip(t.stride(), t.shape) if n > 1):
            if step != size:
                return False
            size *= n
        return True

    def _watch(self):
        """One tensor of every storage: held, so that the memory stays where a tensor's .data is replaced, and looked at by
        every call, since the storage itself may be resized.  A look takes 0.04 us; at all 300 tensors of one buffer it took a
        call that scales 3M values from 18 to 40."""
        first = {}
        for t in self.tensors + (self.out or []):
            if t.numel():
                first.setdefault(t.untyped_storage().data_ptr(), t)
        self._watched = list(first.values())
        self._held = [t.detach() for t in self._watched]
        self._where = self.torch.Tensor.data_ptr
        self._at = list(map(self._where, self._held))

    def _moved(self):
        """A call that finds a tensor elsewhere than it was when the object was made."""
        if list(map(self._where, self._held)) != self._at:
            raise RuntimeError("GradientClip: the memory of a tensor was freed or moved since the object was made")
        warnings.warn("GradientClip: a tensor's .data was replaced, and the object goes on with the memory that it had; "
                      "make a new object", RuntimeWarning, stacklevel=3)

    def _norm(self, out):
        if out is None:
            return self.torch.empty((), dtype=self.torch.float32, device=self.device)
        if out.numel() != 1 or out.dtype != self.torch.float32 or out.device != self.device:
            raise ValueError("out: one float32 on the tensors' device needed")
        return out

    def norm(self, scale: float = 1.0, out=None):
        """|scale| * the norm, as a float32 on the device."""
        if list(map(self._where, self._watched)) != self._at:
            self._moved()
        out = self._norm(out)
        self._call(self.lib.tt_emb_grad_norm, self._in, len(self._in), float(scale), out.data_ptr(), self._ws_ptr,
                   self.workspace_bytes)
        return out

    def clip(self, max_norm: float, scale: float = 1.0, eps: float = 1e-6, out=None):
        """Scales the tensors by scale and down to max_norm; returns the norm before, |scale| included."""
        if not self._apart:
            raise ValueError("tensors that overlap cannot be scaled in place")
        if list(map(self._where, self._watched)) != self._at:
            self._moved()
        out = self._norm(out)
        self._call(self.lib.tt_emb_grad_clip, self._in, self._out, len(self._in), float(scale), float(max_norm), float(eps),
                   out.data_ptr(), self._ws_ptr, self.workspace_bytes)
        return out


class TokenResult(NamedTuple):
    """What TokenScores.forward returns; None: not asked for."""
    logprobs: Any = None      # [n] log probabilities of the tokens
    entropy: Any = None       # [n]
    top_ids: Any = None       # [n, top] the likeliest tokens, int64; -1: none
    top_logprobs: Any = None  # [n, top]
    state: Any = None         # for backward


class TokenScores(_OnDevice):
    """Scores of rows of logits [n, columns] (a vocabulary, classes): log probability of a token for each row, entropy, the
    likeliest tokens; and the logits' gradient.

    p = softmax(scale * logits); scale: 1 / temperature.  Logits: float32, bfloat16 or float16, values of a row side by side.
    tokens: int64, one a row; a row whose token is no column (-1, -100, ...) is left out: its logits are not read, its log
    probability, entropy and gradient are 0.  Logits of -infinity have probability 0; a row of them alone has log probability
    -infinity, entropy 0 and no gradient; NaN and +infinity make a row's numbers NaN.  Must not be used from two
    threads or streams at once (the workspace)."""

    def __init__(self, scale: float = 1.0, device="cuda:0"):
        import torch
        device = torch.device(device)
        if device.type == "cuda" and device.index is None:
            device = torch.device("cuda", torch.cuda.current_device())
        super().__init__(device)
        self.scale = float(scale)
        if not 0.0 < self.scale <= 1e38:
            raise ValueError(f"scale {scale}: a positive number up to 1e38 needed")
        rc, nbytes = tt_emb_token_workspace_bytes()
        if rc:
            raise TTEmbError(rc, "tt_emb_token_workspace_bytes")
        self._make_workspace(nbytes)

    def _vector(self, t, n, kind, name):
        if t.dtype != kind or t.device != self.device or t.shape != (n,) or not t.is_contiguous():
            raise ValueError(f"{name}: contiguous {kind} [{n}] on {self.device} needed, not {t.dtype} {tuple(t.shape)} on "
                             f"{t.device}")
        return t.data_ptr()

    def _empty(self, *shape, dtype=None):
        return self.torch.empty(shape, dtype=dtype or self.torch.float32, device=self.device)

    def _out(self, logits, out, dtype):
        if out is None:
            return self.torch.empty(logits.shape, dtype=dtype or logits.dtype, device=self.device)
        if out.shape != logits.shape or dtype not in (None, out.dtype):
            raise ValueError(f"out: {tuple(logits.shape)} of {dtype or out.dtype} needed, not {tuple(out.shape)}")
        return out

    def forward(self, logits, tokens=None, entropy: bool = False, top: int = 0, state: bool = False):
        """A TokenResult: log probabilities of tokens (without tokens all rows count and there are none), entropies, the
        `top` (up to 64) likeliest tokens, the lowest first among equals, and what backward needs."""
        x = self._matrix(logits)
        n, torch = x.rows, self.torch
        ptr = 0 if tokens is None else self._vector(tokens, n, torch.int64, "tokens")
        if not 0 <= top <= 64:
            raise ValueError(f"top {top}: 0 to 64 needed")
        if tokens is None and not (entropy or top or state):
            raise ValueError("tokens, entropy, top or state needed")
        logprobs = None if tokens is None else self._empty(n)
        h = self._empty(n) if entropy else None
        kept = self._empty(2, n) if state else None
        ids, values = (self._empty(n, top, dtype=torch.int64), self._empty(n, top)) if top else (None, None)
        at = [0 if t is None else t.data_ptr() for t in (logprobs, h, kept, ids, values)]
        self._call(self.lib.tt_emb_token_scores, byref(x), ptr, self.scale, byref(TTEmbTokenOut(*at, top, 0)), self._ws_ptr,
                   self.workspace_bytes)
        return TokenResult(logprobs, h, ids, values, (kept, h) if state else None)

    def backward(self, logits, tokens, state, d_logprobs=None, d_entropy=None, out=None, dtype=None):
        """Gradient of a forward(..., state=True) of the same logits and tokens with respect to the logits, for
        gradients of the log probabilities and (with entropy=True there) of the entropies, float32 [n].  out: may be the
        logits themselves, which are overwritten."""
        x = self._matrix(logits)
        n, torch = x.rows, self.torch
        if d_logprobs is None and d_entropy is None:
            raise ValueError("d_logprobs or d_entropy needed")
        if tokens is None and d_logprobs is not None:
            raise ValueError("d_logprobs needs tokens")
        kept, h = state
        if kept.shape != (2, n) or not kept.is_contiguous() or kept.dtype != torch.float32 or kept.device != self.device:
            raise ValueError(f"state of {n} rows on {self.device} needed")
        if d_entropy is not None and h is None:
            raise ValueError("d_entropy needs the state of a forward with entropy=True")
        at = [0 if d is None else self._vector(d, n, torch.float32, name) for d, name in
              ((h if d_entropy is not None else None, "entropy"), (d_logprobs, "d_logprobs"), (d_entropy, "d_entropy"))]
        ptr = 0 if tokens is None else self._vector(tokens, n, torch.int64, "tokens")
        out = self._out(logits, out, dtype)
        self._call(self.lib.tt_emb_token_backward, byref(x), ptr, self.scale, kept.data_ptr(), *at,
                   byref(self._matrix(out)))
        return out

    def loss(self, logits, tokens, weights=1.0, out=None, dtype=None):
        """Log probabilities of the tokens, and the gradient of the loss -sum(weights * log probabilities) with respect to the
        logits, in one call.  weights: a number, or float32 [n].  out: as in backward."""
        x = self._matrix(logits)
        n, torch = x.rows, self.torch
        ptr = self._vector(tokens, n, torch.int64, "tokens")
        each, one = (self._vector(weights, n, torch.float32, "weights"), 1.0) if isinstance(weights, torch.Tensor) else (
            0, float(weights))
        out, logprobs = self._out(logits, out, dtype), self._empty(n)
        self._call(self.lib.tt_emb_token_loss, byref(x), ptr, self.scale, each, one, logprobs.data_ptr(),
                   byref(self._matrix(out)), self._ws_ptr, self.workspace_bytes)
        return logprobs, out


class PositionBias(_OnDevice):
    """A learned bias of attention by distance: table [buckets, heads], looked up by the bucket of every distance of a key
    from a query, alone or added to scores [batch, heads, queries, keys]; and the table's gradient.

    The distance of key j from query i is j - i + offset, offset: the first key's position less the first query's, a
    number, or int64 [batch] with one for each sequence.  (A query that follows a cache of n keys, its own among them: 1 - n.)
    bucket_of: int32 [2 * span + 1], the buckets of the distances -span to span, whose ends also stand for all beyond; a
    number outside the table: no bucket, where `fill` (-inf: a mask) stands for the bias.  An infinite bias replaces the score
    that it would be added to, whatever that is.  weight (float32, bfloat16 or float16, values of a row side by side) and bucket_of
    are borrowed, and taken as they are at the time of a call.  Must not be used from two threads or streams
    at once (the workspace of backward)."""

    def __init__(self, weight, bucket_of, fill: float = 0.0):
        super().__init__(weight.device)
        self.weight, self.bucket_of, self.fill = weight, bucket_of, float(fill)
        if self.fill != self.fill:
            raise ValueError("fill: a number needed")
        self._spaces, self.workspace_bytes = [], 0
        self._make_workspace(256)
        self._matrix(weight)
        self._distances(0, 1)

    @staticmethod
    def log_buckets(buckets: int, max_distance: int, bidirectional: bool = True):
        """bucket_of (on the CPU) for buckets that widen with the distance: half of a side's buckets hold one distance each,
        from 0 on; the others grow by a constant factor up to max_distance, and the last holds all beyond.  Bucket e + k starts at
        the smallest whole number that is at least e (max_distance / e) ** (k / (side - e)), e the first half's size.
        bidirectional: the first half of the buckets is for keys at and before a query, the second for keys after it; else
        keys after a query have no bucket (-1)."""
        import torch
        side = buckets // 2 if bidirectional else buckets
        near = side // 2
        if near < 1 or bidirectional and buckets % 2 or max_distance <= near:
            raise ValueError(f"{buckets} buckets up to distance {max_distance}: at least two a side, an even number for "
                             "both sides, and a distance beyond the first half needed")
        far, starts = side - near, []
        for k in range(1, far):
            # the smallest n with n ** far >= near ** (far - k) * max_distance ** k, in whole numbers
            power = near ** (far - k) * max_distance ** k
            low, high = near, max_distance
            while low < high:
                middle = (low + high) // 2
                low, high = (low, middle) if middle ** far >= power else (middle + 1, high)
            starts.append(low)
        distance = torch.arange(max_distance + 1)
        before = torch.where(distance < near, distance, near + torch.bucketize(distance, torch.tensor(starts, dtype=torch.int64),
                                                                               right=True))
        after = side + before[1:] if bidirectional else torch.full((max_distance,), -1)
        return torch.cat([before.flip(0), after]).to(torch.int32)

    def _distances(self, offset, batch):
        of, torch = self.bucket_of, self.torch
        if of.dtype != torch.int32 or of.device != self.device or of.dim() != 1 or not of.is_contiguous() or of.numel() % 2 == 0:
            raise ValueError(f"bucket_of: contiguous int32 [2 * span + 1] on {self.device} needed")
        at, number = 0, 0
        if isinstance(offset, torch.Tensor):
            if offset.dtype != torch.int64 or offset.device != self.device or offset.shape != (batch,) or \
                    not offset.is_contiguous():
                raise ValueError(f"offset: a number, or contiguous int64 [{batch}] on {self.device} needed")
            at = offset.data_ptr()
        else:
            number = max(-(1 << 60), min(1 << 60, int(offset)))  # far beyond all distances
        return TTEmbDistances(of.data_ptr(), at, number, of.numel() // 2, 0)

    def _pairs(self, t, written=False):
        if t.dim() != 4 or t.device != self.device:
            raise ValueError(f"[batch, heads, queries, keys] on {self.device} needed: shape {tuple(t.shape)} on {t.device}")
        b, h, q, k = t.shape
        steps = t.stride()
        if k > 1 and steps[3] != 1:
            raise ValueError(f"strides {steps}: keys side by side needed")
        if h != self.weight.shape[1]:
            raise ValueError(f"{h} heads, not the table's {self.weight.shape[1]}")
        if written and t.numel():
            size = 1
            for step, n in sorted((s, n) for s, n in zip(steps, t.shape) if n > 1):
                if step < size:
                    raise ValueError(f"strides {steps}: values that do not overlap needed")
                size = step * (n - 1) + size
        return TTEmbPairs(t.data_ptr(), steps[0] if b > 1 else 0, steps[1] if h > 1 else 0, steps[2] if q > 1 else 0, q, k, b, h,
                          self._type(t), 0)

    def forward(self, queries: int, keys: int, offset=0, out=None, dtype=None):
        """The bias, [batch, heads, queries, keys], in the table's type unless out or dtype says otherwise.  batch: that of out or
        of the offsets, or 1."""
        torch, table = self.torch, self._matrix(self.weight)
        if out is None:
            batch = offset.numel() if isinstance(offset, torch.Tensor) else 1
            out = torch.empty((batch, table.cols, queries, keys), dtype=dtype or self.weight.dtype, device=self.device)
        elif out.shape[2:] != (queries, keys) or dtype not in (None, out.dtype):
            raise ValueError(f"out: [batch, heads, {queries}, {keys}] of {dtype or out.dtype} needed, not {tuple(out.shape)}")
        to = self._pairs(out, True)
        self._call(self.lib.tt_emb_bias_forward, byref(table), byref(self._distances(offset, to.batch)), self.fill, None,
                   byref(to))
        return out

    def add_to(self, scores, offset=0, out=None):
        """scores + bias, in out, or (None) in place.  out: the scores themselves, or a tensor that shares no memory with them; within
        their range it has the same pitches in bytes (columns or rows beside theirs in one buffer)."""
        if out is None:
            out = scores
        elif out.shape != scores.shape:
            raise ValueError(f"out: {tuple(scores.shape)} needed, not {tuple(out.shape)}")
        table, to = self._matrix(self.weight), self._pairs(out, True)
        given = to if out is scores else self._pairs(scores)
        self._call(self.lib.tt_emb_bias_forward, byref(table), byref(self._distances(offset, to.batch)), self.fill,
                   byref(given), byref(to))
        return out

    def backward(self, grad, offset=0, out=None, dtype=None, add: bool = False):
        """Gradient with respect to the table, [buckets, heads], for the gradient of the bias or of the scores that it was added
        to.  With add, it is added to out."""
        g, weight = self._pairs(grad), self.weight
        if out is None:
            if add:
                raise ValueError("add needs out")
            out = self.torch.empty(weight.shape, dtype=dtype or weight.dtype, device=self.device)
        elif out.shape != weight.shape or dtype not in (None, out.dtype):
            raise ValueError(f"out: {tuple(weight.shape)} of {dtype or out.dtype} needed, not {tuple(out.shape)}")
        d = self._distances(offset, g.batch)
        rc, nbytes = tt_emb_bias_workspace_bytes(g, d.span)
        if rc:
            raise TTEmbError(rc, "tt_emb_bias_workspace_bytes")
        if nbytes > self.workspace_bytes:  # sizes that rise in small steps do not make one each
            self._make_workspace(max(nbytes, self.workspace_bytes * 3 // 2))
        if self._capturing() and not any(space is self.workspace for space in self._spaces):
            self._spaces.append(self.workspace)  # the graph goes on using it when a larger one has been made
        self._call(self.lib.tt_emb_bias_backward, byref(g), byref(d), byref(self._matrix(out)), 1 if add else 0, self._ws_ptr,
                   self.workspace_bytes)
        return out
