"""ctypes binding of ``include/adasd.h``: same names, argument marshalling only.

The raw functions (``adasd_verify`` ...) take device addresses as Python ints and
return the library's status code.  :class:`Context` wraps them for torch tensors
(``tensor.data_ptr()``, the current CUDA stream) and raises :class:`AdasdError` on a
non-zero code.  Nothing here computes anything.
"""
from __future__ import annotations

import ctypes as C
import functools
import os
from typing import Optional

from .build import LIB, build

ADASD_BF16, ADASD_FP32 = 0, 1
ADASD_FUSE_UPDATE = 1
ADASD_KMAX_LIMIT = 32
STATUS_CAPACITY, STATUS_TIMEOUT, STATUS_NAN = 1, 2, 4
PREF_SIGMOID, PREF_SQUARED, PREF_HINGE = 0, 1, 2
PREF_SCRATCH_PER_ROW = 16
ADAMW_BLOCK = 256
_PREF_RULES = {"sigmoid": PREF_SIGMOID, "squared": PREF_SQUARED, "hinge": PREF_HINGE}
ERR_NULL, ERR_ALIGN, ERR_SHAPE, ERR_DTYPE, ERR_CAPACITY, ERR_CUDA, ERR_DEVICE = -1, -2, -3, -4, -5, -7, -9


class AdasdError(RuntimeError):
    def __init__(self, code: int, where: str):
        self.code = code
        super().__init__(f"{where}: {adasd_strerror(code)} ({code})")


class AdasdConfig(C.Structure):
    _fields_ = [("B", C.c_int32), ("V", C.c_int32), ("Kmax", C.c_int32), ("dtype", C.c_int32),
                ("list_capacity", C.c_int32), ("kde_bandwidth", C.c_int32),
                ("reject_rule", C.c_int32), ("min_kde_samples", C.c_int32),
                ("cluster_size", C.c_int32), ("device", C.c_int32)]


class RoundRecord(C.Structure):
    """Host struct of device array addresses (``adasd_round_record``)."""
    _fields_ = [(n, C.c_void_p) for n in ("H_d", "H_t", "lse_d", "lse_t", "jsd", "dist", "p_acc",
                                          "y", "draft_len", "accept_len", "rejected")]


class PolicyOptions(C.Structure):
    _fields_ = [(n, C.c_float) for n in ("clip_low", "clip_high", "kl_coef", "entropy_coef", "scale")]


class PreferenceOptions(C.Structure):
    _fields_ = [("rule", C.c_int32), ("average", C.c_int32), ("beta", C.c_float), ("margin", C.c_float),
                ("label_smoothing", C.c_float), ("scale", C.c_float)]


class CrossEntropyOptions(C.Structure):
    _fields_ = [(n, C.c_float) for n in ("label_smoothing", "z_loss", "scale")]


class AdamwTensor(C.Structure):
    _fields_ = [(n, C.c_void_p) for n in ("param", "grad", "exp_avg", "exp_avg_sq", "avg_scale", "sq_scale", "param_copy")] + [
        ("n", C.c_int64), ("weight_decay", C.c_float), ("param_dtype", C.c_int32), ("grad_dtype", C.c_int32), ("state_bits", C.c_int32)]


class AdamwOptions(C.Structure):
    _fields_ = [(n, C.c_double) for n in ("lr", "beta1", "beta2", "eps", "grad_scale")] + [
        ("step", C.c_int32), ("stochastic", C.c_int32), ("seed", C.c_uint32), ("lr_dev", C.c_void_p), ("grad_scale_dev", C.c_void_p),
        ("step_dev", C.c_void_p)]


def library_path() -> str:
    return LIB


@functools.lru_cache(maxsize=None)
def lib() -> C.CDLL:
    """Loads libadasd.so, building it first if the sources are newer.  Raises if it
    cannot be built or loaded: there is no fallback."""
    path = build()
    if not os.path.exists(path):
        raise RuntimeError(f"{path} is missing: build the CUDA library first")
    L = C.CDLL(path)
    P, I32, I64, U32 = C.c_void_p, C.c_int32, C.c_int64, C.c_uint32
    sigs = {
        "adasd_create": [C.POINTER(P), C.POINTER(AdasdConfig)],
        "adasd_destroy": [P],
        "adasd_reset": [P, P, I32, P],
        "adasd_draft_entropy": [P, P, I64, P, P, P, P, P, P, P, P],
        "adasd_verify": [P, P, P, I64, I64, I64, I64, P, P, P, P, P, P, C.POINTER(RoundRecord),
                         U32, P],
        "adasd_update_thresholds": [P, C.POINTER(RoundRecord), P],
        "adasd_vanilla_verify": [P, P, P, I64, I64, I64, I64, P, P, P, P, P, P, P, P],
        "adasd_vanilla_verify_static": [I32, I32, I32, I32, P, P, I64, I64, I64, I64, P, P, P, P,
                                        P, P, P, P, P],
        "adasd_greedy_verify": [P, P, I64, I64, P, P, P, P, P, P],
        "adasd_gen_only_update": [P, P, P, P, P],
        "adasd_selftest_expired_wait": [P, P, I64, I32, P, P, P, P],
        "adasd_token_logprob": [P, P, I64, P, I32, P, P, P, P],
        "adasd_token_logprob_grad": [P, P, I64, P, I32, P, P, P, I64, P],
        "adasd_policy_loss": [P, P, I64, P, I32, P, P, P, P, C.POINTER(PolicyOptions), P, P, P, P, P, P, I64, P],
        "adasd_preference_loss": [P, P, I64, P, I32, P, I32, P, P, C.POINTER(PreferenceOptions), P, P, P, P, P,
                                  I64, P],
        "adasd_head_scratch": [P, I32, I32, I32, C.POINTER(C.c_size_t)],
        "adasd_head_logprob": [P, P, I64, P, I64, I32, P, I32, P, C.c_size_t, P, P, P, P],
        "adasd_head_logprob_grad": [P, P, I64, P, I64, I32, P, I32, P, P, P, P, P, C.c_size_t, P, I64, P, I64, P],
        "adasd_head_cross_entropy": [P, P, I64, P, I64, I32, P, I32, P, C.POINTER(CrossEntropyOptions), P, C.c_size_t, P, P, P, P, P,
                                     I64, P, I64, P],
        "adasd_adamw_step": [P, C.POINTER(AdamwTensor), I32, C.POINTER(AdamwOptions), P],
        "adasd_set_warpers": [P, C.c_float, I32, C.c_float],
        "adasd_get_thresholds": [P, P, P, P, P, P],
        "adasd_state_export": [P, I32, P, C.POINTER(C.c_size_t)],
        "adasd_state_import": [P, I32, P, C.c_size_t],
        "adasd_status": [P, C.POINTER(U32)],
    }
    for name, args in sigs.items():
        fn = getattr(L, name)
        fn.argtypes = args
        fn.restype = C.c_int
    L.adasd_strerror.argtypes = [C.c_int]
    L.adasd_strerror.restype = C.c_char_p
    return L


# ------------------------------------------------------------------ raw calls, same names

def adasd_strerror(code: int) -> str:
    return lib().adasd_strerror(code).decode()


def adasd_create(cfg: AdasdConfig):
    """Returns (code, ctx handle)."""
    h = C.c_void_p()
    rc = lib().adasd_create(C.byref(h), C.byref(cfg))
    return rc, h


def adasd_destroy(ctx) -> int:
    return lib().adasd_destroy(ctx)


def adasd_reset(ctx, seq_ids_dev, n, stream) -> int:
    return lib().adasd_reset(ctx, seq_ids_dev, n, stream)


def adasd_draft_entropy(ctx, logits_dev, row_stride, u_dev, active_inout_dev, H_out_dev,
                        lse_out_dev, token_out_dev, stop_out_dev, draft_len_inout_dev, stream) -> int:
    return lib().adasd_draft_entropy(ctx, logits_dev, row_stride, u_dev, active_inout_dev,
                                     H_out_dev, lse_out_dev, token_out_dev, stop_out_dev,
                                     draft_len_inout_dev, stream)


def adasd_verify(ctx, draft_logits_dev, target_logits_dev, d_seq_stride, d_row_stride,
                 t_seq_stride, t_row_stride, draft_tokens_dev, draft_len_dev, u_target_dev,
                 u_accept_dev, accept_len_dev, next_token_dev, record, flags, stream) -> int:
    return lib().adasd_verify(ctx, draft_logits_dev, target_logits_dev, d_seq_stride,
                              d_row_stride, t_seq_stride, t_row_stride, draft_tokens_dev,
                              draft_len_dev, u_target_dev, u_accept_dev, accept_len_dev,
                              next_token_dev, C.byref(record) if record is not None else None,
                              flags, stream)


def adasd_update_thresholds(ctx, record, stream) -> int:
    return lib().adasd_update_thresholds(ctx, C.byref(record) if record is not None else None,
                                         stream)


def adasd_vanilla_verify(ctx, draft_logits_dev, target_logits_dev, d_seq_stride, d_row_stride,
                         t_seq_stride, t_row_stride, draft_tokens_dev, draft_len_dev,
                         u_accept_dev, u_resample_dev, accept_len_dev, next_token_dev,
                         alpha_out_dev, stream) -> int:
    return lib().adasd_vanilla_verify(ctx, draft_logits_dev, target_logits_dev, d_seq_stride,
                                      d_row_stride, t_seq_stride, t_row_stride, draft_tokens_dev,
                                      draft_len_dev, u_accept_dev, u_resample_dev, accept_len_dev,
                                      next_token_dev, alpha_out_dev, stream)


def adasd_vanilla_verify_static(B, V, Kmax, dtype, draft_logits_dev, target_logits_dev,
                                d_seq_stride, d_row_stride, t_seq_stride, t_row_stride,
                                draft_tokens_dev, draft_len_dev, u_accept_dev, u_resample_dev,
                                accept_len_dev, next_token_dev, alpha_out_dev, status_out_dev,
                                stream) -> int:
    """Context-free vanilla verification whose scratch is a fixed array inside the library:
    for callers that may not allocate device memory.  Same arguments as the C function."""
    return lib().adasd_vanilla_verify_static(B, V, Kmax, dtype, draft_logits_dev,
                                             target_logits_dev, d_seq_stride, d_row_stride,
                                             t_seq_stride, t_row_stride, draft_tokens_dev,
                                             draft_len_dev, u_accept_dev, u_resample_dev,
                                             accept_len_dev, next_token_dev, alpha_out_dev,
                                             status_out_dev, stream)


def adasd_greedy_verify(ctx, target_logits_dev, t_seq_stride, t_row_stride, draft_tokens_dev,
                        draft_len_dev, accept_len_dev, next_token_dev, argmax_out_dev, stream) -> int:
    return lib().adasd_greedy_verify(ctx, target_logits_dev, t_seq_stride, t_row_stride, draft_tokens_dev,
                                     draft_len_dev, accept_len_dev, next_token_dev, argmax_out_dev, stream)


def adasd_gen_only_update(ctx, H_draft_dev, draft_len_dev, accept_len_dev, stream) -> int:
    return lib().adasd_gen_only_update(ctx, H_draft_dev, draft_len_dev, accept_len_dev, stream)


def adasd_set_warpers(ctx, temperature, top_k, top_p) -> int:
    return lib().adasd_set_warpers(ctx, temperature, top_k, top_p)


def adasd_selftest_expired_wait(ctx, logits_dev, row_stride, row, u_dev, H_out_dev, token_out_dev, stream) -> int:
    return lib().adasd_selftest_expired_wait(ctx, logits_dev, row_stride, row, u_dev, H_out_dev, token_out_dev,
                                             stream)


def adasd_token_logprob(ctx, logits_dev, row_stride, tokens_dev, n_rows, logp_out_dev, entropy_out_dev, lse_out_dev,
                        stream) -> int:
    return lib().adasd_token_logprob(ctx, logits_dev, row_stride, tokens_dev, n_rows, logp_out_dev, entropy_out_dev,
                                     lse_out_dev, stream)


def adasd_token_logprob_grad(ctx, logits_dev, row_stride, tokens_dev, n_rows, grad_logp_dev, grad_entropy_dev,
                             grad_logits_dev, grad_row_stride, stream) -> int:
    return lib().adasd_token_logprob_grad(ctx, logits_dev, row_stride, tokens_dev, n_rows, grad_logp_dev,
                                          grad_entropy_dev, grad_logits_dev, grad_row_stride, stream)


def adasd_policy_loss(ctx, logits_dev, row_stride, tokens_dev, n_rows, advantage_dev, old_logp_dev, ref_logp_dev,
                      weight_dev, options, row_loss_out_dev, loss_out_dev, logp_out_dev, entropy_out_dev, kl_out_dev,
                      grad_logits_dev, grad_row_stride, stream) -> int:
    return lib().adasd_policy_loss(ctx, logits_dev, row_stride, tokens_dev, n_rows, advantage_dev, old_logp_dev,
                                   ref_logp_dev, weight_dev, C.byref(options) if options is not None else None,
                                   row_loss_out_dev, loss_out_dev, logp_out_dev, entropy_out_dev, kl_out_dev,
                                   grad_logits_dev, grad_row_stride, stream)


def adasd_preference_loss(ctx, logits_dev, row_stride, tokens_dev, n_rows, seq_start_dev, n_pairs, ref_logp_dev,
                          pair_weight_dev, options, scratch_dev, seq_logp_out_dev, pair_loss_out_dev, loss_out_dev,
                          grad_logits_dev, grad_row_stride, stream) -> int:
    return lib().adasd_preference_loss(ctx, logits_dev, row_stride, tokens_dev, n_rows, seq_start_dev, n_pairs,
                                       ref_logp_dev, pair_weight_dev,
                                       C.byref(options) if options is not None else None, scratch_dev,
                                       seq_logp_out_dev, pair_loss_out_dev, loss_out_dev, grad_logits_dev,
                                       grad_row_stride, stream)


def adasd_head_scratch(ctx, n_rows, dim, with_grad):
    """Returns (code, bytes)."""
    n = C.c_size_t(0)
    rc = lib().adasd_head_scratch(ctx, n_rows, dim, with_grad, C.byref(n))
    return rc, n.value


def adasd_head_logprob(ctx, hidden_dev, hidden_stride, weight_dev, weight_stride, dim, tokens_dev, n_rows, scratch_dev, scratch_bytes,
                       logp_out_dev, entropy_out_dev, lse_out_dev, stream) -> int:
    return lib().adasd_head_logprob(ctx, hidden_dev, hidden_stride, weight_dev, weight_stride, dim, tokens_dev, n_rows, scratch_dev,
                                    scratch_bytes, logp_out_dev, entropy_out_dev, lse_out_dev, stream)


def adasd_head_logprob_grad(ctx, hidden_dev, hidden_stride, weight_dev, weight_stride, dim, tokens_dev, n_rows, lse_dev, entropy_dev,
                            grad_logp_dev, grad_entropy_dev, scratch_dev, scratch_bytes, grad_hidden_dev, grad_hidden_stride,
                            grad_weight_dev, grad_weight_stride, stream) -> int:
    return lib().adasd_head_logprob_grad(ctx, hidden_dev, hidden_stride, weight_dev, weight_stride, dim, tokens_dev, n_rows, lse_dev,
                                         entropy_dev, grad_logp_dev, grad_entropy_dev, scratch_dev, scratch_bytes, grad_hidden_dev,
                                         grad_hidden_stride, grad_weight_dev, grad_weight_stride, stream)


def adasd_head_cross_entropy(ctx, hidden_dev, hidden_stride, weight_dev, weight_stride, dim, tokens_dev, n_rows, row_weight_dev, options,
                             scratch_dev, scratch_bytes, row_loss_out_dev, loss_out_dev, logp_out_dev, lse_out_dev, grad_hidden_dev,
                             grad_hidden_stride, grad_weight_dev, grad_weight_stride, stream) -> int:
    return lib().adasd_head_cross_entropy(ctx, hidden_dev, hidden_stride, weight_dev, weight_stride, dim, tokens_dev, n_rows,
                                          row_weight_dev, C.byref(options) if options is not None else None, scratch_dev,
                                          scratch_bytes, row_loss_out_dev, loss_out_dev, logp_out_dev, lse_out_dev, grad_hidden_dev,
                                          grad_hidden_stride, grad_weight_dev, grad_weight_stride, stream)


def adasd_adamw_step(ctx, tensors, n_tensors, options, stream) -> int:
    """tensors: a ctypes array of AdamwTensor."""
    return lib().adasd_adamw_step(ctx, tensors, n_tensors, C.byref(options) if options is not None else None, stream)


def adasd_get_thresholds(ctx, T_G_dev, nE_dev, nA_dev, nR_dev, stream) -> int:
    return lib().adasd_get_thresholds(ctx, T_G_dev, nE_dev, nA_dev, nR_dev, stream)


def adasd_state_export(ctx, seq: int, host_buf, bytes_inout) -> int:
    return lib().adasd_state_export(ctx, seq, host_buf, bytes_inout)


def adasd_state_import(ctx, seq: int, host_buf, nbytes: int) -> int:
    return lib().adasd_state_import(ctx, seq, host_buf, nbytes)


def adasd_status(ctx):
    """Returns (code, status bits); clears the sticky word."""
    s = C.c_uint32(0)
    rc = lib().adasd_status(ctx, C.byref(s))
    return rc, s.value


# ------------------------------------------------------------------ torch convenience

def _ptr(t) -> Optional[int]:
    return None if t is None else t.data_ptr()


class AdamwTable:
    """The tensors of an AdamW step, checked and laid out once (:meth:`Context.adamw_table`); keeps them alive."""

    def __init__(self, entries, owned):
        self.entries, self.n, self._owned = entries, len(entries), owned


class Context:
    """Owns one ``adasd_ctx``; methods take torch CUDA tensors and use the current stream."""

    def __init__(self, B: int, V: int, Kmax: int, dtype: int = ADASD_BF16,
                 list_capacity: int = 1 << 14, kde_bandwidth: int = 0, reject_rule: int = 0,
                 min_kde_samples: int = 2, cluster_size: int = 0, device: int = 0):
        import torch
        if not torch.cuda.is_available():
            raise RuntimeError("the AdaSD library needs a CUDA device; there is no CPU path")
        self.torch = torch
        self.cfg = AdasdConfig(B, V, Kmax, dtype, list_capacity, kde_bandwidth, reject_rule,
                               min_kde_samples, cluster_size, device)
        self.device = torch.device("cuda", device)
        rc, self.handle = adasd_create(self.cfg)
        if rc != 0:
            self.handle = None
            raise AdasdError(rc, "adasd_create")
        self.B, self.V, self.Kmax = B, V, Kmax
        # What every hot call needs, looked up once: an engine issues these calls between two kernels of
        # a few microseconds each, so the marshalling is kept to the address of each tensor.
        L = lib()
        self._draft_entropy, self._verify = L.adasd_draft_entropy, L.adasd_verify
        self._vanilla_verify, self._greedy_verify = L.adasd_vanilla_verify, L.adasd_greedy_verify
        self._token_logprob, self._token_logprob_grad = L.adasd_token_logprob, L.adasd_token_logprob_grad
        self._policy_loss, self._preference_loss = L.adasd_policy_loss, L.adasd_preference_loss
        self._adamw_step = L.adasd_adamw_step
        self._head_logprob, self._head_logprob_grad = L.adasd_head_logprob, L.adasd_head_logprob_grad
        self._head_cross_entropy, self._bf16 = L.adasd_head_cross_entropy, torch.bfloat16
        self._logit_dtype = torch.bfloat16 if dtype == ADASD_BF16 else torch.float32
        self._i32, self._f32, self._index = torch.int32, torch.float32, self.device.index
        self._raw_stream = torch._C._cuda_getCurrentRawStream
        self._rec = None                           # the last record's addresses and their struct

    def close(self) -> None:
        if getattr(self, "handle", None):
            adasd_destroy(self.handle)
            self.handle = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    def _stream(self) -> int:
        return self._raw_stream(self.device.index)

    @staticmethod
    def _check(rc: int, where: str) -> None:
        if rc != 0:
            raise AdasdError(rc, where)

    def new_record(self) -> dict:
        """Device tensors for every field of a round record."""
        t, B, K = self.torch, self.B, self.Kmax
        f = dict(dtype=t.float32, device=self.device)
        i = dict(dtype=t.int32, device=self.device)
        return dict(H_d=t.full((B, K), float("nan"), **f), H_t=t.full((B, K + 1), float("nan"), **f),
                    lse_d=t.full((B, K), float("nan"), **f), lse_t=t.full((B, K + 1), float("nan"), **f),
                    jsd=t.full((B, K), float("nan"), **f), dist=t.full((B, K), float("nan"), **f),
                    p_acc=t.full((B, K), float("nan"), **f), y=t.full((B, K + 1), -2, **i),
                    draft_len=t.zeros(B, **i), accept_len=t.zeros(B, **i), rejected=t.zeros(B, **i))

    @staticmethod
    def record_struct(rec: Optional[dict]) -> Optional[RoundRecord]:
        if rec is None:
            return None
        return RoundRecord(**{k: (v.data_ptr() if v is not None else None) for k, v in rec.items()})

    def reset(self, seq_ids=None) -> None:
        n = self.B if seq_ids is None else seq_ids.numel()
        self._check(adasd_reset(self.handle, _ptr(seq_ids), n, self._stream()), "adasd_reset")

    def draft_entropy(self, logits, H_out, u=None, token_out=None, active=None, lse_out=None,
                      stop_out=None, draft_len=None, row_stride: Optional[int] = None) -> None:
        rc = self._draft_entropy(self.handle, logits.data_ptr(),
                                 logits.stride(0) if row_stride is None else row_stride,
                                 None if u is None else u.data_ptr(),
                                 None if active is None else active.data_ptr(), H_out.data_ptr(),
                                 None if lse_out is None else lse_out.data_ptr(),
                                 None if token_out is None else token_out.data_ptr(),
                                 None if stop_out is None else stop_out.data_ptr(),
                                 None if draft_len is None else draft_len.data_ptr(),
                                 self._raw_stream(self.device.index))
        if rc:
            raise AdasdError(rc, "adasd_draft_entropy")

    def _record_ref(self, rec: Optional[dict]):
        """The C struct of a record of device tensors; the struct of the last record is used again
        when the addresses are the same.  Addresses and struct are kept as one object, and the call
        works on its own reference to it: another thread's record never gets into this call."""
        if rec is None:
            return None
        key = [(k, v.data_ptr()) if v is not None else (k, None) for k, v in rec.items()]
        last = self._rec
        if last is None or last[0] != key:
            self._rec = last = (key, C.byref(RoundRecord(**dict(key))))
        return last[1]

    def verify(self, draft_logits, target_logits, draft_tokens, u_target, u_accept, accept_len,
               next_token, draft_len=None, record: Optional[dict] = None,
               fuse_update: bool = True) -> None:
        ds, ts = draft_logits.stride(), target_logits.stride()
        rc = self._verify(self.handle, draft_logits.data_ptr(), target_logits.data_ptr(), ds[0], ds[1],
                          ts[0], ts[1], draft_tokens.data_ptr(),
                          None if draft_len is None else draft_len.data_ptr(), u_target.data_ptr(),
                          u_accept.data_ptr(), accept_len.data_ptr(), next_token.data_ptr(),
                          self._record_ref(record), ADASD_FUSE_UPDATE if fuse_update else 0,
                          self._raw_stream(self.device.index))
        if rc:
            raise AdasdError(rc, "adasd_verify")

    def update_thresholds(self, record: dict) -> None:
        self._check(adasd_update_thresholds(self.handle, self.record_struct(record), self._stream()),
                    "adasd_update_thresholds")

    def vanilla_verify(self, draft_logits, target_logits, draft_tokens, u_accept, u_resample,
                       accept_len, next_token, draft_len=None, alpha_out=None) -> None:
        ds, ts = draft_logits.stride(), target_logits.stride()
        rc = self._vanilla_verify(self.handle, draft_logits.data_ptr(), target_logits.data_ptr(), ds[0],
                                  ds[1], ts[0], ts[1], draft_tokens.data_ptr(),
                                  None if draft_len is None else draft_len.data_ptr(), u_accept.data_ptr(),
                                  u_resample.data_ptr(), accept_len.data_ptr(), next_token.data_ptr(),
                                  None if alpha_out is None else alpha_out.data_ptr(),
                                  self._raw_stream(self.device.index))
        if rc:
            raise AdasdError(rc, "adasd_vanilla_verify")

    def greedy_verify(self, target_logits, draft_tokens, accept_len, next_token, draft_len=None,
                      argmax_out=None) -> None:
        ts = target_logits.stride()
        rc = self._greedy_verify(self.handle, target_logits.data_ptr(), ts[0], ts[1], draft_tokens.data_ptr(),
                                 None if draft_len is None else draft_len.data_ptr(), accept_len.data_ptr(),
                                 next_token.data_ptr(), None if argmax_out is None else argmax_out.data_ptr(),
                                 self._raw_stream(self.device.index))
        if rc:
            raise AdasdError(rc, "adasd_greedy_verify")

    def gen_only_update(self, H_draft, accept_len, draft_len=None) -> None:
        self._check(adasd_gen_only_update(self.handle, H_draft.data_ptr(), _ptr(draft_len),
                                          accept_len.data_ptr(), self._stream()), "adasd_gen_only_update")

    def set_warpers(self, temperature: float = 1.0, top_k: int = 0, top_p: float = 1.0) -> None:
        self._check(adasd_set_warpers(self.handle, float(temperature), int(top_k), float(top_p)),
                    "adasd_set_warpers")

    # ---- scoring and training on given tokens: rows of logits [n, V], their tokens [n] ----------------
    # (Every check is a call into torch of 60 to 100 ns, and a launch takes about as long as ten of them on the host: the
    # checks are kept to one pass over the arguments.)

    def _rows(self, where: str, logits):
        """(address, row stride, rows) of logits, after the checks that addresses alone do not allow."""
        if logits.dtype is not self._logit_dtype:
            raise AdasdError(ERR_DTYPE, where)
        if logits.get_device() != self._index:
            raise AdasdError(ERR_DEVICE, where)
        shape, strides, V = logits.shape, logits.stride(), self.V
        if len(shape) != 2 or shape[1] != V or (strides[1] != 1 and V > 1):
            raise AdasdError(ERR_SHAPE, where)
        n, stride = shape[0], strides[0]
        return logits.data_ptr(), stride if n > 1 or stride > V else V, n      # (the stride of a single row says nothing)

    def _arrays(self, where: str, dtype, n: int, arrays) -> list:
        """Addresses of contiguous device arrays of at least n entries; None for None."""
        index, got = self._index, []
        for t in arrays:
            if t is None:
                got.append(None)
            elif t.dtype is dtype and t.get_device() == index and t.numel() >= n and t.is_contiguous():
                got.append(t.data_ptr())
            else:
                raise AdasdError(ERR_DTYPE if t.dtype is not dtype else ERR_DEVICE if t.get_device() != index else ERR_SHAPE,
                                 where)
        return got

    def token_logprob(self, logits, tokens, logp_out, entropy_out=None, lse_out=None) -> None:
        z, stride, n = self._rows("adasd_token_logprob", logits)
        tok, = self._arrays("adasd_token_logprob", self._i32, n, (tokens,))
        lp, ent, lse = self._arrays("adasd_token_logprob", self._f32, n, (logp_out, entropy_out, lse_out))
        rc = self._token_logprob(self.handle, z, stride, tok, n, lp, ent, lse, self._raw_stream(self._index))
        if rc:
            raise AdasdError(rc, "adasd_token_logprob")

    def token_logprob_grad(self, logits, tokens, grad_logp, grad_out, grad_entropy=None) -> None:
        where = "adasd_token_logprob_grad"
        (z, stride, n), (g, g_stride, n_out) = self._rows(where, logits), self._rows(where, grad_out)
        if n_out != n:
            raise AdasdError(ERR_SHAPE, where)
        tok, = self._arrays(where, self._i32, n, (tokens,))
        dl, dH = self._arrays(where, self._f32, n, (grad_logp, grad_entropy))
        rc = self._token_logprob_grad(self.handle, z, stride, tok, n, dl, dH, g, g_stride, self._raw_stream(self._index))
        if rc:
            raise AdasdError(rc, where)

    def policy_loss(self, logits, tokens, advantage, row_loss_out, old_logp=None, ref_logp=None, weight=None,
                    clip_low: float = 0.2, clip_high: float = 0.2, kl_coef: float = 0.0, entropy_coef: float = 0.0,
                    scale: float = 1.0, loss_out=None, logp_out=None, entropy_out=None, kl_out=None,
                    grad_out=None) -> None:
        where = "adasd_policy_loss"
        (z, stride, n), g, g_stride = self._rows(where, logits), None, 0
        if grad_out is not None:
            g, g_stride, n_out = self._rows(where, grad_out)
            if n_out != n:
                raise AdasdError(ERR_SHAPE, where)
        tok, = self._arrays(where, self._i32, n, (tokens,))
        adv, rl, old, ref, w, lp, ent, kl = self._arrays(where, self._f32, n, (advantage, row_loss_out, old_logp, ref_logp,
                                                                              weight, logp_out, entropy_out, kl_out))
        total, = self._arrays(where, self._f32, 1, (loss_out,))
        rc = self._policy_loss(self.handle, z, stride, tok, n, adv, old, ref, w,
                               PolicyOptions(clip_low, clip_high, kl_coef, entropy_coef, scale), rl, total, lp, ent, kl,
                               g, g_stride, self._raw_stream(self._index))
        if rc:
            raise AdasdError(rc, where)

    def preference_loss(self, logits, tokens, seq_start, pair_loss_out, seq_logp_out, scratch, ref_logp=None,
                        pair_weight=None, rule: str = "sigmoid", beta: float = 0.1, margin: float = 0.0,
                        label_smoothing: float = 0.0, average: bool = False, scale: float = 1.0, loss_out=None,
                        grad_out=None) -> None:
        """rule: "sigmoid", "squared" or "hinge"; scratch: a device tensor of PREF_SCRATCH_PER_ROW bytes a row."""
        where = "adasd_preference_loss"
        (z, stride, n), g, g_stride = self._rows(where, logits), None, 0
        if grad_out is not None:
            g, g_stride, n_out = self._rows(where, grad_out)
            if n_out != n:
                raise AdasdError(ERR_SHAPE, where)
        starts = seq_start.numel()
        pairs = starts // 2
        if starts % 2 == 0:
            raise AdasdError(ERR_SHAPE, where)
        if rule not in _PREF_RULES:
            raise AdasdError(ERR_DTYPE, where)
        tok, = self._arrays(where, self._i32, n, (tokens,))
        start, = self._arrays(where, self._i32, 1, (seq_start,))
        seq, ref = self._arrays(where, self._f32, 2 * pairs, (seq_logp_out, ref_logp))
        pl, pw = self._arrays(where, self._f32, pairs, (pair_loss_out, pair_weight))
        total, = self._arrays(where, self._f32, 1, (loss_out,))
        sc, = self._arrays(where, scratch.dtype, -(-PREF_SCRATCH_PER_ROW * n // scratch.element_size()), (scratch,))
        rc = self._preference_loss(self.handle, z, stride, tok, n, start, pairs, ref, pw,
                                   PreferenceOptions(_PREF_RULES[rule], 1 if average else 0, beta, margin, label_smoothing,
                                                     scale),
                                   sc, seq, pl, total, g, g_stride, self._raw_stream(self._index))
        if rc:
            raise AdasdError(rc, where)

    # ---- scoring and training from hidden states [n, dim] and the head's weight [V, dim] -----------------

    def head_scratch(self, n_rows: int, dim: int, grad: bool = False) -> int:
        """Bytes of the scratch tensor (any dtype) that the calls below need for up to n_rows rows."""
        rc, n = adasd_head_scratch(self.handle, n_rows, dim, 1 if grad else 0)
        self._check(rc, "adasd_head_scratch")
        return n

    def _matrix(self, where: str, t, rows: int, dim: int):
        """(address, row stride) of a bf16 matrix; (None, 0) for None."""
        if t is None:
            return None, 0
        if t.dtype is not self._bf16:
            raise AdasdError(ERR_DTYPE, where)
        if t.get_device() != self._index:
            raise AdasdError(ERR_DEVICE, where)
        shape, strides = t.shape, t.stride()
        if len(shape) != 2 or shape[0] != rows or shape[1] != dim or (strides[1] != 1 and dim > 1):
            raise AdasdError(ERR_SHAPE, where)
        return t.data_ptr(), strides[0] if rows > 1 or strides[0] > dim else dim      # (the stride of a single row says nothing)

    def _head(self, where: str, hidden, weight, tokens, scratch):
        """The arguments that the head calls share, and rows and width."""
        if len(hidden.shape) != 2:
            raise AdasdError(ERR_SHAPE, where)
        n, dim = hidden.shape
        (h, hs), (w, ws) = self._matrix(where, hidden, n, dim), self._matrix(where, weight, self.V, dim)
        tok, = self._arrays(where, self._i32, n, (tokens,))
        sc, = self._arrays(where, scratch.dtype, 0, (scratch,))
        return (self.handle, h, hs, w, ws, dim, tok, n), (sc, scratch.numel() * scratch.element_size()), n, dim

    def head_logprob(self, hidden, weight, tokens, logp_out, scratch, entropy_out=None, lse_out=None) -> None:
        where = "adasd_head_logprob"
        first, sc, n, _ = self._head(where, hidden, weight, tokens, scratch)
        rc = self._head_logprob(*first, *sc, *self._arrays(where, self._f32, n, (logp_out, entropy_out, lse_out)), self._raw_stream(self._index))
        if rc:
            raise AdasdError(rc, where)

    def head_logprob_grad(self, hidden, weight, tokens, lse, grad_logp, scratch, entropy=None, grad_entropy=None, grad_hidden_out=None,
                          grad_weight_out=None) -> None:
        """lse and entropy: what :meth:`head_logprob` reported for the same rows."""
        where = "adasd_head_logprob_grad"
        first, sc, n, dim = self._head(where, hidden, weight, tokens, scratch)
        rc = self._head_logprob_grad(*first, *self._arrays(where, self._f32, n, (lse, entropy, grad_logp, grad_entropy)), *sc,
                                     *self._matrix(where, grad_hidden_out, n, dim), *self._matrix(where, grad_weight_out, self.V, dim),
                                     self._raw_stream(self._index))
        if rc:
            raise AdasdError(rc, where)

    def head_cross_entropy(self, hidden, weight, tokens, row_loss_out, scratch, row_weight=None, label_smoothing: float = 0.0,
                           z_loss: float = 0.0, scale: float = 1.0, loss_out=None, logp_out=None, lse_out=None, grad_hidden_out=None,
                           grad_weight_out=None) -> None:
        where = "adasd_head_cross_entropy"
        first, sc, n, dim = self._head(where, hidden, weight, tokens, scratch)
        rw, rl, lp, lse = self._arrays(where, self._f32, n, (row_weight, row_loss_out, logp_out, lse_out))
        total, = self._arrays(where, self._f32, 1, (loss_out,))
        rc = self._head_cross_entropy(*first, rw, CrossEntropyOptions(label_smoothing, z_loss, scale), *sc, rl, total, lp, lse,
                                      *self._matrix(where, grad_hidden_out, n, dim), *self._matrix(where, grad_weight_out, self.V, dim),
                                      self._raw_stream(self._index))
        if rc:
            raise AdasdError(rc, where)

    # ---- AdamW -----------------------------------------------------------------------------------------

    def adamw_table(self, tensors) -> AdamwTable:
        """tensors: dicts of device tensors ``param``, ``grad``, ``exp_avg``, ``exp_avg_sq``, with states in 8 bits ``avg_scale`` and
        ``sq_scale``, and optionally ``param_copy`` (bf16) and the number ``weight_decay``.  States are float32, or float8_e4m3fn (exp_avg) and
        float8_e5m2 (exp_avg_sq).  Every tensor is contiguous; no two may overlap.  The table holds addresses: make it again when a
        tensor moves."""
        t, where = self.torch, "adasd_adamw_step"
        dtypes = {t.bfloat16: ADASD_BF16, t.float32: ADASD_FP32}
        array, ranges = (AdamwTensor * max(1, len(tensors)))(), []
        for e, d in zip(array, tensors):
            n, bits = d["param"].numel(), 32 if d["exp_avg"].dtype is t.float32 else 8
            want = [("param", dtypes, n), ("grad", dtypes, n), ("exp_avg", (t.float32 if bits == 32 else t.float8_e4m3fn,), n),
                    ("exp_avg_sq", (t.float32 if bits == 32 else t.float8_e5m2,), n)]
            if bits == 8:
                want += [(k, (t.float32,), -(-n // ADAMW_BLOCK)) for k in ("avg_scale", "sq_scale")]
            if d.get("param_copy") is not None:
                want.append(("param_copy", (t.bfloat16,), n))
            for name, types, size in want:
                a = d[name]
                if a.dtype not in types:
                    raise AdasdError(ERR_DTYPE, where)
                if a.get_device() != self._index:
                    raise AdasdError(ERR_DEVICE, where)
                if a.numel() != size or not a.is_contiguous():
                    raise AdasdError(ERR_SHAPE, where)
                setattr(e, name, a.data_ptr() if size else None)
                if size:
                    ranges.append((a.data_ptr(), a.data_ptr() + size * a.element_size()))
            e.n, e.weight_decay, e.state_bits = n, float(d.get("weight_decay", 0.0)), bits
            e.param_dtype, e.grad_dtype = dtypes[d["param"].dtype], dtypes[d["grad"].dtype]
        ranges.sort()
        if any(b[0] < a[1] for a, b in zip(ranges, ranges[1:])):
            raise AdasdError(ERR_SHAPE, where)
        table = AdamwTable(array, [dict(d) for d in tensors])
        table.n = len(tensors)
        return table

    def adamw_step(self, table: AdamwTable, lr, step, betas=(0.9, 0.999), eps: float = 1e-8, grad_scale=1.0, rounding: str = "nearest",
                   seed: int = 0, grad_scale_dev=None) -> None:
        """lr (float32) and step (int32) may be device tensors of one element, which are read when the step runs, as grad_scale_dev
        is; rounding: "nearest" or "stochastic"."""
        if rounding not in ("nearest", "stochastic"):
            raise AdasdError(ERR_DTYPE, "adasd_adamw_step")
        lr_dev = step_dev = scale_dev = None
        if hasattr(lr, "data_ptr"):
            (lr_dev,), lr = self._arrays("adasd_adamw_step", self._f32, 1, (lr,)), 0.0
        if hasattr(step, "data_ptr"):
            (step_dev,), step = self._arrays("adasd_adamw_step", self._i32, 1, (step,)), 1
        if grad_scale_dev is not None:
            scale_dev, = self._arrays("adasd_adamw_step", self._f32, 1, (grad_scale_dev,))
        rc = self._adamw_step(self.handle, table.entries, table.n,
                              AdamwOptions(lr, betas[0], betas[1], eps, grad_scale, step, rounding == "stochastic", seed, lr_dev,
                                           scale_dev, step_dev), self._raw_stream(self._index))
        if rc:
            raise AdasdError(rc, "adasd_adamw_step")

    def get_thresholds(self):
        """(T_G, nE, nA, nR) as new device tensors."""
        t = self.torch
        T = t.empty(self.B, dtype=t.float32, device=self.device)
        n = [t.empty(self.B, dtype=t.int32, device=self.device) for _ in range(3)]
        self._check(adasd_get_thresholds(self.handle, T.data_ptr(), n[0].data_ptr(), n[1].data_ptr(),
                                         n[2].data_ptr(), self._stream()), "adasd_get_thresholds")
        return T, n[0], n[1], n[2]

    def state_export(self, seq: int) -> dict:
        """Host copy of one sequence's state: dict(T_G, LE, LA, LR) with numpy arrays."""
        import numpy as np
        nbytes = C.c_size_t(0)
        self._check(adasd_state_export(self.handle, seq, None, C.byref(nbytes)), "adasd_state_export")
        buf = (C.c_char * nbytes.value)()
        self._check(adasd_state_export(self.handle, seq, buf, C.byref(nbytes)), "adasd_state_export")
        raw = bytes(buf)
        nE, nA, nR, _ = np.frombuffer(raw[:16], dtype=np.int32)
        T_G = float(np.frombuffer(raw[16:20], dtype=np.float32)[0])
        body = np.frombuffer(raw[24:], dtype=np.float32)
        return dict(T_G=T_G, LE=body[:nE].copy(), LA=body[nE:nE + nA].copy(),
                    LR=body[nE + nA:nE + nA + nR].copy())

    def state_import(self, seq: int, T_G: float, LE, LA, LR) -> None:
        import numpy as np
        LE, LA, LR = (np.ascontiguousarray(a, dtype=np.float32) for a in (LE, LA, LR))
        raw = (np.array([LE.size, LA.size, LR.size, 0], dtype=np.int32).tobytes() +
               np.array([T_G, 0.0], dtype=np.float32).tobytes() + LE.tobytes() + LA.tobytes() +
               LR.tobytes())
        self._check(adasd_state_import(self.handle, seq, raw, len(raw)), "adasd_state_import")

    def status(self) -> int:
        rc, bits = adasd_status(self.handle)
        self._check(rc, "adasd_status")
        return bits
