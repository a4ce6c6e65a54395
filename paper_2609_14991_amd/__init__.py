"""Python binding of the MI355X shallow-fusion library (libfusion.so).

Argument marshalling only: every step of the decode path runs in the HIP
kernels behind the C ABI declared in ``include/fusion.h``.  PyTorch supplies
device memory and the HIP stream.  The library must have been built
(``__graft_entry__.build()`` or ``python paper_2609_14991_amd/build.py``);
importing a function of this module without it raises an error, there is no
fallback.
"""

from __future__ import annotations

import atexit
import contextlib
import ctypes
import os
import sys
import weakref

import numpy as np

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libfusion.so")

FUSION_OK = 0
FUSION_E_ARG = -1
FUSION_E_NOMEM = -2
FUSION_E_HIP = -3
FUSION_E_LM_FORMAT = -4
FUSION_E_PHRASES = -5
FUSION_E_UNSUPPORTED = -6
FUSION_BLANK_AM = 0
FUSION_BLANK_COMPETE = 1
FUSION_STATUS_BAD_LM_STATE = 1
FUSION_STATUS_BAD_BOOST_STATE = 2
FUSION_STATUS_BAD_TOKEN = 8

FUSION_F32, FUSION_BF16, FUSION_F16 = 0, 1, 2

FUSION_MAX_LMS = 2
FUSION_RUN_RECOMBINE = 1

EXPORTS = ("ngram_load", "ngram_bos_state", "ngram_info", "ngram_free", "boost_build", "boost_info",
           "boost_free", "fusion_step", "fusion_run", "fusion_step_lms", "fusion_run_lms",
           "fusion_run_lms_noalloc", "fusion_run_projected",
           "fusion_end_scores", "joint_project", "token_logprobs", "token_logprobs_backward",
           "joint_logprobs_workspace", "joint_logprobs", "mx_quantize", "mx_dequantize", "joint_project_mx",
           "fusion_last_error", "fusion_device_status")


class FusionError(RuntimeError):
    def __init__(self, code, msg):
        super().__init__(f"fusion error {code}: {msg}")
        self.code = code


_lib = None


def lib():
    """The loaded libfusion.so (raises if it was never built)."""
    global _lib
    if _lib is None:
        if not os.path.exists(LIB_PATH):
            raise ImportError(f"{LIB_PATH} is missing: build it with __graft_entry__.build()")
        L = ctypes.CDLL(LIB_PATH)
        vp, i32, i64, f32, f64 = (ctypes.c_void_p, ctypes.c_int32, ctypes.c_int64, ctypes.c_float,
                                  ctypes.c_double)
        P = ctypes.POINTER
        L.ngram_load.restype = ctypes.c_int
        L.ngram_load.argtypes = [i32, i32, i32, P(i64), P(vp), P(vp), P(vp), vp, P(vp)]
        L.ngram_bos_state.restype = ctypes.c_int
        L.ngram_bos_state.argtypes = [vp, P(i32)]
        L.ngram_info.restype = ctypes.c_int
        L.ngram_info.argtypes = [vp, P(i64), P(i64)]
        L.ngram_free.restype = None
        L.ngram_free.argtypes = [vp]
        L.boost_build.restype = ctypes.c_int
        L.boost_build.argtypes = [i32, i32, i32, vp, vp, vp, f32, vp, P(vp)]
        L.boost_info.restype = ctypes.c_int
        L.boost_info.argtypes = [vp, P(i32), P(i32), P(i64)]
        L.boost_free.restype = None
        L.boost_free.argtypes = [vp]
        L.fusion_step.restype = ctypes.c_int
        L.fusion_step.argtypes = [vp, vp, vp, vp, vp, i32, i32, f32, f32, i32, i32, i32, vp, vp, vp,
                                  vp, vp, vp]
        L.fusion_run.restype = ctypes.c_int
        L.fusion_run.argtypes = [vp, vp, vp, i32, i32, i32, i32, i32, f32, f32, i32, i32, vp, vp, vp,
                                 vp, vp, vp, vp, vp]
        L.fusion_step_lms.restype = ctypes.c_int
        L.fusion_step_lms.argtypes = [vp, vp, i32, vp, vp, vp, vp, i32, i32, f32, i32, i32, i32, vp,
                                      vp, vp, vp, vp, vp]
        L.fusion_run_lms.restype = ctypes.c_int
        L.fusion_run_lms.argtypes = [vp, vp, i32, vp, vp, i32, i32, i32, i32, i32, f32, i32, i32, vp,
                                     vp, vp, vp, vp, vp, vp, i32, vp, vp]
        L.fusion_run_lms_noalloc.restype = ctypes.c_int
        L.fusion_run_lms_noalloc.argtypes = L.fusion_run_lms.argtypes
        L.fusion_run_projected.restype = ctypes.c_int
        L.fusion_run_projected.argtypes = [vp, vp, i32, vp, vp, vp, vp, i32, vp, i32, i32, i32, i32, i32, i32, f32, i32,
                                           i32, vp, vp, vp, vp, vp, i32, vp, vp]
        L.fusion_end_scores.restype = ctypes.c_int
        L.fusion_end_scores.argtypes = [vp, vp, i32, vp, i32, vp, vp, vp]
        L.joint_project.restype = ctypes.c_int
        L.joint_project.argtypes = [vp, vp, vp, i32, i32, i32, vp, vp]
        L.token_logprobs.restype = ctypes.c_int
        L.token_logprobs.argtypes = [vp, i32, i64, i32, i32, i32, i32, vp, vp, i32, vp, vp, vp, vp, vp, vp]
        L.token_logprobs_backward.restype = ctypes.c_int
        L.token_logprobs_backward.argtypes = [vp, i32, i64, i32, i32, i32, i32, vp, vp, vp, vp, vp, vp, vp, vp, i64, vp]
        L.joint_logprobs_workspace.restype = ctypes.c_int
        L.joint_logprobs_workspace.argtypes = [i32, i32, i32, P(i64)]
        L.joint_logprobs.restype = ctypes.c_int
        L.joint_logprobs.argtypes = [vp, vp, vp, i32, i32, i32, i32, i32, vp, vp, vp, vp, vp, vp, i64, vp]
        L.mx_quantize.restype = ctypes.c_int
        L.mx_quantize.argtypes = [vp, i32, i64, i32, i32, vp, vp, vp]
        L.mx_dequantize.restype = ctypes.c_int
        L.mx_dequantize.argtypes = [vp, vp, i32, i32, vp, i32, i64, vp]
        L.joint_project_mx.restype = ctypes.c_int
        L.joint_project_mx.argtypes = [vp, vp, vp, vp, vp, i32, i32, i32, vp, vp]
        L.fusion_last_error.restype = ctypes.c_char_p
        L.fusion_last_error.argtypes = []
        L.fusion_device_status.restype = ctypes.c_int
        L.fusion_device_status.argtypes = [vp, P(i32)]
        _lib = L
    return _lib


def fusion_last_error() -> str:
    return lib().fusion_last_error().decode()


def _check(rc):
    if rc != FUSION_OK:
        raise FusionError(rc, fusion_last_error())


def _stream(stream):
    if stream is not None:
        return ctypes.c_void_p(int(stream))
    import torch

    # the current stream's address alone: torch.cuda.current_stream() builds a Stream object
    # for it, a third of the host time of a one-hypothesis step (3.0 us; 0.4 so)
    return ctypes.c_void_p(torch._C._cuda_getCurrentRawStream(torch.cuda.current_device()))


def _ptr(t):
    """Device (or host numpy) pointer of a buffer, None for None."""
    if t is None:
        return None
    if isinstance(t, np.ndarray):
        return ctypes.c_void_p(t.ctypes.data)
    return ctypes.c_void_p(t.data_ptr())


# Device handles still alive when the interpreter begins to shut down are
# released by an atexit hook, while the HIP runtime is certainly still up;
# a handle's __del__ never calls into the library once shutdown has begun
_live = weakref.WeakSet()


def _release_all():
    for h in list(_live):
        h.close()


atexit.register(_release_all)


class _Handle:
    _free_fn = None

    def __init__(self, handle):
        self.h = ctypes.c_void_p(handle)
        _live.add(self)

    def close(self):
        """Release the device memory now (idempotent)."""
        if getattr(self, "h", None) is not None and self.h.value:
            getattr(lib(), self._free_fn)(self.h)
        self.h = None

    def __del__(self, _finalizing=sys.is_finalizing):
        if _finalizing():
            return
        try:
            self.close()
        except Exception:
            pass


class NgramTables(_Handle):
    """Owning handle of device-resident n-gram tables."""

    _free_fn = "ngram_free"

    def __init__(self, handle, order, vocab, blank):
        super().__init__(handle)
        self.order, self.vocab, self.blank = order, vocab, blank


class BoostTrie(_Handle):
    """Owning handle of a device-resident phrase-boosting tree."""

    _free_fn = "boost_free"

    def __init__(self, handle, vocab, blank):
        super().__init__(handle)
        self.vocab, self.blank = vocab, blank


def ngram_load(order, vocab, blank_id, tokens, logp, backoff=None, stream=None) -> NgramTables:
    """tokens/logp/backoff: per-order host arrays (see include/fusion.h)."""
    L = lib()
    order = int(order)
    toks = [np.ascontiguousarray(t, dtype=np.int32) for t in tokens]
    lps = [np.ascontiguousarray(p, dtype=np.float32) for p in logp]
    bos = [None if (backoff is None or b is None) else np.ascontiguousarray(b, dtype=np.float32)
           for b in (backoff if backoff is not None else [None] * order)]
    count = np.array([t.shape[0] for t in toks], dtype=np.int64)
    VP = ctypes.c_void_p * order
    tp = VP(*[t.ctypes.data for t in toks])
    lp = VP(*[p.ctypes.data for p in lps])
    bp = VP(*[None if b is None else b.ctypes.data for b in bos])
    out = ctypes.c_void_p()
    _check(L.ngram_load(order, int(vocab), int(blank_id),
                        count.ctypes.data_as(ctypes.POINTER(ctypes.c_int64)), tp, lp, bp,
                        _stream(stream), ctypes.byref(out)))
    return NgramTables(out.value, order, int(vocab), int(blank_id))


def ngram_load_arrays(lm, stream=None) -> NgramTables:
    """ngram_load from an object with order/vocab/blank/tokens/logp/backoff."""
    return ngram_load(lm.order, lm.vocab, lm.blank, lm.tokens, lm.logp, lm.backoff, stream)


def ngram_bos_state(lm: NgramTables) -> int:
    v = ctypes.c_int32()
    _check(lib().ngram_bos_state(lm.h, ctypes.byref(v)))
    return v.value


def ngram_info(lm: NgramTables):
    n, b = ctypes.c_int64(), ctypes.c_int64()
    _check(lib().ngram_info(lm.h, ctypes.byref(n), ctypes.byref(b)))
    return n.value, b.value


def boost_build(vocab, blank_id, tokens, offsets, completion=None, token_score=1.0,
                stream=None) -> BoostTrie:
    toks = np.ascontiguousarray(tokens, dtype=np.int32)
    offs = np.ascontiguousarray(offsets, dtype=np.int64)
    comp = None if completion is None else np.ascontiguousarray(completion, dtype=np.float32)
    out = ctypes.c_void_p()
    _check(lib().boost_build(int(vocab), int(blank_id), int(offs.size - 1), _ptr(toks), _ptr(offs),
                             _ptr(comp), float(token_score), _stream(stream), ctypes.byref(out)))
    return BoostTrie(out.value, int(vocab), int(blank_id))


def boost_build_phrases(vocab, blank_id, phrases, stream=None) -> BoostTrie:
    return boost_build(vocab, blank_id, phrases.tokens, phrases.offsets, phrases.completion,
                       phrases.token_score, stream)


def boost_info(trie: BoostTrie):
    n, d, b = ctypes.c_int32(), ctypes.c_int32(), ctypes.c_int64()
    _check(lib().boost_info(trie.h, ctypes.byref(n), ctypes.byref(d), ctypes.byref(b)))
    return n.value, d.value, b.value


def _h(x):
    return None if x is None else x.h


def fusion_step(lm, trie, logits, lm_state, boost_state, H, V, lam, beta, blank_id, k, blank_mode,
                fused, tokens, scores, next_lm, next_boost, stream=None):
    """Same arguments as the C call; tensors are CUDA (HIP) tensors."""
    _check(lib().fusion_step(_h(lm), _h(trie), _ptr(logits), _ptr(lm_state), _ptr(boost_state),
                             int(H), int(V), float(lam), float(beta), int(blank_id), int(k),
                             int(blank_mode), _ptr(fused), _ptr(tokens), _ptr(scores),
                             _ptr(next_lm), _ptr(next_boost), _stream(stream)))


def fusion_run(lm, trie, logits, T, S, B, V, k, lam, beta, blank_id, blank_mode, lm_state,
               boost_state, hyp_score, tokens, parents, fused=None, traffic=None, stream=None):
    """Same arguments as the C call; tensors are CUDA (HIP) tensors."""
    _check(lib().fusion_run(_h(lm), _h(trie), _ptr(logits), int(T), int(S), int(B), int(V), int(k),
                            float(lam), float(beta), int(blank_id), int(blank_mode), _ptr(lm_state),
                            _ptr(boost_state), _ptr(hyp_score), _ptr(tokens), _ptr(parents),
                            _ptr(fused), _ptr(traffic), _stream(stream)))


def _lm_arrays(lms, alphas):
    """Host arrays of handles and weights for the several-LM calls."""
    lms, alphas = list(lms), [float(a) for a in alphas]
    if len(lms) != len(alphas):
        raise ValueError("one weight per LM")
    hs = (ctypes.c_void_p * max(1, len(lms)))(*[m.h.value for m in lms])
    al = np.array(alphas if alphas else [0.0], dtype=np.float32)
    return hs, al, len(lms)


def fusion_step_lms(lms, alphas, trie, logits, lm_state, boost_state, H, V, beta, blank_id, k,
                    blank_mode, fused, tokens, scores, next_lm, next_boost, stream=None):
    """Same arguments as the C call; lms and alphas are Python sequences,
    tensors are CUDA (HIP) tensors (lm_state [n_lm, H], next_lm [n_lm, H, k])."""
    hs, al, n = _lm_arrays(lms, alphas)
    _check(lib().fusion_step_lms(ctypes.cast(hs, ctypes.c_void_p), _ptr(al), n, _h(trie), _ptr(logits),
                                 _ptr(lm_state), _ptr(boost_state), int(H), int(V), float(beta),
                                 int(blank_id), int(k), int(blank_mode), _ptr(fused), _ptr(tokens),
                                 _ptr(scores), _ptr(next_lm), _ptr(next_boost), _stream(stream)))


def fusion_run_lms(lms, alphas, trie, logits, T, S, B, V, k, beta, blank_id, blank_mode, lm_state,
                   boost_state, hyp_score, tokens, parents, fused=None, traffic=None, flags=0, hist=None,
                   stream=None):
    """Same arguments as the C call; lms and alphas are Python sequences,
    tensors are CUDA (HIP) tensors (lm_state [n_lm, S*B], hist [S*B] int64)."""
    hs, al, n = _lm_arrays(lms, alphas)
    _check(lib().fusion_run_lms(ctypes.cast(hs, ctypes.c_void_p), _ptr(al), n, _h(trie), _ptr(logits),
                                int(T), int(S), int(B), int(V), int(k), float(beta), int(blank_id),
                                int(blank_mode), _ptr(lm_state), _ptr(boost_state), _ptr(hyp_score),
                                _ptr(tokens), _ptr(parents), _ptr(fused), _ptr(traffic), int(flags),
                                _ptr(hist), _stream(stream)))


def fusion_run_lms_noalloc(lms, alphas, trie, logits, T, S, B, V, k, beta, blank_id, blank_mode, lm_state,
                           boost_state, hyp_score, tokens, parents, fused=None, traffic=None, flags=0, hist=None,
                           stream=None):
    """fusion_run_lms through the entry point that allocates no device memory
    (its beam exchange lives in the library's static per-GPU scratch)."""
    hs, al, n = _lm_arrays(lms, alphas)
    _check(lib().fusion_run_lms_noalloc(ctypes.cast(hs, ctypes.c_void_p), _ptr(al), n, _h(trie), _ptr(logits),
                                        int(T), int(S), int(B), int(V), int(k), float(beta), int(blank_id),
                                        int(blank_mode), _ptr(lm_state), _ptr(boost_state), _ptr(hyp_score),
                                        _ptr(tokens), _ptr(parents), _ptr(fused), _ptr(traffic), int(flags),
                                        _ptr(hist), _stream(stream)))


def fusion_run_projected(lms, alphas, trie, A, W, bias, K, logits, chunk, T, S, B, V, k, beta, blank_id, blank_mode,
                         lm_state, boost_state, hyp_score, tokens, parents, flags=0, hist=None, stream=None):
    """Same arguments as the C call: A [T, S*B, K] and W [V, K] bf16 (int16 bit
    patterns), logits a [chunk, S*B, V] float32 workspace; CUDA (HIP) tensors."""
    hs, al, n = _lm_arrays(lms, alphas)
    _check(lib().fusion_run_projected(ctypes.cast(hs, ctypes.c_void_p), _ptr(al), n, _h(trie), _ptr(A), _ptr(W),
                                      _ptr(bias), int(K), _ptr(logits), int(chunk), int(T), int(S), int(B), int(V), int(k),
                                      float(beta), int(blank_id), int(blank_mode), _ptr(lm_state), _ptr(boost_state),
                                      _ptr(hyp_score), _ptr(tokens), _ptr(parents), int(flags), _ptr(hist),
                                      _stream(stream)))


def fusion_end_scores(lms, alphas, lm_state, H, hyp_score=None, end_term=None, stream=None):
    """Same arguments as the C call; lm_state [n_lm, H] int32, hyp_score / end_term
    [H] float64 CUDA tensors (either may be None, not both)."""
    hs, al, n = _lm_arrays(lms, alphas)
    _check(lib().fusion_end_scores(ctypes.cast(hs, ctypes.c_void_p), _ptr(al), n, _ptr(lm_state), int(H),
                                   _ptr(hyp_score), _ptr(end_term), _stream(stream)))


def joint_project(A, W, bias, M, N, K, out, stream=None):
    """Same arguments as the C call; A and W are int16/uint16 (bf16 bit patterns) or
    bfloat16 CUDA tensors, bias and out float32 CUDA tensors."""
    _check(lib().joint_project(_ptr(A), _ptr(W), _ptr(bias), int(M), int(N), int(K), _ptr(out),
                               _stream(stream)))


_DTYPES = None


def _dtype(t) -> int:
    """FUSION_F32 / FUSION_BF16 / FUSION_F16 of a tensor (anything else: -1, which the library refuses)."""
    global _DTYPES
    if _DTYPES is None:
        import torch

        _DTYPES = {torch.float32: FUSION_F32, torch.bfloat16: FUSION_BF16, torch.float16: FUSION_F16}
    return _DTYPES.get(t.dtype, -1)


def _at(t):
    """A tensor's device address as a plain int (ctypes turns it into the pointer), None for None."""
    return None if t is None else t.data_ptr()


_current = None


def _on(stream):
    """``_stream`` as a plain int, torch's functions looked up once."""
    global _current
    if stream is not None:
        return int(stream)
    if _current is None:
        import torch

        _current = torch._C._cuda_getCurrentRawStream, torch.cuda.current_device
    return _current[0](_current[1]())


_unchanged = contextlib.nullcontext()


def _made_for(stream):
    """Tensors made inside are made on ``stream`` (an address; None: the current stream): their memory goes from one
    use on that stream to the next one there, and not to the current stream's work while ``stream`` still uses it."""
    if stream is None:
        return _unchanged
    import torch

    return torch.cuda.stream(torch.cuda.ExternalStream(int(stream)))


def token_logprobs(logits, stride, T, S, B, V, tokens, parents, k, logp, entropy, lse, top_tokens=None, top_logp=None,
                   stream=None):
    """Same arguments as the C call, the dtype taken from logits; CUDA (HIP) tensors, float32 outputs."""
    _check(lib().token_logprobs(_at(logits), _dtype(logits), int(stride), int(T), int(S), int(B), int(V), _at(tokens),
                                _at(parents), int(k), _at(logp), _at(entropy), _at(lse), _at(top_tokens),
                                _at(top_logp), _on(stream)))


def token_logprobs_backward(logits, stride, T, S, B, V, tokens, parents, logp, entropy, lse, grad_logp, grad_entropy,
                            grad_logits, grad_stride, stream=None):
    """Same arguments as the C call, the dtype taken from logits (grad_logits has the same); CUDA (HIP) tensors."""
    if grad_logits.dtype != logits.dtype:
        raise ValueError("grad_logits must have the type of logits")
    _check(lib().token_logprobs_backward(_at(logits), _dtype(logits), int(stride), int(T), int(S), int(B), int(V),
                                         _at(tokens), _at(parents), _at(logp), _at(entropy), _at(lse),
                                         _at(grad_logp), _at(grad_entropy), _at(grad_logits), int(grad_stride),
                                         _on(stream)))


def joint_logprobs_workspace(M, V, K) -> int:
    """float32 elements that joint_logprobs needs as its workspace for M = T * S * B rows."""
    v = ctypes.c_int64()
    _check(lib().joint_logprobs_workspace(int(M), int(V), int(K), ctypes.byref(v)))
    return v.value


def joint_logprobs(A, W, bias, K, T, S, B, V, tokens, parents, logp, entropy, lse, workspace, stream=None):
    """Same arguments as the C call (the workspace's size is its tensor's, float32 or any other type in order); A and W
    bfloat16 (or int16 bit patterns)."""
    _check(lib().joint_logprobs(_at(A), _at(W), _at(bias), int(K), int(T), int(S), int(B), int(V), _at(tokens),
                                _at(parents), _at(logp), _at(entropy), _at(lse), _at(workspace),
                                workspace.numel() * workspace.element_size() // 4, _on(stream)))


def mx_scale_stride(K) -> int:
    """Scale bytes of a row of K values (FUSION_MX_SCALE_STRIDE)."""
    return (int(K) // 32 + 7) // 8 * 8


def mx_quantize(x, stride, R, K, q, scales, stream=None):
    """Same arguments as the C call, the dtype taken from x; q [R, K // 2] and scales [R, mx_scale_stride(K)] uint8."""
    _check(lib().mx_quantize(_at(x), _dtype(x), int(stride), int(R), int(K), _at(q), _at(scales), _on(stream)))


def mx_dequantize(q, scales, R, K, out, stride, stream=None):
    """Same arguments as the C call, the dtype taken from out."""
    _check(lib().mx_dequantize(_at(q), _at(scales), int(R), int(K), _at(out), _dtype(out), int(stride),
                               _on(stream)))


def joint_project_mx(A, A_scales, W, W_scales, bias, M, N, K, out, stream=None):
    """Same arguments as the C call; operands as mx_quantize writes them, bias and out float32 CUDA tensors."""
    _check(lib().joint_project_mx(_at(A), _at(A_scales), _at(W), _at(W_scales), _at(bias), int(M), int(N), int(K),
                                  _at(out), _on(stream)))


def fusion_device_status(stream=None) -> int:
    v = ctypes.c_int32()
    _check(lib().fusion_device_status(_stream(stream), ctypes.byref(v)))
    return v.value


# ---------------------------------------------------------------------------
# conveniences that allocate the outputs with torch (still no compute here)
#
# ``stream`` is the address of the stream to work on.  What they return was made on it, as a tensor of
# ``with torch.cuda.stream(...)``: another stream that uses it waits for this one and calls record_stream.
# ---------------------------------------------------------------------------
def step(lm, trie, logits, lm_state, boost_state, lam, beta, blank_id, k, blank_mode,
         want_fused=False, stream=None):
    import torch

    H, V = logits.shape
    dev = logits.device
    with _made_for(stream):
        out = dict(
            tokens=torch.empty((H, k), dtype=torch.int32, device=dev),
            scores=torch.empty((H, k), dtype=torch.float32, device=dev),
            next_lm=torch.empty((H, k), dtype=torch.int32, device=dev),
            next_boost=torch.empty((H, k), dtype=torch.int32, device=dev),
            fused=torch.empty((H, V), dtype=torch.float32, device=dev) if want_fused else None,
        )
    fusion_step(lm, trie, logits, lm_state, boost_state, H, V, lam, beta, blank_id, k, blank_mode,
                out["fused"], out["tokens"], out["scores"], out["next_lm"], out["next_boost"], stream)
    return out


def project(A, W, bias=None, stream=None):
    """logits [M, N] fp32 of A [M, K] and W [N, K] (bf16 CUDA tensors)."""
    import torch

    M, K = A.shape
    N = W.shape[0]
    with _made_for(stream):
        out = torch.empty((M, N), dtype=torch.float32, device=A.device)
    joint_project(A, W, bias, M, N, K, out, stream)
    return out


def _here(t) -> bool:
    """Whether a tensor is on the current device, where a call's kernels run."""
    import torch

    return t.is_cuda and t.get_device() == torch.cuda.current_device()


def _want(t, what, dtype, shape):
    """A tensor on the current device of this type and shape (None in a shape: any size), its elements in order."""
    if not _here(t) or t.dtype != dtype or not t.is_contiguous() or len(t.shape) != len(shape) or any(
            n is not None and n != m for n, m in zip(shape, t.shape)):
        raise ValueError(f"{what}: a contiguous tensor of {dtype} on the current CUDA device, shape {list(shape)}, is wanted")
    return t


def _rows(logits, what="logits"):
    """T, H, V and the distance of the rows of logits [T, H, V], which may lie apart."""
    if not _here(logits) or logits.dim() != 3 or _dtype(logits) < 0:
        raise ValueError(f"{what}: a tensor [T, S * B, V] of float32, bfloat16 or float16 on the current CUDA device is wanted")
    T, H, V = logits.shape
    # (a dimension of one row says nothing about their distance)
    stride = logits.stride(1) if H > 1 else logits.stride(0) if T > 1 else V
    if logits.numel() and ((V > 1 and logits.stride(2) != 1) or stride < V or (T > 1 and logits.stride(0) != H * stride)):
        raise ValueError(f"{what}: rows one distance apart, each in order, are wanted")
    return T, H, V, stride


def _slots(H, B):
    """S of S * B slots a frame."""
    if B < 1 or H % B != 0:
        raise ValueError("S * B rows a frame are wanted")
    return H // B


def score(logits, tokens=None, parents=None, B=1, k=0, stream=None):
    """Log probabilities [T, S * B] of the tokens that a decode (``run``) chose from logits [T, S * B, V],
    the entropies and log sum exps of the rows they were chosen on, and the k best alternatives
    ``top`` and ``top_logp`` [T, S * B, k].  Without tokens the rows alone.  Nothing is recorded for
    autograd, whether logits require a gradient or not: ``score_backward`` gives it."""
    import torch

    T, H, V, stride = _rows(logits)
    S = _slots(H, B)
    for t, what in ((tokens, "tokens"), (parents, "parents")):
        if t is not None:
            _want(t, what, torch.int32, (T, H))
    new = lambda dt, *n: torch.empty((T, H) + n, dtype=dt, device=logits.device)  # noqa: E731
    with _made_for(stream):
        out = dict(logp=None if tokens is None else new(torch.float32), entropy=new(torch.float32), lse=new(torch.float32),
                   top=new(torch.int32, k) if k else None, top_logp=new(torch.float32, k) if k else None)
    token_logprobs(logits, stride, T, S, B, V, tokens, parents, k, out["logp"], out["entropy"], out["lse"], out["top"],
                   out["top_logp"], stream)
    return out


def score_backward(logits, scored, tokens=None, parents=None, B=1, grad_logp=None, grad_entropy=None, in_place=False,
                   stream=None):
    """The gradient with respect to logits of what ``score`` gave (``scored``) for the same arguments, of the
    logits' type; ``in_place`` writes it over them (an autograd graph that saved them then refuses its backward
    pass, as after any operation in place)."""
    import torch

    T, H, V, stride = _rows(logits)
    S = _slots(H, B)
    for t, what, dt in ((tokens, "tokens", torch.int32), (parents, "parents", torch.int32), (grad_logp, "grad_logp", torch.float32),
                        (grad_entropy, "grad_entropy", torch.float32)):
        if t is not None:
            _want(t, what, dt, (T, H))
    for n in ("logp", "entropy", "lse"):
        if scored[n] is not None:
            _want(scored[n], n, torch.float32, (T, H))
    with _made_for(stream):
        grad = logits if in_place else torch.empty((T, H, V), dtype=logits.dtype, device=logits.device)
    token_logprobs_backward(logits, stride, T, S, B, V, tokens, parents, scored["logp"], scored["entropy"], scored["lse"],
                            grad_logp, grad_entropy, grad, stride if in_place else V, stream)
    if in_place and not logits.is_inference():
        torch.autograd.graph.increment_version(logits)
    return grad


def score_projected(A, W, bias=None, tokens=None, parents=None, B=1, stream=None):
    """``score`` (without alternatives) straight from the hidden states A [T, S * B, K] and the output layer
    W [V, K] (bf16) and bias: the logits are never stored."""
    import torch

    T, H, K = A.shape
    V = W.shape[0]
    _want(A, "A", torch.bfloat16, (None, None, K))
    _want(W, "W", torch.bfloat16, (None, K))
    if bias is not None:
        _want(bias, "bias", torch.float32, (V,))
    S = _slots(H, B)
    for t, what in ((tokens, "tokens"), (parents, "parents")):
        if t is not None:
            _want(t, what, torch.int32, (T, H))
    new = lambda: torch.empty((T, H), dtype=torch.float32, device=A.device)  # noqa: E731
    with _made_for(stream):
        out = dict(logp=None if tokens is None else new(), entropy=new(), lse=new())
        work = torch.empty(joint_logprobs_workspace(T * H, V, K), dtype=torch.float32, device=A.device)
    joint_logprobs(A, W, bias, K, T, S, B, V, tokens, parents, out["logp"], out["entropy"], out["lse"], work, stream)
    return out


def quantize(x, stream=None):
    """x [R, K] (float32, bfloat16 or float16; rows may lie apart) in microscaled 4-bit floating point: the
    packed elements [R, K // 2] and scale bytes [R, mx_scale_stride(K)], both uint8."""
    import torch

    if x.dim() != 2:
        raise ValueError("x: rows [R, K] are wanted")
    _, R, K, stride = _rows(x.unsqueeze(0), "x")
    with _made_for(stream):
        q = torch.empty((R, K // 2), dtype=torch.uint8, device=x.device)
        s = torch.empty((R, mx_scale_stride(K)), dtype=torch.uint8, device=x.device)
    mx_quantize(x, stride, R, K, q, s, stream)
    return q, s


def dequantize(q, scales, dtype=None, stream=None):
    """The values [R, K] that ``quantize``'s result stands for, float32 or another type."""
    import torch

    R, K = q.shape[0], 2 * q.shape[1]
    _want(q, "q", torch.uint8, (R, K // 2))
    _want(scales, "scales", torch.uint8, (R, mx_scale_stride(K)))
    with _made_for(stream):
        out = torch.empty((R, K), dtype=torch.float32 if dtype is None else dtype, device=q.device)
    mx_dequantize(q, scales, R, K, out, K, stream)
    return out


def project_mx(A, W, bias=None, stream=None):
    """``project`` with both operands as ``quantize`` gives them; A may also be the states [M, K] themselves,
    which are then quantised first."""
    import torch

    (qw, sw), (qa, sa) = W, A if isinstance(A, tuple) else quantize(A, stream)
    M, N, K = qa.shape[0], qw.shape[0], 2 * qw.shape[1]
    for t, what, shape in ((qa, "A", (M, K // 2)), (sa, "A's scales", (M, mx_scale_stride(K))), (qw, "W", (N, K // 2)),
                           (sw, "W's scales", (N, mx_scale_stride(K)))):
        _want(t, what, torch.uint8, shape)
    if bias is not None:
        _want(bias, "bias", torch.float32, (N,))
    with _made_for(stream):
        out = torch.empty((M, N), dtype=torch.float32, device=qa.device)
    joint_project_mx(qa, sa, qw, sw, bias, M, N, K, out, stream)
    return out


def run(lm, trie, logits, S, B, k, lam, beta, blank_id, blank_mode, lm_state, boost_state,
        hyp_score=None, want_fused=False, traffic=None, stream=None):
    """Decode all frames of logits [T, S*B, V]; lm_state / boost_state /
    hyp_score are updated in place (they are the carried decoder state)."""
    import torch

    T, H, V = logits.shape
    dev = logits.device
    with _made_for(stream):
        tokens = torch.empty((T, H), dtype=torch.int32, device=dev)
        parents = torch.empty((T, H), dtype=torch.int32, device=dev) if B > 1 else None
        fused = torch.zeros((T, H, V), dtype=torch.float32, device=dev) if want_fused else None
    fusion_run(lm, trie, logits, T, S, B, V, k, lam, beta, blank_id, blank_mode, lm_state,
               boost_state, hyp_score, tokens, parents, fused, traffic, stream)
    return dict(tokens=tokens, parents=parents, fused=fused)


def step_lms(lms, alphas, trie, logits, lm_state, boost_state, beta, blank_id, k, blank_mode,
             want_fused=False, stream=None):
    """``step`` with several LMs: lm_state [n_lm, H]; next_lm comes back [n_lm, H, k]."""
    import torch

    H, V = logits.shape
    dev = logits.device
    n = len(lms)
    with _made_for(stream):
        out = dict(
            tokens=torch.empty((H, k), dtype=torch.int32, device=dev),
            scores=torch.empty((H, k), dtype=torch.float32, device=dev),
            next_lm=torch.empty((n, H, k), dtype=torch.int32, device=dev),
            next_boost=torch.empty((H, k), dtype=torch.int32, device=dev),
            fused=torch.empty((H, V), dtype=torch.float32, device=dev) if want_fused else None,
        )
    fusion_step_lms(lms, alphas, trie, logits, lm_state, boost_state, H, V, beta, blank_id, k,
                    blank_mode, out["fused"], out["tokens"], out["scores"], out["next_lm"],
                    out["next_boost"], stream)
    return out


def run_lms(lms, alphas, trie, logits, S, B, k, beta, blank_id, blank_mode, lm_state, boost_state,
            hyp_score=None, want_fused=False, traffic=None, recombine=False, hist=None, stream=None):
    """``run`` with several LMs: lm_state [n_lm, S*B] is updated in place;
    ``recombine`` merges beam candidates that reach the same history (``hist``,
    an int64 [S*B] tensor or None, carries the history hashes across calls)."""
    import torch

    T, H, V = logits.shape
    dev = logits.device
    with _made_for(stream):
        tokens = torch.empty((T, H), dtype=torch.int32, device=dev)
        parents = torch.empty((T, H), dtype=torch.int32, device=dev) if B > 1 else None
        fused = torch.zeros((T, H, V), dtype=torch.float32, device=dev) if want_fused else None
    fusion_run_lms(lms, alphas, trie, logits, T, S, B, V, k, beta, blank_id, blank_mode, lm_state,
                   boost_state, hyp_score, tokens, parents, fused, traffic,
                   FUSION_RUN_RECOMBINE if recombine else 0, hist, stream)
    return dict(tokens=tokens, parents=parents, fused=fused)
