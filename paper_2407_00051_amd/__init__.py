"""Python binding of libsagips.so, the MI355X (gfx950) implementation of one
rank's SAGIPS sample -> discriminate -> backward step (arXiv 2407.00051).

The binding only marshals arguments: every step runs in the library's HIP
kernels.  PyTorch supplies device memory and the stream (the context runs on
torch's current stream of its device unless another is set).  There is no
CPU fallback: if the library is missing or fails to load, importing the
calls raises.
"""
from __future__ import annotations

import ctypes
import os
from typing import Dict, List, Optional, Sequence

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libsagips.so")
MAX_LAYERS = 8
MAX_TENSORS = 16
MAX_TOP = 32
_INT32 = (1 << 31) - 1   # the ABI's 32-bit fields take what is beyond modulo 2^32
_W_NAMES = [f"W[{l}]" for l in range(MAX_LAYERS)]
_B_NAMES = [f"b[{l}]" for l in range(MAX_LAYERS)]

OK, E_INVAL, E_ARCH, E_NOMEM, E_HIP, E_UNSUPPORTED = 0, -1, -2, -3, -4, -5
F32, BF16 = 0, 1
FEAT_IDENTITY, FEAT_HD8, FEAT_PROXY2 = 0, 1, 2
CRITIC_BUFFER, CRITIC_QUADRATIC = 0, 1
MEAN_EVENTS, MEAN_ROWS = 0, 1
SCALE_NONE, SCALE_SHAPE, SCALE_RMS = 0, 1, 2
NS_COEF = (3.4445, -4.7750, 2.0315)

EXPORTED = ("sagips_create", "sagips_destroy", "sagips_set_stream", "sagips_set_bf16_chunk_rows",
            "sagips_last_error", "sagips_set_timing",
            "sagips_kernel_times", "sagips_sample_events", "sagips_disc_fwd_bwd", "sagips_param_grad",
            "sagips_bootstrap", "sagips_bootstrap_rows", "sagips_gen_forward", "sagips_gen_backward", "sagips_ensemble_response",
            "sagips_adam_step", "sagips_disc_fwd_bwd_noalloc", "sagips_noalloc_scratch_bytes",
            "sagips_group_advantage", "sagips_policy_loss", "sagips_preference_loss", "sagips_orthogonalise",
            "sagips_muon_step",
            "sagips_choice_logprob", "sagips_choice_backward", "sagips_route", "sagips_dispatch", "sagips_combine",
            "sagips_combine_backward", "sagips_gen_forward_routed", "sagips_gen_backward_routed")


class SagipsError(RuntimeError):
    def __init__(self, status: int, message: str):
        super().__init__(f"sagips status {status}: {message}")
        self.status = status


class Source(ctypes.Structure):
    _fields_ = [("theta", ctypes.c_void_p), ("n_theta", ctypes.c_int32), ("d", ctypes.c_int32),
                ("events_per_theta", ctypes.c_int64), ("seed", ctypes.c_uint64),
                ("counter_base", ctypes.c_uint64), ("stream", ctypes.c_uint32)]


class Mlp(ctypes.Structure):
    _fields_ = [("n_layers", ctypes.c_int32), ("width", ctypes.c_int32 * (MAX_LAYERS + 1)),
                ("W", ctypes.c_void_p * MAX_LAYERS), ("b", ctypes.c_void_p * MAX_LAYERS),
                ("leaky_slope", ctypes.c_float), ("precision", ctypes.c_int32), ("features", ctypes.c_int32)]


class GenStack(ctypes.Structure):
    _fields_ = [("n_layers", ctypes.c_int32), ("width", ctypes.c_int32 * (MAX_LAYERS + 1)),
                ("W", ctypes.c_void_p * MAX_LAYERS), ("b", ctypes.c_void_p * MAX_LAYERS),
                ("n_members", ctypes.c_int32), ("leaky_slope", ctypes.c_float)]


class ParamSet(ctypes.Structure):
    _fields_ = [("n_tensors", ctypes.c_int32), ("param", ctypes.c_void_p * MAX_TENSORS),
                ("grad", ctypes.c_void_p * MAX_TENSORS), ("m", ctypes.c_void_p * MAX_TENSORS),
                ("v", ctypes.c_void_p * MAX_TENSORS), ("size", ctypes.c_int64 * MAX_TENSORS)]


class Policy(ctypes.Structure):
    _fields_ = [("theta", ctypes.c_void_p), ("theta_old", ctypes.c_void_p), ("theta_ref", ctypes.c_void_p),
                ("n_theta", ctypes.c_int32), ("d", ctypes.c_int32), ("events_per_theta", ctypes.c_int64),
                ("clip_low", ctypes.c_double), ("clip_high", ctypes.c_double), ("kl_coef", ctypes.c_double),
                ("average", ctypes.c_int32)]


class Preference(ctypes.Structure):
    _fields_ = [("theta", ctypes.c_void_p), ("theta_ref", ctypes.c_void_p), ("n_theta", ctypes.c_int32),
                ("d", ctypes.c_int32), ("pairs_per_theta", ctypes.c_int64), ("len_chosen", ctypes.c_int64),
                ("len_rejected", ctypes.c_int64), ("beta", ctypes.c_double), ("label_smoothing", ctypes.c_double)]


class NewtonSchulz(ctypes.Structure):
    _fields_ = [("steps", ctypes.c_int32), ("coef", ctypes.c_double * 3), ("eps", ctypes.c_double)]


class MatrixSet(ctypes.Structure):
    _fields_ = [("n_tensors", ctypes.c_int32), ("grad_type", ctypes.c_int32), ("param", ctypes.c_void_p * MAX_TENSORS),
                ("grad", ctypes.c_void_p * MAX_TENSORS), ("m", ctypes.c_void_p * MAX_TENSORS),
                ("count", ctypes.c_int32 * MAX_TENSORS), ("rows", ctypes.c_int32 * MAX_TENSORS),
                ("cols", ctypes.c_int32 * MAX_TENSORS)]


class Muon(ctypes.Structure):
    _fields_ = [("lr", ctypes.c_double), ("momentum", ctypes.c_double), ("weight_decay", ctypes.c_double),
                ("nesterov", ctypes.c_int32), ("scale", ctypes.c_int32), ("ns", NewtonSchulz)]


class Choices(ctypes.Structure):
    _fields_ = [("logits", ctypes.c_void_p), ("rows", ctypes.c_int64), ("stride", ctypes.c_int64),
                ("n_choices", ctypes.c_int32), ("type", ctypes.c_int32), ("top", ctypes.c_int32), ("scale", ctypes.c_double)]


class ChoiceGrads(ctypes.Structure):
    _fields_ = [("choice", ctypes.c_void_p), ("logp", ctypes.c_void_p), ("entropy", ctypes.c_void_p),
                ("top_choice", ctypes.c_void_p), ("stats", ctypes.c_void_p), ("d_logp", ctypes.c_void_p),
                ("d_entropy", ctypes.c_void_p), ("d_top", ctypes.c_void_p)]


class Routed(ctypes.Structure):
    _fields_ = [("place", ctypes.c_void_p), ("rows", ctypes.c_int64), ("slots", ctypes.c_int32), ("width", ctypes.c_int32),
                ("type", ctypes.c_int32)]


class DiscOut(ctypes.Structure):
    _fields_ = [("logits_fake", ctypes.c_void_p), ("logits_real", ctypes.c_void_p),
                ("loss_d", ctypes.c_void_p), ("loss_g", ctypes.c_void_p),
                ("dW", ctypes.c_void_p * MAX_LAYERS), ("db", ctypes.c_void_p * MAX_LAYERS),
                ("dLg_dx", ctypes.c_void_p), ("dLg_dtheta", ctypes.c_void_p)]


_lib = None


def load_library(path: str = LIB_PATH) -> ctypes.CDLL:
    """Load libsagips.so (once) and declare its signatures."""
    global _lib
    if _lib is not None:
        return _lib
    if not os.path.exists(path):
        raise ImportError(f"{path} is not built; run python -m paper_2407_00051_amd.build")
    lib = ctypes.CDLL(path)
    vp, i32, i64 = ctypes.c_void_p, ctypes.c_int, ctypes.c_int64
    lib.sagips_create.argtypes = [ctypes.POINTER(vp), i32, vp]
    lib.sagips_destroy.argtypes = [vp]
    lib.sagips_set_stream.argtypes = [vp, vp]
    lib.sagips_set_bf16_chunk_rows.argtypes = [vp, i64]
    lib.sagips_last_error.argtypes = [vp]
    lib.sagips_last_error.restype = ctypes.c_char_p
    lib.sagips_set_timing.argtypes = [vp, i32]
    lib.sagips_kernel_times.argtypes = [vp, ctypes.POINTER(ctypes.c_char_p), ctypes.POINTER(i64),
                                        ctypes.POINTER(ctypes.c_double), i32]
    lib.sagips_sample_events.argtypes = [vp, ctypes.POINTER(Source), vp, vp]
    lib.sagips_disc_fwd_bwd.argtypes = [vp, ctypes.POINTER(Mlp), vp, ctypes.POINTER(Source), i64, vp, i64,
                                        ctypes.POINTER(DiscOut)]
    lib.sagips_disc_fwd_bwd_noalloc.argtypes = lib.sagips_disc_fwd_bwd.argtypes
    lib.sagips_noalloc_scratch_bytes.argtypes = []
    lib.sagips_noalloc_scratch_bytes.restype = ctypes.c_size_t
    lib.sagips_param_grad.argtypes = [vp, ctypes.POINTER(Source), i32, vp, vp, vp]
    lib.sagips_bootstrap.argtypes = [vp, vp, i64, i32, ctypes.c_uint64, ctypes.c_uint32, i64, vp, vp]
    lib.sagips_bootstrap_rows.argtypes = lib.sagips_bootstrap.argtypes
    lib.sagips_gen_forward.argtypes = [vp, ctypes.POINTER(GenStack), vp, i64, vp]
    lib.sagips_gen_backward.argtypes = [vp, ctypes.POINTER(GenStack), vp, i64, vp, ctypes.POINTER(vp),
                                        ctypes.POINTER(vp)]
    lib.sagips_ensemble_response.argtypes = [vp, ctypes.POINTER(GenStack), vp, i64, vp, vp, vp, vp]
    lib.sagips_adam_step.argtypes = [vp, ctypes.POINTER(ParamSet), i32, ctypes.c_double, ctypes.c_double,
                                     ctypes.c_double, ctypes.c_double]
    lib.sagips_group_advantage.argtypes = [vp, vp, vp, ctypes.c_int32, i64, i32, ctypes.c_double, vp]
    lib.sagips_policy_loss.argtypes = [vp, ctypes.POINTER(Policy), vp, vp, vp, vp, vp, vp, vp]
    lib.sagips_orthogonalise.argtypes = [vp, ctypes.POINTER(NewtonSchulz), ctypes.c_int32, vp, ctypes.c_int32,
                                         ctypes.c_int32, ctypes.c_int32, vp]
    lib.sagips_muon_step.argtypes = [vp, ctypes.POINTER(MatrixSet), ctypes.POINTER(Muon)]
    lib.sagips_preference_loss.argtypes = [vp, ctypes.POINTER(Preference), vp, vp, vp, vp, vp, vp, vp]
    lib.sagips_choice_logprob.argtypes = [vp, ctypes.POINTER(Choices), vp, vp, vp, vp, vp, vp]
    lib.sagips_choice_backward.argtypes = [vp, ctypes.POINTER(Choices), ctypes.POINTER(ChoiceGrads), vp, i64]
    lib.sagips_route.argtypes = [vp, vp, i64, ctypes.c_int32, ctypes.c_int32, vp, vp, vp]
    lib.sagips_dispatch.argtypes = [vp, ctypes.POINTER(Routed), vp, vp]
    lib.sagips_combine.argtypes = [vp, ctypes.POINTER(Routed), vp, vp, vp]
    lib.sagips_combine_backward.argtypes = [vp, ctypes.POINTER(Routed), vp, vp, vp, vp, vp]
    lib.sagips_gen_forward_routed.argtypes = [vp, ctypes.POINTER(GenStack), vp, vp, i64, vp]
    lib.sagips_gen_backward_routed.argtypes = [vp, ctypes.POINTER(GenStack), vp, vp, i64, vp, ctypes.POINTER(vp),
                                               ctypes.POINTER(vp), vp]
    for name in ("sagips_create", "sagips_destroy", "sagips_set_stream", "sagips_set_bf16_chunk_rows",
                 "sagips_set_timing",
                 "sagips_kernel_times", "sagips_sample_events", "sagips_disc_fwd_bwd", "sagips_param_grad",
                 "sagips_bootstrap", "sagips_bootstrap_rows", "sagips_gen_forward", "sagips_gen_backward", "sagips_ensemble_response",
                 "sagips_adam_step", "sagips_disc_fwd_bwd_noalloc", "sagips_group_advantage", "sagips_policy_loss",
                 "sagips_preference_loss", "sagips_orthogonalise", "sagips_muon_step", "sagips_choice_logprob",
                 "sagips_choice_backward", "sagips_route", "sagips_dispatch", "sagips_combine", "sagips_combine_backward",
                 "sagips_gen_forward_routed", "sagips_gen_backward_routed"):
        getattr(lib, name).restype = ctypes.c_int
    _lib = lib
    return lib


def _ptr(t) -> Optional[int]:
    return None if t is None else t.data_ptr()


def _check_tensor(t, name, dtype=None, shape=None, device=None):
    if t is None:
        return
    try:                        # the usual case first; what fails here is named below
        if (t.is_cuda and (device is None or t.get_device() == device) and t.is_contiguous()
                and (dtype is None or t.dtype is dtype) and (shape is None or t.shape == shape)):
            return
    except (AttributeError, TypeError):
        pass
    import torch
    if not isinstance(t, torch.Tensor):
        raise TypeError(f"{name} must be a torch.Tensor")
    if not t.is_cuda:
        raise ValueError(f"{name} must be on a GPU device")
    if device is not None and t.get_device() != device:
        raise ValueError(f"{name} is on cuda:{t.get_device()}, the context on cuda:{device}")
    if not t.is_contiguous():
        raise ValueError(f"{name} must be contiguous")
    if dtype is not None and t.dtype != dtype:
        raise TypeError(f"{name} must be {dtype}, got {t.dtype}")
    if shape is not None and t.shape != shape and tuple(t.shape) != tuple(shape):
        raise ValueError(f"{name} must have shape {tuple(shape)}, got {tuple(t.shape)}")


def _raw_stream(device: int) -> int:
    """The handle of torch's current stream of the device."""
    import torch
    try:
        return torch._C._cuda_getCurrentRawStream(device)
    except AttributeError:
        return torch.cuda.current_stream(device).cuda_stream


class Context:
    """A library context on one GPU.

    Without a stream it follows torch: every call runs on torch's current stream
    of the device at the time of the call, the stream on which the binding also
    allocates the outputs it returns.  With an explicit stream every call runs
    there, and outputs the binding allocates are marked as used by that stream
    (record_stream), so that torch's caching allocator does not hand their memory
    out again before the library's kernels are done with it."""

    def __init__(self, device: int = 0, stream=None):
        import torch
        self._torch = torch
        self.lib = load_library()
        self.device = device
        self._follow = stream is None
        if stream is None:
            stream = torch.cuda.current_stream(device)
        self._stream = stream
        self._raw = stream.cuda_stream
        h = ctypes.c_void_p()
        st = self.lib.sagips_create(ctypes.byref(h), device, ctypes.c_void_p(stream.cuda_stream))
        if st != OK:
            raise SagipsError(st, self.lib.sagips_last_error(None).decode())
        self.h = h

    # -- plumbing -------------------------------------------------------------
    def _check(self, st: int):
        if st != OK:
            raise SagipsError(st, self.lib.sagips_last_error(self.h).decode())

    def close(self):
        if getattr(self, "h", None):
            self.lib.sagips_destroy(self.h)
            self.h = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    @property
    def stream(self):
        return self._stream

    def set_stream(self, stream):
        """Run later calls on `stream` (and stop following torch's current stream)."""
        self._check(self.lib.sagips_set_stream(self.h, ctypes.c_void_p(stream.cuda_stream)))
        self._stream = stream
        self._raw = stream.cuda_stream
        self._follow = False

    def _enter(self):
        """Before a call: in follow mode, switch to torch's current stream if it changed."""
        if self._follow and _raw_stream(self.device) != self._raw:
            import torch
            cur = torch.cuda.current_stream(self.device)
            self._check(self.lib.sagips_set_stream(self.h, ctypes.c_void_p(cur.cuda_stream)))
            self._stream = cur
            self._raw = cur.cuda_stream

    def _owned(self, *tensors):
        """Tensors that belong to torch's current stream (outputs the binding allocated there, inputs
        that the caller may drop), used by the library's stream."""
        if self._follow:
            return
        import torch
        if torch.cuda.current_stream(self.device).cuda_stream == self._stream.cuda_stream:
            return
        for t in tensors:
            if isinstance(t, (list, tuple)):
                self._owned(*t)
            elif t is not None:
                t.record_stream(self._stream)

    def set_bf16_chunk_rows(self, rows: int = 0):
        """Rows per chunk of the bf16 discriminator (0: the default, 4,194,304)."""
        self._check(self.lib.sagips_set_bf16_chunk_rows(self.h, int(rows)))

    def set_timing(self, enable: bool):
        self._check(self.lib.sagips_set_timing(self.h, 1 if enable else 0))

    def kernel_times(self) -> Dict[str, tuple]:
        """{kernel name: (launches, total ms)} since the last call; syncs the stream."""
        cap = 64
        names = (ctypes.c_char_p * cap)()
        launches = (ctypes.c_int64 * cap)()
        ms = (ctypes.c_double * cap)()
        n = self.lib.sagips_kernel_times(self.h, names, launches, ms, cap)
        if n < 0:
            self._check(n)
        return {names[i].decode(): (int(launches[i]), float(ms[i])) for i in range(min(n, cap))}

    def source(self, theta, events_per_theta: int, seed: int, counter_base: int = 0, stream: int = 0) -> Source:
        import torch
        _check_tensor(theta, "theta", torch.float32, device=self.device)
        if theta.dim() != 2 or theta.shape[1] not in (4, 6):
            raise ValueError("theta must be [n_theta][4] or [n_theta][6]")
        return Source(theta.data_ptr(), theta.shape[0], theta.shape[1] // 2, int(events_per_theta), int(seed),
                      int(counter_base), int(stream))

    # -- 1. parameters -> events ---------------------------------------------------
    def sample_events(self, theta, events_per_theta: int, seed: int, counter_base: int = 0, stream: int = 0,
                      want_x: bool = True, want_words: bool = False, out=None, words_out=None):
        """Events [N][d] fp32 (and optionally the raw Philox words [N][4] int32)."""
        import torch
        self._enter()
        src = self.source(theta, events_per_theta, seed, counter_base, stream)
        N = src.n_theta * src.events_per_theta
        x = None
        w = None
        if want_x:
            x = out if out is not None else torch.empty((N, src.d), dtype=torch.float32, device=theta.device)
            _check_tensor(x, "out", torch.float32, (N, src.d), self.device)
        if want_words:
            w = words_out if words_out is not None else torch.empty((N, 4), dtype=torch.int32, device=theta.device)
            _check_tensor(w, "words_out", torch.int32, (N, 4), self.device)
        self._owned(x if out is None else None, w if words_out is None else None)
        self._check(self.lib.sagips_sample_events(self.h, ctypes.byref(src), _ptr(x), _ptr(w)))
        self._keep = (theta,)
        if want_words and want_x:
            return x, w
        return x if want_x else w

    # -- 4. reference data -> bootstrapped sub-sample --------------------------------
    def bootstrap(self, data, n_out: int, seed: int, step: int, want_idx: bool = False, out=None, idx_out=None,
                  row_order: bool = False):
        """The step's sub-sample [n_out][d] of the rows of data (drawn with replacement), and
        optionally the drawn row indices [n_out] int64; with row_order the same multiset in
        ascending row order."""
        import torch
        self._enter()
        _check_tensor(data, "data", torch.float32, None, self.device)
        if data.dim() != 2 or data.shape[1] not in (2, 3):
            raise ValueError("data must be [n_data][d] with d in {2, 3}")
        d = data.shape[1]
        x = out if out is not None else torch.empty((n_out, d), dtype=torch.float32, device=data.device)
        _check_tensor(x, "out", torch.float32, (n_out, d), self.device)
        idx = None
        if want_idx:
            idx = idx_out if idx_out is not None else torch.empty(n_out, dtype=torch.int64, device=data.device)
            _check_tensor(idx, "idx_out", torch.int64, (n_out,), self.device)
        self._owned(x if out is None else None, idx if idx_out is None else None)
        fn = self.lib.sagips_bootstrap_rows if row_order else self.lib.sagips_bootstrap
        self._check(fn(self.h, _ptr(data), data.shape[0], d, seed & (2**64 - 1), step & 0xFFFFFFFF, n_out, _ptr(x),
                       _ptr(idx)))
        self._keep = (data,)
        return (x, idx) if want_idx else x

    # -- generator (noise -> parameters) and the ensemble response -------------------
    def _gen(self, W: Sequence, b: Sequence, slope: float):
        """GenStack for stacked members: W[l] is [M][out][in] (or [out][in] for one member),
        b[l] is [M][out] (or [out])."""
        import torch
        n_layers = len(W)
        if n_layers != len(b) or not 2 <= n_layers <= MAX_LAYERS:
            raise ValueError("W and b must have the same length, 2..8")
        W3 = [w if w.dim() == 3 else w.unsqueeze(0) for w in W]
        b2 = [v if v.dim() == 2 else v.unsqueeze(0) for v in b]
        M = W3[0].shape[0]
        g = GenStack()
        g.n_layers = n_layers
        g.n_members = M
        g.leaky_slope = float(slope)
        g.width[0] = W3[0].shape[2]
        for l in range(n_layers):
            _check_tensor(W3[l], f"W[{l}]", torch.float32, (M, W3[l].shape[1], g.width[l]), self.device)
            g.width[l + 1] = W3[l].shape[1]
            _check_tensor(b2[l], f"b[{l}]", torch.float32, (M, g.width[l + 1]), self.device)
            g.W[l] = W3[l].data_ptr()
            g.b[l] = b2[l].data_ptr()
        return g, M

    def gen_forward(self, W: Sequence, b: Sequence, noise, slope: float = 0.2, out=None):
        """theta [M][k][out] = 1 + softplus(G_m(noise)) for every member m."""
        import torch
        self._enter()
        g, M = self._gen(W, b, slope)
        _check_tensor(noise, "noise", torch.float32, (noise.shape[0], g.width[0]), self.device)
        k = noise.shape[0]
        th = out if out is not None else torch.empty((M, k, g.width[g.n_layers]), dtype=torch.float32,
                                                     device=noise.device)
        _check_tensor(th, "out", torch.float32, (M, k, g.width[g.n_layers]), self.device)
        self._owned(th if out is None else None)
        self._check(self.lib.sagips_gen_forward(self.h, ctypes.byref(g), noise.data_ptr(), k, th.data_ptr()))
        return th

    def gen_backward(self, W: Sequence, b: Sequence, noise, dL_dtheta, slope: float = 0.2, dW=None, db=None):
        """Gradients (dW, db), shaped like W and b, of sum <dL/dtheta, theta> per member."""
        import torch
        self._enter()
        g, M = self._gen(W, b, slope)
        _check_tensor(noise, "noise", torch.float32, (noise.shape[0], g.width[0]), self.device)
        k = noise.shape[0]
        n_out = g.width[g.n_layers]
        if M > 1 or dL_dtheta.dim() == 3:
            _check_tensor(dL_dtheta, "dL_dtheta", torch.float32, (M, k, n_out), self.device)
        else:
            _check_tensor(dL_dtheta, "dL_dtheta", torch.float32, (k, n_out), self.device)
        new_dW, new_db = dW is None, db is None
        dW = dW if dW is not None else [torch.empty_like(w) for w in W]
        db = db if db is not None else [torch.empty_like(v) for v in b]
        self._owned(dW if new_dW else None, db if new_db else None)
        for l in range(g.n_layers):
            _check_tensor(dW[l], f"dW[{l}]", torch.float32, tuple(W[l].shape), self.device)
            _check_tensor(db[l], f"db[{l}]", torch.float32, tuple(b[l].shape), self.device)
        pw = (ctypes.c_void_p * MAX_LAYERS)(*[t.data_ptr() for t in dW])
        pb = (ctypes.c_void_p * MAX_LAYERS)(*[t.data_ptr() for t in db])
        self._check(self.lib.sagips_gen_backward(self.h, ctypes.byref(g), noise.data_ptr(), k,
                                                 dL_dtheta.data_ptr(), pw, pb))
        return dW, db

    def ensemble_response(self, W: Sequence, b: Sequence, noise, p_true=None, slope: float = 0.2) -> dict:
        """p_hat and sigma [out] averaged over the noise batch, and r_hat = (p_true - p_hat) / p_true."""
        import torch
        self._enter()
        g, M = self._gen(W, b, slope)
        _check_tensor(noise, "noise", torch.float32, (noise.shape[0], g.width[0]), self.device)
        n_out = g.width[g.n_layers]
        f32 = dict(dtype=torch.float32, device=noise.device)
        o = {"p_hat": torch.empty(n_out, **f32), "sigma": torch.empty(n_out, **f32), "r_hat": None}
        if p_true is not None:
            _check_tensor(p_true, "p_true", torch.float32, (n_out,), self.device)
            o["r_hat"] = torch.empty(n_out, **f32)
        self._owned(o["p_hat"], o["sigma"], o["r_hat"])
        self._check(self.lib.sagips_ensemble_response(self.h, ctypes.byref(g), noise.data_ptr(), noise.shape[0],
                                                      _ptr(p_true), o["p_hat"].data_ptr(), o["sigma"].data_ptr(),
                                                      _ptr(o["r_hat"])))
        return o

    # -- optimiser ------------------------------------------------------------------
    def adam_step(self, params: Sequence, grads: Sequence, m: Sequence, v: Sequence, step: int, lr: float,
                  beta1: float = 0.9, beta2: float = 0.999, eps: float = 1e-8) -> None:
        """In-place Adam step on up to 16 fp32 tensors (m, v start at zero; step counts from 1)."""
        import torch
        self._enter()
        n = len(params)
        if not (n == len(grads) == len(m) == len(v)) or not 1 <= n <= MAX_TENSORS:
            raise ValueError("params, grads, m, v must have the same length, 1..16")
        ps = ParamSet()
        ps.n_tensors = n
        for i in range(n):
            for t, name in ((params[i], "param"), (grads[i], "grad"), (m[i], "m"), (v[i], "v")):
                _check_tensor(t, f"{name}[{i}]", torch.float32, tuple(params[i].shape), self.device)
            ps.param[i], ps.grad[i] = params[i].data_ptr(), grads[i].data_ptr()
            ps.m[i], ps.v[i] = m[i].data_ptr(), v[i].data_ptr()
            ps.size[i] = params[i].numel()
        self._check(self.lib.sagips_adam_step(self.h, ctypes.byref(ps), int(step), lr, beta1, beta2, eps))

    # -- 2. events -> discriminator -> BCE -> backward -------------------------------
    def disc_fwd_bwd(self, W: Sequence, b: Sequence, real_x, fake_x=None, fake_source: Optional[dict] = None,
                     precision: int = F32, features: int = FEAT_IDENTITY, slope: float = 0.2,
                     want_logits: bool = True, want_grads: bool = True, want_dx: bool = True,
                     want_dtheta: bool = True, outputs: Optional[dict] = None, no_alloc: bool = False) -> dict:
        """One discriminator step.  fake_source = dict(theta=, events_per_theta=, seed=[, counter_base=, stream=])
        samples the fake events inside the kernel and also returns dLg_dtheta.  With no_alloc the
        library takes its workspace from its fixed per-device scratch (sagips_disc_fwd_bwd_noalloc)
        instead of allocating; pass every output in `outputs` so that the binding allocates nothing
        either."""
        import torch
        self._enter()
        n_layers = len(W)
        if n_layers != len(b) or not 1 <= n_layers <= MAX_LAYERS:
            raise ValueError("W and b must have the same length, 1..8")
        widths = [W[0].shape[1]] + [w.shape[0] for w in W]
        for l in range(n_layers):
            _check_tensor(W[l], _W_NAMES[l], torch.float32, (widths[l + 1], widths[l]), self.device)
            _check_tensor(b[l], _B_NAMES[l], torch.float32, (widths[l + 1],), self.device)
        mlp = Mlp(n_layers, tuple(widths), tuple([w.data_ptr() for w in W]), tuple([v.data_ptr() for v in b]),
                  float(slope), int(precision), int(features))
        dev = real_x.device
        _check_tensor(real_x, "real_x", torch.float32, device=self.device)
        src = None
        if fake_source is not None:
            fs = dict(fake_source)
            src = self.source(fs.pop("theta"), fs.pop("events_per_theta"), fs.pop("seed"), **fs)
            n_fake = src.n_theta * src.events_per_theta
            d = src.d
        elif fake_x is not None:
            _check_tensor(fake_x, "fake_x", torch.float32, device=self.device)
            n_fake = fake_x.shape[0]
            d = fake_x.shape[1]
        else:                       # no fake input: the library rejects the call
            n_fake, d = 0, widths[0]
        n_real = real_x.shape[0]
        d_in = widths[0] if features == FEAT_IDENTITY else 3
        if (fake_x is not None and d != d_in) or real_x.dim() != 2 or real_x.shape[1] != d_in:
            raise ValueError(f"events must be [n][{d_in}] for this network and feature map")
        o = dict(outputs or {})
        new = []                    # outputs the binding allocates: only those not given

        def want(k, *shape):
            if k not in o:
                o[k] = torch.empty(shape, dtype=torch.float32, device=dev)
                new.append(o[k])

        if want_logits:
            want("logits_fake", max(n_fake, 1))
            want("logits_real", n_real)
        want("loss_d", 1)
        want("loss_g", 1)
        if want_grads:
            for k, like in (("dW", W), ("db", b)):
                if k not in o:
                    o[k] = [torch.empty_like(t) for t in like]
                    new.append(o[k])
        if want_dx:
            want("dLg_dx", max(n_fake, 1), d)
        if want_dtheta and src is not None:
            want("dLg_dtheta", src.n_theta, 2 * src.d)
        if new:
            self._owned(*new)
        out = DiscOut()
        for k in ("logits_fake", "logits_real", "loss_d", "loss_g", "dLg_dx", "dLg_dtheta"):
            t = o.get(k)
            if t is not None:
                _check_tensor(t, k, torch.float32, device=self.device)
                setattr(out, k, t.data_ptr())
        if "dW" in o:
            dW, db = o["dW"], o["db"]
            out.dW = tuple([dW[l].data_ptr() for l in range(n_layers)])
            out.db = tuple([db[l].data_ptr() for l in range(n_layers)])
        fn = self.lib.sagips_disc_fwd_bwd_noalloc if no_alloc else self.lib.sagips_disc_fwd_bwd
        st = fn(self.h, ctypes.byref(mlp), _ptr(fake_x), ctypes.byref(src) if src is not None else None, n_fake,
                real_x.data_ptr(), n_real, ctypes.byref(out))
        self._check(st)
        return o

    # -- 3. dL/dx -> pathwise dx/dtheta -> per-parameter reduction ---------------------------
    def param_grad(self, theta, events_per_theta: int, seed: int, dL_dx=None, counter_base: int = 0,
                   stream: int = 0, out=None, loss_out=None, want_loss: bool = True):
        """dL/dtheta [n_theta][2d]; with dL_dx None the quadratic critic is used and its loss returned too."""
        import torch
        self._enter()
        src = self.source(theta, events_per_theta, seed, counter_base, stream)
        g = out if out is not None else torch.empty((src.n_theta, 2 * src.d), dtype=torch.float32, device=theta.device)
        _check_tensor(g, "out", torch.float32, (src.n_theta, 2 * src.d), self.device)
        loss = None
        if dL_dx is None:
            critic = CRITIC_QUADRATIC
            if want_loss:
                loss = loss_out if loss_out is not None else torch.empty(1, dtype=torch.float32, device=theta.device)
        else:
            critic = CRITIC_BUFFER
            _check_tensor(dL_dx, "dL_dx", torch.float32, (src.n_theta * src.events_per_theta, src.d), self.device)
        self._owned(g if out is None else None, loss if loss_out is None else None)
        self._check(self.lib.sagips_param_grad(self.h, ctypes.byref(src), critic, _ptr(dL_dx), g.data_ptr(),
                                               _ptr(loss)))
        return (g, loss) if critic == CRITIC_QUADRATIC else g


    # -- training without a differentiable pipeline ------------------------------------------
    def _rows(self, t, name, like=None):
        """A table of parameter rows [n_theta][4] or [n_theta][6]."""
        import torch
        if like is not None:
            return _check_tensor(t, name, torch.float32, like.shape, self.device)
        _check_tensor(t, name, torch.float32, None, self.device)
        if t.dim() != 2 or t.shape[1] not in (4, 6):
            raise ValueError(f"{name} must be [n_theta][4] or [n_theta][6]")

    def _mask(self, mask, shape):
        import torch
        if mask is None:
            return None
        _check_tensor(mask, "mask", None, shape, self.device)
        if mask.dtype not in (torch.bool, torch.uint8):
            raise TypeError(f"mask must be torch.bool or torch.uint8, got {mask.dtype}")
        return mask.data_ptr()

    def group_advantage(self, reward, mask=None, normalise: bool = True, eps: float = 1e-6, out=None):
        """Advantages [n_rows][E]: each row's rewards less their mean, over their deviation plus eps if
        normalise, among the events that the mask (bool or uint8, like reward) leaves; 0 elsewhere."""
        import torch
        self._enter()
        _check_tensor(reward, "reward", torch.float32, None, self.device)
        if reward.dim() != 2:
            raise ValueError("reward must be [n_rows][events_per_row]")
        m = self._mask(mask, reward.shape)
        adv = out if out is not None else torch.empty_like(reward)
        if out is not None:
            _check_tensor(out, "out", torch.float32, reward.shape, self.device)
        self._owned(adv if out is None else None, reward, mask)
        self._check(self.lib.sagips_group_advantage(self.h, reward.data_ptr(), m, reward.shape[0], reward.shape[1],
                                                    1 if normalise else 0, eps, adv.data_ptr()))
        return adv

    def policy_loss(self, theta, theta_old, x, adv, theta_ref=None, mask=None, clip_low: float = 0.2,
                    clip_high: float = 0.2, kl_coef: float = 0.0, average: str = "events", want_grad: bool = True) -> dict:
        """Clipped policy loss of events x [n_theta][E][d] drawn at theta_old with advantages adv
        [n_theta][E], and its gradient with respect to theta; the KL term needs theta_ref.
        average: "events" or "rows".  Returns loss, kl, clip_frac [1] and dtheta."""
        import torch
        self._enter()
        f32, dev = torch.float32, self.device
        self._rows(theta, "theta")
        self._rows(theta_old, "theta_old", theta)
        if theta_ref is not None:
            self._rows(theta_ref, "theta_ref", theta)
        n, d = theta.shape[0], theta.shape[1] // 2
        _check_tensor(adv, "adv", f32, None, dev)
        if adv.dim() != 2 or adv.shape[0] != n:
            raise ValueError(f"adv must be [{n}][events_per_theta]")
        E = adv.shape[1]
        _check_tensor(x, "x", f32, (n, E, d), dev)
        m = self._mask(mask, adv.shape)
        if average not in ("events", "rows"):
            raise ValueError("average must be 'events' or 'rows'")
        P = Policy(theta.data_ptr(), theta_old.data_ptr(), _ptr(theta_ref), n, d, E, clip_low, clip_high, kl_coef,
                   MEAN_ROWS if average == "rows" else MEAN_EVENTS)
        scalars = theta.new_empty(3, 1)
        dtheta = torch.empty_like(theta) if want_grad else None
        self._owned(scalars, dtheta, theta, theta_old, theta_ref, x, adv, mask)
        at = scalars.data_ptr()
        self._check(self.lib.sagips_policy_loss(self.h, ctypes.byref(P), x.data_ptr(), adv.data_ptr(), m, at, at + 4,
                                                at + 8, _ptr(dtheta)))
        loss, kl, clip_frac = scalars.unbind()           # [1] each
        return {"loss": loss, "kl": kl, "clip_frac": clip_frac, "dtheta": dtheta}

    def preference_loss(self, theta, theta_ref, chosen, rejected, len_chosen=None, len_rejected=None, beta: float = 0.1,
                        label_smoothing: float = 0.0, want_grad: bool = True) -> dict:
        """Preference loss over pairs of event sets, chosen [n_pairs][T][d] against rejected
        [n_pairs][T'][d] with n_pairs a multiple of n_theta (row i's pairs follow each other), of which
        the first len_* [n_pairs] int32 events count.  Returns loss [1], margin [n_pairs] and dtheta."""
        import torch
        self._enter()
        f32, dev = torch.float32, self.device
        self._rows(theta, "theta")
        self._rows(theta_ref, "theta_ref", theta)
        n, d = theta.shape[0], theta.shape[1] // 2
        _check_tensor(chosen, "chosen", f32, None, dev)
        _check_tensor(rejected, "rejected", f32, None, dev)
        P = chosen.shape[0]
        if chosen.dim() != 3 or rejected.dim() != 3 or rejected.shape[0] != P or chosen.shape[2] != d or rejected.shape[2] != d:
            raise ValueError(f"chosen and rejected must be [n_pairs][events][{d}]")
        if n == 0 or P == 0 or P % n:
            raise ValueError("the number of pairs must be a multiple of the number of rows")
        for t, name in ((len_chosen, "len_chosen"), (len_rejected, "len_rejected")):
            _check_tensor(t, name, torch.int32, (P,), dev)
        a = Preference(theta.data_ptr(), theta_ref.data_ptr(), n, d, P // n, chosen.shape[1], rejected.shape[1], beta,
                       label_smoothing)
        loss, margin = theta.new_empty(1), theta.new_empty(P)
        dtheta = torch.empty_like(theta) if want_grad else None
        self._owned(loss, margin, dtheta, theta, theta_ref, chosen, rejected, len_chosen, len_rejected)
        self._check(self.lib.sagips_preference_loss(self.h, ctypes.byref(a), chosen.data_ptr(), _ptr(len_chosen),
                                                    rejected.data_ptr(), _ptr(len_rejected), loss.data_ptr(),
                                                    margin.data_ptr(), _ptr(dtheta)))
        return {"loss": loss, "margin": margin, "dtheta": dtheta}

    # -- orthogonalised updates ----------------------------------------------------------------
    @staticmethod
    def _stack(t):
        """(count, rows, cols) of a matrix or a stack of matrices."""
        if t.dim() == 2:
            return 1, t.shape[0], t.shape[1]
        if t.dim() == 3:
            return tuple(t.shape)
        raise ValueError("matrices must be [rows][cols] or [count][rows][cols]")

    @staticmethod
    def _newton_schulz(steps, coef, eps):
        if steps < 1:
            raise ValueError("steps must be >= 1")
        if len(coef) != 3:
            raise ValueError(f"coef must be three numbers, got {len(coef)}")
        return NewtonSchulz(steps, (ctypes.c_double * 3)(*coef), eps)

    def orthogonalise(self, x, steps: int = 5, coef: Sequence[float] = NS_COEF, eps: float = 1e-7, out=None):
        """Newton-Schulz steps on every matrix of x, [rows][cols] or [count][rows][cols], fp32 or bf16:
        singular values to a band around 1, singular vectors kept.  out may be x."""
        import torch
        self._enter()
        _check_tensor(x, "x", None, None, self.device)
        if x.dtype not in (torch.float32, torch.bfloat16):
            raise TypeError(f"x must be torch.float32 or torch.bfloat16, got {x.dtype}")
        count, rows, cols = self._stack(x)
        o = out if out is not None else torch.empty_like(x)
        if out is not None:
            _check_tensor(out, "out", x.dtype, x.shape, self.device)
        ns = self._newton_schulz(steps, coef, eps)
        self._owned(o if out is None else None, x)
        self._check(self.lib.sagips_orthogonalise(self.h, ctypes.byref(ns), F32 if x.dtype == torch.float32 else BF16,
                                                  x.data_ptr(), count, rows, cols, o.data_ptr()))
        return o

    def muon_step(self, params: Sequence, grads: Sequence, momenta: Sequence, lr: float, momentum: float = 0.95,
                  nesterov: bool = True, weight_decay: float = 0.0, scale: int = SCALE_SHAPE, steps: int = 5,
                  coef: Sequence[float] = NS_COEF, eps: float = 1e-7) -> None:
        """In-place step on up to 16 fp32 matrices or stacks of matrices: momentum (fp32, starting at
        zero), then the parameters move along the orthogonalised momentum.  grads are fp32 or bf16."""
        import torch
        self._enter()
        n = len(params)
        if not (n == len(grads) == len(momenta)) or not 1 <= n <= MAX_TENSORS:
            raise ValueError("params, grads and momenta must have the same length, 1..16")
        ns = self._newton_schulz(steps, coef, eps)
        dtype = grads[0].dtype
        if dtype not in (torch.float32, torch.bfloat16):
            raise TypeError(f"grads must be torch.float32 or torch.bfloat16, got {dtype}")
        ms = MatrixSet()
        ms.n_tensors = n
        ms.grad_type = F32 if dtype == torch.float32 else BF16
        for i in range(n):
            p = params[i]
            _check_tensor(p, f"params[{i}]", torch.float32, None, self.device)
            _check_tensor(grads[i], f"grads[{i}]", dtype, p.shape, self.device)
            _check_tensor(momenta[i], f"momenta[{i}]", torch.float32, p.shape, self.device)
            ms.count[i], ms.rows[i], ms.cols[i] = self._stack(p)
            ms.param[i], ms.grad[i], ms.m[i] = p.data_ptr(), grads[i].data_ptr(), momenta[i].data_ptr()
        self._owned(params, grads, momenta)
        o = Muon(lr, momentum, weight_decay, 1 if nesterov else 0, scale, ns)
        self._check(self.lib.sagips_muon_step(self.h, ctypes.byref(ms), ctypes.byref(o)))

    # -- choices, and a mixture of members -----------------------------------------------------
    def _choices(self, logits, top, scale) -> Choices:
        torch = self._torch
        dtype = logits.dtype
        if dtype is torch.float32:
            kind = F32
        elif dtype is torch.bfloat16:
            kind = BF16
        else:
            raise TypeError(f"logits must be torch.float32 or torch.bfloat16, got {dtype}")
        if logits.get_device() != self.device or not logits.is_cuda:
            raise ValueError(f"logits must be on cuda:{self.device}")
        shape = logits.shape
        if len(shape) != 2 or shape[0] < 1 or shape[1] < 1:
            raise ValueError("logits must be [rows][choices]")
        n, V = shape
        rows, each = logits.stride()
        if n == 1:
            rows = max(rows, V)
        if (each != 1 and V > 1) or rows < V:
            raise ValueError("the choices of a row must follow each other, and rows must not overlap")
        return Choices(logits.data_ptr(), n, rows, V, kind, top, scale)

    def choice_logprob(self, logits, choice=None, top: int = 0, scale: float = 1.0) -> dict:
        """Of the categorical distribution softmax(scale * logits) of every row of logits [rows][choices]
        (fp32 or bf16; rows may be strided, -inf masks a choice): logp [rows] of the given choice [rows]
        int32 (0 for a row whose choice is outside the range; None without choice), entropy [rows], the
        `top` (up to 32) most likely alternatives top_choice [rows][top] int32 (-1 where there are
        fewer) and their top_logp, and stats [rows][2] for choice_backward."""
        torch = self._torch
        self._enter()
        if not 0 <= top <= MAX_TOP:
            raise ValueError(f"top must be in [0, {MAX_TOP}]")
        C = self._choices(logits, top, scale)
        n = C.rows
        # one allocation for the fp32 results: a call is short
        held = logits.new_empty(n * (4 + top), dtype=torch.float32)
        logp, entropy, stats, top_logp = held.split_with_sizes((n, n, 2 * n, n * top))
        top_choice = logits.new_empty((n, top), dtype=torch.int32)
        if choice is not None:
            _check_tensor(choice, "choice", torch.int32, (n,), self.device)
        if not self._follow:
            self._owned(held, top_choice, logits, choice)
        at = held.data_ptr()
        self._check(self.lib.sagips_choice_logprob(
            self.h, ctypes.byref(C), None if choice is None else choice.data_ptr(), None if choice is None else at,
            at + 4 * n, top_choice.data_ptr() if top else None, at + 16 * n if top else None, at + 8 * n))
        return {"logp": None if choice is None else logp, "entropy": entropy, "top_choice": top_choice,
                "top_logp": top_logp.view(n, top), "stats": stats.view(n, 2)}

    def choice_backward(self, logits, fwd: dict, choice=None, d_logp=None, d_entropy=None, d_top=None, scale: float = 1.0,
                        out=None):
        """dL/dlogits [rows][choices] in the logits' type, from what choice_logprob returned (fwd) for the
        same logits, choice and scale, and the derivatives d_logp, d_entropy [rows], d_top [rows][top] of
        the loss (None: not in it).  out may be the logits, and rows of it may be strided."""
        torch = self._torch
        self._enter()
        f32, dev = torch.float32, self.device
        tops = fwd["top_choice"]
        top = 0 if d_top is None else tops.shape[1]
        C = self._choices(logits, top, scale)
        n = C.rows
        g = ChoiceGrads()
        stats = fwd["stats"]
        _check_tensor(stats, "fwd['stats']", f32, (n, 2), dev)
        g.stats = stats.data_ptr()
        if d_logp is not None:
            if choice is None or fwd["logp"] is None:
                raise ValueError("d_logp needs the choice, in choice_logprob too")
            _check_tensor(d_logp, "d_logp", f32, (n,), dev)
            _check_tensor(choice, "choice", torch.int32, (n,), dev)
            _check_tensor(fwd["logp"], "fwd['logp']", f32, (n,), dev)
            g.d_logp, g.choice, g.logp = d_logp.data_ptr(), choice.data_ptr(), fwd["logp"].data_ptr()
        if d_entropy is not None:
            _check_tensor(d_entropy, "d_entropy", f32, (n,), dev)
            _check_tensor(fwd["entropy"], "fwd['entropy']", f32, (n,), dev)
            g.d_entropy, g.entropy = d_entropy.data_ptr(), fwd["entropy"].data_ptr()
        if top:
            _check_tensor(d_top, "d_top", f32, (n, top), dev)
            _check_tensor(tops, "fwd['top_choice']", torch.int32, (n, top), dev)
            g.d_top, g.top_choice = d_top.data_ptr(), tops.data_ptr()
        stride = C.n_choices
        if out is None:
            out = logits.new_empty((n, stride))
        else:
            if out.dtype != logits.dtype or out.shape != logits.shape:
                raise ValueError("out must have the logits' shape and type")
            stride = self._choices(out, top, scale).stride
        if not self._follow:
            self._owned(out, logits, choice, d_logp, d_entropy, d_top, [fwd[k] for k in ("logp", "entropy", "stats", "top_choice")])
        self._check(self.lib.sagips_choice_backward(self.h, ctypes.byref(C), ctypes.byref(g), out.data_ptr(), stride))
        return out

    def route(self, member, n_members: int) -> dict:
        """Items sorted by the member that they are given to: of member [rows][slots] int32 (or [rows]; values
        outside [0, n_members) give the item to none) the plan offsets [n_members + 1], order [rows * slots]
        (the item row * slots + slot at each sorted position, then -1) and place [rows][slots] (each item's
        sorted position, or -1), all int32."""
        self._enter()
        _check_tensor(member, "member", self._torch.int32, None, self.device)
        shape = member.shape
        if len(shape) not in (1, 2):
            raise ValueError("member must be [rows][slots] or [rows]")
        rows, slots = shape[0], shape[1] if len(shape) == 2 else 1
        if slots > _INT32 or not -_INT32 <= n_members <= _INT32:
            raise ValueError(f"slots = {slots} or n_members = {n_members} does not fit in 32 bits")
        offsets, order, place = member.new_empty(max(0, n_members) + 1), member.new_empty(rows * slots), member.new_empty((rows, slots))
        if not self._follow:
            self._owned(offsets, order, place, member)
        self._check(self.lib.sagips_route(self.h, member.data_ptr(), rows, slots, n_members, offsets.data_ptr(),
                                          order.data_ptr(), place.data_ptr()))
        return {"offsets": offsets, "order": order, "place": place}

    def _routed(self, plan, t, name, items: bool) -> Routed:
        """The plan for rows like t, [rows][width] or (items) [rows * slots][width]."""
        torch = self._torch
        place = plan["place"]
        _check_tensor(place, "place", torch.int32, None, self.device)
        _check_tensor(t, name, None, None, self.device)
        dtype = t.dtype
        if dtype is not torch.float32 and dtype is not torch.bfloat16:
            raise TypeError(f"{name} must be torch.float32 or torch.bfloat16, got {dtype}")
        if place.dim() != 2:
            raise ValueError("place must be [rows][slots]")
        (rows, slots), shape = place.shape, t.shape
        want = rows * slots if items else rows
        if len(shape) != 2 or shape[0] != want:
            raise ValueError(f"{name} must be [{want}][width]")
        if slots > _INT32 or shape[1] > _INT32:
            raise ValueError(f"slots = {slots} or width = {shape[1]} does not fit in 32 bits")
        return Routed(place.data_ptr(), rows, slots, shape[1], F32 if dtype is torch.float32 else BF16)

    def dispatch(self, x, plan: dict, out=None):
        """x [rows][width] (fp32 or bf16) laid out by member: out[place[r][k]] = x[r], [rows * slots][width].
        Positions from plan["offsets"][-1] on are left as they were.  Its gradient is combine without
        weights."""
        self._enter()
        R = self._routed(plan, x, "x", False)
        shape = (R.rows * R.slots, R.width)
        if out is None:
            out = x.new_empty(shape)
        else:
            _check_tensor(out, "out", x.dtype, shape, self.device)
        if not self._follow:
            self._owned(out, x, plan["place"])
        self._check(self.lib.sagips_dispatch(self.h, ctypes.byref(R), x.data_ptr(), out.data_ptr()))
        return out

    def combine(self, y, plan: dict, weight=None, out=None):
        """Rows put back: out[r] = sum_k weight[r][k] y[place[r][k]], [rows][width], of y [rows * slots][width]
        (fp32 or bf16) and weight [rows][slots] fp32 (None: 1)."""
        self._enter()
        R = self._routed(plan, y, "y", True)
        if weight is not None:
            _check_tensor(weight, "weight", self._torch.float32, (R.rows, R.slots), self.device)
        if out is None:
            out = y.new_empty((R.rows, R.width))
        else:
            _check_tensor(out, "out", y.dtype, (R.rows, R.width), self.device)
        if not self._follow:
            self._owned(out, y, weight, plan["place"])
        self._check(self.lib.sagips_combine(self.h, ctypes.byref(R), y.data_ptr(), _ptr(weight), out.data_ptr()))
        return out

    def combine_backward(self, dout, y, plan: dict, weight=None, want_dweight: bool = True, dy=None):
        """Gradient of combine: dy [rows * slots][width] (positions of no item are left as they were) and, if
        wanted, dweight [rows][slots], which alone needs y."""
        self._enter()
        R = self._routed(plan, dout, "dout", False)
        shape, f32 = (R.rows * R.slots, R.width), self._torch.float32
        if weight is not None:
            _check_tensor(weight, "weight", f32, (R.rows, R.slots), self.device)
        if dy is None:
            dy = dout.new_empty(shape)
        else:
            _check_tensor(dy, "dy", dout.dtype, shape, self.device)
        dw = None
        if want_dweight:
            if y is None:
                raise ValueError("dweight needs y")
            _check_tensor(y, "y", dout.dtype, shape, self.device)
            dw = dout.new_empty((R.rows, R.slots), dtype=f32)
        if not self._follow:
            self._owned(dy, dw, dout, y, weight, plan["place"])
        self._check(self.lib.sagips_combine_backward(self.h, ctypes.byref(R), dout.data_ptr(), _ptr(y) if want_dweight else None,
                                                     _ptr(weight), dy.data_ptr(), _ptr(dw)))
        return dy, dw

    def gen_forward_routed(self, W: Sequence, b: Sequence, x, offsets, slope: float = 0.2, out=None):
        """theta [n][out] = 1 + softplus(G_m(x)) with the member m that each row of x [n][in] belongs to:
        offsets[m] .. offsets[m + 1] - 1 (route's, [n_members + 1] int32).  Rows of no member are left as
        they were."""
        import torch
        self._enter()
        g, M = self._gen(W, b, slope)
        _check_tensor(x, "x", torch.float32, (x.shape[0], g.width[0]), self.device)
        _check_tensor(offsets, "offsets", torch.int32, (M + 1,), self.device)
        shape = (x.shape[0], g.width[g.n_layers])
        th = out if out is not None else x.new_empty(shape)
        if out is not None:
            _check_tensor(out, "out", torch.float32, shape, self.device)
        self._owned(th if out is None else None, W, b, x, offsets)
        self._check(self.lib.sagips_gen_forward_routed(self.h, ctypes.byref(g), x.data_ptr(), offsets.data_ptr(), x.shape[0],
                                                       th.data_ptr()))
        return th

    def gen_backward_routed(self, W: Sequence, b: Sequence, x, offsets, dL_dtheta, slope: float = 0.2, dW=None, db=None,
                            want_dx: bool = False, dx=None):
        """Gradients of sum <dL/dtheta, theta> for gen_forward_routed: (dW, db, dx) shaped like W, b and x;
        dx (None unless wanted or given) keeps its rows of no member."""
        import torch
        self._enter()
        g, M = self._gen(W, b, slope)
        _check_tensor(x, "x", torch.float32, (x.shape[0], g.width[0]), self.device)
        _check_tensor(offsets, "offsets", torch.int32, (M + 1,), self.device)
        _check_tensor(dL_dtheta, "dL_dtheta", torch.float32, (x.shape[0], g.width[g.n_layers]), self.device)
        new = []
        if dW is None:
            dW = [torch.empty_like(w) for w in W]
            new += dW
        if db is None:
            db = [torch.empty_like(v) for v in b]
            new += db
        if dx is not None:
            _check_tensor(dx, "dx", torch.float32, x.shape, self.device)
        elif want_dx:
            dx = torch.empty_like(x)
            new.append(dx)
        for l in range(g.n_layers):
            _check_tensor(dW[l], f"dW[{l}]", torch.float32, tuple(W[l].shape), self.device)
            _check_tensor(db[l], f"db[{l}]", torch.float32, tuple(b[l].shape), self.device)
        self._owned(new, W, b, x, offsets, dL_dtheta)
        pw = (ctypes.c_void_p * MAX_LAYERS)(*[t.data_ptr() for t in dW])
        pb = (ctypes.c_void_p * MAX_LAYERS)(*[t.data_ptr() for t in db])
        self._check(self.lib.sagips_gen_backward_routed(self.h, ctypes.byref(g), x.data_ptr(), offsets.data_ptr(), x.shape[0],
                                                        dL_dtheta.data_ptr(), pw, pb, _ptr(dx)))
        return dW, db, dx


_default: Dict[int, Context] = {}


def default_context(device: int = 0) -> Context:
    if device not in _default:
        _default[device] = Context(device)
    return _default[device]


def sample_events(theta, events_per_theta: int, seed: int, **kw):
    return default_context(theta.device.index).sample_events(theta, events_per_theta, seed, **kw)


def disc_fwd_bwd(W, b, real_x, **kw):
    return default_context(real_x.device.index).disc_fwd_bwd(W, b, real_x, **kw)


def param_grad(theta, events_per_theta: int, seed: int, **kw):
    return default_context(theta.device.index).param_grad(theta, events_per_theta, seed, **kw)
