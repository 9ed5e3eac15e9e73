"""ctypes binding of libmfmg.so (include/mfmg.h).  Argument marshalling only.

Every function here has the name of the C entry point it wraps.  Torch is
used for device memory, the current stream and pointers; all arithmetic of
the meta-gradient runs in the library's HIP kernels.  Loading fails loudly
when the library has not been built.
"""
from __future__ import annotations

import ctypes
import os
from ctypes import POINTER, c_char_p, c_double, c_float, c_int, c_int64, c_size_t, c_void_p

HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(HERE, "libmfmg.so")

MAX_LAYERS = 16
OK, ERR_INVALID_ARGUMENT, ERR_UNSUPPORTED, ERR_WORKSPACE, ERR_HIP, ERR_NUMERIC = 0, 1, 2, 3, 4, 5

EXPORTED = [
    "mfmg_problem_create", "mfmg_problem_destroy", "mfmg_query_sizes", "mfmg_inner_step",
    "mfmg_hvp_fwd_over_rev", "mfmg_meta_grad", "mfmg_status_string", "mfmg_last_error_message",
    "mfmg_timing_enable", "mfmg_timing_read", "mfmg_check_finite", "mfmg_meta_grad_noalloc",
    "mfmg_attn_create", "mfmg_attn_destroy", "mfmg_attn_ws_bytes", "mfmg_seq_plan_bytes",
    "mfmg_seq_plan", "mfmg_qk_rope_fwd", "mfmg_qk_rope_bwd", "mfmg_attn_fwd", "mfmg_attn_bwd",
]
ROPE_PLAIN, ROPE_LINEAR, ROPE_BASE, ROPE_PARTS = 0, 1, 2, 3
NOALLOC_SCRATCH_BYTES = 64 * 1024 * 1024   # MFMG_NOALLOC_SCRATCH_BYTES


class mfmg_problem_desc(ctypes.Structure):
    _fields_ = [
        ("kind", c_int), ("n_layers", c_int), ("widths", c_int * (MAX_LAYERS + 1)),
        ("act", c_int), ("loss", c_int), ("optimizer", c_int), ("meta", c_int),
        ("precision", c_int), ("has_bias", c_int), ("rows", c_int), ("val_rows", c_int),
        ("sgd_lr", c_float), ("adam_b1", c_float), ("adam_b2", c_float), ("adam_eps", c_float),
        ("d_model", c_int), ("n_heads", c_int), ("d_ff", c_int), ("vocab", c_int), ("seq", c_int),
        ("n_blocks", c_int), ("meta_hidden", c_int), ("ln_eps", c_float), ("rope_base", c_float),
        ("map_steps", c_int), ("ckpt_segment", c_int), ("fused_attention", c_int),
        ("block_remat", c_int), ("n_kv_heads", c_int), ("qk_norm", c_int), ("rope_dims", c_int),
        ("rope_interleaved", c_int), ("rope_scaling", c_int), ("rope_factor", c_float),
        ("rope_train_len", c_float), ("rope_slow", c_float), ("rope_fast", c_float),
        ("rope_mscale", c_float), ("docs", c_int), ("val_docs", c_int),
    ]


class mfmg_sizes(ctypes.Structure):
    _fields_ = [("n_theta", c_size_t), ("n_opt_state", c_size_t), ("n_eta", c_size_t),
                ("workspace_bytes", c_size_t), ("static_bytes", c_size_t),
                ("dynamic_bytes", c_size_t), ("step_workspace_bytes", c_size_t)]


class mfmg_batch(ctypes.Structure):
    _fields_ = [("x", c_void_p), ("y", c_void_p), ("rows", c_int64)]


class mfmg_attn_desc(ctypes.Structure):
    _fields_ = [("heads", c_int), ("kv_heads", c_int), ("head_dim", c_int), ("precision", c_int),
                ("scale", c_float), ("qk_norm", c_int), ("norm_eps", c_float), ("rope_dims", c_int),
                ("rope_interleaved", c_int), ("rope_base", c_float), ("rope_scaling", c_int),
                ("rope_factor", c_float), ("rope_train_len", c_float), ("rope_slow", c_float),
                ("rope_fast", c_float), ("rope_mscale", c_float)]


class mfmg_qkv(ctypes.Structure):   # mfmg_qkv and mfmg_qkv_out
    _fields_ = [("q", c_void_p), ("k", c_void_p), ("v", c_void_p),
                ("ldq", c_int64), ("ldk", c_int64), ("ldv", c_int64)]


class MfmgError(RuntimeError):
    def __init__(self, status: int, message: str):
        super().__init__(f"{message} (status {status})")
        self.status = status


_lib = None


def lib() -> ctypes.CDLL:
    """The loaded library; raises if it has not been built."""
    global _lib
    if _lib is not None:
        return _lib
    if not os.path.exists(LIB_PATH):
        raise RuntimeError(f"{LIB_PATH} is missing: build it with "
                           "`python -m paper_2505_00793_amd.build`")
    L = ctypes.CDLL(LIB_PATH)
    P = POINTER
    L.mfmg_problem_create.argtypes = [P(mfmg_problem_desc), P(c_void_p)]
    L.mfmg_problem_destroy.argtypes = [c_void_p]
    L.mfmg_problem_destroy.restype = None
    L.mfmg_query_sizes.argtypes = [c_void_p, c_int, P(mfmg_sizes)]
    L.mfmg_inner_step.argtypes = [c_void_p, c_void_p, c_void_p, c_void_p, P(mfmg_batch), c_int,
                                  c_void_p, c_void_p, c_void_p, c_void_p, c_void_p, c_size_t,
                                  c_void_p]
    L.mfmg_hvp_fwd_over_rev.argtypes = [c_void_p, c_void_p, c_void_p, P(mfmg_batch), c_int,
                                        c_void_p, c_void_p, c_void_p, c_void_p, c_void_p,
                                        c_size_t, c_void_p]
    L.mfmg_meta_grad.argtypes = [c_void_p, c_void_p, c_void_p, c_void_p, P(mfmg_batch), c_int,
                                 P(mfmg_batch), c_void_p, c_void_p, P(c_size_t), c_void_p,
                                 c_size_t, c_void_p]
    L.mfmg_meta_grad_noalloc.argtypes = [c_void_p, c_void_p, c_void_p, c_void_p, P(mfmg_batch),
                                         c_int, P(mfmg_batch), c_void_p, c_void_p, P(c_size_t),
                                         c_void_p]
    L.mfmg_check_finite.argtypes = [c_void_p, c_size_t, P(c_size_t), c_void_p, c_size_t,
                                    c_void_p]
    L.mfmg_status_string.argtypes = [c_int]
    L.mfmg_status_string.restype = c_char_p
    L.mfmg_last_error_message.argtypes = []
    L.mfmg_last_error_message.restype = c_char_p
    L.mfmg_timing_enable.argtypes = [c_int]
    L.mfmg_timing_read.argtypes = [c_int, P(c_int), P(c_double)]
    L.mfmg_attn_create.argtypes = [P(mfmg_attn_desc), P(c_void_p)]
    L.mfmg_attn_destroy.argtypes = [c_void_p]
    L.mfmg_attn_destroy.restype = None
    L.mfmg_attn_ws_bytes.argtypes = [c_void_p, c_int64, P(c_size_t)]
    L.mfmg_seq_plan_bytes.argtypes = [c_int64, c_int, P(c_size_t)]
    L.mfmg_seq_plan.argtypes = [c_void_p, c_int, c_int64, c_void_p, c_void_p, c_size_t, c_void_p]
    rows = [c_void_p, c_void_p, c_int64]   # an array, its tangent, their leading dimension
    head = [c_void_p, c_void_p, c_int64, c_int]   # handle, plan, n_tokens, n_seqs
    ws = [c_void_p, c_size_t, c_void_p]   # workspace, its bytes, stream
    L.mfmg_qk_rope_fwd.argtypes = head + rows + [c_void_p, c_void_p] + rows + [c_void_p]
    L.mfmg_qk_rope_bwd.argtypes = (head + rows + [c_void_p, c_void_p] + rows + rows
                                   + [c_void_p, c_void_p] + ws)
    L.mfmg_attn_fwd.argtypes = head + [P(mfmg_qkv), P(mfmg_qkv)] + rows + [c_void_p, c_void_p]
    L.mfmg_attn_bwd.argtypes = (head + [P(mfmg_qkv), P(mfmg_qkv)] + rows + [c_void_p] + rows
                                + [P(mfmg_qkv), P(mfmg_qkv)] + ws)
    for name in ("mfmg_attn_create", "mfmg_attn_ws_bytes", "mfmg_seq_plan_bytes", "mfmg_seq_plan",
                 "mfmg_qk_rope_fwd", "mfmg_qk_rope_bwd", "mfmg_attn_fwd", "mfmg_attn_bwd",
                 "mfmg_problem_create", "mfmg_query_sizes", "mfmg_inner_step",
                 "mfmg_hvp_fwd_over_rev", "mfmg_meta_grad", "mfmg_timing_enable",
                 "mfmg_timing_read", "mfmg_check_finite", "mfmg_meta_grad_noalloc"):
        getattr(L, name).restype = c_int
    _lib = L
    return L


def check(status: int) -> None:
    if status != OK:
        msg = lib().mfmg_last_error_message().decode()
        raise MfmgError(status, f"{lib().mfmg_status_string(status).decode()}: {msg}")


def _ptr(t):
    return None if t is None else c_void_p(t.data_ptr())


def _batch(x, y):
    """mfmg_batch of a CUDA tensor x (rows = its first dimension) and y (None: NULL)."""
    return mfmg_batch(x.data_ptr(), None if y is None else y.data_ptr(), x.shape[0])


def _stream():
    import torch
    return torch.cuda.current_stream().cuda_stream


def make_desc(*, widths, act=0, loss=1, optimizer=0, meta=0, precision=0, has_bias=True, rows=1,
              val_rows=1, sgd_lr=0.1, adam_b1=0.9, adam_b2=0.999, adam_eps=1e-8,
              kind=0, **transformer) -> mfmg_problem_desc:
    d = mfmg_problem_desc()
    d.kind = kind
    d.n_layers = len(widths) - 1
    for i, w in enumerate(widths):
        d.widths[i] = int(w)
    d.act, d.loss, d.optimizer, d.meta, d.precision = act, loss, optimizer, meta, precision
    d.has_bias = int(bool(has_bias))
    d.rows, d.val_rows = rows, val_rows
    d.sgd_lr, d.adam_b1, d.adam_b2, d.adam_eps = sgd_lr, adam_b1, adam_b2, adam_eps
    for k, v in transformer.items():
        setattr(d, k, v)
    return d


class Problem:
    """Owns an mfmg_problem_t handle."""

    def __init__(self, desc: mfmg_problem_desc):
        self._h = c_void_p()
        check(lib().mfmg_problem_create(ctypes.byref(desc), ctypes.byref(self._h)))
        self.desc = desc

    def __del__(self):
        h = getattr(self, "_h", None)
        if h is not None and h.value and _lib is not None:
            _lib.mfmg_problem_destroy(h)
            self._h = c_void_p()

    @property
    def handle(self):
        return self._h

    def mfmg_query_sizes(self, T: int) -> mfmg_sizes:
        s = mfmg_sizes()
        check(lib().mfmg_query_sizes(self._h, T, ctypes.byref(s)))
        return s

    def workspace(self, nbytes: int, device="cuda"):
        """A 256-byte-aligned uint8 CUDA tensor of at least nbytes (torch allocation)."""
        import torch
        return torch.empty(max(int(nbytes), 1), dtype=torch.uint8, device=device)

    def mfmg_inner_step(self, theta, opt_state, eta, x, y, step_index, theta_next,
                        opt_state_next=None, grad_out=None, loss_out=None, ws=None):
        b = _batch(x, y)
        if ws is None:
            ws = self.workspace(self.mfmg_query_sizes(1).step_workspace_bytes, theta.device)
        check(lib().mfmg_inner_step(self._h, _ptr(theta), _ptr(opt_state), _ptr(eta),
                                    ctypes.byref(b), step_index, _ptr(theta_next),
                                    _ptr(opt_state_next), _ptr(grad_out), _ptr(loss_out),
                                    _ptr(ws), ws.numel(), _stream()))

    def mfmg_hvp_fwd_over_rev(self, theta, eta, x, y, step_index, v, grad_out, hvp_out,
                              mvp_out=None, ws=None):
        b = _batch(x, y)
        if ws is None:
            ws = self.workspace(self.mfmg_query_sizes(1).step_workspace_bytes, theta.device)
        check(lib().mfmg_hvp_fwd_over_rev(self._h, _ptr(theta), _ptr(eta), ctypes.byref(b),
                                          step_index, _ptr(v), _ptr(grad_out), _ptr(hvp_out),
                                          _ptr(mvp_out), _ptr(ws), ws.numel(), _stream()))

    def mfmg_meta_grad(self, theta0, opt_state0, eta, xs, ys, vx, vy, d_eta_out,
                       val_loss_out=None, ws=None) -> int:
        """Returns peak bytes."""
        T = len(xs)
        arr = (mfmg_batch * T)(*[_batch(x, y) for x, y in zip(xs, ys)])
        vb = _batch(vx, vy)
        if ws is None:
            ws = self.workspace(self.mfmg_query_sizes(T).workspace_bytes, theta0.device)
        peak = c_size_t(0)
        check(lib().mfmg_meta_grad(self._h, _ptr(theta0), _ptr(opt_state0), _ptr(eta), arr, T,
                                   ctypes.byref(vb), _ptr(d_eta_out), _ptr(val_loss_out),
                                   ctypes.byref(peak), _ptr(ws), ws.numel(), _stream()))
        return peak.value

    def mfmg_meta_grad_noalloc(self, theta0, opt_state0, eta, xs, ys, vx, vy, d_eta_out,
                               val_loss_out=None) -> int:
        """mfmg_meta_grad on the library's static scratch (no workspace); returns peak bytes."""
        T = len(xs)
        arr = (mfmg_batch * T)(*[_batch(x, y) for x, y in zip(xs, ys)])
        vb = _batch(vx, vy)
        peak = c_size_t(0)
        check(lib().mfmg_meta_grad_noalloc(self._h, _ptr(theta0), _ptr(opt_state0), _ptr(eta),
                                           arr, T, ctypes.byref(vb), _ptr(d_eta_out),
                                           _ptr(val_loss_out), ctypes.byref(peak), _stream()))
        return peak.value


def make_attn_desc(*, heads, kv_heads=None, head_dim, precision=0, scale=0.0, qk_norm=False,
                   norm_eps=1e-6, rope_dims=0, rope_interleaved=False, rope_base=10000.0,
                   rope_scaling=ROPE_PLAIN, rope_factor=1.0, rope_train_len=0.0, rope_slow=1.0,
                   rope_fast=32.0, rope_mscale=0.0) -> mfmg_attn_desc:
    return mfmg_attn_desc(heads, heads if kv_heads is None else kv_heads, head_dim, precision, scale,
                          int(bool(qk_norm)), norm_eps, rope_dims, int(bool(rope_interleaved)),
                          rope_base, rope_scaling, rope_factor, rope_train_len, rope_slow, rope_fast,
                          rope_mscale)


def _bad(message: str):
    return MfmgError(ERR_INVALID_ARGUMENT, f"MFMG_ERR_INVALID_ARGUMENT: {message}")


def _check_dev(name, t, dtype, device: int):
    """t is a tensor of dtype on the device (None passes)."""
    if t is None:
        return
    if t.dtype != dtype:
        raise _bad(f"{name}: {t.dtype}, expected {dtype}")
    if t.get_device() != device:
        raise _bad(f"{name} is on {t.device}, expected the current device")


def _addr(t):
    return None if t is None else t.data_ptr()


def _device() -> int:
    """The current CUDA device (0 where there is none: no tensor is on it)."""
    import torch
    return torch.cuda.current_device() if torch.cuda.is_initialized() else 0


def _raw_stream(device: int) -> int:
    """The current stream's handle, without a stream object where torch offers it."""
    import torch
    raw = getattr(torch._C, "_cuda_getCurrentRawStream", None)
    return raw(device) if raw else torch.cuda.current_stream(device).cuda_stream


class SeqPlan:
    """The plan of a batch's sequences (mfmg_seq_plan): device memory with its sizes."""

    def __init__(self, data, n_tokens: int, n_seqs: int):
        self.data, self.n_tokens, self.n_seqs = data, n_tokens, n_seqs


def mfmg_seq_plan(cu_seqlens, n_tokens: int, positions=None, plan=None) -> SeqPlan:
    """Plan of n_tokens rows holding len(cu_seqlens) - 1 sequences; `plan` reuses the device
    memory of an earlier one of the same sizes."""
    import torch
    device = _device()
    _check_dev("cu_seqlens", cu_seqlens, torch.int32, device)
    _check_dev("positions", positions, torch.int32, device)
    m = cu_seqlens.numel() - 1
    if m < 0 or not cu_seqlens.is_contiguous():
        raise _bad("cu_seqlens must be contiguous with at least one entry")
    if positions is not None and (positions.numel() != n_tokens or not positions.is_contiguous()):
        raise _bad("positions must be contiguous, one per token")
    if plan is None:
        n = c_size_t(0)
        check(lib().mfmg_seq_plan_bytes(n_tokens, m, ctypes.byref(n)))
        plan = SeqPlan(torch.empty(n.value, dtype=torch.uint8, device=cu_seqlens.device), n_tokens, m)
    elif (plan.n_tokens, plan.n_seqs) != (n_tokens, m):
        raise _bad("the plan to reuse is of other sizes")
    _check_dev("plan", plan.data, torch.uint8, device)
    check(lib().mfmg_seq_plan(_addr(cu_seqlens), m, n_tokens, _addr(positions), _addr(plan.data),
                              plan.data.numel(), _stream()))
    return plan


class Attention:
    """Owns an mfmg_attn_t handle.  Row arguments are 2-D tensors [n_tokens][columns] whose rows
    are contiguous (views of wider rows pass); optional ones may be None as in the C calls."""

    def __init__(self, desc: mfmg_attn_desc):
        import torch
        self._h = c_void_p()
        check(lib().mfmg_attn_create(ctypes.byref(desc), ctypes.byref(self._h)))
        self.desc = desc
        self.dtype = torch.bfloat16 if desc.precision == 1 else torch.float32
        self.float32 = torch.float32
        self.uint8 = torch.uint8
        self.q_cols = desc.heads * desc.head_dim
        self.kv_cols = desc.kv_heads * desc.head_dim
        self.cols = self.q_cols + 2 * self.kv_cols
        self.gain_shape = (2, desc.head_dim)

    def __del__(self):
        h = getattr(self, "_h", None)
        if h is not None and h.value and _lib is not None:
            _lib.mfmg_attn_destroy(h)
            self._h = c_void_p()

    def mfmg_attn_ws_bytes(self, n_tokens: int) -> int:
        n = c_size_t(0)
        check(lib().mfmg_attn_ws_bytes(self._h, n_tokens, ctypes.byref(n)))
        return n.value

    def workspace(self, n_tokens: int, device="cuda"):
        """A workspace of the backward calls (torch allocation)."""
        import torch
        return torch.empty(max(self.mfmg_attn_ws_bytes(n_tokens), 1), dtype=torch.uint8, device=device)

    @staticmethod
    def _rows(name, t, cols, dtype, n, device):
        """The leading dimension of row tensor t."""
        if t.dtype != dtype or t.get_device() != device:
            _check_dev(name, t, dtype, device)
        if t.shape != (n, cols):
            raise _bad(f"{name}: shape {tuple(t.shape)}, expected ({n}, {cols})")
        if n < 2:
            return cols
        ld, one = t.stride()
        if one != 1:
            raise _bad(f"{name}: rows are not contiguous")
        return ld

    def _pair(self, name, t, td, cols, dtype, n, device):
        """The one leading dimension of an array and its tangent (either may be None)."""
        ld = 0 if t is None else self._rows(name, t, cols, dtype, n, device)
        if td is not None:
            ldd = self._rows(name + "d", td, cols, dtype, n, device)
            if t is not None and ld != ldd:
                raise _bad(f"{name} and {name}d have different row strides")
            ld = ldd
        return ld

    def _gains(self, device, *ts):
        for name, t in zip(("gain", "gaind", "dgain", "dgaind"), ts):
            if t is not None:
                _check_dev(name, t, self.float32, device)
                if t.shape != self.gain_shape or not t.is_contiguous():
                    raise _bad(f"{name}: expected a contiguous {self.gain_shape}")

    def _qkv(self, name, q, k, v, n, device):
        """mfmg_qkv of three row tensors; None if none is given."""
        if q is None and k is None and v is None:
            return None
        if q is None or k is None or v is None:
            raise _bad(f"{name}: q, k and v go together")
        rows = self._rows
        return ctypes.byref(mfmg_qkv(
            q.data_ptr(), k.data_ptr(), v.data_ptr(),
            rows(name + ".q", q, self.q_cols, self.dtype, n, device),
            rows(name + ".k", k, self.kv_cols, self.dtype, n, device),
            rows(name + ".v", v, self.kv_cols, self.dtype, n, device)))

    def _head(self, plan, device, ws=None):
        """The first arguments of every call."""
        _check_dev("plan", plan.data, self.uint8, device)
        _check_dev("ws", ws, self.uint8, device)
        return self._h, plan.data.data_ptr(), plan.n_tokens, plan.n_seqs

    def mfmg_qk_rope_fwd(self, plan, x, y, gain=None, xd=None, gaind=None, yd=None):
        n, w, dev = plan.n_tokens, self.cols, _device()
        ldx = self._pair("x", x, xd, w, self.float32, n, dev)
        ldy = self._pair("y", y, yd, w, self.dtype, n, dev)
        self._gains(dev, gain, gaind)
        check(lib().mfmg_qk_rope_fwd(*self._head(plan, dev), _addr(x), _addr(xd), ldx, _addr(gain),
                                     _addr(gaind), _addr(y), _addr(yd), ldy, _raw_stream(dev)))

    def mfmg_qk_rope_bwd(self, plan, dy, dx, x=None, gain=None, dgain=None, dyd=None, dxd=None,
                         xd=None, gaind=None, dgaind=None, ws=None):
        n, w, dev = plan.n_tokens, self.cols, _device()
        ldx = self._pair("x", x, xd, w, self.float32, n, dev)
        lddy = self._pair("dy", dy, dyd, w, self.dtype, n, dev)
        lddx = self._pair("dx", dx, dxd, w, self.dtype, n, dev)
        self._gains(dev, gain, gaind, dgain, dgaind)
        if ws is None:
            ws = self.workspace(n, dy.device)
        check(lib().mfmg_qk_rope_bwd(*self._head(plan, dev, ws), _addr(x), _addr(xd), ldx, _addr(gain),
                                     _addr(gaind), _addr(dy), _addr(dyd), lddy, _addr(dx), _addr(dxd),
                                     lddx, _addr(dgain), _addr(dgaind), _addr(ws), ws.numel(), _raw_stream(dev)))

    def _stats(self, stats, n, device):
        _check_dev("stats", stats, self.float32, device)
        if stats.numel() != 2 * self.desc.heads * n or not stats.is_contiguous():
            raise _bad(f"stats: expected a contiguous (2, {self.desc.heads}, {n})")
        return stats.data_ptr()

    def mfmg_attn_fwd(self, plan, q, k, v, o, stats, qd=None, kd=None, vd=None, od=None):
        n, dev = plan.n_tokens, _device()
        ldo = self._pair("o", o, od, self.q_cols, self.dtype, n, dev)
        check(lib().mfmg_attn_fwd(*self._head(plan, dev), self._qkv("x", q, k, v, n, dev),
                                  self._qkv("xd", qd, kd, vd, n, dev), _addr(o), _addr(od), ldo,
                                  self._stats(stats, n, dev), _raw_stream(dev)))

    def mfmg_attn_bwd(self, plan, q, k, v, o, stats, g, dq, dk, dv, qd=None, kd=None, vd=None,
                      od=None, dod=None, dqd=None, dkd=None, dvd=None, ws=None):
        n, dev = plan.n_tokens, _device()
        ldo = self._pair("o", o, od, self.q_cols, self.dtype, n, dev)
        ldg = self._pair("g", g, dod, self.q_cols, self.dtype, n, dev)
        if ws is None:
            ws = self.workspace(n, o.device)
        check(lib().mfmg_attn_bwd(*self._head(plan, dev, ws), self._qkv("x", q, k, v, n, dev),
                                  self._qkv("xd", qd, kd, vd, n, dev), _addr(o), _addr(od), ldo,
                                  self._stats(stats, n, dev), _addr(g), _addr(dod), ldg,
                                  self._qkv("dx", dq, dk, dv, n, dev),
                                  self._qkv("dxd", dqd, dkd, dvd, n, dev), _addr(ws), ws.numel(),
                                  _raw_stream(dev)))


def mfmg_check_finite(x, ws=None) -> int:
    """Number of NaN / infinite entries of the float32 CUDA tensor x (synchronises the
    current stream); raises MfmgError (status ERR_NUMERIC) when it is not zero."""
    import torch
    if ws is None:
        ws = torch.empty(256, dtype=torch.uint8, device=x.device)
    n = c_size_t(0)
    check(lib().mfmg_check_finite(_ptr(x), x.numel(), ctypes.byref(n), _ptr(ws), ws.numel(),
                                  _stream()))
    return n.value


def mfmg_timing_enable(enable: bool) -> None:
    check(lib().mfmg_timing_enable(int(enable)))


def mfmg_timing_read(kernel_class: int):
    n = c_int(0)
    ms = c_double(0.0)
    check(lib().mfmg_timing_read(kernel_class, ctypes.byref(n), ctypes.byref(ms)))
    return n.value, ms.value
