"""Thin binding of libhoccl.so: same names as include/hoccl.h, argument marshalling only (the diagnostics of
include/hoccl_diag.h are bound in diag.py).  The calls of a program's inner loop (collectives, send/recv) are marshalled in C
(csrc/calls.c), everything else with ctypes; both use the one library that lib() loads.

Buffers are given as objects with a `data_ptr()` method (torch tensors) or as integer device
addresses; streams as `torch.cuda.Stream`, raw integer handles or None (the current torch stream).
Nothing here computes: every step of a collective runs inside the library.  If the library cannot
be built or loaded the import of `lib()` raises; there is no fallback.
"""
from __future__ import annotations

import ctypes
from typing import Optional, Sequence

from . import build as _build

OK, ERR_INVALID_ARG, ERR_UNSUPPORTED, ERR_CUDA, ERR_MISMATCH, ERR_PENDING, ERR_SCRATCH, ERR_INTERNAL, ERR_TIMEOUT = range(9)
FLOAT32, BFLOAT16 = 0, 1
SUM = 0
PATH_CE, PATH_SM, PATH_CE_HOST = 0, 1, 2

DTYPES = {"fp32": FLOAT32, "bf16": BFLOAT16}
STATES = {"fp32": 0, "8bit": 1}   # how the averages of an AdamW step are kept
STATE_BLOCK = 256                 # elements that share a scale in 8-bit states

EXPORTS = [   # every function include/hoccl.h declares
    "hoccl_comm_init", "hoccl_comm_destroy", "hoccl_scratch_bytes", "hoccl_scratch_bytes_direct",
    "hoccl_comm_set_scratch", "hoccl_comm_set_staging", "hoccl_comm_set_host_staging", "hoccl_comm_set_path",
    "hoccl_comm_set_param", "hoccl_comm_get_param", "hoccl_allreduce", "hoccl_reduce_scatter", "hoccl_allgather",
    "hoccl_alltoall", "hoccl_alltoallv", "hoccl_send", "hoccl_recv", "hoccl_comm_pending", "hoccl_comm_async_error",
    "hoccl_comm_handshakes", "hoccl_comm_proxy_stats", "hoccl_host_allreduce", "hoccl_error_string", "hoccl_last_cuda_error", "hoccl_last_stats",
    "hoccl_profile_reset", "hoccl_allreduce_static", "hoccl_sched_build", "hoccl_sched_destroy",
    "hoccl_sched_num_stages", "hoccl_sched_stage_tau", "hoccl_sched_total_tau", "hoccl_sched_lower_bound",
    "hoccl_sched_matrix", "hoccl_sched_num_flows", "hoccl_sched_get_flow", "hoccl_sched_queue_len",
    "hoccl_sched_queue_get", "hoccl_adamw_create", "hoccl_adamw_destroy", "hoccl_adamw_step", "hoccl_sharded_adamw",
    "hoccl_grad_norm_scratch_bytes", "hoccl_grad_norm", "hoccl_route_scratch_bytes", "hoccl_route", "hoccl_route_backward",
]


class Stats(ctypes.Structure):
    _fields_ = [
        ("host_launch_us", ctypes.c_double), ("n_moves", ctypes.c_long), ("n_move_launches", ctypes.c_long),
        ("n_sum_launches", ctypes.c_long), ("max_sum_ctas", ctypes.c_long), ("max_copy_ctas", ctypes.c_long),
        ("n_pieces", ctypes.c_long), ("graph_hit", ctypes.c_long), ("sum_kernel_ms", ctypes.c_double),
        ("sum_kernel_launches_timed", ctypes.c_long), ("sum_kernel_bytes", ctypes.c_double),
        ("copy_kernel_ms", ctypes.c_double), ("copy_kernel_launches_timed", ctypes.c_long), ("copy_kernel_bytes", ctypes.c_double),
        ("n_order_launches", ctypes.c_long),
    ]

    def as_dict(self):
        return {k: getattr(self, k) for k, _ in self._fields_}


class SchedFlow(ctypes.Structure):
    _fields_ = [("src", ctypes.c_int), ("dst", ctypes.c_int), ("cls", ctypes.c_int), ("origin_src", ctypes.c_int),
                ("origin_dst", ctypes.c_int), ("bytes", ctypes.c_uint64), ("origin_offset", ctypes.c_uint64)]


class AdamTensor(ctypes.Structure):
    _fields_ = [("param", ctypes.c_void_p), ("grad", ctypes.c_void_p), ("exp_avg", ctypes.c_void_p), ("exp_avg_sq", ctypes.c_void_p),
                ("master", ctypes.c_void_p), ("exp_avg_scale", ctypes.c_void_p), ("exp_avg_sq_scale", ctypes.c_void_p),
                ("count", ctypes.c_size_t), ("weight_decay", ctypes.c_float)]


FLOW_NATIVE, FLOW_RDMA, FLOW_FWD_SEND, FLOW_FWD_RECV = 0, 1, 2, 3


class HocclError(RuntimeError):
    def __init__(self, code: int, what: str, detail: str = ""):
        self.code = code
        super().__init__("%s failed: %s (code %d)%s" % (what, error_string(code), code, (": " + detail) if detail else ""))


_lib = None
_calls = None   # the module built from csrc/calls.c


def library_path() -> str:
    """Path of libhoccl.so (built first if it is missing or stale)."""
    return _build.build()


def lib() -> ctypes.CDLL:
    """Builds (if stale) and loads libhoccl.so.  Raises if that is not possible."""
    global _lib, _calls
    if _lib is not None:
        return _lib
    path = _build.build()
    L = ctypes.CDLL(path)
    vp, vpp, sz, i, l = ctypes.c_void_p, ctypes.POINTER(ctypes.c_void_p), ctypes.c_size_t, ctypes.c_int, ctypes.c_long
    sigs = {
        "hoccl_comm_init": (i, [vpp, i, i]),
        "hoccl_comm_destroy": (i, [vp]),
        "hoccl_scratch_bytes": (sz, [i, sz, i]),
        "hoccl_scratch_bytes_direct": (sz, [i, sz, i]),
        "hoccl_comm_set_scratch": (i, [vp, vp, sz]),
        "hoccl_comm_set_staging": (i, [vp, vp, sz]),
        "hoccl_comm_set_host_staging": (i, [vp, vp, sz]),
        "hoccl_comm_set_path": (i, [vp, i]),
        "hoccl_comm_set_param": (i, [vp, ctypes.c_char_p, l]),
        "hoccl_comm_get_param": (i, [vp, ctypes.c_char_p, ctypes.POINTER(l)]),
        "hoccl_allreduce": (i, [vpp, vpp, sz, i, i, vp, vp]),
        "hoccl_reduce_scatter": (i, [vpp, vpp, sz, i, i, vp, vp]),
        "hoccl_allgather": (i, [vpp, vpp, sz, i, vp, vp]),
        "hoccl_alltoall": (i, [vpp, vpp, sz, i, vp, vp]),
        "hoccl_alltoallv": (i, [vpp, ctypes.POINTER(sz), ctypes.POINTER(sz), vpp, ctypes.POINTER(sz), i, vp, vp]),
        "hoccl_sched_build": (i, [vpp, i, i, ctypes.c_double, ctypes.c_double, ctypes.POINTER(ctypes.c_uint64), ctypes.c_uint64]),
        "hoccl_sched_destroy": (None, [vp]),
        "hoccl_sched_num_stages": (i, [vp]),
        "hoccl_sched_stage_tau": (ctypes.c_double, [vp, i]),
        "hoccl_sched_total_tau": (ctypes.c_double, [vp]),
        "hoccl_sched_lower_bound": (ctypes.c_double, [vp]),
        "hoccl_sched_matrix": (i, [vp, i, ctypes.POINTER(ctypes.c_uint64)]),
        "hoccl_sched_num_flows": (i, [vp, i]),
        "hoccl_sched_get_flow": (i, [vp, i, i, ctypes.POINTER(SchedFlow)]),
        "hoccl_sched_queue_len": (i, [vp, i, i]),
        "hoccl_sched_queue_get": (i, [vp, i, i, i, ctypes.POINTER(i), ctypes.POINTER(ctypes.c_uint64), ctypes.POINTER(ctypes.c_uint64)]),
        "hoccl_send": (i, [vp, sz, i, i, i, vp, vp]),
        "hoccl_recv": (i, [vp, sz, i, i, i, vp, vp]),
        "hoccl_comm_pending": (i, [vp]),
        "hoccl_comm_async_error": (i, [vp, i]),
        "hoccl_comm_handshakes": (l, [vp]),
        "hoccl_comm_proxy_stats": (i, [vp, ctypes.POINTER(ctypes.c_double), ctypes.POINTER(ctypes.c_double), i]),
        "hoccl_host_allreduce": (i, [vpp, vpp, sz, i, i, vp, vp]),
        "hoccl_allreduce_static": (i, [vpp, vpp, sz, i, i, i, vp]),
        "hoccl_adamw_create": (i, [vpp, ctypes.POINTER(AdamTensor), i, i, i, i]),
        "hoccl_adamw_destroy": (None, [vp]),
        "hoccl_grad_norm_scratch_bytes": (sz, []),
        "hoccl_route_scratch_bytes": (sz, [i, sz, i]),
        "hoccl_error_string": (ctypes.c_char_p, [i]),
        "hoccl_last_cuda_error": (ctypes.c_char_p, [vp]),
        "hoccl_last_stats": (i, [vp, ctypes.POINTER(Stats)]),
        "hoccl_profile_reset": (i, [vp]),
    }
    for name, (res, args) in sigs.items():
        fn = getattr(L, name)
        fn.restype = res
        fn.argtypes = args
    from . import _calls as calls

    calls.bind(*[ctypes.cast(getattr(L, "hoccl_" + name), vp).value for name in _INNER_LOOP])
    _lib, _calls = L, calls
    return L


# functions called through csrc/calls.c, in the order its bind() takes them
_INNER_LOOP = ["allreduce", "reduce_scatter", "host_allreduce", "allgather", "alltoall", "alltoallv", "send", "recv", "allreduce_static",
               "adamw_step", "sharded_adamw", "grad_norm", "route", "route_backward"]


def error_string(code: int) -> str:
    return lib().hoccl_error_string(code).decode()


def _ptr(x) -> int:
    if x is None:
        return 0
    if hasattr(x, "data_ptr"):
        return int(x.data_ptr())
    return int(x)


def _ptr_array(xs: Sequence):
    arr = (ctypes.c_void_p * len(xs))()
    for k, x in enumerate(xs):
        arr[k] = _ptr(x)
    return arr


def _stream(s) -> int:
    if s is None:
        import torch

        return int(torch.cuda.current_stream().cuda_stream)
    if hasattr(s, "cuda_stream"):
        return int(s.cuda_stream)
    return int(s)


def _dtype(d) -> int:
    if isinstance(d, str):
        return DTYPES[d]
    return int(d)


def _state(s) -> int:
    return STATES[s] if isinstance(s, str) else int(s)


def _count_of(x, k: int, counts) -> int:
    return int(counts[k]) if counts is not None else int(x.numel())


def _check_elements(x, what: str, count: int, size: int) -> None:
    """A tensor that the library is to take for `count` elements of `size` bytes; an address cannot be checked."""
    if hasattr(x, "element_size") and (not x.is_contiguous() or x.numel() < count or x.element_size() != size):
        raise ValueError("%s: %d contiguous elements of %d bytes are wanted" % (what, count, size))


# bytes of an element, by the library's numbers for dtypes and states; of numbers that it does not know none is checked: it refuses them
_DTYPE_SIZE, _STATE_SIZE = {FLOAT32: 4, BFLOAT16: 2}, {0: 4, 1: 1}


class Tensors:
    """A list of vectors marshalled once (grad_norm): their addresses, their lengths (of contiguous tensors, or `counts`) and dtype."""

    def __init__(self, xs: Sequence, dtype, counts: Optional[Sequence[int]] = None):
        self.n, self.dtype, self._keep = len(xs), _dtype(dtype), list(xs)
        self._ptrs = _ptr_array(xs)
        self._counts = (ctypes.c_size_t * self.n)(*[_count_of(x, k, counts) for k, x in enumerate(xs)])
        if self.dtype in _DTYPE_SIZE:
            for k, x in enumerate(xs):
                _check_elements(x, "tensor %d" % k, self._counts[k], _DTYPE_SIZE[self.dtype])
        self._at = ctypes.addressof(self._ptrs), ctypes.addressof(self._counts)


class AdamTensors:
    """The table of one hoccl_adamw_plan_t: lists of as many tensors (or addresses, with `counts`) as there are weights.

    state "fp32" or "8bit" (then with scales); weight_decay: one number, or one for each tensor.  The tensors are kept alive."""

    def __init__(self, params: Sequence, grads: Sequence, exp_avg: Sequence, exp_avg_sq: Sequence, param_dtype, grad_dtype, state="fp32", master=None,
                 exp_avg_scale=None, exp_avg_sq_scale=None, weight_decay=0.0, counts: Optional[Sequence[int]] = None):
        self._h = ctypes.c_void_p()
        n = len(params)
        lists = {"param": params, "grad": grads, "exp_avg": exp_avg, "exp_avg_sq": exp_avg_sq, "master": master, "exp_avg_scale": exp_avg_scale,
                 "exp_avg_sq_scale": exp_avg_sq_scale}
        table = (AdamTensor * max(n, 1))()
        for k in range(n):
            table[k].count = _count_of(params[k], k, counts)
            table[k].weight_decay = float(weight_decay[k]) if hasattr(weight_decay, "__getitem__") else float(weight_decay)
        blocks = [(table[k].count + STATE_BLOCK - 1) // STATE_BLOCK for k in range(n)]
        param_dtype, grad_dtype, state = _dtype(param_dtype), _dtype(grad_dtype), _state(state)
        known = param_dtype in _DTYPE_SIZE and grad_dtype in _DTYPE_SIZE and state in _STATE_SIZE
        size = {"param": _DTYPE_SIZE.get(param_dtype), "grad": _DTYPE_SIZE.get(grad_dtype), "exp_avg": _STATE_SIZE.get(state), "exp_avg_sq": _STATE_SIZE.get(state)}
        for name, xs in lists.items():
            if xs is None:
                continue
            if len(xs) != n:
                raise ValueError("%d %s tensors, %d wanted" % (len(xs), name, n))
            for k, x in enumerate(xs):
                if known and (state == STATES["8bit"] or not name.endswith("_scale")):   # (scales beside binary32 states are not read)
                    _check_elements(x, "%s[%d]" % (name, k), blocks[k] if name.endswith("_scale") else table[k].count, size.get(name, 4))
                setattr(table[k], name, _ptr(x))
        rc = lib().hoccl_adamw_create(ctypes.byref(self._h), table, n, param_dtype, grad_dtype, state)
        if rc != OK:
            raise HocclError(rc, "hoccl_adamw_create")
        self._keep = {name: list(xs) for name, xs in lists.items() if xs is not None}

    def destroy(self):
        if self._h:
            lib().hoccl_adamw_destroy(self._h)
            self._h = ctypes.c_void_p()

    def __del__(self):
        try:
            self.destroy()
        except Exception:
            pass


def adamw_rates(lr: float, step: int, beta1: float = 0.9, beta2: float = 0.999, seed: int = 0):
    """The record that a captured AdamW step reads (hoccl_adamw_rates_t) as a CPU tensor of four 32-bit words, to be copied to the device between replays."""
    import math
    import struct

    import torch

    bias = [-math.expm1(step * math.log(b)) if b else 1.0 for b in (beta1, beta2)]
    return torch.frombuffer(bytearray(struct.pack("<fffI", lr, *bias, seed & 0xFFFFFFFF)), dtype=torch.int32)


class Comm:
    """Owner of one hoccl_comm_t.  Methods carry the C names without the prefix."""

    def __init__(self, R: int, device: int = 0):
        self._h = ctypes.c_void_p()
        self.R = R
        rc = lib().hoccl_comm_init(ctypes.byref(self._h), R, device)
        if rc != OK:
            self._h = ctypes.c_void_p()
            raise HocclError(rc, "hoccl_comm_init")
        self._keep = []

    # -- helpers
    def _check(self, rc: int, what: str):
        if rc != OK:
            raise HocclError(rc, what, self.last_cuda_error() if rc == ERR_CUDA else "")

    def last_cuda_error(self) -> str:
        return lib().hoccl_last_cuda_error(self._h).decode()

    def destroy(self):
        if self._h:
            rc = lib().hoccl_comm_destroy(self._h)
            if rc != ERR_PENDING:      # PENDING is the one case in which nothing was freed
                self._h = ctypes.c_void_p()
            return rc
        return OK

    def __del__(self):
        try:
            if self._h:
                lib().hoccl_comm_destroy(self._h)
        except Exception:
            pass

    # -- configuration
    def set_scratch(self, buf, nbytes: Optional[int] = None):
        if nbytes is None:
            nbytes = buf.numel() * buf.element_size() if buf is not None else 0
        self._keep = [b for b in self._keep if b[0] != "scratch"] + [("scratch", buf)]
        self._check(lib().hoccl_comm_set_scratch(self._h, _ptr(buf), nbytes), "hoccl_comm_set_scratch")

    def set_staging(self, buf, nbytes: Optional[int] = None):
        if nbytes is None:
            nbytes = buf.numel() * buf.element_size() if buf is not None else 0
        self._keep = [b for b in self._keep if b[0] != "staging"] + [("staging", buf)]
        self._check(lib().hoccl_comm_set_staging(self._h, _ptr(buf), nbytes), "hoccl_comm_set_staging")

    def set_host_staging(self, pinned, nbytes: Optional[int] = None):
        """Pinned host memory (e.g. a torch tensor created with pin_memory()) for the CE_HOST path."""
        if nbytes is None:
            nbytes = pinned.numel() * pinned.element_size() if pinned is not None else 0
        self._keep = [b for b in self._keep if b[0] != "host_staging"] + [("host_staging", pinned)]
        self._check(lib().hoccl_comm_set_host_staging(self._h, _ptr(pinned), nbytes), "hoccl_comm_set_host_staging")

    def set_path(self, path: int):
        self._check(lib().hoccl_comm_set_path(self._h, path), "hoccl_comm_set_path")

    def set_param(self, key: str, value: int):
        self._check(lib().hoccl_comm_set_param(self._h, key.encode(), value), "hoccl_comm_set_param(%s)" % key)

    def get_param(self, key: str) -> int:
        v = ctypes.c_long()
        self._check(lib().hoccl_comm_get_param(self._h, key.encode(), ctypes.byref(v)), "hoccl_comm_get_param(%s)" % key)
        return v.value

    # -- collectives (raise on error; the *_rc variants return the code)
    def allreduce_rc(self, send, recv, count, dtype, stream=None, op=SUM) -> int:
        return _calls.allreduce(self._h.value, send, recv, count, dtype, op, stream)

    def reduce_scatter_rc(self, send, recv, count, dtype, stream=None, op=SUM) -> int:
        return _calls.reduce_scatter(self._h.value, send, recv, count, dtype, op, stream)

    def allgather_rc(self, send, recv, count, dtype, stream=None) -> int:
        return _calls.allgather(self._h.value, send, recv, count, dtype, stream)

    def alltoall_rc(self, send, recv, count, dtype, stream=None) -> int:
        return _calls.alltoall(self._h.value, send, recv, count, dtype, stream)

    def alltoall(self, send, recv, count, dtype, stream=None):
        self._check(self.alltoall_rc(send, recv, count, dtype, stream), "hoccl_alltoall")

    def alltoallv_rc(self, send, sendcounts, sdispls, recv, rdispls, dtype, stream=None) -> int:
        return _calls.alltoallv(self._h.value, self.R, send, sendcounts, sdispls, recv, rdispls, dtype, stream)

    def alltoallv(self, send, sendcounts, sdispls, recv, rdispls, dtype, stream=None):
        self._check(self.alltoallv_rc(send, sendcounts, sdispls, recv, rdispls, dtype, stream), "hoccl_alltoallv")

    def allreduce(self, send, recv, count, dtype, stream=None, op=SUM):
        self._check(self.allreduce_rc(send, recv, count, dtype, stream, op), "hoccl_allreduce")

    def reduce_scatter(self, send, recv, count, dtype, stream=None, op=SUM):
        self._check(self.reduce_scatter_rc(send, recv, count, dtype, stream, op), "hoccl_reduce_scatter")

    def allgather(self, send, recv, count, dtype, stream=None):
        self._check(self.allgather_rc(send, recv, count, dtype, stream), "hoccl_allgather")

    def host_allreduce(self, h_send, h_recv, count, dtype, stream=None, op=SUM):
        self._check(_calls.host_allreduce(self._h.value, h_send, h_recv, count, dtype, op, stream), "hoccl_host_allreduce")

    # -- operators of a training step
    def _check_tokens(self, tokens):
        if len(tokens) != self.R:   # the library sees R of them: a missing one would be a rank without tokens
            raise ValueError("%d numbers of tokens, %d wanted" % (len(tokens), self.R))

    def adamw(self, tensors: AdamTensors, lr, step, beta1=0.9, beta2=0.999, eps=1e-8, grad_scale=1.0, factor=None, rates=None, seed=0, stream=None):
        """hoccl_adamw_step.  factor: device float (grad_norm's out[1:]); rates: device record (adamw_rates) in place of lr, step and seed."""
        self._check(_calls.adamw_step(self._h.value, tensors._h.value, lr, step, beta1, beta2, eps, grad_scale, factor, rates, seed, stream), "hoccl_adamw_step")

    def sharded_adamw(self, grads, params, exp_avg, exp_avg_sq, count, param_dtype, grad_dtype, lr, step, state="fp32", master=None, exp_avg_scale=None,
                      exp_avg_sq_scale=None, beta1=0.9, beta2=0.999, eps=1e-8, weight_decay=0.0, grad_scale=1.0, factor=None, rates=None, seed=0, stream=None):
        self._check(_calls.sharded_adamw(self._h.value, grads, params, exp_avg, exp_avg_sq, master, exp_avg_scale, exp_avg_sq_scale, count, param_dtype, grad_dtype,
                                         _state(state), weight_decay, lr, step, beta1, beta2, eps, grad_scale, factor, rates, seed, stream), "hoccl_sharded_adamw")

    def grad_norm(self, grads: Tensors, out, max_norm=float("inf"), stream=None):
        """out: two device floats, the norm and the factor that clips to max_norm, both of the gradients as they lie in memory (sums over R ranks that adamw scales
        by 1 / R: max_norm = R * the mean's)."""
        self._check(_calls.grad_norm(self._h.value, grads._at[0], grads._at[1], grads.n, grads.dtype, max_norm, out, stream), "hoccl_grad_norm")

    def route(self, logits, tokens, experts, topk, dtype, indices, weights, counts, loss, saved, balance_coef=0.01, z_coef=0.0, normalize=True, per_rank=False,
              ld=None, stream=None):
        """ld: elements from one row of the logits to the next (None: experts)."""
        self._check_tokens(tokens)
        self._check(_calls.route(self._h.value, logits, experts if ld is None else ld, tokens, experts, topk, dtype, normalize, per_rank, balance_coef, z_coef, indices,
                                 weights, counts, loss, saved, stream), "hoccl_route")

    def route_backward(self, logits, tokens, experts, topk, dtype, indices, saved, dweights, dloss, dlogits, normalize=True, per_rank=False, ld=None, dld=None,
                       stream=None):
        self._check_tokens(tokens)
        self._check(_calls.route_backward(self._h.value, logits, experts if ld is None else ld, tokens, experts, topk, dtype, normalize, per_rank, indices, saved, dweights,
                                          dloss, dlogits, experts if dld is None else dld, stream), "hoccl_route_backward")

    # -- point to point
    def send_rc(self, buf, count, dtype, src, dst, stream=None) -> int:
        return _calls.send(self._h.value, buf, count, dtype, src, dst, stream)

    def recv_rc(self, buf, count, dtype, src, dst, stream=None) -> int:
        return _calls.recv(self._h.value, buf, count, dtype, src, dst, stream)

    def send(self, buf, count, dtype, src, dst, stream=None):
        self._check(self.send_rc(buf, count, dtype, src, dst, stream), "hoccl_send")

    def recv(self, buf, count, dtype, src, dst, stream=None):
        self._check(self.recv_rc(buf, count, dtype, src, dst, stream), "hoccl_recv")

    def pending(self) -> int:
        return lib().hoccl_comm_pending(self._h)

    def async_error(self, clear: bool = False) -> int:
        return lib().hoccl_comm_async_error(self._h, int(clear))

    def handshakes(self) -> int:
        return int(lib().hoccl_comm_handshakes(self._h))

    def proxy_stats(self, reset: bool = False):
        """(busy_us, span_us) of the proxy thread: see hoccl_comm_proxy_stats."""
        b, s = ctypes.c_double(), ctypes.c_double()
        self._check(lib().hoccl_comm_proxy_stats(self._h, ctypes.byref(b), ctypes.byref(s), int(reset)), "hoccl_comm_proxy_stats")
        return b.value, s.value

    # -- diagnostics
    def last_stats(self) -> dict:
        st = Stats()
        self._check(lib().hoccl_last_stats(self._h, ctypes.byref(st)), "hoccl_last_stats")
        return st.as_dict()

    def profile_reset(self):
        self._check(lib().hoccl_profile_reset(self._h), "hoccl_profile_reset")

STATIC_SCRATCH_BYTES = 32 << 20


def allreduce_static(send, recv, count, dtype, R, stream=None, op=SUM) -> int:
    """hoccl_allreduce_static: all-reduce that allocates nothing and uses the library's fixed scratch array.
    Returns the result code (OK, or ERR_SCRATCH when the buffers are too large for the fixed array)."""
    lib()
    return _calls.allreduce_static(send, recv, count, dtype, op, R, stream)


def scratch_bytes(R: int, max_count: int, dtype) -> int:
    return int(lib().hoccl_scratch_bytes(R, max_count, _dtype(dtype)))


def scratch_bytes_direct(R: int, max_count: int, dtype) -> int:
    """Scratch bound with "rs_direct" set (R-1 inbox slots per rank)."""
    return int(lib().hoccl_scratch_bytes_direct(R, max_count, _dtype(dtype)))


def grad_norm_scratch_bytes() -> int:
    return int(lib().hoccl_grad_norm_scratch_bytes())


def route_scratch_bytes(R: int, max_tokens: int, experts: int) -> int:
    return int(lib().hoccl_route_scratch_bytes(R, max_tokens, experts))


class Schedule:
    """Host-only view of the collective scheduler's output for a traffic matrix C (G x G bytes, row = source)."""

    def __init__(self, C, gpus_per_node, bw_nvlink=400e9, bw_rdma=50e9, chunk_bytes=1 << 20):
        import numpy as np

        C = np.ascontiguousarray(C, dtype=np.uint64)
        G = C.shape[0]
        assert C.shape == (G, G)
        L = lib()
        h = ctypes.c_void_p()
        rc = L.hoccl_sched_build(ctypes.byref(h), G, gpus_per_node, bw_nvlink, bw_rdma, C.ctypes.data_as(ctypes.POINTER(ctypes.c_uint64)),
                                 chunk_bytes)
        if rc != OK:
            raise HocclError(rc, "hoccl_sched_build")
        self.G = G

        def mat(which):
            out = np.zeros((G, G), dtype=np.uint64)
            assert L.hoccl_sched_matrix(h, which, out.ctypes.data_as(ctypes.POINTER(ctypes.c_uint64))) == OK
            return out

        self.C, self.T = mat(-2), mat(-1)
        self.total_tau = L.hoccl_sched_total_tau(h)
        self.lower_bound = L.hoccl_sched_lower_bound(h)
        self.stages = []
        for s in range(L.hoccl_sched_num_stages(h)):
            flows = []
            for k in range(L.hoccl_sched_num_flows(h, s)):
                f = SchedFlow()
                assert L.hoccl_sched_get_flow(h, s, k, ctypes.byref(f)) == OK
                flows.append({name: getattr(f, name) for name, _ in SchedFlow._fields_})
            queues = []
            for g in range(G):
                q = []
                for k in range(L.hoccl_sched_queue_len(h, s, g)):
                    fl, off, nb = ctypes.c_int(), ctypes.c_uint64(), ctypes.c_uint64()
                    assert L.hoccl_sched_queue_get(h, s, g, k, ctypes.byref(fl), ctypes.byref(off), ctypes.byref(nb)) == OK
                    q.append((fl.value, off.value, nb.value))
                queues.append(q)
            self.stages.append({"matrix": mat(s), "tau": L.hoccl_sched_stage_tau(h, s), "flows": flows, "queues": queues})
        L.hoccl_sched_destroy(h)
