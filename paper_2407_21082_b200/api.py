"""Python binding of the C ABI in include/eexit.h: argument marshalling only.

Tensors are torch CUDA tensors (torch supplies device memory and the current stream); bf16 tensors may be
passed as torch.bfloat16 or as int16/uint16 bit patterns.  Every function launches on torch's current
stream and returns without synchronising, exactly like the C calls underneath.
"""
from __future__ import annotations

import torch

from . import _lib

EE_PATH_AUTO, EE_PATH_STREAM, EE_PATH_TCGEN05, EE_PATH_SKINNY = 0, 1, 2, 3


class EExitError(RuntimeError):
    def __init__(self, code: int, where: str):
        self.code = int(code)
        msg = _lib.load().ee_status_string(int(code)).decode()
        super().__init__(f"{where}: {msg} (ee_status {int(code)})")


def _check(code: int, where: str) -> None:
    if code != 0:
        raise EExitError(code, where)


def _ptr(t):
    return None if t is None else t.data_ptr()


def _stream():
    # torch.cuda.current_stream() builds a Stream object, four to five microseconds a call; this is the handle it would hold
    return torch._C._cuda_getCurrentRawStream(torch._C._cuda_getDevice())


def _bf16(t: torch.Tensor) -> torch.Tensor:
    if t.dtype in (torch.int16, torch.uint16):
        t = t.view(torch.bfloat16)
    if t.dtype != torch.bfloat16:
        raise TypeError(f"expected bf16 (or its 16-bit patterns), got {t.dtype}")
    return t


def _dev(t: torch.Tensor, name: str) -> torch.Tensor:
    if not t.is_cuda:
        raise ValueError(f"{name} must be a CUDA tensor")
    return t


def ee_exit_head_workspace_bytes(M: int, d: int, V: int) -> int:
    return int(_lib.load().ee_exit_head_workspace_bytes(int(M), int(d), int(V)))


def ee_exit_head_launches(M: int, d: int, V: int, path: int = EE_PATH_AUTO) -> int:
    return int(_lib.load().ee_exit_head_launches(int(M), int(d), int(V), int(path)))


def ee_workspace_init(workspace: torch.Tensor) -> None:
    _check(_lib.load().ee_workspace_init(_ptr(workspace), workspace.numel() * workspace.element_size(), _stream()),
           "ee_workspace_init")


def new_workspace(M: int, d: int, V: int, device="cuda") -> torch.Tensor:
    """Allocates (through torch) and initialises a workspace for ee_exit_head at these sizes."""
    nbytes = ee_exit_head_workspace_bytes(M, d, V)
    if nbytes == 0:
        raise EExitError(2, "ee_exit_head_workspace_bytes")
    ws = torch.empty(nbytes, dtype=torch.uint8, device=device)
    ee_workspace_init(ws)
    return ws


def new_outputs(M: int, device="cuda") -> dict:
    return dict(argmax=torch.empty(M, dtype=torch.int32, device=device),
                entropy=torch.empty(M, dtype=torch.float32, device=device),
                maxprob=torch.empty(M, dtype=torch.float32, device=device),
                exit_mask=torch.empty(M, dtype=torch.uint8, device=device))


_OUT_DTYPES = dict(argmax=torch.int32, entropy=torch.float32, maxprob=torch.float32, exit_mask=torch.uint8)


def _check_head_tensors(h, gamma, beta, W, tau, out=None):
    """Host-side checks shared by the single-head wrappers: everything the kernels take on trust (shapes, strides,
    dtypes, devices) is verified here, so that a bad argument raises ValueError instead of reaching the device.
    Returns h and W as bf16 tensors and (M, d, V)."""
    h, W = _bf16(_dev(h, "h")), _bf16(_dev(W, "W"))
    if h.dim() != 2 or W.dim() != 2:
        raise ValueError("h must be [M, d] and W [V, d]")
    M, d = h.shape
    V = W.shape[0]
    if W.shape[1] != d or not W.is_contiguous() or (M > 0 and h.stride(1) != 1):
        raise ValueError("W must be contiguous [V, d] and h row-major [M, d]")
    for name, t in (("gamma", gamma), ("beta", beta)):
        if not (isinstance(t, torch.Tensor) and t.is_cuda and t.dtype == torch.float32 and t.is_contiguous() and t.numel() == d):
            raise ValueError(f"{name} must be a contiguous float32 CUDA tensor of d = {d} elements")
        if t.device != h.device:
            raise ValueError(f"{name} is on {t.device}, h on {h.device}")
    if W.device != h.device:
        raise ValueError(f"W is on {W.device}, h on {h.device}")
    if isinstance(tau, torch.Tensor):
        if not (tau.is_cuda and tau.device == h.device and tau.dtype == torch.float32 and tau.is_contiguous() and tau.numel() == M):
            raise ValueError(f"a per-row tau must be a contiguous float32 CUDA tensor of M = {M} elements")
    if out is not None:
        for name, dtype in _OUT_DTYPES.items():
            t = out.get(name)
            if not (isinstance(t, torch.Tensor) and t.is_cuda and t.device == h.device and t.dtype == dtype and
                    t.is_contiguous() and t.numel() >= M):
                raise ValueError(f"out[{name!r}] must be a contiguous {dtype} CUDA tensor of at least M = {M} elements")
    return h, W, (M, d, V)


def _exit_head_args(h, gamma, beta, ln_eps, W, tau, out, workspace, path):
    h, W, (M, d, V) = _check_head_tensors(h, gamma, beta, W, tau, out)
    out = out if out is not None else new_outputs(M, h.device)
    workspace = workspace if workspace is not None else new_workspace(M, d, V, h.device)
    tau_t, tau_f = (tau, 0.0) if isinstance(tau, torch.Tensor) else (None, float(tau))
    args = (_ptr(h), h.stride(0) if M > 1 else max(h.stride(0), d), _ptr(gamma), _ptr(beta), float(ln_eps), _ptr(W),
            M, d, V, _ptr(tau_t), tau_f, _ptr(out["argmax"]), _ptr(out["entropy"]), _ptr(out["maxprob"]),
            _ptr(out["exit_mask"]), _ptr(workspace), workspace.numel(), _stream(), int(path))
    return args, out, (h, gamma, beta, W, tau_t, out, workspace)


def ee_exit_head(h, gamma, beta, ln_eps, W, tau, *, out=None, workspace=None, path=EE_PATH_AUTO) -> dict:
    """LayerNorm + exit-head projection + entropy / argmax / max-prob + exit decision for the rows of h.

    tau is a float (nats) or a float32 CUDA tensor [M] of per-row thresholds.  `out` (see new_outputs) and
    `workspace` (see new_workspace) are allocated when not given.
    """
    args, out, _ = _exit_head_args(h, gamma, beta, ln_eps, W, tau, out, workspace, path)
    _check(_lib.load().ee_exit_head_path(*args), "ee_exit_head")
    return out


class PreparedCall:
    """A C-ABI call with its arguments marshalled once, for loops that repeat the same call.

    Holds references to the tensors so that their memory stays alive; the stream is the one that was current
    at preparation time.  Calling it launches and returns, like the function it wraps.
    """
    __slots__ = ("_fn", "_args", "_where", "_keep", "out")

    def __init__(self, fn, args, where, keep, out):
        import ctypes as C
        self._fn = fn
        self._args = tuple(C.c_void_p(a) if (t is C.c_void_p) else t(a) for a, t in zip(args, fn.argtypes))
        self._where, self._keep, self.out = where, keep, out

    def __call__(self):
        code = self._fn(*self._args)
        if code:
            raise EExitError(code, self._where)
        return self.out


def ee_exit_head_multi_workspace_bytes(n_heads: int, M: int, d: int, V: int) -> int:
    return int(_lib.load().ee_exit_head_multi_workspace_bytes(int(n_heads), int(M), int(d), int(V)))


def ee_exit_head_multi_launches(n_heads: int, M: int, d: int, V: int) -> int:
    return int(_lib.load().ee_exit_head_multi_launches(int(n_heads), int(M), int(d), int(V)))


def _multi_args(heads, ln_eps, workspace):
    """heads: list of dicts with h, gamma, beta, W, tau and optionally out (see new_outputs)."""
    n = len(heads)
    arr = (_lib.EEHead * n)()
    keep, outs = [], []
    M, d = _bf16(heads[0]["h"]).shape
    V = heads[0]["W"].shape[0]
    for i, hd in enumerate(heads):
        h, W = _bf16(_dev(hd["h"], "h")), _bf16(_dev(hd["W"], "W"))
        if h.shape != (M, d) or W.shape != (V, d) or not W.is_contiguous() or h.stride(1) != 1:
            raise ValueError("all heads must share M, d, V; W contiguous [V, d]; h row-major [M, d]")
        out = hd.get("out") or new_outputs(M, h.device)
        tau = hd["tau"]
        tau_t, tau_f = (tau, 0.0) if isinstance(tau, torch.Tensor) else (None, float(tau))
        e = arr[i]
        e.h, e.ld_h, e.gamma, e.beta, e.W = _ptr(h), (h.stride(0) if M > 1 else max(h.stride(0), d)), _ptr(hd["gamma"]), _ptr(hd["beta"]), _ptr(W)
        e.tau_per_row, e.tau = _ptr(tau_t), tau_f
        e.argmax, e.entropy, e.maxprob, e.exit_mask = (_ptr(out[k]) for k in ("argmax", "entropy", "maxprob", "exit_mask"))
        keep.append((h, W, hd["gamma"], hd["beta"], tau_t, out))
        outs.append(out)
    if workspace is None:
        nbytes = ee_exit_head_multi_workspace_bytes(n, M, d, V)
        workspace = torch.empty(nbytes, dtype=torch.uint8, device=heads[0]["h"].device)
        ee_workspace_init(workspace)
    args = (arr, n, float(ln_eps), M, d, V, _ptr(workspace), workspace.numel(), _stream())
    return args, outs, (arr, keep, workspace)


def ee_exit_head_multi(heads, ln_eps, *, workspace=None) -> list:
    """ee_exit_head for several heads on batches of the same shape in one call; returns one output dict per head."""
    args, outs, _ = _multi_args(heads, ln_eps, workspace)
    _check(_lib.load().ee_exit_head_multi(*args), "ee_exit_head_multi")
    return outs


class PreparedMulti:
    """ee_exit_head_multi for a loop that repeats the call: the host work (argument checks, tensor maps, launch shapes)
    is done once here (ee_exit_head_plan_init) and a call only launches (ee_exit_head_plan_run) on the stream that was
    current at preparation time.  More heads than a plan takes fall back to ee_exit_head_multi with its argument
    block built once."""
    __slots__ = ("_args", "_keep", "out", "_plan", "_stream", "_run")

    def __init__(self, heads, ln_eps, workspace=None):
        import ctypes as C
        self._args, self.out, self._keep = _multi_args(heads, ln_eps, workspace)
        self._plan = None
        arr, n, eps, M, d, V, ws, ws_bytes, stream = self._args
        if 1 <= n <= _lib.EE_PLAN_MAX_HEADS and M >= 1:
            self._plan = _lib.EEExitHeadPlan()
            _check(_lib.load().ee_exit_head_plan_init(C.byref(self._plan), arr, n, eps, M, d, V, ws, ws_bytes), "ee_exit_head_plan_init")
            self._stream = C.c_void_p(stream)
            self._plan = C.byref(self._plan), self._plan          # the reference passed to C, and the object it refers to
            self._run = _lib.load().ee_exit_head_plan_run

    def __call__(self):
        code = self._run(self._plan[0], self._stream) if self._plan is not None else _lib.load().ee_exit_head_multi(*self._args)
        if code:
            raise EExitError(code, "ee_exit_head_multi")
        return self.out


def ee_exit_head_top2(h, gamma, beta, ln_eps, W, tau, *, out=None, workspace=None) -> dict:
    """ee_exit_head plus out["top2gap"]: the difference between the two largest probabilities of every row."""
    h, W, (M, d, V) = _check_head_tensors(h, gamma, beta, W, tau, out)
    if out is None:
        out = new_outputs(M, h.device)
        out["top2gap"] = torch.empty(M, dtype=torch.float32, device=h.device)
    if workspace is None:
        workspace = new_workspace(M, d, V, h.device)
    tau_t, tau_f = (tau, 0.0) if isinstance(tau, torch.Tensor) else (None, float(tau))
    _check(_lib.load().ee_exit_head_top2(
        _ptr(h), h.stride(0) if M > 1 else max(h.stride(0), d), _ptr(gamma), _ptr(beta), float(ln_eps), _ptr(W), M, d, V,
        _ptr(tau_t), tau_f, _ptr(out["argmax"]), _ptr(out["entropy"]), _ptr(out["maxprob"]), _ptr(out["top2gap"]),
        _ptr(out["exit_mask"]), _ptr(workspace), workspace.numel(), _stream()), "ee_exit_head_top2")
    return out


def ee_exit_head_results_bytes(n_heads: int, M: int) -> int:
    return int(_lib.load().ee_exit_head_results_bytes(n_heads, M))


def results_views(block: torch.Tensor, n_heads: int, M: int) -> list:
    """Views (no copies) of a packed result block (uint8, host or device) as one output dict per head."""
    stride = ee_exit_head_results_bytes(1, M)
    outs = []
    for k in range(n_heads):
        b = block[k * stride:(k + 1) * stride]
        outs.append(dict(argmax=b[0:4 * M].view(torch.int32), entropy=b[4 * M:8 * M].view(torch.float32),
                         maxprob=b[8 * M:12 * M].view(torch.float32), exit_mask=b[12 * M:13 * M]))
    return outs


class PreparedMultiHost:
    """ee_exit_head_multi_host with its argument block built once.

    heads: list of dicts with gamma, beta, W, tau (device tensors / floats).  h_host: pinned bf16
    [n_heads, M, d].  The staging buffers and the pinned result block are created here, once; `out_host`
    and `out_dev` are per-head views into the packed result blocks.
    """
    __slots__ = ("_args", "_keep", "out_host", "out_dev", "h_dev", "h2d_bytes", "d2h_bytes", "_plan")

    def __init__(self, heads, ln_eps, h_host, workspace):
        n, (_, M, d) = len(heads), h_host.shape
        V = heads[0]["W"].shape[0]
        dev = workspace.device
        arr = (_lib.EEHead * n)()
        keep = []
        for i, hd in enumerate(heads):
            W = _bf16(_dev(hd["W"], "W"))
            tau = hd["tau"]
            tau_t, tau_f = (tau, 0.0) if isinstance(tau, torch.Tensor) else (None, float(tau))
            e = arr[i]
            e.gamma, e.beta, e.W, e.tau_per_row, e.tau = _ptr(hd["gamma"]), _ptr(hd["beta"]), _ptr(W), _ptr(tau_t), tau_f
            keep.append((W, hd["gamma"], hd["beta"], tau_t))
        import ctypes as C
        nbytes = ee_exit_head_results_bytes(n, M)
        self.h_dev = torch.empty((n, M, d), dtype=torch.bfloat16, device=dev)
        res_dev = torch.zeros(nbytes, dtype=torch.uint8, device=dev)
        res_host = torch.zeros(nbytes, dtype=torch.uint8).pin_memory()
        self.out_dev, self.out_host = results_views(res_dev, n, M), results_views(res_host, n, M)
        self.h2d_bytes, self.d2h_bytes = h_host.numel() * 2, nbytes
        self._args = (arr, n, float(ln_eps), M, d, V, _ptr(h_host), _ptr(self.h_dev), _ptr(res_host), _ptr(res_dev),
                      _ptr(workspace), workspace.numel(), _stream())
        self._keep = (arr, keep, h_host, res_dev, res_host, workspace)
        self._plan = None
        if 1 <= n <= _lib.EE_PLAN_MAX_HEADS and M >= 1:
            # the plan's heads read their rows from the staging buffer and write into the packed device results
            for i in range(n):
                e, o = arr[i], self.out_dev[i]
                e.h, e.ld_h = self.h_dev[i].data_ptr(), d
                e.argmax, e.entropy, e.maxprob, e.exit_mask = (_ptr(o[k]) for k in ("argmax", "entropy", "maxprob", "exit_mask"))
            plan = _lib.EEExitHeadPlan()
            _check(_lib.load().ee_exit_head_plan_init(C.byref(plan), arr, n, float(ln_eps), M, d, V, _ptr(workspace), workspace.numel()),
                   "ee_exit_head_plan_init")
            self._plan = (C.byref(plan), plan, C.c_void_p(_ptr(h_host)), C.c_void_p(_ptr(self.h_dev)), C.c_size_t(self.h2d_bytes),
                          C.c_void_p(_ptr(res_host)), C.c_void_p(_ptr(res_dev)), C.c_size_t(nbytes), C.c_void_p(_stream()))

    def __call__(self):
        if self._plan is not None:
            p = self._plan
            code = _lib.load().ee_exit_head_plan_run_host(p[0], p[2], p[3], p[4], p[5], p[6], p[7], p[8])
        else:
            code = _lib.load().ee_exit_head_multi_host(*self._args)
        if code:
            raise EExitError(code, "ee_exit_head_multi_host")
        return self.out_host


def prepare_exit_head(h, gamma, beta, ln_eps, W, tau, *, out=None, workspace=None, path=EE_PATH_AUTO) -> PreparedCall:
    """ee_exit_head with the arguments marshalled once; see PreparedCall."""
    args, out, keep = _exit_head_args(h, gamma, beta, ln_eps, W, tau, out, workspace, path)
    return PreparedCall(_lib.load().ee_exit_head_path, args, "ee_exit_head", keep, out)


EE_STATIC_MAX_ROWS = 32


def ee_exit_head_static(h, gamma, beta, ln_eps, W, tau, *, out: dict) -> dict:
    """ee_exit_head for callers that may not allocate: no workspace argument, at most EE_STATIC_MAX_ROWS rows.

    The library's built-in scratch array is used, so nothing is allocated by the call.  `out` must be given
    (see new_outputs) -- this wrapper creates no tensors either.  Calls sharing a GPU must not overlap.
    """
    h, W, (M, d, V) = _check_head_tensors(h, gamma, beta, W, tau, out)
    tau_t, tau_f = (tau, 0.0) if isinstance(tau, torch.Tensor) else (None, float(tau))
    _check(_lib.load().ee_exit_head_static(
        _ptr(h), h.stride(0) if M > 1 else max(h.stride(0), d), _ptr(gamma), _ptr(beta), float(ln_eps), _ptr(W),
        M, d, V, _ptr(tau_t), tau_f, _ptr(out["argmax"]), _ptr(out["entropy"]), _ptr(out["maxprob"]),
        _ptr(out["exit_mask"]), _stream()), "ee_exit_head_static")
    return out


def ee_exit_head_static_query_error() -> int:
    """ee_query_async_error for the built-in array of ee_exit_head_static: synchronises the current stream; 0, or
    EE_ERR_TIMEOUT after putting the array's control block back to its initial state."""
    return int(_lib.load().ee_exit_head_static_query_error(_stream()))


def ee_exit_head_static_selftest_timeout() -> None:
    """Makes one bounded wait give up against the built-in array (see include/eexit.h)."""
    _check(_lib.load().ee_exit_head_static_selftest_timeout(_stream()), "ee_exit_head_static_selftest_timeout")


def _exit_head_host_args(h_host, h_dev, gamma, beta, ln_eps, W, tau, out_host, out_dev, workspace):
    W = _bf16(W)
    M, d = h_host.shape
    tau_t, tau_f = (tau, 0.0) if isinstance(tau, torch.Tensor) else (None, float(tau))
    args = (_ptr(h_host), _ptr(h_dev), _ptr(gamma), _ptr(beta), float(ln_eps), _ptr(W), M, d, W.shape[0], _ptr(tau_t), tau_f,
            _ptr(out_host["argmax"]), _ptr(out_host["entropy"]), _ptr(out_host["maxprob"]), _ptr(out_host["exit_mask"]),
            _ptr(out_dev["argmax"]), _ptr(out_dev["entropy"]), _ptr(out_dev["maxprob"]), _ptr(out_dev["exit_mask"]),
            _ptr(workspace), workspace.numel(), _stream())
    return args, (h_host, h_dev, gamma, beta, W, tau_t, out_host, out_dev, workspace)


def ee_exit_head_host(h_host, h_dev, gamma, beta, ln_eps, W, tau, out_host: dict, out_dev: dict, workspace) -> None:
    """Host-buffer variant: copies h_host (pinned CPU tensor) in, runs the head, copies the outputs to out_host."""
    args, _ = _exit_head_host_args(h_host, h_dev, gamma, beta, ln_eps, W, tau, out_host, out_dev, workspace)
    _check(_lib.load().ee_exit_head_host(*args), "ee_exit_head_host")


def prepare_exit_head_host(h_host, h_dev, gamma, beta, ln_eps, W, tau, out_host, out_dev, workspace) -> PreparedCall:
    args, keep = _exit_head_host_args(h_host, h_dev, gamma, beta, ln_eps, W, tau, out_host, out_dev, workspace)
    return PreparedCall(_lib.load().ee_exit_head_host, args, "ee_exit_head_host", keep, out_host)


def ee_compact(exit_mask, h=None, *, gather=True, out=None) -> dict:
    """Indices (ascending) and count of the rows with exit_mask == 0, and a dense copy of their rows of h."""
    args, out, _ = _compact_args(exit_mask, h, gather, out)
    _check(_lib.load().ee_compact(*args), "ee_compact")
    return out


def prepare_compact(exit_mask, h=None, *, gather=True, out=None) -> PreparedCall:
    args, out, keep = _compact_args(exit_mask, h, gather, out)
    return PreparedCall(_lib.load().ee_compact, args, "ee_compact", keep, out)


def _compact_args(exit_mask, h, gather, out):
    M = exit_mask.numel()
    dev = exit_mask.device
    gather = gather and h is not None
    if gather:
        h = _bf16(_dev(h, "h"))
    d = h.shape[1] if h is not None else 0
    if out is None:
        out = dict(kept_idx=torch.empty(M, dtype=torch.int32, device=dev),
                   kept_count=torch.empty(1, dtype=torch.int32, device=dev))
        if gather:
            out["h_out"] = torch.empty((M, d), dtype=torch.bfloat16, device=dev)
    ld = (h.stride(0) if M > 1 else max(h.stride(0), d)) if gather else 0
    args = (_ptr(exit_mask), _ptr(h) if gather else None, ld, M, d, _ptr(out["kept_idx"]),
            _ptr(out["kept_count"]), _ptr(out.get("h_out")) if gather else None, _stream())
    return args, out, (exit_mask, h, out)


def dssd_accept(draft_tok, draft_exit_mask, verify_tok, *, out=None) -> dict:
    """Draft length, accepted prefix length and next token per sequence (see include/eexit.h)."""
    args, out, _ = _accept_args(draft_tok, draft_exit_mask, verify_tok, out)
    _check(_lib.load().dssd_accept(*args), "dssd_accept")
    return out


def prepare_accept(draft_tok, draft_exit_mask, verify_tok, *, out=None) -> PreparedCall:
    args, out, keep = _accept_args(draft_tok, draft_exit_mask, verify_tok, out)
    return PreparedCall(_lib.load().dssd_accept, args, "dssd_accept", keep, out)


def _compact_accept_args(exit_mask, h, draft_tok, draft_exit_mask, verify_tok, gather, out):
    c_args, c_out, c_keep = _compact_args(exit_mask, h, gather, None if out is None else out["compact"])
    a_args, a_out, a_keep = _accept_args(draft_tok, draft_exit_mask, verify_tok, None if out is None else out["accept"])
    return c_args[:-1] + a_args, dict(compact=c_out, accept=a_out), (c_keep, a_keep)


def ee_compact_accept(exit_mask, h, draft_tok, draft_exit_mask, verify_tok, *, gather=True, out=None) -> dict:
    """`ee_compact` and `dssd_accept` in one launch; returns dict(compact=..., accept=...) of their results."""
    args, out, _ = _compact_accept_args(exit_mask, h, draft_tok, draft_exit_mask, verify_tok, gather, out)
    _check(_lib.load().ee_compact_accept(*args), "ee_compact_accept")
    return out


def prepare_compact_accept(exit_mask, h, draft_tok, draft_exit_mask, verify_tok, *, gather=True, out=None) -> PreparedCall:
    args, out, keep = _compact_accept_args(exit_mask, h, draft_tok, draft_exit_mask, verify_tok, gather, out)
    return PreparedCall(_lib.load().ee_compact_accept, args, "ee_compact_accept", keep, out)


def ee_cascade_workspace_bytes(M: int, d: int, V: int) -> int:
    return int(_lib.load().ee_cascade_workspace_bytes(int(M), int(d), int(V)))


def ee_calibrate_workspace_bytes(n: int) -> int:
    return int(_lib.load().ee_calibrate_workspace_bytes(int(n)))


def ee_head_kl_workspace_bytes(M: int, d: int, V: int) -> int:
    return int(_lib.load().ee_head_kl_workspace_bytes(int(M), int(d), int(V)))


def _head_kl_args(head, teacher, ln_eps, out, workspace, labels=None):
    hh, Wh = _bf16(_dev(head["h"], "h")), _bf16(_dev(head["W"], "W"))
    ht, Wt = _bf16(_dev(teacher["h"], "h")), _bf16(_dev(teacher["W"], "W"))
    M, d = hh.shape
    V = Wh.shape[0]
    if ht.shape != (M, d) or Wt.shape != (V, d) or not (Wh.is_contiguous() and Wt.is_contiguous()):
        raise ValueError("head and teacher must share M, d, V; W contiguous [V, d]")
    dev = hh.device
    if out is None:
        out = dict(kl=torch.empty(M, dtype=torch.float32, device=dev), loss=torch.zeros(2, dtype=torch.float32, device=dev))
        if labels is not None:
            out["ce"] = torch.empty(M, dtype=torch.float32, device=dev)
    if labels is not None and (labels.dtype != torch.int32 or not labels.is_contiguous() or labels.numel() != M):
        raise TypeError("labels must be a contiguous int32 tensor [M]")
    if workspace is None:
        workspace = torch.empty(int(_lib.load().ee_head_kl_workspace_bytes(M, d, V)), dtype=torch.uint8, device=dev)
        ee_workspace_init(workspace)

    def ld(h):
        return h.stride(0) if M > 1 else max(h.stride(0), d)

    args = (_ptr(hh), ld(hh), _ptr(head["gamma"]), _ptr(head["beta"]), _ptr(Wh), _ptr(ht), ld(ht), _ptr(teacher["gamma"]),
            _ptr(teacher["beta"]), _ptr(Wt), float(ln_eps), M, d, V, _ptr(labels), _ptr(out["kl"]),
            _ptr(out.get("ce")) if labels is not None else None, _ptr(out.get("loss")), _ptr(workspace), workspace.numel(), _stream())
    return args, out, (hh, Wh, ht, Wt, head, teacher, workspace, out, labels)


def ee_head_kl(head, teacher, ln_eps, *, labels=None, out=None, workspace=None) -> dict:
    """KL divergence of a head's distribution from the teacher's, per token and mean (see include/eexit.h); with
    `labels` also the cross-entropy per token (out["ce"]) and its mean (out["loss"][1]).
    head / teacher: dicts with h, gamma, beta, W."""
    args, out, _ = _head_kl_args(head, teacher, ln_eps, out, workspace, labels)
    _check(_lib.load().ee_head_kl(*args), "ee_head_kl")
    return out


def prepare_head_kl(head, teacher, ln_eps, *, labels=None, out=None, workspace=None) -> PreparedCall:
    args, out, keep = _head_kl_args(head, teacher, ln_eps, out, workspace, labels)
    return PreparedCall(_lib.load().ee_head_kl, args, "ee_head_kl", keep, out)


def _workspace_of(nbytes: int, where: str, device) -> torch.Tensor:
    if nbytes == 0:
        raise EExitError(2, where)
    ws = torch.empty(nbytes, dtype=torch.uint8, device=device)
    ee_workspace_init(ws)
    return ws


# The checks of the calls below are a few attribute reads per tensor: these calls take ten to twenty microseconds on the device, and
# a wrapper that takes as long sets the pace of a decoding loop that does not prepare its calls.
def _device_of(t, name: str) -> int:
    """Ordinal of the CUDA device t is on.  The library launches on the current device: a tensor of another one is refused."""
    if not isinstance(t, torch.Tensor):
        raise ValueError(f"{name} must be a CUDA tensor")
    dev = t.get_device()
    if dev < 0:
        raise ValueError(f"{name} must be a CUDA tensor")
    if dev != torch._C._cuda_getDevice():
        raise ValueError(f"{name} is on {t.device}, the current device is cuda:{torch.cuda.current_device()}")
    return dev


def _vector(t, name: str, dtype, n: int, dev: int):
    """t, a contiguous tensor of n elements on device `dev`."""
    if not isinstance(t, torch.Tensor) or t.dtype is not dtype or t.get_device() != dev or t.numel() != n or not t.is_contiguous():
        raise ValueError(f"{name} must be a contiguous {dtype} tensor of {n} elements on cuda:{dev}")
    return t


def _matrix(t, name: str, dtype, rows: int, cols: int, dev: int):
    """t, a contiguous tensor [rows, cols] on device `dev`."""
    if not isinstance(t, torch.Tensor) or t.dtype is not dtype or t.get_device() != dev or t.shape != (rows, cols) or not t.is_contiguous():
        raise ValueError(f"{name} must be a contiguous {dtype} tensor [{rows}, {cols}] on cuda:{dev}")
    return t


def _row_stride(t, name: str, rows: int, cols: int, dev: int) -> int:
    """Row stride of t, a row-major bf16 matrix [rows, cols] on device `dev`."""
    if not isinstance(t, torch.Tensor) or t.dtype is not torch.bfloat16 or t.get_device() != dev or t.shape != (rows, cols):
        raise ValueError(f"{name} must be a bfloat16 tensor [{rows}, {cols}] on cuda:{dev}")
    if rows == 0:
        return cols
    ld, one = t.stride()
    if one != 1 and cols > 1:
        raise ValueError(f"{name} must be row-major")
    return ld if rows > 1 else max(ld, cols)


def _scratch(workspace, dev: int):
    if not isinstance(workspace, torch.Tensor) or workspace.dtype is not torch.uint8 or workspace.get_device() != dev or not workspace.is_contiguous():
        raise ValueError(f"workspace must be a contiguous uint8 tensor on cuda:{dev}")
    return workspace


def ee_head_ce_workspace_bytes(M: int, d: int, V: int) -> int:
    return int(_lib.load().ee_head_ce_workspace_bytes(int(M), int(d), int(V)))


def ee_head_ce_grad_workspace_bytes(M: int, d: int, V: int) -> int:
    return int(_lib.load().ee_head_ce_grad_workspace_bytes(int(M), int(d), int(V)))


def new_head_ce_workspace(M: int, d: int, V: int, device="cuda") -> torch.Tensor:
    """Allocates (through torch) and initialises a workspace for ee_head_ce at these sizes."""
    return _workspace_of(ee_head_ce_workspace_bytes(M, d, V), "ee_head_ce_workspace_bytes", device)


def new_head_ce_grad_workspace(M: int, d: int, V: int, device="cuda") -> torch.Tensor:
    """The same for ee_head_ce_grad; it serves ee_head_ce as well."""
    return _workspace_of(ee_head_ce_grad_workspace_bytes(M, d, V), "ee_head_ce_grad_workspace_bytes", device)


def _head_ce_inputs(head, labels):
    h, W = _bf16(head["h"]), _bf16(head["W"])
    dev = _device_of(h, "h")
    if h.dim() != 2 or W.dim() != 2:
        raise ValueError("h must be [M, d] and W [V, d]")
    M, d = h.shape
    V = W.shape[0]
    ld = _row_stride(h, "h", M, d, dev)
    _matrix(W, "W", torch.bfloat16, V, d, dev)
    _vector(head["gamma"], "gamma", torch.float32, d, dev)
    _vector(head["beta"], "beta", torch.float32, d, dev)
    _vector(labels, "labels", torch.int32, M, dev)
    return h, W, ld, M, d, V, dev


def _head_ce_args(head, labels, ln_eps, out, workspace):
    h, W, ld, M, d, V, dev = _head_ce_inputs(head, labels)
    if out is None:
        f32 = torch.float32
        out = dict(ce=torch.empty(M, dtype=f32, device=h.device), lse=torch.empty(M, dtype=f32, device=h.device),
                   loss=torch.empty(2, dtype=f32, device=h.device))
    else:
        for name, n in (("ce", M), ("lse", M), ("loss", 2)):
            _vector(out.get(name), f"out[{name!r}]", torch.float32, n, dev)
    workspace = new_head_ce_workspace(M, d, V, h.device) if workspace is None else _scratch(workspace, dev)
    args = (h.data_ptr(), ld, head["gamma"].data_ptr(), head["beta"].data_ptr(), ln_eps, W.data_ptr(), M, d, V, labels.data_ptr(),
            out["ce"].data_ptr(), out["lse"].data_ptr(), out["loss"].data_ptr(), workspace.data_ptr(), workspace.numel(), _stream())
    return args, out, (h, W, head, labels, out, workspace)


def ee_head_ce(head, labels, ln_eps, *, out=None, workspace=None) -> dict:
    """Cross-entropy of a head (a dict with h, gamma, beta, W) at int32 `labels` [M], without keeping the logits (see
    include/eexit.h): dict(ce [M], lse [M], loss [2] = mean over the counted rows and their number).  Labels outside
    [0, V) mark rows that are not counted."""
    args, out, _ = _head_ce_args(head, labels, ln_eps, out, workspace)
    _check(_lib.load().ee_head_ce(*args), "ee_head_ce")
    return out


def prepare_head_ce(head, labels, ln_eps, *, out=None, workspace=None) -> PreparedCall:
    args, out, keep = _head_ce_args(head, labels, ln_eps, out, workspace)
    return PreparedCall(_lib.load().ee_head_ce, args, "ee_head_ce", keep, out)


def _head_ce_grad_args(head, labels, ln_eps, forward, dce, dloss, accumulate, out, workspace):
    h, W, ld, M, d, V, dev = _head_ce_inputs(head, labels)
    lse, loss = _vector(forward["lse"], "lse", torch.float32, M, dev), _vector(forward["loss"], "loss", torch.float32, 2, dev)
    ce = forward.get("ce")
    if ce is not None:
        _vector(ce, "ce", torch.float32, M, dev)
    if dce is not None:
        _vector(dce, "dce", torch.float32, M, dev)
    if dloss is not None:
        _vector(dloss, "dloss", torch.float32, 1, dev)
    bf16 = torch.bfloat16
    ld_dh = d
    if out is None:
        if accumulate:
            raise ValueError("accumulate needs the buffers to add to (out)")
        out = dict(dh=torch.empty((M, d), dtype=bf16, device=h.device), dW=torch.empty((V, d), dtype=bf16, device=h.device),
                   dgamma=torch.empty(d, dtype=bf16, device=h.device), dbeta=torch.empty(d, dtype=bf16, device=h.device))
    else:
        if out.get("dh") is not None:
            ld_dh = _row_stride(out["dh"], "out['dh']", M, d, dev)
        if out.get("dW") is not None:
            _matrix(out["dW"], "out['dW']", bf16, V, d, dev)
        for name in ("dgamma", "dbeta"):
            if out.get(name) is not None:
                _vector(out[name], f"out[{name!r}]", bf16, d, dev)
    workspace = new_head_ce_grad_workspace(M, d, V, h.device) if workspace is None else _scratch(workspace, dev)
    args = (h.data_ptr(), ld, head["gamma"].data_ptr(), head["beta"].data_ptr(), ln_eps, W.data_ptr(), M, d, V, labels.data_ptr(),
            _ptr(ce), lse.data_ptr(), loss.data_ptr(), _ptr(dce), _ptr(dloss), _ptr(out.get("dh")), ld_dh, _ptr(out.get("dW")), _ptr(out.get("dgamma")),
            _ptr(out.get("dbeta")), int(bool(accumulate)), workspace.data_ptr(), workspace.numel(), _stream())
    return args, out, (h, W, head, labels, forward, dce, dloss, out, workspace)


def ee_head_ce_grad(head, labels, ln_eps, forward, *, dce=None, dloss=None, accumulate=False, out=None, workspace=None) -> dict:
    """Gradient of the cross-entropy (see include/eexit.h): dict(dh, dW, dgamma, dbeta), bf16.  `forward` is what
    ee_head_ce returned for the same inputs (its lse and loss, and its ce if it is there: with it the gradient of a nearly certain
    row keeps its digits).  By default the gradient of the mean, times the device
    scalar `dloss` if given; `dce` [M] gives every row's own weight instead.  With `out`, entries left out or None are
    not computed; accumulate=True adds dW, dgamma and dbeta to the buffers in it."""
    args, out, _ = _head_ce_grad_args(head, labels, ln_eps, forward, dce, dloss, accumulate, out, workspace)
    _check(_lib.load().ee_head_ce_grad_of(*args), "ee_head_ce_grad")
    return out


def prepare_head_ce_grad(head, labels, ln_eps, forward, *, dce=None, dloss=None, accumulate=False, out=None, workspace=None) -> PreparedCall:
    args, out, keep = _head_ce_grad_args(head, labels, ln_eps, forward, dce, dloss, accumulate, out, workspace)
    return PreparedCall(_lib.load().ee_head_ce_grad_of, args, "ee_head_ce_grad", keep, out)


def _packed(weights, kind):
    """Weights packed in the form `kind`: the two 4-bit forms have the same attributes, and sizes that fit one another."""
    if not isinstance(weights, kind):
        raise TypeError(f"expected {kind.__name__}, got {type(weights).__name__}")
    return weights


class Q4Weights:
    """A head's weights in 4 bits (see include/eexit.h): the packed bytes (a device tensor) and what they are of."""
    __slots__ = ("data", "V", "d", "group")

    def __init__(self, data: torch.Tensor, V: int, d: int, group: int):
        need = ee_head_q4_bytes(V, d, group)
        if need == 0:
            raise EExitError(2, "ee_head_q4_bytes")
        if not (isinstance(data, torch.Tensor) and data.is_cuda and data.dtype == torch.uint8 and data.is_contiguous() and data.numel() >= need):
            raise ValueError(f"data must be a contiguous uint8 CUDA tensor of at least {need} bytes")
        self.data, self.V, self.d, self.group = data, int(V), int(d), int(group)


def ee_head_q4_bytes(V: int, d: int, group: int) -> int:
    return int(_lib.load().ee_head_q4_bytes(int(V), int(d), int(group)))


def ee_head_q4_pack(W, group: int = 64, *, out: Q4Weights | None = None) -> Q4Weights:
    """Writes a head's weights (bf16 [V, d]) in 4 bits with a scale per row and `group` columns (see include/eexit.h)."""
    W = _bf16(W)
    dev = _device_of(W, "W")
    if W.dim() != 2 or not W.is_contiguous():
        raise ValueError("W must be contiguous [V, d]")
    V, d = W.shape
    if out is None:
        nbytes = ee_head_q4_bytes(V, d, group)
        if nbytes == 0:
            raise EExitError(2, "ee_head_q4_pack")
        out = Q4Weights(torch.empty(nbytes, dtype=torch.uint8, device=W.device), V, d, group)
    elif (_packed(out, Q4Weights).V, out.d, out.group) != (V, d, group) or out.data.get_device() != dev:
        raise ValueError("out was made for other weights")
    _check(_lib.load().ee_head_q4_pack(W.data_ptr(), V, d, int(group), out.data.data_ptr(), out.data.numel(), _stream()), "ee_head_q4_pack")
    return out


def ee_head_q4_unpack(q4: Q4Weights, *, out=None) -> torch.Tensor:
    """What the packed weights stand for, bf16 [V, d]."""
    dev = _device_of(_packed(q4, Q4Weights).data, "q4")
    if out is None:
        out = torch.empty((q4.V, q4.d), dtype=torch.bfloat16, device=q4.data.device)
    else:
        _matrix(out, "out", torch.bfloat16, q4.V, q4.d, dev)
    _check(_lib.load().ee_head_q4_unpack(q4.data.data_ptr(), q4.data.numel(), q4.V, q4.d, q4.group, out.data_ptr(), _stream()),
           "ee_head_q4_unpack")
    return out


def ee_exit_head_q4_workspace_bytes(M: int, d: int, V: int) -> int:
    return int(_lib.load().ee_exit_head_q4_workspace_bytes(int(M), int(d), int(V)))


def new_exit_head_q4_workspace(M: int, q4: Q4Weights) -> torch.Tensor:
    """Allocates (through torch) and initialises a workspace for ee_exit_head_q4 with these weights."""
    return _workspace_of(ee_exit_head_q4_workspace_bytes(M, q4.d, q4.V), "ee_exit_head_q4_workspace_bytes", q4.data.device)


def _exit_head_4bit_args(h, gamma, beta, ln_eps, q4, tau, out, workspace, new_workspace):
    h = _bf16(h)
    dev = _device_of(h, "h")
    d = q4.d
    if h.dim() != 2:
        raise ValueError(f"h must be row-major [M, d = {d}]")
    M = h.shape[0]
    if M > _INT_MAX:
        raise EExitError(2, "an exit head of 4-bit weights")
    ld = _row_stride(h, "h", M, d, dev)
    data = q4.data
    if data.get_device() != dev:
        raise ValueError(f"the weights are on {data.device}, h on {h.device}")
    _vector(gamma, "gamma", torch.float32, d, dev)
    _vector(beta, "beta", torch.float32, d, dev)
    tau_t = tau_ptr = None
    if isinstance(tau, torch.Tensor):
        tau_t, tau = _vector(tau, "a per-row tau", torch.float32, M, dev), 0.0
        tau_ptr = tau_t.data_ptr()
    if out is None:
        out = new_outputs(M, h.device)
    else:
        for name, dtype in _OUT_DTYPES.items():
            t = out.get(name)
            if not isinstance(t, torch.Tensor) or t.dtype is not dtype or t.get_device() != dev or not t.is_contiguous() or t.numel() < M:
                raise ValueError(f"out[{name!r}] must be a contiguous {dtype} tensor of at least M = {M} elements on cuda:{dev}")
    workspace = new_workspace(M, q4) if workspace is None else _scratch(workspace, dev)
    args = (h.data_ptr(), ld, gamma.data_ptr(), beta.data_ptr(), ln_eps, data.data_ptr(), data.numel(), q4.group, M, d, q4.V, tau_ptr, tau,
            out["argmax"].data_ptr(), out["entropy"].data_ptr(), out["maxprob"].data_ptr(), out["exit_mask"].data_ptr(),
            workspace.data_ptr(), workspace.numel(), _stream())
    return args, out, (h, gamma, beta, q4, tau_t, out, workspace)


def ee_exit_head_q4(h, gamma, beta, ln_eps, q4: Q4Weights, tau, *, out=None, workspace=None) -> dict:
    """ee_exit_head with weights held in 4 bits (ee_head_q4_pack); see there for the arguments."""
    args, out, _ = _exit_head_4bit_args(h, gamma, beta, ln_eps, _packed(q4, Q4Weights), tau, out, workspace, new_exit_head_q4_workspace)
    _check(_lib.load().ee_exit_head_q4(*args), "ee_exit_head_q4")
    return out


def prepare_exit_head_q4(h, gamma, beta, ln_eps, q4: Q4Weights, tau, *, out=None, workspace=None) -> PreparedCall:
    args, out, keep = _exit_head_4bit_args(h, gamma, beta, ln_eps, _packed(q4, Q4Weights), tau, out, workspace, new_exit_head_q4_workspace)
    return PreparedCall(_lib.load().ee_exit_head_q4, args, "ee_exit_head_q4", keep, out)


class Fp4Weights:
    """A head's weights in microscaled 4-bit floating point (see include/eexit.h): the packed bytes (a device tensor) and what they are of."""
    __slots__ = ("data", "V", "d", "group")

    def __init__(self, data: torch.Tensor, V: int, d: int, group: int):
        need = ee_head_fp4_bytes(V, d, group)
        if need == 0:
            raise EExitError(2, "ee_head_fp4_bytes")
        if not (isinstance(data, torch.Tensor) and data.is_cuda and data.dtype == torch.uint8 and data.is_contiguous() and data.numel() >= need):
            raise ValueError(f"data must be a contiguous uint8 CUDA tensor of at least {need} bytes")
        self.data, self.V, self.d, self.group = data, int(V), int(d), int(group)


# ctypes cuts an int off at 32 bits, and what is left of an invalid size may be a valid one.
_INT_MAX = 2 ** 31 - 1


def _are_ints(*sizes) -> bool:
    return all(-_INT_MAX <= n <= _INT_MAX for n in sizes)


def ee_head_fp4_bytes(V: int, d: int, group: int) -> int:
    if not _are_ints(V, d, group):
        return 0
    return int(_lib.load().ee_head_fp4_bytes(int(V), int(d), int(group)))


def ee_head_fp4_pack(W, group: int = 16, *, out: Fp4Weights | None = None) -> Fp4Weights:
    """Writes a head's weights (bf16 [V, d]) in 4-bit floating point with a scale per row and 16 or 32 columns (see include/eexit.h)."""
    W = _bf16(W)
    dev = _device_of(W, "W")
    if W.dim() != 2 or not W.is_contiguous():
        raise ValueError("W must be contiguous [V, d]")
    V, d = W.shape
    if out is None:
        nbytes = ee_head_fp4_bytes(V, d, group)
        if nbytes == 0:
            raise EExitError(2, "ee_head_fp4_pack")
        out = Fp4Weights(torch.empty(nbytes, dtype=torch.uint8, device=W.device), V, d, group)
    elif (_packed(out, Fp4Weights).V, out.d, out.group) != (V, d, group) or out.data.get_device() != dev:
        raise ValueError("out was made for other weights")
    _check(_lib.load().ee_head_fp4_pack(W.data_ptr(), V, d, int(group), out.data.data_ptr(), out.data.numel(), _stream()), "ee_head_fp4_pack")
    return out


def ee_head_fp4_unpack(fp4: Fp4Weights, *, out=None) -> torch.Tensor:
    """What the packed weights stand for, bf16 [V, d]."""
    dev = _device_of(_packed(fp4, Fp4Weights).data, "fp4")
    if out is None:
        out = torch.empty((fp4.V, fp4.d), dtype=torch.bfloat16, device=fp4.data.device)
    else:
        _matrix(out, "out", torch.bfloat16, fp4.V, fp4.d, dev)
    _check(_lib.load().ee_head_fp4_unpack(fp4.data.data_ptr(), fp4.data.numel(), fp4.V, fp4.d, fp4.group, out.data_ptr(), _stream()),
           "ee_head_fp4_unpack")
    return out


def ee_exit_head_fp4_workspace_bytes(M: int, d: int, V: int, group: int) -> int:
    if not _are_ints(M, d, V, group):
        return 0
    return int(_lib.load().ee_exit_head_fp4_workspace_bytes(int(M), int(d), int(V), int(group)))


def new_exit_head_fp4_workspace(M: int, fp4: Fp4Weights) -> torch.Tensor:
    """Allocates (through torch) and initialises a workspace for ee_exit_head_fp4 with these weights, for up to M rows."""
    return _workspace_of(ee_exit_head_fp4_workspace_bytes(M, fp4.d, fp4.V, fp4.group), "ee_exit_head_fp4_workspace_bytes", fp4.data.device)


def ee_exit_head_fp4(h, gamma, beta, ln_eps, fp4: Fp4Weights, tau, *, out=None, workspace=None) -> dict:
    """ee_exit_head with weights held in 4-bit floating point (ee_head_fp4_pack) and activations in the same form; see there for the
    arguments."""
    args, out, _ = _exit_head_4bit_args(h, gamma, beta, ln_eps, _packed(fp4, Fp4Weights), tau, out, workspace, new_exit_head_fp4_workspace)
    _check(_lib.load().ee_exit_head_fp4(*args), "ee_exit_head_fp4")
    return out


def prepare_exit_head_fp4(h, gamma, beta, ln_eps, fp4: Fp4Weights, tau, *, out=None, workspace=None) -> PreparedCall:
    args, out, keep = _exit_head_4bit_args(h, gamma, beta, ln_eps, _packed(fp4, Fp4Weights), tau, out, workspace, new_exit_head_fp4_workspace)
    return PreparedCall(_lib.load().ee_exit_head_fp4, args, "ee_exit_head_fp4", keep, out)


def new_token_loss_workspace(device="cuda") -> torch.Tensor:
    """Allocates (through torch) and initialises a workspace for ee_policy_loss and ee_preference_loss, of any size."""
    return _workspace_of(int(_lib.load().ee_token_loss_workspace_bytes()), "ee_token_loss_workspace_bytes", device)


def new_policy_loss_outputs(M: int, device="cuda") -> dict:
    return dict(loss=torch.empty(4, dtype=torch.float32, device=device), dce=torch.empty(M, dtype=torch.float32, device=device))


def new_preference_loss_outputs(M: int, P: int, device="cuda") -> dict:
    return dict(loss=torch.empty(4, dtype=torch.float32, device=device), margin=torch.empty(P, dtype=torch.float32, device=device),
                dce=torch.empty(M, dtype=torch.float32, device=device))


def _token_loss_inputs(forward, labels, V, seq_start, units_per, ref_ce, out):
    """ce, M, device ordinal and the number of units that seq_start delimits (None without it)."""
    ce = forward["ce"]
    dev = _device_of(ce, "ce")
    M = ce.numel()
    if M > _INT_MAX or not -_INT_MAX <= V <= _INT_MAX:
        raise EExitError(2, "a loss over tokens")
    f32 = torch.float32
    _vector(ce, "ce", f32, M, dev)
    _vector(labels, "labels", torch.int32, M, dev)
    if ref_ce is not None:
        _vector(ref_ce, "ref_ce", f32, M, dev)
    units = None
    if seq_start is not None:
        if not isinstance(seq_start, torch.Tensor):
            raise ValueError("seq_start must be an int32 CUDA tensor")
        n = seq_start.numel()
        if n < 1 + units_per or (n - 1) % units_per:
            raise ValueError(f"seq_start must have 1 + {units_per} n elements, n >= 1" if units_per > 1 else "seq_start must have at least two elements")
        _vector(seq_start, "seq_start", torch.int32, n, dev)
        units = (n - 1) // units_per
        if units > _INT_MAX:
            raise EExitError(2, "a loss over tokens")
    if out is not None:
        _vector(out.get("loss"), "out['loss']", f32, 4, dev)
        _vector(out.get("dce"), "out['dce']", f32, M, dev)
    return ce, M, dev, units


def _policy_loss_args(forward, labels, V, old_ce, adv, ref_ce, kl_weight, clip, seq_start, out, workspace):
    ce, M, dev, S = _token_loss_inputs(forward, labels, V, seq_start, 1, ref_ce, out)
    f32 = torch.float32
    _vector(old_ce, "old_ce", f32, M, dev)
    _vector(adv, "adv", f32, M if S is None else S, dev)
    counted = None
    if S is None:
        counted = _vector(forward["loss"], "loss", f32, 2, dev)
    if out is None:
        out = new_policy_loss_outputs(M, ce.device)
    workspace = new_token_loss_workspace(ce.device) if workspace is None else _scratch(workspace, dev)
    args = (ce.data_ptr(), old_ce.data_ptr(), _ptr(ref_ce), adv.data_ptr(), labels.data_ptr(), M, V, _ptr(seq_start), S or 0, _ptr(counted),
            clip[0], clip[1], kl_weight, out["dce"].data_ptr(), out["loss"].data_ptr(), workspace.data_ptr(), workspace.numel(), _stream())
    return args, out, (ce, old_ce, ref_ce, adv, labels, seq_start, counted, out, workspace)


def ee_policy_loss(forward, labels, V: int, old_ce, adv, *, ref_ce=None, kl_weight: float = 0.0, clip=(0.2, 0.2), seq_start=None, out=None,
                   workspace=None) -> dict:
    """Clipped policy loss over drafted tokens (see include/eexit.h): dict(loss [4], dce [M]).  `forward` is what ee_head_ce returned for the
    tokens at `labels`, old_ce their cross-entropies when they were drafted, ref_ce those of a reference head.  Without seq_start every counted
    token counts alike and adv is [M]; with it (int32 [S + 1]) every sequence does, and adv is [S].  dce goes to ee_head_ce_grad as dce."""
    args, out, _ = _policy_loss_args(forward, labels, V, old_ce, adv, ref_ce, kl_weight, clip, seq_start, out, workspace)
    _check(_lib.load().ee_policy_loss(*args), "ee_policy_loss")
    return out


def prepare_policy_loss(forward, labels, V: int, old_ce, adv, *, ref_ce=None, kl_weight: float = 0.0, clip=(0.2, 0.2), seq_start=None, out=None,
                        workspace=None) -> PreparedCall:
    args, out, keep = _policy_loss_args(forward, labels, V, old_ce, adv, ref_ce, kl_weight, clip, seq_start, out, workspace)
    return PreparedCall(_lib.load().ee_policy_loss, args, "ee_policy_loss", keep, out)


def _preference_loss_args(forward, labels, V, seq_start, ref_ce, beta, smoothing, out, workspace):
    if seq_start is None:
        raise ValueError("seq_start must be an int32 CUDA tensor")
    ce, M, dev, P = _token_loss_inputs(forward, labels, V, seq_start, 2, ref_ce, out)
    if out is None:
        out = new_preference_loss_outputs(M, P, ce.device)
    else:
        _vector(out.get("margin"), "out['margin']", torch.float32, P, dev)
    workspace = new_token_loss_workspace(ce.device) if workspace is None else _scratch(workspace, dev)
    args = (ce.data_ptr(), _ptr(ref_ce), labels.data_ptr(), M, V, seq_start.data_ptr(), P, beta, smoothing, out["dce"].data_ptr(),
            out["margin"].data_ptr(), out["loss"].data_ptr(), workspace.data_ptr(), workspace.numel(), _stream())
    return args, out, (ce, ref_ce, labels, seq_start, out, workspace)


def ee_preference_loss(forward, labels, V: int, seq_start, *, ref_ce=None, beta: float = 0.1, smoothing: float = 0.0, out=None, workspace=None) -> dict:
    """Loss of pairs of sequences 2p (preferred) and 2p + 1 (rejected), delimited by seq_start int32 [2 P + 1] (see include/eexit.h):
    dict(loss [4], margin [P], dce [M]).  `forward` is what ee_head_ce returned for their tokens, ref_ce a reference head's
    cross-entropies; dce goes to ee_head_ce_grad as dce."""
    args, out, _ = _preference_loss_args(forward, labels, V, seq_start, ref_ce, beta, smoothing, out, workspace)
    _check(_lib.load().ee_preference_loss(*args), "ee_preference_loss")
    return out


def prepare_preference_loss(forward, labels, V: int, seq_start, *, ref_ce=None, beta: float = 0.1, smoothing: float = 0.0, out=None,
                            workspace=None) -> PreparedCall:
    args, out, keep = _preference_loss_args(forward, labels, V, seq_start, ref_ce, beta, smoothing, out, workspace)
    return PreparedCall(_lib.load().ee_preference_loss, args, "ee_preference_loss", keep, out)


_GRAD_TYPES = {torch.bfloat16: _lib.EE_BFLOAT16, torch.float16: _lib.EE_FLOAT16, torch.float32: _lib.EE_FLOAT32}


class GradClip:
    """The norm over a list of gradients (contiguous bf16, fp16 or fp32 tensors that do not overlap) and their scaling, with the list marshalled once: gradient
    buffers are the same from step to step (see ee_grad_norm and ee_grad_clip in include/eexit.h).  Calling it with max_norm computes the norm,
    scales the gradients, in place or into `out` (a list of tensors like them), and returns the norm, fp32 [1] on the device.  norm() and
    scale(max_norm) are its two halves, for a sum over several GPUs in between: scale reads self.value.  It launches on the
    stream that is current when it is called, the first time behind what was queued where it was made; value and workspace are its own, so that its
    calls must not run at the same time."""

    def __init__(self, grads, *, out=None, workspace=None):
        import ctypes as C
        grads = list(grads)
        dev = _device_of(grads[0], "grads[0]") if grads else torch.cuda.current_device()
        spans = []
        self._tensors = (_lib.EETensor * max(1, len(grads)))()
        for i, g in enumerate(grads):
            self._one(g, f"grads[{i}]", dev)
            at, n = g.data_ptr(), g.numel()
            spans.append((at, at + n * g.element_size(), "grads", i))
            self._tensors[i].data, self._tensors[i].n, self._tensors[i].type = at or None, n, _GRAD_TYPES[g.dtype]
        self._out = None
        if out is not None:
            out = list(out)
            if len(out) != len(grads):
                raise ValueError("out must have a tensor for each of grads")
            self._out = (C.c_void_p * max(1, len(grads)))()
            for i, (o, g) in enumerate(zip(out, grads)):
                self._one(o, f"out[{i}]", dev)
                if o.dtype is not g.dtype or o.numel() != g.numel():
                    raise ValueError(f"out[{i}] must be like grads[{i}]")
                at = o.data_ptr()
                self._out[i] = at or None
                if at != spans[i][0]:                                    # (an out equal to its tensor is that tensor in place)
                    spans.append((at, at + o.numel() * o.element_size(), "out", i))
        # Tensors are read, scaled and written piece by piece in no order: one that lies in another would be scaled twice, or read after it was.
        spans = sorted(s for s in spans if s[0] < s[1])
        for a, b in zip(spans, spans[1:]):
            if b[0] < a[1]:
                raise ValueError(f"{a[2]}[{a[3]}] and {b[2]}[{b[3]}] overlap")
        self._n, self._dev, self._keep = len(grads), dev, grads
        self.out = grads if out is None else out
        self._made_on = _stream()
        self._ordered = {self._made_on}                                  # streams that are behind the making of value and workspace
        self.value = torch.empty(1, dtype=torch.float32, device=torch.device("cuda", dev))
        self.workspace = new_grad_norm_workspace(grads, self.value.device) if workspace is None else _scratch(workspace, dev)
        lib, value = _lib.load(), C.c_void_p(self.value.data_ptr())
        self._norm_fn, self._norm_args = lib.ee_grad_norm, (self._tensors, self._n, value, C.c_void_p(self.workspace.data_ptr()), C.c_size_t(self.workspace.numel()))
        self._clip_fn, self._clip_args = lib.ee_grad_clip, (self._tensors, self._out, self._n, value)

    @staticmethod
    def _one(t, name, dev):
        if not isinstance(t, torch.Tensor) or t.dtype not in _GRAD_TYPES or t.get_device() != dev or not t.is_contiguous():
            raise ValueError(f"{name} must be a contiguous bfloat16, float16 or float32 tensor on cuda:{dev}")

    def _here(self):
        if torch._C._cuda_getDevice() != self._dev:
            raise ValueError(f"the gradients are on cuda:{self._dev}, the current device is cuda:{torch.cuda.current_device()}")
        stream = _stream()
        if stream not in self._ordered:
            self._order(stream)
        return stream

    def _order(self, stream):
        """The workspace is cleared, and the memory of both is free, only behind what is queued on the stream that the object was made on: the first
        call on another one waits for that.  (A capture cannot wait for what is outside of it; torch synchronises before it begins one.)"""
        if not torch.cuda.is_current_stream_capturing():
            torch.cuda.current_stream().wait_stream(torch.cuda.ExternalStream(self._made_on, device=self._dev))
            self._ordered.add(stream)

    def norm(self) -> torch.Tensor:
        _check(self._norm_fn(*self._norm_args, self._here()), "ee_grad_norm")
        return self.value

    def scale(self, max_norm: float) -> None:
        tensors, out, n, value = self._clip_args
        _check(self._clip_fn(tensors, out, n, max_norm, value, self._here()), "ee_grad_clip")

    def __call__(self, max_norm: float) -> torch.Tensor:
        stream = self._here()
        _check(self._norm_fn(*self._norm_args, stream), "ee_grad_norm")
        tensors, out, n, value = self._clip_args
        _check(self._clip_fn(tensors, out, n, max_norm, value, stream), "ee_grad_clip")
        return self.value


def new_grad_norm_workspace(grads, device="cuda") -> torch.Tensor:
    """Allocates (through torch) and initialises a workspace for the norm over these gradients (a list, or their number)."""
    n = grads if isinstance(grads, int) else len(grads)
    return _workspace_of(int(_lib.load().ee_grad_norm_workspace_bytes(n)), "ee_grad_norm_workspace_bytes", device)


def ee_grad_norm(grads, *, workspace=None) -> torch.Tensor:
    """The norm over all elements of a list of gradients, fp32 [1] on the device (see include/eexit.h)."""
    return GradClip(grads, workspace=workspace).norm()


def ee_grad_clip(grads, max_norm: float, *, out=None, workspace=None) -> torch.Tensor:
    """Scales a list of gradients by min(1, max_norm / (norm + 1e-6)), in place or into `out`; returns their norm before that, fp32 [1] on the
    device.  A loop keeps a GradClip instead."""
    return GradClip(grads, out=out, workspace=workspace)(max_norm)


def _embed_args(table, tokens, scale, out):
    table = _bf16(table)
    dev = _device_of(table, "table")
    if table.dim() != 2 or not table.is_contiguous():
        raise ValueError("table must be contiguous [V, d]")
    V, d = table.shape
    n = tokens.numel()
    _vector(tokens, "tokens", torch.int32, n, dev)
    if out is None:
        out, ld = table.new_empty((n, d)), d
    else:
        ld = _row_stride(out, "out", n, d, dev)
    args = (table.data_ptr(), V, d, tokens.data_ptr(), n, scale, out.data_ptr(), ld, _stream())
    return args, out, (table, tokens, out)


def ee_embed(table, tokens, scale: float = 1.0, *, out=None) -> torch.Tensor:
    """Rows of `table` (bf16 [V, d]) at int32 `tokens` [n], times `scale`, rounded once; zero rows for tokens outside
    [0, V)."""
    args, out, _ = _embed_args(table, tokens, scale, out)
    _check(_lib.load().ee_embed(*args), "ee_embed")
    return out


def prepare_embed(table, tokens, scale: float = 1.0, *, out=None) -> PreparedCall:
    args, out, keep = _embed_args(table, tokens, scale, out)
    return PreparedCall(_lib.load().ee_embed, args, "ee_embed", keep, out)


def ee_embed_grad_workspace_bytes(n: int, d: int, V: int) -> int:
    return int(_lib.load().ee_embed_grad_workspace_bytes(int(n), int(d), int(V)))


def new_embed_grad_workspace(n: int, d: int, V: int, device="cuda") -> torch.Tensor:
    """Allocates (through torch) a workspace for ee_embed_grad at these sizes; it needs no initialisation."""
    nbytes = ee_embed_grad_workspace_bytes(n, d, V)
    if nbytes == 0:
        raise EExitError(2, "ee_embed_grad_workspace_bytes")
    return torch.empty(nbytes, dtype=torch.uint8, device=device)


def _embed_grad_args(dout, tokens, V, scale, dtype, out, accumulate, workspace):
    dout = _bf16(dout)
    dev = _device_of(dout, "dout")
    if dout.dim() != 2:
        raise ValueError("dout must be [n, d]")
    n, d = dout.shape
    ld = _row_stride(dout, "dout", n, d, dev)
    _vector(tokens, "tokens", torch.int32, n, dev)
    if out is not None:
        dtype = out.dtype
    if dtype is not torch.bfloat16 and dtype is not torch.float32:
        raise ValueError("the table's gradient is bfloat16 or float32")
    if out is None:
        if accumulate:
            raise ValueError("accumulate needs the table to add to (out)")
        out = torch.empty((V, d), dtype=dtype, device=dout.device)
    else:
        _matrix(out, "out", dtype, V, d, dev)
    workspace = new_embed_grad_workspace(n, d, V, dout.device) if workspace is None else _scratch(workspace, dev)
    args = (dout.data_ptr(), ld, tokens.data_ptr(), n, V, d, scale, out.data_ptr(), 1 if dtype is torch.float32 else 0, 1 if accumulate else 0,
            workspace.data_ptr(), workspace.numel(), _stream())
    return args, out, (dout, tokens, out, workspace)


def ee_embed_grad(dout, tokens, V: int, scale: float = 1.0, *, dtype=torch.bfloat16, out=None, accumulate=False, workspace=None) -> torch.Tensor:
    """Gradient of ee_embed's table [V, d]: per token the sum of its rows of `dout` (bf16 [n, d]) times `scale`, in bf16
    or fp32 (`dtype`, or that of `out`); accumulate=True adds to `out` and touches no other rows."""
    args, out, _ = _embed_grad_args(dout, tokens, V, scale, dtype, out, accumulate, workspace)
    _check(_lib.load().ee_embed_grad(*args), "ee_embed_grad")
    return out


def prepare_embed_grad(dout, tokens, V: int, scale: float = 1.0, *, dtype=torch.bfloat16, out=None, accumulate=False, workspace=None) -> PreparedCall:
    args, out, keep = _embed_grad_args(dout, tokens, V, scale, dtype, out, accumulate, workspace)
    return PreparedCall(_lib.load().ee_embed_grad, args, "ee_embed_grad", keep, out)


def ee_selftest_wait_timeout(workspace) -> None:
    """Makes one bounded device-side wait give up (see include/eexit.h); ee_query_async_error then reports it."""
    _check(_lib.load().ee_selftest_wait_timeout(_ptr(workspace), workspace.numel(), _stream()), "ee_selftest_wait_timeout")


def ee_selftest_read_stream(buffer, workspace) -> None:
    """Reads `buffer` (a device tensor) once with the kernels' weight-streaming mechanism (see include/eexit.h);
    the caller times it."""
    _check(_lib.load().ee_selftest_read_stream(_ptr(buffer), buffer.numel() * buffer.element_size(), _ptr(workspace),
                                               workspace.numel(), _stream()), "ee_selftest_read_stream")


def _cascade_args(heads, ln_eps, out, workspace):
    n = len(heads)
    arr = (_lib.EEHead * n)()
    keep = []
    M, d = _bf16(heads[0]["h"]).shape
    V = heads[0]["W"].shape[0]
    dev = heads[0]["h"].device
    for i, hd in enumerate(heads):
        h, W = _bf16(_dev(hd["h"], "h")), _bf16(_dev(hd["W"], "W"))
        if h.shape != (M, d) or W.shape != (V, d) or not W.is_contiguous() or h.stride(1) != 1:
            raise ValueError("all heads must share M, d, V; W contiguous [V, d]; h row-major [M, d]")
        e = arr[i]
        e.h, e.ld_h, e.gamma, e.beta, e.W = _ptr(h), (h.stride(0) if M > 1 else max(h.stride(0), d)), _ptr(hd["gamma"]), _ptr(hd["beta"]), _ptr(W)
        e.tau_per_row, e.tau = None, float(hd["tau"])
        keep.append((h, W, hd["gamma"], hd["beta"]))
    if out is None:
        out = dict(exit_head=torch.empty(M, dtype=torch.int32, device=dev), token=torch.empty(M, dtype=torch.int32, device=dev),
                   entropy=torch.empty(M, dtype=torch.float32, device=dev), rows_in=torch.empty(n, dtype=torch.int32, device=dev))
    if workspace is None:
        workspace = torch.empty(int(_lib.load().ee_cascade_workspace_bytes(M, d, V)), dtype=torch.uint8, device=dev)
        ee_workspace_init(workspace)
    args = (arr, n, float(ln_eps), M, d, V, _ptr(out["exit_head"]), _ptr(out["token"]), _ptr(out["entropy"]), _ptr(out["rows_in"]),
            _ptr(workspace), workspace.numel(), _stream())
    return args, out, (arr, keep, workspace, out)


def ee_cascade(heads, ln_eps, *, out=None, workspace=None) -> dict:
    """Cascade of heads on a batch (see include/eexit.h): heads is a list of dicts with h, gamma, beta, W, tau."""
    args, out, _ = _cascade_args(heads, ln_eps, out, workspace)
    _check(_lib.load().ee_cascade(*args), "ee_cascade")
    return out


class PreparedCascade:
    """ee_cascade with its argument block built once (see PreparedCall)."""
    __slots__ = ("_args", "_keep", "out")

    def __init__(self, heads, ln_eps, out=None, workspace=None):
        self._args, self.out, self._keep = _cascade_args(heads, ln_eps, out, workspace)

    def __call__(self):
        code = _lib.load().ee_cascade(*self._args)
        if code:
            raise EExitError(code, "ee_cascade")
        return self.out


def _calibrate_args(entropy, argmax_head, argmax_final, epsilon, out, workspace):
    n = entropy.numel()
    dev = entropy.device
    if not (entropy.dtype == torch.float32 and argmax_head.dtype == torch.int32 and argmax_final.dtype == torch.int32):
        raise TypeError("entropy must be float32, the argmax arrays int32")
    if not (entropy.is_contiguous() and argmax_head.is_contiguous() and argmax_final.is_contiguous()):
        raise ValueError("calibration arrays must be contiguous")
    if out is None:
        out = dict(tau=torch.empty(1, dtype=torch.float32, device=dev), counts=torch.empty(3, dtype=torch.int32, device=dev))
    if workspace is None:
        workspace = torch.empty(int(_lib.load().ee_calibrate_workspace_bytes(n)), dtype=torch.uint8, device=dev)
    args = (_ptr(entropy), _ptr(argmax_head), _ptr(argmax_final), n, float(epsilon), _ptr(out["tau"]), _ptr(out["counts"]),
            _ptr(workspace), workspace.numel(), _stream())
    return args, out, (entropy, argmax_head, argmax_final, workspace, out)


def ee_calibrate(entropy, argmax_head, argmax_final, epsilon, *, out=None, workspace=None) -> dict:
    """Threshold of one head from a calibration set (see include/eexit.h): dict(tau [1], counts [3]) on the device."""
    args, out, _ = _calibrate_args(entropy, argmax_head, argmax_final, epsilon, out, workspace)
    _check(_lib.load().ee_calibrate(*args), "ee_calibrate")
    return out


def prepare_calibrate(entropy, argmax_head, argmax_final, epsilon, *, out=None, workspace=None) -> PreparedCall:
    args, out, keep = _calibrate_args(entropy, argmax_head, argmax_final, epsilon, out, workspace)
    return PreparedCall(_lib.load().ee_calibrate, args, "ee_calibrate", keep, out)


def dssd_commit(draft_tok, draft_exit_mask, verify_tok, eos_token, state: dict, *, out=None) -> dict:
    """Commit step of a DSSD round (see include/eexit.h).  `state` holds the sequences' device tensors: out_tok
    int32 [S, capacity], seq_len int32 [S], finished uint8 [S], stats int64 [4]; they are updated in place."""
    S, k = draft_tok.shape
    kv = verify_tok.shape[1]
    dev = draft_tok.device
    if not (draft_tok.is_contiguous() and verify_tok.is_contiguous() and state["out_tok"].is_contiguous()):
        raise ValueError("token arrays must be contiguous")
    if out is None:
        out = {n: torch.empty(S, dtype=torch.int32, device=dev) for n in ("draft_len", "accept_len", "next_tok")}
    _check(_lib.load().dssd_commit(_ptr(draft_tok), _ptr(draft_exit_mask), _ptr(verify_tok), S, k, kv, int(eos_token),
                                   _ptr(state["out_tok"]), state["out_tok"].shape[1], _ptr(state["seq_len"]),
                                   _ptr(state["finished"]), _ptr(out["draft_len"]), _ptr(out["accept_len"]),
                                   _ptr(out["next_tok"]), _ptr(state["stats"]), _stream()), "dssd_commit")
    return out


class TableModel:
    """Stand-in model for dssd_round served by the library itself (ee_hidden_from_tables in include/eexit.h): the
    hidden state after a token is that token's row of a table, one table per draft head's layer (`draft_table`: a
    tensor, or a list of K tensors, shallowest first) and `verify_table` for the verification pass, bf16 [V, d]
    device tensors.  Pass it to DssdRound as `hidden_fn`.  chained=True launches its kernel with programmatic stream
    serialization (early trigger, wait before the tokens are read)."""

    def __init__(self, draft_table, verify_table, chained: bool = False):
        drafts = list(draft_table) if isinstance(draft_table, (list, tuple)) else [draft_table]
        self.tables = tuple(_bf16(_dev(t, "table")) for t in drafts + [verify_table])
        if len(drafts) > _lib.EE_ROUND_MAX_DRAFT_HEADS:
            raise ValueError(f"at most {_lib.EE_ROUND_MAX_DRAFT_HEADS} draft tables")
        if any(t.shape != self.tables[0].shape for t in self.tables) or not all(t.is_contiguous() for t in self.tables):
            raise ValueError("tables must be contiguous and of one shape [V, d]")
        V, d = self.tables[0].shape
        self.struct = _lib.EEHiddenTables()
        for i, t in enumerate(self.tables):
            self.struct.table[i] = _ptr(t)
        self.struct.d, self.struct.V, self.struct.chained = d, V, int(bool(chained))


class DssdRound:
    """dssd_round (see include/eexit.h) with its argument block built once.

    draft_head: a dict with gamma, beta, W, tau, or a list of K such dicts (shallowest head first: per position the
    first confident one supplies the token); verify_head: dict with gamma, beta, W.  hidden_fn(tokens, which, h_out) is
    the caller's model: `tokens` int32 [n_rows] and `h_out` bf16 [n_rows, d] are device tensors (views into the
    workspace); it must fill h_out on the current stream with the hidden states at draft head `which`'s layer
    (which < K) or the full model's (which = K).  all_layers=True asks for ONE call per drafting step instead of K:
    which = -1 and h_out bf16 [K, n_rows, d], layer by layer (the library's TableModel is always driven that way).
    `state`: last_tok, out_tok, seq_len, finished, stats.  With a list
    of heads, self.head_use (int64 [K]) accumulates the positions each head supplied."""

    def __init__(self, draft_head, verify_head, ln_eps, k, eos_token, hidden_fn, state, workspace=None, all_layers=None):
        import ctypes as C
        S = state["last_tok"].numel()
        multi = isinstance(draft_head, (list, tuple))
        drafts = list(draft_head) if multi else [draft_head]
        K = len(drafts)
        Wd = [_bf16(_dev(h["W"], "W")) for h in drafts]
        Wv = _bf16(_dev(verify_head["W"], "W"))
        V, d = Wd[0].shape
        dev = Wd[0].device
        if workspace is None:
            workspace = torch.empty(int(_lib.load().dssd_round_multi_workspace_bytes(S, k, d, V, K)), dtype=torch.uint8, device=dev)
            ee_workspace_init(workspace)
        self.workspace, self.state = workspace, state
        self.out = {n: torch.empty(S, dtype=torch.int32, device=dev) for n in ("draft_len", "accept_len", "next_tok")}
        self.head_use = torch.zeros(K, dtype=torch.int64, device=dev) if multi else None
        base = workspace.data_ptr()

        def trampoline(user, tokens_ptr, n_rows, which, h_ptr, stream):
            try:
                tokens = workspace[tokens_ptr - base:tokens_ptr - base + 4 * n_rows].view(torch.int32)
                layers = K if which < 0 else 1
                h_out = workspace[h_ptr - base:h_ptr - base + 2 * layers * n_rows * d].view(torch.bfloat16)
                h_out = h_out.view(K, n_rows, d) if which < 0 else h_out.view(n_rows, d)
                hidden_fn(tokens, which, h_out)
                return 0
            except Exception:                    # an exception must not cross the C boundary
                import traceback
                traceback.print_exc()
                return 1

        native = isinstance(hidden_fn, TableModel)
        if native and (hidden_fn.tables[0].shape != (V, d) or len(hidden_fn.tables) != K + 1):
            raise ValueError("the table model needs one [V, d] table per draft head and one for the verification pass")
        self._cb = C.cast(_lib.load().ee_hidden_from_tables, _lib.HIDDEN_FN) if native else _lib.HIDDEN_FN(trampoline)
        a = _lib.EEDssdRoundArgs()
        a.S, a.k, a.d, a.V, a.ln_eps, a.eos_token = S, int(k), d, V, float(ln_eps), int(eos_token)
        arr = (_lib.EEHead * K)()
        for dst, src, W in [(arr[i], drafts[i], Wd[i]) for i in range(K)] + [(a.draft_head, drafts[0], Wd[0]), (a.verify_head, verify_head, Wv)]:
            dst.gamma, dst.beta, dst.W, dst.tau = _ptr(src["gamma"]), _ptr(src["beta"]), _ptr(W), float(src.get("tau", 0.0))
        if multi:
            a.n_draft_heads, a.draft_heads, a.head_use = K, arr, _ptr(self.head_use)
        a.hidden, a.hidden_user = self._cb, (C.cast(C.pointer(hidden_fn.struct), C.c_void_p) if native else None)
        a.hidden_all_layers = int(native if all_layers is None else bool(all_layers))
        a.last_tok, a.out_tok, a.capacity = _ptr(state["last_tok"]), _ptr(state["out_tok"]), state["out_tok"].shape[1]
        a.seq_len, a.finished, a.stats = _ptr(state["seq_len"]), _ptr(state["finished"]), _ptr(state["stats"])
        a.draft_len, a.accept_len, a.next_tok = (_ptr(self.out[n]) for n in ("draft_len", "accept_len", "next_tok"))
        a.workspace, a.workspace_bytes, a.stream = _ptr(workspace), workspace.numel(), _stream()
        self._args, self._keep = a, (Wd, Wv, drafts, verify_head, C, hidden_fn, arr)

    def __call__(self):
        import ctypes as C
        code = _lib.load().dssd_round(C.byref(self._args))
        if code:
            raise EExitError(code, "dssd_round")
        return self.out


def _accept_args(draft_tok, draft_exit_mask, verify_tok, out):
    S, k = draft_tok.shape
    kv = verify_tok.shape[1]
    dev = draft_tok.device
    if not (draft_tok.is_contiguous() and verify_tok.is_contiguous()):
        raise ValueError("token arrays must be contiguous")
    if out is None:
        out = {n: torch.empty(S, dtype=torch.int32, device=dev) for n in ("draft_len", "accept_len", "next_tok")}
    args = (_ptr(draft_tok), _ptr(draft_exit_mask), _ptr(verify_tok), S, k, kv,
            _ptr(out["draft_len"]), _ptr(out["accept_len"]), _ptr(out["next_tok"]), _stream())
    return args, out, (draft_tok, draft_exit_mask, verify_tok, out)


def ee_query_async_error(workspace) -> int:
    """Synchronises the current stream; 0 if no bounded wait gave up since the last query, else EE_ERR_TIMEOUT."""
    return int(_lib.load().ee_query_async_error(_ptr(workspace), _stream()))
