"""Python binding of the C ABI declared in include/rpd.h.

Argument marshalling only: torch tensors supply device memory and the
current stream; every step of the commit step runs in the HIP library
``librpd.so``. The library is loaded on first use and its absence is an
error (there is no other implementation behind these functions).
"""
from __future__ import annotations

import ctypes
import os
from dataclasses import dataclass

import torch

_LIB_PATH = os.path.join(os.path.dirname(os.path.abspath(__file__)), "librpd.so")

DTYPE_BF16 = 0
DTYPE_F32 = 1
DTYPE_F16 = 2   # the operators beside the commit step only

FLAG_CANDIDATE = 1
FLAG_HIGH_CONF = 2
FLAG_STABLE = 4
FLAG_COMMITTED = 8
FLAG_FALLBACK = 16

DEVICE_STATUS_MASKED_OVERFLOW = 1
ABI_VERSION = 3   # RPD_ABI_VERSION: the layouts and entry points this binding marshals for
PARAM_LAZY = 1
PARAM_LAZY_ALL = 2

STATUS_NAMES = {0: "RPD_OK", 1: "RPD_ERR_NULL_POINTER", 2: "RPD_ERR_BAD_SHAPE", 3: "RPD_ERR_BAD_PARAM",
                4: "RPD_ERR_WORKSPACE_TOO_SMALL", 5: "RPD_ERR_UNSUPPORTED", 6: "RPD_ERR_HIP"}


class RpdProblem(ctypes.Structure):
    _fields_ = [("K", ctypes.c_int32), ("B", ctypes.c_int32), ("L", ctypes.c_int32),
                ("d", ctypes.c_int32), ("V", ctypes.c_int32), ("dtype", ctypes.c_int32),
                ("hidden", ctypes.c_void_p), ("w_u", ctypes.c_void_p), ("mask", ctypes.c_void_p),
                ("max_masked", ctypes.c_int32), ("norm_weight", ctypes.c_void_p), ("norm_eps", ctypes.c_float),
                ("norm_final", ctypes.c_int32)]


class RpdParams(ctypes.Structure):
    _fields_ = [("theta_h", ctypes.c_float), ("theta_c", ctypes.c_float), ("theta_s", ctypes.c_float),
                ("w", ctypes.c_float), ("k_max", ctypes.c_int32), ("beta", ctypes.c_float),
                ("window", ctypes.c_int32), ("flags", ctypes.c_uint32), ("block", ctypes.c_int32),
                ("logit_scale", ctypes.c_float)]


class RpdQuantHead(ctypes.Structure):
    _fields_ = [(n, ctypes.c_int32) for n in ("V", "d", "group", "dtype", "has_zeros")]


class RpdVerify(ctypes.Structure):
    _fields_ = [("B", ctypes.c_int32), ("T", ctypes.c_int32), ("V", ctypes.c_int32), ("dtype", ctypes.c_int32),
                ("target", ctypes.c_void_p), ("target_batch_stride", ctypes.c_int64),
                ("target_row_stride", ctypes.c_int64),
                ("draft", ctypes.c_void_p), ("draft_batch_stride", ctypes.c_int64),
                ("draft_row_stride", ctypes.c_int64),
                ("token", ctypes.c_void_p), ("len", ctypes.c_void_p), ("u", ctypes.c_void_p), ("r", ctypes.c_void_p),
                ("target_scale", ctypes.c_float), ("draft_scale", ctypes.c_float), ("flags", ctypes.c_uint32),
                ("out_token", ctypes.c_void_p), ("n_accept", ctypes.c_void_p), ("accept", ctypes.c_void_p)]


class RpdDistill(ctypes.Structure):
    _fields_ = [("N", ctypes.c_int32), ("V", ctypes.c_int32), ("k", ctypes.c_int32), ("dtype", ctypes.c_int32),
                ("teacher_dtype", ctypes.c_int32),
                ("logits", ctypes.c_void_p), ("logits_stride", ctypes.c_int64), ("id", ctypes.c_void_p),
                ("teacher", ctypes.c_void_p), ("teacher_lse", ctypes.c_void_p), ("weight", ctypes.c_void_p),
                ("grad_loss", ctypes.c_void_p), ("logit_scale", ctypes.c_float), ("loss", ctypes.c_void_p),
                ("state", ctypes.c_void_p), ("grad", ctypes.c_void_p), ("grad_stride", ctypes.c_int64)]


_OUT_FIELDS = ["commit", "token", "entropy", "confidence", "persistence", "drop", "stability", "flags",
               "upstream_entropy", "n_commit", "layer_argmax", "layer_conf", "layer_entropy", "status"]


class RpdOutputs(ctypes.Structure):
    _fields_ = [(n, ctypes.c_void_p) for n in _OUT_FIELDS]


@dataclass(frozen=True)
class Params:
    """Commit-rule hyperparameters (Table 4, Appendix A.6)."""
    theta_h: float = 0.9
    theta_c: float = 0.6
    theta_s: float = 3.5
    w: float = 15.0
    k_max: int = 6
    beta: float = 4.0
    window: int = 32
    block: int = 0     # 0: full RPD; > 0: RPD-block with blocks of this many positions
    logit_scale: float = 1.0   # inverse temperature of the scoring softmax
    lazy: bool = False         # lazy layerwise projection (RPD_PARAM_LAZY)
    lazy_all: bool = False     # with lazy: every masked position walks its layers (RPD_PARAM_LAZY_ALL)

    @staticmethod
    def llada() -> "Params":
        return Params(theta_s=3.5, w=15.0)

    @staticmethod
    def dream() -> "Params":
        return Params(theta_s=2.5, w=20.0)

    @staticmethod
    def strict(K: int, beta: float = 1.0) -> "Params":
        """All K layers agree and the final probability is the peak (Eq. 4
        with w = 1, K_max >= K, theta_s = K)."""
        return Params(theta_s=float(K), w=1.0, k_max=max(K, 6), beta=beta)

    def to_c(self) -> RpdParams:
        flags = (PARAM_LAZY if self.lazy else 0) | (PARAM_LAZY_ALL if self.lazy_all else 0)
        return RpdParams(self.theta_h, self.theta_c, self.theta_s, self.w, int(self.k_max), self.beta,
                         int(self.window), flags, int(self.block), float(self.logit_scale))


class RpdError(RuntimeError):
    def __init__(self, status: int, detail: str):
        super().__init__(f"{STATUS_NAMES.get(status, status)}: {detail}")
        self.status = status


_lib = None


def lib() -> ctypes.CDLL:
    global _lib
    if _lib is None:
        if not os.path.exists(_LIB_PATH):
            raise RuntimeError(f"{_LIB_PATH} is missing: build it with __graft_entry__.build() "
                               "(the commit step has no other implementation)")
        L = ctypes.CDLL(_LIB_PATH)
        L.rpd_workspace_size.restype = ctypes.c_size_t
        L.rpd_workspace_size.argtypes = [ctypes.POINTER(RpdProblem)]
        L.rpd_score_commit.restype = ctypes.c_int
        L.rpd_score_commit.argtypes = [ctypes.POINTER(RpdProblem), ctypes.POINTER(RpdParams),
                                       ctypes.POINTER(RpdOutputs), ctypes.c_void_p, ctypes.c_size_t,
                                       ctypes.c_void_p]
        L.rpd_score_commit_timed.restype = ctypes.c_int
        L.rpd_score_commit_timed.argtypes = [ctypes.POINTER(RpdProblem), ctypes.POINTER(RpdParams),
                                             ctypes.POINTER(RpdOutputs), ctypes.c_void_p, ctypes.c_size_t,
                                             ctypes.c_void_p, ctypes.POINTER(ctypes.c_void_p), ctypes.c_int32]
        L.rpd_score_commit_noalloc.restype = ctypes.c_int
        L.rpd_score_commit_noalloc.argtypes = [ctypes.POINTER(RpdProblem), ctypes.POINTER(RpdParams),
                                               ctypes.POINTER(RpdOutputs), ctypes.c_void_p]
        L.rpd_gate_commit.restype = ctypes.c_int
        L.rpd_gate_commit.argtypes = [ctypes.c_int32, ctypes.c_int32, ctypes.c_int32, ctypes.c_void_p,
                                      ctypes.c_void_p, ctypes.c_void_p, ctypes.c_void_p,
                                      ctypes.POINTER(RpdParams), ctypes.POINTER(RpdOutputs), ctypes.c_void_p]
        L.rpd_apply_commit.restype = ctypes.c_int
        L.rpd_apply_commit.argtypes = [ctypes.c_int32, ctypes.c_int32, ctypes.c_void_p, ctypes.c_void_p,
                                       ctypes.c_void_p, ctypes.c_void_p, ctypes.c_void_p, ctypes.c_int32,
                                       ctypes.c_void_p, ctypes.c_void_p]
        v, i32, i64, size = ctypes.c_void_p, ctypes.c_int32, ctypes.c_int64, ctypes.c_size_t
        head, ver, dis = ctypes.POINTER(RpdQuantHead), ctypes.POINTER(RpdVerify), ctypes.POINTER(RpdDistill)
        for name, res, args in (
                ("rpd_quant_packed_size", size, [head]),
                ("rpd_quant_pack", ctypes.c_int, [head, v, v, v, v, size, v]),
                ("rpd_quant_workspace_size", size, [head, i32, i32]),
                ("rpd_quant_project", ctypes.c_int,
                 [head, v, i32, v, i64, v, i64, i32, v, v, v, ctypes.c_float, v, size, v]),
                ("rpd_verify_workspace_size", size, [ver]),
                ("rpd_verify_draft", ctypes.c_int, [ver, v, size, v]),
                ("rpd_distill_workspace_size", size, [dis]),
                ("rpd_distill_loss", ctypes.c_int, [dis, v, size, v]),
                ("rpd_distill_grad", ctypes.c_int, [dis, v])):
            f = getattr(L, name)
            f.restype, f.argtypes = res, args
        L.rpd_status_string.restype = ctypes.c_char_p
        L.rpd_status_string.argtypes = [ctypes.c_int]
        L.rpd_last_error.restype = ctypes.c_char_p
        L.rpd_last_error.argtypes = []
        L.rpd_projection_variant.restype = ctypes.c_int32
        L.rpd_projection_variant.argtypes = [ctypes.POINTER(RpdProblem)]
        L.rpd_abi_version.restype = ctypes.c_int32
        L.rpd_abi_version.argtypes = []
        if L.rpd_abi_version() != ABI_VERSION:
            raise RuntimeError(f"{_LIB_PATH} has ABI version {L.rpd_abi_version()}, this binding needs "
                               f"{ABI_VERSION}: rebuild the library")
        _lib = L
    return _lib


def status_string(s: int) -> str:
    return lib().rpd_status_string(s).decode()


def last_error() -> str:
    return lib().rpd_last_error().decode()


def abi_version() -> int:
    return int(lib().rpd_abi_version())


def _check(status: int) -> None:
    if status != 0:
        raise RpdError(status, last_error())


def _ptr(t: torch.Tensor | None) -> int | None:
    return None if t is None else t.data_ptr()


def _dtype_code(t: torch.Tensor) -> int:
    if t.dtype == torch.bfloat16:
        return DTYPE_BF16
    if t.dtype == torch.float32:
        return DTYPE_F32
    raise TypeError(f"unsupported dtype {t.dtype} (bfloat16 or float32)")


def make_problem(K, B, L, d, V, dtype_code, hidden=None, w_u=None, mask=None, max_masked=-1,
                 norm_weight=None, norm_eps: float = 0.0, norm_final: bool = False) -> RpdProblem:
    nw = norm_weight if isinstance(norm_weight, (int, type(None))) else _ptr(norm_weight)
    return RpdProblem(K, B, L, d, V, dtype_code, _ptr(hidden), _ptr(w_u), _ptr(mask), int(max_masked),
                      nw, float(norm_eps), int(bool(norm_final)))


def workspace_size(K: int, B: int, L: int, d: int, V: int, dtype: torch.dtype | int,
                   max_masked: int = -1, norm: bool = False) -> int:
    code = dtype if isinstance(dtype, int) else (DTYPE_BF16 if dtype == torch.bfloat16 else DTYPE_F32)
    p = make_problem(K, B, L, d, V, code, max_masked=max_masked, norm_weight=1 if norm else None)
    return int(lib().rpd_workspace_size(ctypes.byref(p)))


PROJ_VARIANTS = {0: "bf16_s32", 1: "bf16_s64", 3: "f32", 4: "bf16_big", 6: "bf16_big192", 7: "bf16_big128"}


def projection_variant(K: int, B: int, L: int, d: int, V: int, dtype: torch.dtype | int,
                       max_masked: int = -1) -> str:
    """Name of the projection kernel variant rpd_score_commit launches for
    this shape (rpd_projection_variant)."""
    code = dtype if isinstance(dtype, int) else (DTYPE_BF16 if dtype == torch.bfloat16 else DTYPE_F32)
    p = make_problem(K, B, L, d, V, code, max_masked=max_masked)
    v = int(lib().rpd_projection_variant(ctypes.byref(p)))
    if v < 0:
        raise RpdError(2, f"invalid shape or dtype for a plan: K={K} B={B} L={L} d={d} V={V} dtype={code}")
    return PROJ_VARIANTS[v]


def alloc_outputs(K: int, B: int, L: int, device, layer_stats: bool = False) -> dict:
    e = dict(device=device)
    o = {
        "commit": torch.empty((B, L), dtype=torch.uint8, **e),
        "token": torch.empty((B, L), dtype=torch.int32, **e),
        "entropy": torch.empty((B, L), dtype=torch.float32, **e),
        "confidence": torch.empty((B, L), dtype=torch.float32, **e),
        "persistence": torch.empty((B, L), dtype=torch.int32, **e),
        "drop": torch.empty((B, L), dtype=torch.float32, **e),
        "stability": torch.empty((B, L), dtype=torch.float32, **e),
        "flags": torch.empty((B, L), dtype=torch.uint8, **e),
        "upstream_entropy": torch.empty((B, L), dtype=torch.float32, **e),
        "n_commit": torch.empty((B,), dtype=torch.int32, **e),
        "status": torch.empty((1,), dtype=torch.int32, **e),
    }
    if layer_stats:
        o["layer_argmax"] = torch.empty((K, B, L), dtype=torch.int32, **e)
        o["layer_conf"] = torch.empty((K, B, L), dtype=torch.float32, **e)
        o["layer_entropy"] = torch.empty((K, B, L), dtype=torch.float32, **e)
    return o


def _outputs_struct(o: dict) -> RpdOutputs:
    return RpdOutputs(*[_ptr(o.get(n)) for n in _OUT_FIELDS])


def _stream_handle(stream) -> int | None:
    s = torch.cuda.current_stream() if stream is None else stream
    return s.cuda_stream or None


def _check_dev(name: str, t: torch.Tensor, shape: tuple, dtypes) -> None:
    if not t.is_cuda:
        raise ValueError(f"{name} must be a device tensor")
    if tuple(t.shape) != tuple(shape):
        raise ValueError(f"{name} has shape {tuple(t.shape)}, expected {tuple(shape)}")
    if t.dtype not in dtypes:
        raise TypeError(f"{name} has dtype {t.dtype}")
    if not t.is_contiguous():
        raise ValueError(f"{name} must be contiguous")


class ScoreCommit:
    """A reusable call of ``rpd_score_commit`` for one problem shape: the
    outputs and the workspace are allocated once (by torch) and every
    ``__call__`` only enqueues the library's kernels."""

    def __init__(self, hidden: torch.Tensor, w_u: torch.Tensor, mask: torch.Tensor, params: Params,
                 max_masked: int | None = None, layer_stats: bool = False, norm_weight: torch.Tensor | None = None,
                 norm_eps: float = 1e-5, norm_final: bool = False):
        K, B, L, d = hidden.shape
        V = w_u.shape[0]
        code = _dtype_code(hidden)
        _check_dev("hidden", hidden, (K, B, L, d), (hidden.dtype,))
        _check_dev("w_u", w_u, (V, d), (hidden.dtype,))
        _check_dev("mask", mask, (B, L), (torch.uint8, torch.bool))
        if norm_weight is not None:
            _check_dev("norm_weight", norm_weight, (d,), (hidden.dtype,))
        mm = -1 if max_masked is None else int(max_masked)
        self.problem = make_problem(K, B, L, d, V, code, hidden, w_u, mask.view(torch.uint8), mm,
                                    norm_weight, norm_eps, norm_final)
        self.params = params.to_c()
        self.out = alloc_outputs(K, B, L, hidden.device, layer_stats)
        self.out_c = _outputs_struct(self.out)
        nbytes = int(lib().rpd_workspace_size(ctypes.byref(self.problem)))
        if nbytes == 0:
            raise ValueError("invalid problem shape")
        self.workspace = torch.empty(nbytes, dtype=torch.uint8, device=hidden.device)
        self._keep = (hidden, w_u, mask, norm_weight)

    def __call__(self, stream=None, events=None) -> dict:
        """Enqueue one call. ``events``: optional list of up to five
        ``torch.cuda.Event`` (or None) recorded at the stage boundaries
        (``rpd_score_commit_timed``)."""
        if events is None:
            _check(lib().rpd_score_commit(ctypes.byref(self.problem), ctypes.byref(self.params),
                                          ctypes.byref(self.out_c), self.workspace.data_ptr(),
                                          self.workspace.numel(), _stream_handle(stream)))
        else:
            arr = (ctypes.c_void_p * len(events))(*[None if e is None else e.cuda_event for e in events])
            _check(lib().rpd_score_commit_timed(ctypes.byref(self.problem), ctypes.byref(self.params),
                                                ctypes.byref(self.out_c), self.workspace.data_ptr(),
                                                self.workspace.numel(), _stream_handle(stream), arr,
                                                len(events)))
        return self.out


def score_commit(hidden: torch.Tensor, w_u: torch.Tensor, mask: torch.Tensor, params: Params,
                 max_masked: int | None = None, layer_stats: bool = False, stream=None,
                 norm_weight: torch.Tensor | None = None, norm_eps: float = 1e-5, norm_final: bool = False) -> dict:
    """``rpd_score_commit``: the whole commit step of one decoding iteration.

    hidden [K][B][L][d] and w_u [V][d] (bfloat16 or float32, same dtype,
    device, contiguous), mask [B][L] uint8/bool; optional norm_weight [d]
    (the gain of the model's final normalization, applied to layers 0..K-2,
    and to K-1 with norm_final). Returns the output tensors (see
    include/rpd.h), valid once the stream has run."""
    return ScoreCommit(hidden, w_u, mask, params, max_masked, layer_stats, norm_weight, norm_eps,
                       norm_final)(stream)


NOALLOC_SCRATCH_BYTES = 64 << 20   # RPD_NOALLOC_SCRATCH_BYTES


def score_commit_noalloc(hidden: torch.Tensor, w_u: torch.Tensor, mask: torch.Tensor, params: Params,
                         max_masked: int | None = None, layer_stats: bool = False, stream=None,
                         norm_weight: torch.Tensor | None = None, norm_eps: float = 1e-5, norm_final: bool = False,
                         out: dict | None = None) -> dict:
    """``rpd_score_commit_noalloc``: the commit step on the library's static
    scratch array instead of a workspace (for callers that cannot allocate
    device memory; calls that overlap on one GPU race). ``out``: output
    tensors from a previous call or ``alloc_outputs`` (allocated here if
    None). Returns the output tensors."""
    K, B, L, d = hidden.shape
    V = w_u.shape[0]
    _check_dev("hidden", hidden, (K, B, L, d), (hidden.dtype,))
    _check_dev("w_u", w_u, (V, d), (hidden.dtype,))
    _check_dev("mask", mask, (B, L), (torch.uint8, torch.bool))
    if norm_weight is not None:
        _check_dev("norm_weight", norm_weight, (d,), (hidden.dtype,))
    mm = -1 if max_masked is None else int(max_masked)
    problem = make_problem(K, B, L, d, V, _dtype_code(hidden), hidden, w_u, mask.view(torch.uint8), mm,
                           norm_weight, norm_eps, norm_final)
    o = alloc_outputs(K, B, L, hidden.device, layer_stats) if out is None else out
    q = params.to_c()
    oc = _outputs_struct(o)
    _check(lib().rpd_score_commit_noalloc(ctypes.byref(problem), ctypes.byref(q), ctypes.byref(oc),
                                          _stream_handle(stream)))
    return o


def gate_commit(mask: torch.Tensor, layer_argmax: torch.Tensor, layer_conf: torch.Tensor,
                layer_entropy: torch.Tensor, params: Params, stream=None) -> dict:
    """``rpd_gate_commit``: scoring and commitment from per-layer statistics
    ([K][B][L] int32 / float32 / float32 device tensors)."""
    K, B, L = layer_argmax.shape
    _check_dev("mask", mask, (B, L), (torch.uint8, torch.bool))
    _check_dev("layer_argmax", layer_argmax, (K, B, L), (torch.int32,))
    _check_dev("layer_conf", layer_conf, (K, B, L), (torch.float32,))
    _check_dev("layer_entropy", layer_entropy, (K, B, L), (torch.float32,))
    out = alloc_outputs(K, B, L, mask.device, False)
    oc = _outputs_struct(out)
    q = params.to_c()
    _check(lib().rpd_gate_commit(K, B, L, mask.view(torch.uint8).data_ptr(), layer_argmax.data_ptr(),
                                 layer_conf.data_ptr(), layer_entropy.data_ptr(), ctypes.byref(q),
                                 ctypes.byref(oc), _stream_handle(stream)))
    return out


def apply_commit(mask: torch.Tensor, canvas: torch.Tensor, commit: torch.Tensor, token: torch.Tensor,
                 progress: torch.Tensor | None = None, step: torch.Tensor | None = None, stream=None) -> None:
    """``rpd_apply_commit``: committed positions take their token in the
    canvas and leave the mask (in place). mask [B][L] uint8/bool, canvas and
    token [B][L] int32, commit [B][L] uint8; optional progress int32
    [1 + n] (call counter, then the masked count left after each call) and
    step int32 [B][L] (the call index at which each position was filled)."""
    B, L = mask.shape
    _check_dev("mask", mask, (B, L), (torch.uint8, torch.bool))
    _check_dev("canvas", canvas, (B, L), (torch.int32,))
    _check_dev("commit", commit, (B, L), (torch.uint8,))
    _check_dev("token", token, (B, L), (torch.int32,))
    n = 0
    if progress is not None:
        if progress.dim() != 1 or progress.numel() < 1:
            raise ValueError("progress must be a 1-d tensor of at least one element")
        _check_dev("progress", progress, (progress.numel(),), (torch.int32,))
        n = progress.numel() - 1
    if step is not None:
        _check_dev("step", step, (B, L), (torch.int32,))
    _check(lib().rpd_apply_commit(B, L, mask.view(torch.uint8).data_ptr(), canvas.data_ptr(), commit.data_ptr(),
                                  token.data_ptr(), _ptr(progress), n, _ptr(step), _stream_handle(stream)))


class Decoder:
    """Iterations of the commit step until no position is masked (Section
    3.2): each iteration is ``rpd_score_commit`` followed by
    ``rpd_apply_commit`` on the same stream, over hidden states that stay
    fixed between iterations (they stand in for the forward passes of the
    model, which this library does not run).

    Every iteration commits at least one masked position (the progress
    fallback), so after t iterations at most n0 - t positions are masked; that
    bound is the ``max_masked`` of the call, and the masked count left after
    each iteration is recorded on the device (``progress``) and read back
    only every ``sync_every`` iterations, to tighten the bound and to stop.
    Iterations that find the canvas already full change nothing. With
    ``graph=True`` one iteration is captured in a HIP graph per plan and
    replayed: a plan is made for the first bound that needs it and serves
    every smaller bound of the same projection variant (down to half its
    bound for the variants whose grid grows with the rows). Plans are kept
    across ``reset()``, so repeated decodes replay the same graphs. A lazy
    call reads counts back while its bound exceeds 256 positions, so those
    iterations run eagerly and the rest replay graphs."""

    def __init__(self, hidden: torch.Tensor, w_u: torch.Tensor, mask: torch.Tensor, params: Params,
                 norm_weight: torch.Tensor | None = None, norm_eps: float = 1e-5, norm_final: bool = False,
                 graph: bool = True, sync_every: int = 8):
        K, B, L, d = hidden.shape
        _check_dev("mask", mask, (B, L), (torch.uint8, torch.bool))
        self.hidden, self.w_u, self.params = hidden, w_u, params
        self.norm = dict(norm_weight=norm_weight, norm_eps=norm_eps, norm_final=norm_final)
        self.sync_every = max(1, int(sync_every))
        self.shape = (K, B, L, d, w_u.shape[0])
        dev = hidden.device
        self.mask0 = mask.view(torch.uint8).clone()
        self.mask = self.mask0.clone()
        self.n0 = int(self.mask0.sum().item())
        self.graph = bool(graph)
        self.canvas = torch.full((B, L), -1, dtype=torch.int32, device=dev)
        self.step = torch.full((B, L), -1, dtype=torch.int32, device=dev)
        self.progress = torch.zeros(1 + max(self.n0, 1), dtype=torch.int32, device=dev)
        self._plans: dict[tuple, list] = {}   # (variant, captured) -> [(bound, ScoreCommit, graph or None)]
        self.captures = 0
        self.bounds: list[int] = []    # the max_masked of each enqueued iteration

    def reset(self) -> None:
        """Start a new decode from the initial mask (the plans are kept)."""
        self.mask.copy_(self.mask0)
        self.canvas.fill_(-1)
        self.step.fill_(-1)
        self.progress.zero_()
        self.bounds = []

    def _iteration(self, sc: ScoreCommit, events=None) -> None:
        o = sc(events=events)
        apply_commit(self.mask, self.canvas, o["commit"], o["token"], self.progress, self.step)

    def _plan_for(self, bound: int):
        K, B, L, d, V = self.shape
        variant = projection_variant(K, B, L, d, V, self.hidden.dtype, max_masked=bound)
        # a lazy call reads counts back (and cannot be captured) while its bound exceeds 256
        capture = self.graph and (not self.params.lazy or bound <= 256)
        plans = self._plans.setdefault((variant, capture), [])
        fits = [p for p in plans if p[0] >= bound and (variant.startswith("bf16_s") or 2 * bound > p[0])]
        if fits:
            return min(fits, key=lambda p: p[0])
        sc = ScoreCommit(self.hidden, self.w_u, self.mask, self.params, max_masked=bound, **self.norm)
        g = None
        if capture:
            g = torch.cuda.CUDAGraph()
            with torch.cuda.graph(g):
                self._iteration(sc)
            self.captures += 1
        plans.append((bound, sc, g))
        return plans[-1]

    def run(self, max_iter: int | None = None, stage_events: bool = False) -> dict:
        """Decode until the canvas is full (or ``max_iter`` iterations);
        returns the canvas (-1 where never filled), the iteration at which
        each position was filled (``step``, -1 if never), the number of
        iterations that committed something (``iterations``, the NFE of the
        loop), the masked count left after each of them (``left``) and the
        number of enqueued iterations (``calls``). With ``stage_events``
        every iteration runs eagerly with events around its projection stage
        and ``proj_ms`` lists the projection time of each iteration."""
        limit = self.n0 if max_iter is None else min(int(max_iter), self.n0)
        t, known, t_known = 0, self.n0, 0
        ev = []
        while t < limit and known > 0:
            chunk = min(self.sync_every, limit - t)
            for _ in range(chunk):
                bound = max(known - (t - t_known), 1)
                bnd, sc, g = self._plan_for(bound)
                self.bounds.append(bnd)
                if stage_events:
                    pair = (torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True))
                    for e in pair:         # torch creates the HIP event at its first record
                        e.record()
                    ev.append(pair)
                    self._iteration(sc, events=[None, pair[0], pair[1]])
                elif g is not None:
                    g.replay()
                else:
                    self._iteration(sc)
                t += 1
            known, t_known = int(self.progress[t].item()), t
        left = self.progress[1:1 + t].cpu().tolist()
        iters = next((i + 1 for i, n in enumerate(left) if n == 0), t)
        out = {"canvas": self.canvas, "step": self.step, "mask": self.mask, "iterations": iters,
               "left": left[:iters], "calls": t}
        if stage_events:
            torch.cuda.synchronize()
            out["proj_ms"] = [a.elapsed_time(b) for a, b in ev]
        return out


# ------------------------------------------------ operators beside the commit step --

_FLOAT_CODES = {torch.bfloat16: DTYPE_BF16, torch.float32: DTYPE_F32, torch.float16: DTYPE_F16}
VERIFY_GREEDY = 1
DISTILL_MAX_K = 256
DISTILL_STATE = 8


def _float_code(name: str, t: torch.Tensor) -> int:
    if t.dtype not in _FLOAT_CODES:
        raise TypeError(f"{name} has dtype {t.dtype} (bfloat16, float16 or float32)")
    return _FLOAT_CODES[t.dtype]


def _one_device(first: str, t: torch.Tensor, **others) -> torch.device:
    """The device that t and every other tensor given are on."""
    if not t.is_cuda:
        raise ValueError(f"{first} must be a device tensor")
    for name, o in others.items():
        if o is not None and o.device != t.device:
            raise ValueError(f"{name} is on {o.device}, {first} on {t.device}")
    return t.device


def _rows(name: str, t: torch.Tensor) -> torch.Tensor:
    """t [..., n] as 2-d rows: the last dimension contiguous, the leading ones of one stride (a view, never a copy)."""
    if t.dim() < 1 or (t.shape[-1] > 1 and t.stride(-1) != 1):
        raise ValueError(f"{name} must be contiguous in its last dimension")
    try:
        r = t.view(-1, t.shape[-1]) if t.dim() != 2 else t
    except RuntimeError as e:
        raise ValueError(f"{name}'s leading dimensions must be rows of one stride (call .contiguous())") from e
    if r.shape[0] > 1 and r.stride(0) < r.shape[1]:
        raise ValueError(f"{name}'s rows overlap")
    return r


def _row_stride(r: torch.Tensor) -> int:
    return r.stride(0) if r.shape[0] > 1 else max(r.shape[1], 1)


def _enqueue(device: torch.device, stream, entry, *args) -> None:
    """entry(*args, stream handle) with ``device`` current, on ``stream`` or that device's current stream."""
    if device.index != torch.cuda.current_device():
        with torch.cuda.device(device):
            return _enqueue(device, stream, entry, *args)
    handle = torch._C._cuda_getCurrentRawStream(device.index) if stream is None else stream.cuda_stream
    _check(entry(*args, handle or None))


class QuantHead:
    """An output head with 4-bit weights and group scales (``rpd_quant_pack``, ``rpd_quant_project``):
    W[v][k] = scales[v][k // group] * (code[v][k] - zeros[v][k // group]).

    codes uint8 [V][d/2] (column 2j in the low nibble of byte j, 2j+1 in the high one), scales [V][ceil(d/group)]
    bfloat16 or float16, optional zeros uint8 of the same shape (values 0..15; 8 everywhere without). Packs them once
    into ``packed`` on the current stream; the inputs are not kept. Outputs and workspaces of the calls are made on
    the current stream as well: another one that is given as ``stream`` has to wait for it beforehand
    (``stream.wait_stream``), as for any tensor of the caller's."""

    def __init__(self, codes: torch.Tensor, scales: torch.Tensor, zeros: torch.Tensor | None = None,
                 group: int = 128):
        self.device = _one_device("codes", codes, scales=scales, zeros=zeros)
        if codes.dim() != 2:
            raise ValueError("codes must be [V][d/2]")
        if scales.dtype not in (torch.bfloat16, torch.float16):
            raise TypeError(f"scales has dtype {scales.dtype} (bfloat16 or float16)")
        V, d = codes.shape[0], 2 * codes.shape[1]
        groups = -(-d // group) if group > 0 else 0
        _check_dev("codes", codes, (V, d // 2), (torch.uint8,))
        _check_dev("scales", scales, (V, groups), (scales.dtype,))
        if zeros is not None:
            _check_dev("zeros", zeros, (V, groups), (torch.uint8,))
        self.V, self.d, self.group, self.dtype = V, d, int(group), scales.dtype
        self.head = RpdQuantHead(V, d, self.group, _FLOAT_CODES[scales.dtype], int(zeros is not None))
        # an invalid head has size 0, and the call below says what is wrong with it
        self.packed = torch.empty(max(int(lib().rpd_quant_packed_size(ctypes.byref(self.head))), 1),
                                  dtype=torch.uint8, device=self.device)
        _enqueue(self.device, None, lib().rpd_quant_pack, ctypes.byref(self.head), codes.data_ptr(),
                 scales.data_ptr(), _ptr(zeros), self.packed.data_ptr(), self.packed.numel())

    def _x(self, x: torch.Tensor) -> torch.Tensor:
        _one_device("x", x, packed=self.packed)
        if x.dtype != self.dtype:
            raise TypeError(f"x has dtype {x.dtype}, the head {self.dtype}")
        if x.shape[-1] != self.d:
            raise ValueError(f"x has {x.shape[-1]} columns, the head {self.d}")
        return _rows("x", x)

    def _workspace(self, M: int, statistics: int, stream) -> tuple[torch.Tensor | None, int]:
        nbytes = int(lib().rpd_quant_workspace_size(ctypes.byref(self.head), M, statistics))
        if nbytes == 0:
            return None, 0
        ws = torch.empty(nbytes, dtype=torch.uint8, device=self.device)
        if stream is not None:
            ws.record_stream(stream)
        return ws, nbytes

    def logits(self, x: torch.Tensor, out_dtype: torch.dtype | None = None, out: torch.Tensor | None = None,
               stream=None) -> torch.Tensor:
        """x [..., d] through the head: [..., V] of type ``out_dtype`` (x's, or float32), into ``out`` if given."""
        r = self._x(x)
        if out is None:
            out = torch.empty((*x.shape[:-1], self.V), dtype=out_dtype or x.dtype, device=x.device)
            out_stride = self.V
        else:
            if tuple(out.shape) != (*x.shape[:-1], self.V) or (out_dtype and out.dtype != out_dtype):
                raise ValueError(f"out has shape {tuple(out.shape)} and dtype {out.dtype}")
            _one_device("out", out, x=x)
            out_stride = _row_stride(_rows("out", out))
        code = _float_code("out", out)
        ws, nbytes = self._workspace(r.shape[0], 0, stream)
        _enqueue(x.device, stream, lib().rpd_quant_project, ctypes.byref(self.head), self.packed.data_ptr(),
                 r.shape[0], r.data_ptr(), _row_stride(r), out.data_ptr(), out_stride, code, None, None, None, 1.0,
                 _ptr(ws), nbytes)
        return out

    def stats(self, x: torch.Tensor, logit_scale: float = 1.0, stream=None) -> dict:
        """The softmax statistics of logit_scale * (x through the head), as ``gate_commit`` takes them for
        x [K][B][L][d]: argmax int32, confidence and entropy float32, of x's leading shape."""
        r = self._x(x)
        e = dict(device=x.device)
        o = {"argmax": torch.empty(x.shape[:-1], dtype=torch.int32, **e),
             "confidence": torch.empty(x.shape[:-1], dtype=torch.float32, **e),
             "entropy": torch.empty(x.shape[:-1], dtype=torch.float32, **e)}
        ws, nbytes = self._workspace(r.shape[0], 1, stream)
        _enqueue(x.device, stream, lib().rpd_quant_project, ctypes.byref(self.head), self.packed.data_ptr(),
                 r.shape[0], r.data_ptr(), _row_stride(r), None, 0, 0, o["argmax"].data_ptr(),
                 o["confidence"].data_ptr(), o["entropy"].data_ptr(), float(logit_scale), _ptr(ws), nbytes)
        return o


class VerifyDraft:
    """A reusable call of ``rpd_verify_draft`` on given tensors: outputs and workspace are allocated once and every
    ``__call__`` only enqueues the library's kernels (on the tensors' values of that time).

    target_logits [B][T+1][V] (bfloat16, float16 or float32; last dimension contiguous), draft_token int32 [B][T],
    u float32 [B][T] and r float32 [B] in [0, 1) (neither with ``greedy``), optional draft_logits [B][T][V] of the
    same type and draft_len int32 [B]. Returns token int32 [B][T+1] (the accepted tokens, the one drawn after them,
    then -1), n_accept int32 [B] and accept float32 [B][T] (see include/rpd.h). The workspace and the outputs are
    this object's: calls that overlap need objects of their own."""

    def __init__(self, target_logits: torch.Tensor, draft_token: torch.Tensor, u: torch.Tensor | None = None,
                 r: torch.Tensor | None = None, draft_logits: torch.Tensor | None = None,
                 draft_len: torch.Tensor | None = None, target_scale: float = 1.0, draft_scale: float = 1.0,
                 greedy: bool = False):
        dev = self.device = _one_device("target_logits", target_logits, draft_token=draft_token, u=u, r=r,
                                        draft_logits=draft_logits, draft_len=draft_len)
        code = _float_code("target_logits", target_logits)
        if target_logits.dim() != 3 or target_logits.shape[1] < 1:
            raise ValueError("target_logits must be [B][T+1][V]")
        B, T, V = target_logits.shape[0], target_logits.shape[1] - 1, target_logits.shape[2]
        _check_dev("draft_token", draft_token, (B, T), (torch.int32,))
        if not greedy and (u is None or r is None):
            raise ValueError("u and r are required (without greedy)")
        if u is not None:
            _check_dev("u", u, (B, T), (torch.float32,))
        if r is not None:
            _check_dev("r", r, (B,), (torch.float32,))
        if draft_len is not None:
            _check_dev("draft_len", draft_len, (B,), (torch.int32,))
        for name, t, shape in (("target_logits", target_logits, (B, T + 1, V)), ("draft_logits", draft_logits, (B, T, V))):
            if t is None:
                continue
            if tuple(t.shape) != shape or t.dtype != target_logits.dtype:
                raise ValueError(f"{name} has shape {tuple(t.shape)} and dtype {t.dtype}, expected {shape}")
            if V > 1 and t.stride(2) != 1:
                raise ValueError(f"{name} must be contiguous in its last dimension")
        q = draft_logits if T > 0 else None
        self.out = {"token": torch.empty((B, T + 1), dtype=torch.int32, device=dev),
                    "n_accept": torch.empty((B,), dtype=torch.int32, device=dev),
                    "accept": torch.empty((B, T), dtype=torch.float32, device=dev)}
        self.problem = RpdVerify(B, T, V, code, target_logits.data_ptr(), target_logits.stride(0),
                                 target_logits.stride(1), _ptr(q), 0 if q is None else q.stride(0),
                                 0 if q is None else q.stride(1), draft_token.data_ptr(), _ptr(draft_len), _ptr(u),
                                 _ptr(r), float(target_scale), float(draft_scale), VERIFY_GREEDY if greedy else 0,
                                 self.out["token"].data_ptr(), self.out["n_accept"].data_ptr(),
                                 self.out["accept"].data_ptr())
        nbytes = int(lib().rpd_verify_workspace_size(ctypes.byref(self.problem)))
        self.workspace = torch.empty(max(nbytes, 1), dtype=torch.uint8, device=dev)
        self._keep = (target_logits, draft_token, u, r, draft_logits, draft_len)

    def __call__(self, stream=None) -> dict:
        """Enqueue one call."""
        _enqueue(self.device, stream, lib().rpd_verify_draft, ctypes.byref(self.problem),
                 self.workspace.data_ptr(), self.workspace.numel())
        return self.out


def verify_draft(target_logits: torch.Tensor, draft_token: torch.Tensor, u: torch.Tensor | None = None,
                 r: torch.Tensor | None = None, draft_logits: torch.Tensor | None = None,
                 draft_len: torch.Tensor | None = None, target_scale: float = 1.0, draft_scale: float = 1.0,
                 greedy: bool = False, stream=None) -> dict:
    """``rpd_verify_draft``: drafted tokens against a target's logits, from given random numbers (see
    ``VerifyDraft``). Returns token, n_accept and accept, valid once the stream has run; a ``stream`` other than the
    current one, on which they are made, has to wait for it beforehand."""
    call = VerifyDraft(target_logits, draft_token, u, r, draft_logits, draft_len, target_scale, draft_scale, greedy)
    if stream is not None:
        call.workspace.record_stream(stream)
    return call(stream)


def _distill_problem(logits, teacher_id, teacher_logit, teacher_lse, weight, logit_scale) -> RpdDistill:
    """The problem of [..., V] logits without its outputs."""
    _one_device("logits", logits, teacher_id=teacher_id, teacher_logit=teacher_logit, teacher_lse=teacher_lse,
                weight=weight)
    code = _float_code("logits", logits)
    r = _rows("logits", logits)
    lead, k = tuple(logits.shape[:-1]), teacher_id.shape[-1] if teacher_id.dim() else 0
    _check_dev("teacher_id", teacher_id, (*lead, k), (torch.int32,))
    _check_dev("teacher_logit", teacher_logit, (*lead, k), tuple(_FLOAT_CODES))
    for name, t in (("teacher_lse", teacher_lse), ("weight", weight)):
        if t is not None:
            _check_dev(name, t, lead, (torch.float32,))
    return RpdDistill(r.shape[0], r.shape[1], k, code, _FLOAT_CODES[teacher_logit.dtype], r.data_ptr(),
                      _row_stride(r), teacher_id.data_ptr(), teacher_logit.data_ptr(), _ptr(teacher_lse),
                      _ptr(weight), None, float(logit_scale), None, None, None, 0)


def _distill_loss(p: RpdDistill, logits: torch.Tensor, stream) -> tuple[torch.Tensor, torch.Tensor]:
    """The loss, and the buffer that begins with the rows' state (then the workspace)."""
    loss = torch.empty(logits.shape[:-1], dtype=torch.float32, device=logits.device)
    at = -(-p.N * DISTILL_STATE * 4 // 256) * 256
    nbytes = int(lib().rpd_distill_workspace_size(ctypes.byref(p)))
    buf = torch.empty(at + nbytes, dtype=torch.uint8, device=logits.device)
    if stream is not None:
        buf.record_stream(stream)
    p.loss, p.state = loss.data_ptr(), buf.data_ptr()
    _enqueue(logits.device, stream, lib().rpd_distill_loss, ctypes.byref(p), (p.state or 0) + at, nbytes)
    return loss, buf


def _grad_like(logits: torch.Tensor, p: RpdDistill) -> torch.Tensor:
    grad = torch.empty(logits.shape, dtype=logits.dtype, device=logits.device)
    p.grad, p.grad_stride = grad.data_ptr(), max(p.V, 1)
    return grad


class _Distill(torch.autograd.Function):
    @staticmethod
    def forward(ctx, logits, teacher_id, teacher_logit, teacher_lse, weight, logit_scale):
        p = _distill_problem(logits, teacher_id, teacher_logit, teacher_lse, weight, logit_scale)
        loss, state = _distill_loss(p, logits, None)
        ctx.save_for_backward(logits, teacher_id, teacher_logit, teacher_lse, weight, state)
        ctx.logit_scale = logit_scale
        return loss

    @staticmethod
    @torch.autograd.function.once_differentiable
    def backward(ctx, grad_loss):
        *inputs, state = ctx.saved_tensors   # perhaps not where they were (saved tensors' hooks)
        p = _distill_problem(*inputs, ctx.logit_scale)
        logits = inputs[0]
        grad = _grad_like(logits, p)
        up = grad_loss.to(torch.float32).contiguous()   # a broadcast upstream gradient has stride 0
        p.grad_loss, p.state, p.loss = up.data_ptr(), state.data_ptr(), None
        _enqueue(logits.device, None, lib().rpd_distill_grad, ctypes.byref(p))
        return grad, None, None, None, None, None


def distill(logits: torch.Tensor, teacher_id: torch.Tensor, teacher_logit: torch.Tensor,
            teacher_lse: torch.Tensor | None = None, weight: torch.Tensor | None = None,
            logit_scale: float = 1.0) -> torch.Tensor:
    """Distillation loss of every row against a teacher's top logits (``rpd_distill_loss``, and
    ``rpd_distill_grad`` in the backward pass).

    logits [..., V] (bfloat16, float16 or float32), teacher_id int32 [..., k] (entries outside 0..V-1 are no part of
    the list), teacher_logit [..., k], optional teacher_lse and weight float32 [...]. Returns float32 [...],
    differentiable once in ``logits`` (the teacher and the weights are constants). A backward pass that is captured into
    a graph must not meet leaves that an earlier backward pass outside it still refers to (as for any torch function)."""
    return _Distill.apply(logits, teacher_id, teacher_logit, teacher_lse, weight, float(logit_scale))


def distill_grad(logits: torch.Tensor, teacher_id: torch.Tensor, teacher_logit: torch.Tensor,
                 teacher_lse: torch.Tensor | None = None, weight: torch.Tensor | None = None,
                 grad_loss: torch.Tensor | None = None, logit_scale: float = 1.0,
                 stream=None) -> tuple[torch.Tensor, torch.Tensor]:
    """Loss and gradient in one call, for a training step that knows the upstream gradient ``grad_loss`` (float32
    [...], 1 if None) beforehand: (loss [...], gradient [..., V] of ``logits``'s type). Not recorded by autograd.
    ``stream`` as in ``verify_draft``."""
    logits = logits.detach()
    p = _distill_problem(logits, teacher_id, teacher_logit, teacher_lse, weight, logit_scale)
    if grad_loss is not None:
        _one_device("logits", logits, grad_loss=grad_loss)
        _check_dev("grad_loss", grad_loss, tuple(logits.shape[:-1]), (torch.float32,))
        p.grad_loss = grad_loss.data_ptr()
    grad = _grad_like(logits, p)
    loss, _ = _distill_loss(p, logits, stream)
    return loss, grad
