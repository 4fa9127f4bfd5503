"""Token-aware verifier hot path on MI355X (Pro-Router, Sec. 3.1).

A thin binding over the C ABI of ``libprouter.so`` (include/prouter.h):
tensors are checked and their device pointers handed to the library, which
runs every step of the path in its own HIP kernels on torch's current
stream. PyTorch only provides device memory and streams here.

    feats = token_features(logits, sampled_ids, temperature, top_p=None)
    agg = request_aggregate(feats, offsets)
    ship, n_ship = route(agg["score"], threshold)

The paper's own verifier input, the per-token tuples (l, m, h, rho) with the
top-K entropy (Sec. 3.1, Eq. 3): :func:`feature_sequence`.

Streaming decode: :class:`StreamState`.

Training the small model on what the routing saw: :func:`policy_loss` and
:func:`preference_loss` over the same logit rows, with their gradients, and
:class:`AdamW`.
"""

from __future__ import annotations

import ctypes as C

import torch

from . import _abi
from ._abi import (FLAG_BAD_ID, FLAG_BAD_TP, FLAG_CLIPPED, FLAG_MASKED, FLAG_NONFINITE,  # noqa: F401
                   FLAG_OUTSIDE_NUCLEUS, ProuterError)

__all__ = ["token_features", "token_features_noalloc", "feature_sequence", "sample_features", "verifier_head", "request_aggregate", "route", "calibrate_threshold",
           "validate_offsets", "StreamState", "policy_loss", "preference_loss", "AdamW",
           "token_features_workspace", "ProuterError", "FEATURE_FLOATS", "FEATURE_INTS", "PAPER_TOP_K"]

PAPER_TOP_K = 20  # K of the paper's top-K entropy (Sec. 3.1)

FEATURE_FLOATS = ("max_logit", "lse", "entropy", "logprob", "maxprob", "margin")
FEATURE_INTS = ("rank", "argmax", "cutoff")
_LINKS = {"identity": 0, "sigmoid": 1}


# What a call costs on the host is most of a small batch's time: pointers go to
# ctypes as plain ints, and the current stream's handle is read without making
# a Stream object (1.5 us a call).
_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None)


def _stream_handle() -> int:
    if _raw_stream is None:
        return torch.cuda.current_stream().cuda_stream
    return _raw_stream(torch.cuda.current_device())


def _ptr(t) -> int | None:
    return None if t is None else t.data_ptr()


def _dtype_code(logits: torch.Tensor) -> int:
    if logits.dtype == torch.float32:
        return _abi.PR_F32
    if logits.dtype == torch.bfloat16:
        return _abi.PR_BF16
    raise TypeError(f"logits must be float32 or bfloat16, got {logits.dtype}")


def _check_rows(logits, sampled_ids, temperature, top_p):
    if not logits.is_cuda or logits.dim() != 2 or logits.stride(1) != 1:
        raise ValueError("logits must be a 2-D CUDA tensor with unit stride along the vocabulary")
    shape = (logits.shape[0],)
    for name, t, dt in (("sampled_ids", sampled_ids, torch.int32), ("temperature", temperature, torch.float32),
                        ("top_p", top_p, torch.float32)):
        if t is not None and (t.dtype != dt or not t.is_cuda or t.shape != shape or not t.is_contiguous()):
            raise ValueError(f"{name} must be a contiguous 1-D {dt} CUDA tensor of length {shape[0]}")


def _check_features(f: dict, device, n: int | None, what: str, fields=_abi.FEATURE_FIELDS):
    """Caller-supplied per-token feature tensors: each of `fields` present,
    1-D, contiguous, on `device`, of its dtype, and n long when n is given
    (a tensor on the host would reach a kernel as a host pointer)."""
    for k in fields:
        t = f.get(k)
        dt = torch.float32 if k in FEATURE_FLOATS else torch.int32
        if (t is None or t.dtype != dt or t.dim() != 1 or t.device != device or not t.is_contiguous()
                or (n is not None and t.shape[0] != n)):
            size = "" if n is None else f" of length {n}"
            raise ValueError(f"{what}['{k}'] must be a contiguous 1-D {dt} tensor{size} on {device}")


def _check_workspace(workspace, device):
    if workspace is not None and (workspace.device != device or not workspace.is_contiguous()):
        raise ValueError(f"workspace must be a contiguous tensor on {device}")


def _check_index_tensor(t, name: str, device, n: int | None = None):
    if (t.dtype != torch.int32 or t.device != device or t.dim() != 1 or not t.is_contiguous()
            or (n is not None and t.shape[0] != n)):
        size = "" if n is None else f" [{n}]"
        raise ValueError(f"{name} must be a contiguous int32{size} tensor on {device}")


def _as_row_tensor(x, n, device):
    if isinstance(x, (int, float)):
        return torch.full((n,), float(x), dtype=torch.float32, device=device)
    return x


_INT_FIELDS = FEATURE_INTS + ("flags",)  # flags: uint32 bits
assert FEATURE_FLOATS + _INT_FIELDS == _abi.FEATURE_FIELDS


def _outputs(k: int, n: int, dtype, device):
    """k tensors of n entries, each 16-byte aligned, from one allocation (ten
    of them took 12.9 us as allocations of their own, 6.3 this way). They are
    tensors of their own: views of one tensor would share a version counter,
    so that writing one in place would invalidate what autograd saved of the
    others, and views of several outputs refuse such writes."""
    pad = -n % 4
    if pad == 0:
        return torch.empty(k * n, dtype=dtype, device=device).unsafe_split_with_sizes([n] * k)
    return torch.empty(k * (n + pad), dtype=dtype, device=device).unsafe_split_with_sizes([n, pad] * k)[::2]


def _alloc_features(n: int, device) -> dict:
    """The ten per-token outputs."""
    out = dict(zip(FEATURE_FLOATS, _outputs(len(FEATURE_FLOATS), n, torch.float32, device)))
    out.update(zip(_INT_FIELDS, _outputs(len(_INT_FIELDS), n, torch.int32, device)))
    return out


def _features_struct(f: dict) -> _abi.TokenFeatures:
    return _abi.TokenFeatures(*[t.data_ptr() if t is not None else None for t in map(f.get, _abi.FEATURE_FIELDS)])


def token_features_workspace(logits: torch.Tensor, top_p_on: bool = False) -> int:
    n, V = logits.shape
    return int(_abi.lib().pr_token_features_workspace(_dtype_code(logits), n, V, int(top_p_on)))


def token_features(logits: torch.Tensor, sampled_ids: torch.Tensor, temperature, top_p=None,
                   out: dict | None = None, workspace: torch.Tensor | None = None) -> dict:
    """Per-token features of each logit row (``pr_token_features``).

    ``logits`` [n_rows, V] float32/bfloat16; ``sampled_ids`` int32 [n_rows];
    ``temperature`` float32 [n_rows] or a Python float; ``top_p`` float32
    [n_rows], a Python float or None. Returns a dict of [n_rows] tensors.
    ``workspace``: optional device scratch of this call, not shared with one
    that may overlap (by default as much as the call can use is allocated).
    """
    n, V = logits.shape
    temperature = _as_row_tensor(temperature, n, logits.device)
    top_p = None if top_p is None else _as_row_tensor(top_p, n, logits.device)
    _check_rows(logits, sampled_ids, temperature, top_p)
    L = _abi.lib()
    code = _dtype_code(logits)
    if out is None:
        out = _alloc_features(n, logits.device)
    else:
        _check_features(out, logits.device, n, "out")
    _check_workspace(workspace, logits.device)
    top_p_on = int(top_p is not None)
    if workspace is None or (workspace.numel() * workspace.element_size()
                             < L.pr_token_features_workspace(code, n, V, top_p_on)):
        full = L.pr_token_features_workspace_full(code, n, V, top_p_on)
        workspace = torch.empty(full, dtype=torch.uint8, device=logits.device) if full else None
    elif top_p_on and workspace.data_ptr() % 16:
        workspace = None  # none is needed
    ws_bytes = 0 if workspace is None else workspace.numel() * workspace.element_size()
    st = L.pr_token_features_ws(_ptr(logits), code, n, V, logits.stride(0), _ptr(sampled_ids), _ptr(temperature),
                                _ptr(top_p), C.byref(_features_struct(out)), _ptr(workspace), ws_bytes,
                                _stream_handle())
    _abi.check("pr_token_features", st)
    return out


def token_features_noalloc(logits: torch.Tensor, sampled_ids: torch.Tensor, temperature, top_p=None,
                           out: dict | None = None) -> dict:
    """``pr_token_features_noalloc``: :func:`token_features` with the library's
    static per-GPU scratch instead of a workspace (nothing is allocated by the
    library; pass ``out`` to allocate nothing here either). Calls that overlap
    on one GPU race on that scratch."""
    n, V = logits.shape
    temperature = _as_row_tensor(temperature, n, logits.device)
    top_p = None if top_p is None else _as_row_tensor(top_p, n, logits.device)
    _check_rows(logits, sampled_ids, temperature, top_p)
    if out is None:
        out = _alloc_features(n, logits.device)
    else:
        _check_features(out, logits.device, n, "out")
    st = _abi.lib().pr_token_features_noalloc(_ptr(logits), _dtype_code(logits), n, V, logits.stride(0),
                                              _ptr(sampled_ids), _ptr(temperature), _ptr(top_p),
                                              C.byref(_features_struct(out)), _stream_handle())
    _abi.check("pr_token_features_noalloc", st)
    return out


def feature_sequence(logits: torch.Tensor, sampled_ids: torch.Tensor, temperature, offsets: torch.Tensor,
                     top_p=None, top_k: int = PAPER_TOP_K, features: bool = False, out: torch.Tensor | None = None):
    """The paper's verifier input sequence X (``pr_feature_sequence``).

    Returns X, a float32 [n_rows, 4] tensor of (log-prob of the sampled token,
    max probability, negated top-K entropy, position fraction t / T) per
    row; request i owns rows ``offsets[i]:offsets[i+1]``. With
    ``features=True`` returns ``(X, feats)``, feats being the dict that
    :func:`token_features` returns, computed in the same pass. ``out``: an
    optional float32 [n_rows, 4] CUDA tensor that receives X.
    """
    n, V = logits.shape
    temperature = _as_row_tensor(temperature, n, logits.device)
    top_p = None if top_p is None else _as_row_tensor(top_p, n, logits.device)
    _check_rows(logits, sampled_ids, temperature, top_p)
    if offsets.dtype != torch.int32 or not offsets.is_cuda or offsets.dim() != 1 or not offsets.is_contiguous():
        raise ValueError("offsets must be a contiguous 1-D int32 CUDA tensor")
    if out is not None and (out.dtype != torch.float32 or tuple(out.shape) != (n, 4) or not out.is_contiguous()
                            or out.device != logits.device):
        raise ValueError(f"out must be a contiguous float32 [{n}, 4] tensor on {logits.device}")
    X = torch.empty(n, 4, dtype=torch.float32, device=logits.device) if out is None else out
    feats = _alloc_features(n, logits.device) if features else None
    fs = C.byref(_features_struct(feats)) if feats is not None else None
    L = _abi.lib()
    code = _dtype_code(logits)
    need = int(L.pr_feature_sequence_workspace(code, n, V, int(top_p is not None)))
    ws = torch.empty(need, dtype=torch.uint8, device=logits.device) if need else None
    st = L.pr_feature_sequence_ws(_ptr(logits), code, n, V, logits.stride(0), _ptr(sampled_ids), _ptr(temperature),
                                  _ptr(top_p), _ptr(offsets), offsets.shape[0] - 1, int(top_k), _ptr(X), fs, _ptr(ws),
                                  need, _stream_handle())
    _abi.check("pr_feature_sequence", st)
    return (X, feats) if features else X


def sample_features(logits: torch.Tensor, temperature, seed: int, offset: int = 0, features: bool = True,
                    offsets: torch.Tensor | None = None, top_k: int = PAPER_TOP_K, ids_out: torch.Tensor | None = None,
                    out: dict | None = None):
    """Fused sample-and-verify (``pr_sample_features``): draws each row's token
    from softmax(logits / T) in the same pass that computes its features.

    Returns ``(ids, feats, X)``: the drawn tokens (int32 [n_rows], -1 where the
    distribution is undefined), the per-token features for them as
    :func:`token_features` returns them (rank written as -1, not available), or None with
    ``features=False``, and the paper's input sequence X for them when
    ``offsets`` is given (else None). The draw is a fixed function of
    (seed, offset, row index, logits, temperature) and of the workgroup size
    the number of rows selects. ``ids_out`` / ``out``: optional preallocated
    outputs (int32 [n_rows]; a features dict as :func:`token_features`
    returns)."""
    n, V = logits.shape
    temperature = _as_row_tensor(temperature, n, logits.device)
    if logits.dim() != 2 or not logits.is_cuda or logits.stride(1) != 1:
        raise ValueError("logits must be a 2-D CUDA tensor with unit column stride")
    if logits.dtype not in (torch.float32, torch.bfloat16):
        raise ValueError("logits must be float32 or bfloat16")
    _check_rows(logits, None, temperature, None)
    if features and out is not None:
        _check_features(out, logits.device, n, "out")
    ids = torch.empty(n, dtype=torch.int32, device=logits.device) if ids_out is None else ids_out
    if ids.dtype != torch.int32 or ids.shape != (n,) or not ids.is_contiguous() or ids.device != logits.device:
        raise ValueError(f"ids_out must be a contiguous int32 [{n}] tensor on {logits.device}")
    feats = (out if out is not None else _alloc_features(n, logits.device)) if features else None
    fs = C.byref(_features_struct(feats)) if feats is not None else None
    X = None
    n_req = 0
    if offsets is not None:
        if offsets.dtype != torch.int32 or not offsets.is_cuda or offsets.dim() != 1 or not offsets.is_contiguous():
            raise ValueError("offsets must be a contiguous 1-D int32 CUDA tensor")
        X = torch.empty(n, 4, dtype=torch.float32, device=logits.device)
        n_req = offsets.shape[0] - 1
    L = _abi.lib()
    code = _dtype_code(logits)
    need = int(L.pr_sample_features_workspace(code, n, V, int(X is not None)))
    ws = torch.empty(need, dtype=torch.uint8, device=logits.device) if need else None
    st = L.pr_sample_features_ws(_ptr(logits), code, n, V, logits.stride(0), _ptr(temperature),
                                 int(seed) & 0xFFFFFFFFFFFFFFFF, int(offset) & 0xFFFFFFFFFFFFFFFF, _ptr(ids), fs,
                                 _ptr(offsets), n_req, int(top_k), _ptr(X), _ptr(ws), need, _stream_handle())
    _abi.check("pr_sample_features", st)
    return ids, feats, X


def verifier_head(X: torch.Tensor, offsets: torch.Tensor, weights: torch.Tensor, max_len: int | None = None,
                  workspace: torch.Tensor | None = None) -> torch.Tensor:
    """The paper's shipping confidence per request from its input sequence
    (``pr_verifier_head``). ``X`` float32 [n_rows, 4] (as returned by
    :func:`feature_sequence`), ``offsets`` int32 [n_req + 1], ``weights``
    float32 [67,329] in the documented layout. ``max_len``: at least the
    longest request's length (default: n_rows). ``workspace``: optional device
    scratch of ``pr_verifier_head_workspace_full(n_rows)`` bytes (or, slower,
    ``pr_verifier_head_workspace(n_rows)``). Returns float32 [n_req]."""
    if X.dtype != torch.float32 or not X.is_cuda or X.dim() != 2 or X.shape[1] != 4 or not X.is_contiguous():
        raise ValueError("X must be a contiguous float32 [n_rows, 4] CUDA tensor")
    if offsets.dtype != torch.int32 or not offsets.is_cuda or offsets.dim() != 1 or not offsets.is_contiguous():
        raise ValueError("offsets must be a contiguous 1-D int32 CUDA tensor")
    if (weights.dtype != torch.float32 or not weights.is_cuda or weights.numel() != _abi.PR_HEAD_WEIGHTS
            or not weights.is_contiguous()):
        raise ValueError(f"weights must be a contiguous float32 CUDA tensor of {_abi.PR_HEAD_WEIGHTS} entries")
    n = X.shape[0]
    n_req = offsets.shape[0] - 1
    _check_workspace(workspace, X.device)
    L = _abi.lib()
    if workspace is None or workspace.numel() * workspace.element_size() < int(L.pr_verifier_head_workspace(n)):
        workspace = torch.empty(int(L.pr_verifier_head_workspace_full(n)), dtype=torch.uint8, device=X.device)
    ws_bytes = 0 if workspace is None else workspace.numel() * workspace.element_size()
    scores = torch.empty(n_req, dtype=torch.float32, device=X.device)
    st = L.pr_verifier_head(_ptr(X), n, _ptr(offsets), n_req, int(max_len if max_len is not None else max(n, 1)),
                            _ptr(weights), _ptr(scores), _ptr(workspace), ws_bytes, _stream_handle())
    _abi.check("pr_verifier_head", st)
    return scores


_default_params = None


def _params(q=0.1, weights=None, bias=0.0, link="identity") -> _abi.AggParams:
    global _default_params
    if _default_params is None:  # the library's defaults, which never change
        p = _abi.AggParams()
        _abi.lib().pr_agg_params_default(C.byref(p))
        _default_params = bytes(p)
    p = _abi.AggParams.from_buffer_copy(_default_params)
    p.q = float(q)
    if weights is not None:
        w = [float(v) for v in torch.as_tensor(weights, dtype=torch.float64).reshape(-1).tolist()]
        if len(w) != 12:
            raise ValueError("weights must have 12 entries (stat-major [mean, min, quant] x 4 features)")
        for i, v in enumerate(w):
            p.w[i] = v
    p.b = float(bias)
    p.link = _LINKS[link]
    return p


def _alloc_agg(n: int, device) -> dict:
    mean, mn, quant = torch.empty((3 * n, 4), dtype=torch.float32, device=device).unsafe_split_with_sizes([n] * 3)
    return {"count": torch.empty(n, dtype=torch.int32, device=device), "mean": mean, "min": mn, "quant": quant,
            "score": torch.empty(n, dtype=torch.float32, device=device)}


def _agg_struct(a: dict) -> _abi.RequestAgg:
    return _abi.RequestAgg(*[t.data_ptr() if t is not None else None for t in map(a.get, _abi.AGG_FIELDS)])


def request_aggregate(feats: dict, offsets: torch.Tensor, q: float = 0.1, weights=None, bias: float = 0.0,
                      link: str = "identity") -> dict:
    """Per-request count, mean/min/q-quantile of (logprob, maxprob, -entropy,
    margin) and the summary score (``pr_request_aggregate``)."""
    if offsets.dtype != torch.int32 or not offsets.is_cuda or offsets.dim() != 1 or not offsets.is_contiguous():
        raise ValueError("offsets must be a contiguous 1-D int32 CUDA tensor")
    n_req = offsets.shape[0] - 1
    _check_features(feats, offsets.device, None, "feats", ("logprob", "maxprob", "entropy", "margin"))
    out = _alloc_agg(n_req, offsets.device)
    params = _params(q, weights, bias, link)
    st = _abi.lib().pr_request_aggregate(C.byref(_features_struct(feats)), _ptr(offsets), n_req, C.byref(params),
                                         C.byref(_agg_struct(out)), _stream_handle())
    _abi.check("pr_request_aggregate", st)
    return out


def route(scores: torch.Tensor, threshold: float):
    """Ship iff score >= threshold (``pr_route``). Returns (ship uint8 [n], n_ship int32 [1])."""
    if scores.dtype != torch.float32 or not scores.is_cuda or not scores.is_contiguous():
        raise ValueError("scores must be a contiguous float32 CUDA tensor")
    n = scores.shape[0]
    ship = torch.empty(n, dtype=torch.uint8, device=scores.device)
    n_ship = torch.empty(1, dtype=torch.int32, device=scores.device)
    st = _abi.lib().pr_route(_ptr(scores), n, float(threshold), _ptr(ship), _ptr(n_ship), _stream_handle())
    _abi.check("pr_route", st)
    return ship, n_ship


def calibrate_threshold(scores: torch.Tensor, ship_fraction: float):
    """Threshold tau for a ship fraction on a validation pool of scores
    (``pr_calibrate_threshold``). Returns (tau float32 [1], n_ship int32 [1])."""
    if scores.dtype != torch.float32 or not scores.is_cuda or not scores.is_contiguous() or scores.dim() != 1:
        raise ValueError("scores must be a 1-D contiguous float32 CUDA tensor")
    n = scores.shape[0]
    tau = torch.empty(1, dtype=torch.float32, device=scores.device)
    n_ship = torch.empty(1, dtype=torch.int32, device=scores.device)
    ws_bytes = _abi.lib().pr_calibrate_workspace(n)
    ws = torch.empty(ws_bytes, dtype=torch.uint8, device=scores.device) if ws_bytes else None
    st = _abi.lib().pr_calibrate_threshold(_ptr(scores), n, float(ship_fraction), _ptr(tau), _ptr(n_ship),
                                          _ptr(ws), ws_bytes, _stream_handle())
    _abi.check("pr_calibrate_threshold", st)
    return tau, n_ship


def validate_offsets(offsets: torch.Tensor, n_rows: int) -> bool:
    """Synchronous check of an offsets array (``pr_validate_offsets``)."""
    if not offsets.is_cuda:
        raise ValueError("offsets must be a CUDA tensor")
    _check_index_tensor(offsets, "offsets", offsets.device)
    st = _abi.lib().pr_validate_offsets(_ptr(offsets), offsets.shape[0] - 1, n_rows, _stream_handle())
    if st == _abi.PR_ERR_INVALID_ARG:
        return False
    _abi.check("pr_validate_offsets", st)
    return True


class StreamState:
    """Device-resident per-request state for streaming decode (``pr_stream_*``).

    ``max_len`` tokens of history per slot give the exact tail quantile;
    ``max_len=0`` keeps P-square markers instead (bounded memory, any length)."""

    def __init__(self, max_slots: int, max_len: int, q: float = 0.1, weights=None, bias: float = 0.0,
                 link: str = "identity"):
        self._h = C.c_void_p()
        params = _params(q, weights, bias, link)
        _abi.check("pr_stream_create", _abi.lib().pr_stream_create(max_slots, max_len, C.byref(params),
                                                                     C.byref(self._h)))
        self.max_slots, self.max_len = max_slots, max_len

    def step(self, logits, slot_ids, sampled_ids, temperature, out: dict | None = None, want_features=False,
             top_p=None):
        n, V = logits.shape
        temperature = _as_row_tensor(temperature, n, logits.device)
        top_p = None if top_p is None else _as_row_tensor(top_p, n, logits.device)
        _check_rows(logits, sampled_ids, temperature, top_p)
        _check_index_tensor(slot_ids, "slot_ids", logits.device, n)
        if out is None and want_features:
            out = _alloc_features(n, logits.device)
        elif out is not None:
            _check_features(out, logits.device, n, "out")
        fs = C.byref(_features_struct(out)) if out is not None else None
        L = _abi.lib()
        code = _dtype_code(logits)
        need = L.pr_stream_step_workspace(code, n, V, 1) if top_p is not None else 0
        ws = torch.empty(need, dtype=torch.uint8, device=logits.device) if need else None
        st = L.pr_stream_step_ws(self._h, _ptr(logits), code, n, V, logits.stride(0), _ptr(slot_ids),
                                 _ptr(sampled_ids), _ptr(temperature), _ptr(top_p), fs, _ptr(ws), need,
                                 _stream_handle())
        _abi.check("pr_stream_step", st)
        return out

    def finish(self, slots: torch.Tensor, threshold: float) -> dict:
        if not slots.is_cuda:
            raise ValueError("slots must be a CUDA tensor")
        _check_index_tensor(slots, "slots", slots.device)
        n = slots.shape[0]
        out = _alloc_agg(n, slots.device)
        ship = torch.empty(n, dtype=torch.uint8, device=slots.device)
        st = _abi.lib().pr_stream_finish(self._h, _ptr(slots), n, float(threshold), C.byref(_agg_struct(out)),
                                         _ptr(ship), _stream_handle())
        _abi.check("pr_stream_finish", st)
        out["ship"] = ship
        return out

    def reset(self, slots: torch.Tensor) -> None:
        if not slots.is_cuda:
            raise ValueError("slots must be a CUDA tensor")
        _check_index_tensor(slots, "slots", slots.device)
        _abi.check("pr_stream_reset_slots",
                   _abi.lib().pr_stream_reset_slots(self._h, _ptr(slots), slots.shape[0], _stream_handle()))

    def close(self) -> None:
        if self._h:
            _abi.lib().pr_stream_destroy(self._h)
            self._h = C.c_void_p()

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass


# ---------------------------------------------------------------------------
# Training: losses over logit rows, and the optimizer's step.

def _check_current(device, what: str) -> int:
    """Launches go to the current device's stream: the tensors have to be there. Returns that stream."""
    current = torch.cuda.current_device() if device.type == "cuda" else None
    if current is None or device.index != current:
        raise ValueError(f"{what} must be on the current CUDA device, got {device}")
    return torch.cuda.current_stream().cuda_stream if _raw_stream is None else _raw_stream(current)


def _check_row_floats(device, n: int, **tensors):
    for name, t in tensors.items():
        if t is not None and (t.dtype != torch.float32 or t.dim() != 1 or t.numel() != n or not t.is_contiguous()
                              or t.device != device):
            raise ValueError(f"{name} must be a contiguous float32 [{n}] tensor on {device}")


def _rows_apart(t, V: int) -> bool:
    """Whether a 2-D tensor's rows are contiguous and do not overlap."""
    return t.stride(1) == 1 and (t.shape[0] <= 1 or t.stride(0) >= V)


def _check_loss(logits, ids, temperature, grad):
    """Checks of a loss's rows. Returns the stream, the device, the type's code, the temperature as a tensor, and the
    gradient to write or None."""
    if logits.dim() != 2:
        raise ValueError("logits must be a 2-D CUDA tensor with unit stride along the vocabulary")
    n, V = logits.shape
    device = logits.device
    code = _dtype_code(logits)
    stream = _check_current(device, "logits")
    if not _rows_apart(logits, V):
        raise ValueError("logits must be a 2-D CUDA tensor with unit stride along the vocabulary and rows apart")
    _check_index_tensor(ids, "ids", device, n)
    if grad is True:
        grad = torch.empty((n, V), dtype=logits.dtype, device=device)
    elif grad is False or grad is None:
        grad = None
    elif (grad.dtype != logits.dtype or grad.shape != logits.shape or grad.device != device
          or not _rows_apart(grad, V)):
        raise ValueError(f"grad must be a {logits.dtype} {list(logits.shape)} tensor on {device} with unit stride along "
                         "the vocabulary and rows apart")
    return stream, device, code, _as_row_tensor(temperature, n, device), grad


def _row_stride(t) -> int:
    """Elements from row to row (a single row may come with any stride)."""
    return t.stride(0) if t.shape[0] > 1 else max(t.stride(0), t.shape[1])


def _loss_outputs(sizes, workspace, need: int, device):
    """Float32 outputs of these sizes and the scratch of a call, from one allocation as tensors of their own (see
    _outputs): the caller's workspace where it serves, else the part before the outputs. Returns the workspace's
    address, its bytes and the outputs."""
    if workspace is not None:
        _check_workspace(workspace, device)
        have = workspace.numel() * workspace.element_size()
        if have >= need and workspace.data_ptr() % 16 == 0:
            out = torch.empty(sum(sizes), dtype=torch.float32, device=device).unsafe_split_with_sizes(sizes)
            return workspace.data_ptr(), have, out
    sizes = [(need + 3) // 4, *sizes]
    scratch, *out = torch.empty(sum(sizes), dtype=torch.float32, device=device).unsafe_split_with_sizes(sizes)
    return scratch.data_ptr(), need, out


def policy_loss(logits: torch.Tensor, ids: torch.Tensor, temperature, weight: torch.Tensor, advantage: torch.Tensor,
                old_logprob: torch.Tensor, ref_logprob: torch.Tensor | None = None, clip_low: float = 0.2,
                clip_high: float = 0.2, kl_coef: float = 0.0, grad=True, grad_scale: float = 1.0,
                workspace: torch.Tensor | None = None) -> dict:
    """Clipped policy loss with a KL term, and its gradient (``pr_policy_loss``).

    ``logits`` [n_rows, V] float32/bfloat16, ``ids`` int32 [n_rows] (the
    tokens that were generated), ``temperature`` float32 [n_rows] or a Python
    float, ``weight`` float32 [n_rows]: a row's weight in the sum, 0 for rows
    that do not count (they are not read). ``advantage``, ``old_logprob``,
    ``ref_logprob`` float32 [n_rows]; without ``ref_logprob`` there is no KL
    term. The loss is the sum over rows of
    weight (kl_coef kl - min(ratio A, clip(ratio, 1 - clip_low, 1 + clip_high) A)),
    ratio = exp(logprob - old_logprob).

    ``grad``: True for a gradient in the logits (of their type, times
    ``grad_scale``), False for none, or the tensor that receives it, which may
    be ``logits``. Returns a dict with ``loss`` (float32 [1]), ``logprob``,
    ``ratio``, ``kl``, ``flags`` ([n_rows]) and, when wanted, ``grad``.
    ``workspace``: optional device scratch of this call, not shared with one
    that may overlap.
    """
    stream, device, code, temperature, grad = _check_loss(logits, ids, temperature, grad)
    n, V = logits.shape
    _check_row_floats(device, n, temperature=temperature, weight=weight, advantage=advantage, old_logprob=old_logprob,
                      ref_logprob=ref_logprob)
    L = _abi.lib()
    ws, ws_bytes, (logprob, ratio, kl, loss) = _loss_outputs((n, n, n, 1), workspace,
                                                             L.pr_policy_loss_workspace(code, n, V), device)
    flags = torch.empty(n, dtype=torch.int32, device=device)
    params = _abi.PolicyParams(clip_low, clip_high, kl_coef, grad_scale)
    tokens = _abi.PolicyTokens(logprob.data_ptr(), ratio.data_ptr(), kl.data_ptr(), flags.data_ptr())
    st = L.pr_policy_loss(logits.data_ptr(), code, n, V, _row_stride(logits), ids.data_ptr(), temperature.data_ptr(),
                          weight.data_ptr(), advantage.data_ptr(), old_logprob.data_ptr(), _ptr(ref_logprob),
                          C.byref(params), loss.data_ptr(), C.byref(tokens), _ptr(grad),
                          0 if grad is None else _row_stride(grad), ws, ws_bytes, stream)
    _abi.check("pr_policy_loss", st)
    out = {"loss": loss, "logprob": logprob, "ratio": ratio, "kl": kl, "flags": flags}
    if grad is not None:
        out["grad"] = grad
    return out


def preference_loss(logits: torch.Tensor, ids: torch.Tensor, temperature, weight: torch.Tensor, offsets: torch.Tensor,
                    ref_logprob: torch.Tensor | None = None, beta: float = 0.1, label_smoothing: float = 0.0,
                    margin: float = 0.0, grad=True, grad_scale: float = 1.0,
                    workspace: torch.Tensor | None = None) -> dict:
    """Preference loss over pairs of requests, and its gradient (``pr_preference_loss``).

    ``logits``, ``ids``, ``temperature``, ``weight``, ``grad``, ``workspace``
    as for :func:`policy_loss`. ``offsets`` int32 [2 n_pairs + 1]: request i
    owns rows ``offsets[i]:offsets[i+1]``; requests 2p and 2p + 1 are the
    chosen and the rejected answer of pair p. With q the sum over a request's
    rows of weight (logprob - ref_logprob) and
    h = beta (q_chosen - q_rejected) - margin, the loss is the mean over pairs
    of -(1 - label_smoothing) log sigmoid(h) - label_smoothing log sigmoid(-h).

    Returns a dict with ``loss`` (float32 [1]), ``pair_loss``, ``pair_logit``
    (h) [n_pairs], ``seq_logratio`` (q) [2 n_pairs], ``logprob``, ``flags``
    [n_rows] and, when wanted, ``grad``.
    """
    stream, device, code, temperature, grad = _check_loss(logits, ids, temperature, grad)
    n, V = logits.shape
    _check_row_floats(device, n, temperature=temperature, weight=weight, ref_logprob=ref_logprob)
    _check_index_tensor(offsets, "offsets", device)
    if offsets.shape[0] % 2 == 0:
        raise ValueError("offsets must have 2 n_pairs + 1 entries")
    n_pairs = offsets.shape[0] // 2
    L = _abi.lib()
    ws, ws_bytes, (logprob, q, pair, h, loss) = _loss_outputs(
        (n, 2 * n_pairs, n_pairs, n_pairs, 1), workspace, L.pr_preference_loss_workspace(code, n, V, n_pairs), device)
    flags = torch.empty(n, dtype=torch.int32, device=device)
    params = _abi.PreferenceParams(beta, label_smoothing, margin, grad_scale)
    values = _abi.PreferenceOut(pair.data_ptr(), h.data_ptr(), q.data_ptr(), logprob.data_ptr(), flags.data_ptr())
    st = L.pr_preference_loss(logits.data_ptr(), code, n, V, _row_stride(logits), ids.data_ptr(),
                              temperature.data_ptr(), weight.data_ptr(), offsets.data_ptr(), n_pairs,
                              _ptr(ref_logprob), C.byref(params), loss.data_ptr(), C.byref(values), _ptr(grad),
                              0 if grad is None else _row_stride(grad), ws, ws_bytes, stream)
    _abi.check("pr_preference_loss", st)
    out = {"loss": loss, "pair_loss": pair, "pair_logit": h, "seq_logratio": q, "logprob": logprob, "flags": flags}
    if grad is not None:
        out["grad"] = grad
    return out


class AdamW:
    """AdamW over many tensors at once (``pr_adamw_*``), states in 32 or 8 bits.

    ``params``: contiguous CUDA tensors, all float32 or all bfloat16 (then
    rounded stochastically). ``grads``: their gradients, when these stay in
    the same memory from step to step; otherwise :meth:`step` takes them.
    ``copies``: bfloat16 tensors that receive float32 parameters rounded to
    nearest. ``states``: a dict per tensor with ``m`` and ``v`` (float32 like
    the parameter; with ``state_bits=8`` uint8 codes, and uint8 ``m_exp`` and
    ``v_exp`` of one entry per 256 elements), as :attr:`states` holds them; by
    default zeros. ``steps``: steps taken so far. ``seed``: of the stochastic
    rounding.

    The tensors given and made here are kept, not copied: a step changes them
    in place, and they must stay where they are (one given another storage
    afterwards is stepped where it was). No two may overlap.

    The device's plan of the tensors is made at construction, or, for want of
    ``grads``, by the first :meth:`step` or :meth:`moments` and again by a
    first step whose gradients are not of the parameters' type: such a call
    allocates and waits for the device, so it cannot be captured into a graph.
    After :meth:`close` there are no more steps.
    """

    def __init__(self, params, grads=None, copies=None, state_bits: int = 32, states=None, seed: int = 0,
                 steps: int = 0):
        self._h = C.c_void_p()
        self._closed = False
        self._plan_dtype = None  # of the gradients that the plan takes
        self.params = list(params)
        if not self.params:
            raise ValueError("params must hold at least one tensor")
        if state_bits not in (8, 32):
            raise ValueError("state_bits must be 8 or 32")
        self.device = self.params[0].device
        _check_current(self.device, "params")
        self.state_bits, self.steps = state_bits, int(steps)
        n = len(self.params)
        self._dtype = self.params[0].dtype
        _dtype_code(self.params[0])
        for p in self.params:
            self._check(p, "params", self._dtype, None)
        self._sizes = [p.numel() for p in self.params]
        self.grads = self._list(grads, "grads", None)
        self._grad_dtype = self.grads[0].dtype if self.grads else None
        self.copies = self._list(copies, "copies", torch.bfloat16)
        if self.copies and self._dtype != torch.float32:
            raise ValueError("copies need float32 params")
        blocks = [-(-k // _abi.PR_ADAMW_BLOCK) for k in self._sizes]
        self._blocks = blocks
        if states is None:
            states = [self._zeros(k, b) for k, b in zip(self._sizes, blocks)]
        self.states = list(states)
        if len(self.states) != n:
            raise ValueError(f"states must have {n} entries")
        kind = torch.float32 if state_bits == 32 else torch.uint8
        names = ("m", "v", "m_exp", "v_exp")[:2 if state_bits == 32 else 4]
        for s, k, b in zip(self.states, self._sizes, blocks):
            for name, size in zip(names, (k, k, b, b)):
                if name not in s:
                    raise ValueError(f"a state of {state_bits} bits needs '{name}'")
                self._check(s[name], f"states' {name}", kind, size)
        self._tensors, self._storages = self._describe(names)
        self._seed = int(seed) & 0xFFFFFFFFFFFFFFFF
        if self._grad_dtype is not None:
            self._plan(self._grad_dtype)

    def _check(self, t, what, dtype, size):
        if t.dtype != dtype or t.device != self.device or not t.is_contiguous() or (size is not None and t.numel() != size):
            count = "" if size is None else f" of {size} elements"
            raise ValueError(f"{what} must be contiguous {dtype} tensors{count} on {self.device}")

    def _list(self, tensors, what, dtype):
        """A list that matches the parameters, or None."""
        if tensors is None:
            return None
        tensors = list(tensors)
        if len(tensors) != len(self._sizes):
            raise ValueError(f"{what} must have {len(self._sizes)} entries")
        if dtype is None:
            dtype = next((t.dtype for t in tensors if t is not None), None)
            if dtype not in (torch.float32, torch.bfloat16):
                raise ValueError(f"{what} must be float32 or bfloat16 tensors")
        for t, size in zip(tensors, self._sizes):
            if t is not None:
                self._check(t, what, dtype, size)
            elif what != "step's grads":
                raise ValueError(f"{what} must have a tensor for every parameter")
        return tensors

    def _zeros(self, n, blocks):
        kind = torch.float32 if self.state_bits == 32 else torch.uint8
        sizes = {"m": n, "v": n}
        if self.state_bits == 8:
            sizes.update(m_exp=blocks, v_exp=blocks)
        return {k: torch.zeros(size, dtype=kind, device=self.device) for k, size in sizes.items()}

    def _describe(self, names):
        """The tensors that were checked, for the plan, and their storages: kept, so that the plan's addresses stay
        allocated when one of the caller's tensors is given another storage."""
        T = (_abi.AdamWTensor * len(self.params))()
        for i, (t, p, s) in enumerate(zip(T, self.params, self.states)):
            t.param, t.n = p.data_ptr(), self._sizes[i]
            t.grad = self.grads[i].data_ptr() if self.grads else None
            t.copy = self.copies[i].data_ptr() if self.copies else None
            for name in names:
                setattr(t, name, s[name].data_ptr())
        lists = (self.params, self.grads or (), self.copies or (), *([s[k] for s in self.states] for k in names))
        return T, [t.untyped_storage() for tensors in lists for t in tensors]

    def _plan(self, grad_dtype):
        """Makes the device's plan for gradients of this type, unless it is there."""
        if self._h and self._plan_dtype == grad_dtype:
            return
        self._destroy()
        code = {torch.float32: _abi.PR_F32, torch.bfloat16: _abi.PR_BF16}
        st = _abi.lib().pr_adamw_create(self._tensors, len(self._tensors), code[self._dtype], code[grad_dtype],
                                        self.state_bits, self._seed, C.byref(self._h))
        _abi.check("pr_adamw_create", st)
        self._plan_dtype = grad_dtype

    def step(self, lr: float, beta1: float = 0.9, beta2: float = 0.999, eps: float = 1e-8, weight_decay: float = 0.01,
             grad_scale: float = 1.0, grads=None) -> None:
        """One step (``pr_adamw_step``) with the gradients given here or at construction; a None among those given
        here leaves its tensor as it is."""
        if self._closed:
            raise ValueError("the optimizer is closed")
        stream = _check_current(self.device, "the optimizer's tensors")
        pointers = None
        if grads is not None:
            grads = self._list(grads, "step's grads", None)
            dtype = next(t.dtype for t in grads if t is not None)
            if self._grad_dtype is None:
                self._plan(dtype)
                self._grad_dtype = dtype
            elif dtype != self._grad_dtype:
                raise ValueError(f"step's grads must be {self._grad_dtype} tensors")
            pointers = (C.c_void_p * len(grads))(*[None if t is None else t.data_ptr() for t in grads])
        elif self.grads is None:
            raise ValueError("step needs grads: none were given at construction")
        p = _abi.AdamWParams(float(lr), float(beta1), float(beta2), float(eps), float(weight_decay), float(grad_scale),
                             self.steps + 1)
        _abi.check("pr_adamw_step", _abi.lib().pr_adamw_step(self._h, pointers, C.byref(p), stream))
        self.steps += 1

    def moments(self, out=None):
        """The values of the states, a list of m and a list of v, each shaped like its parameter.

        32-bit states are returned themselves. 8-bit ones are decoded
        (``pr_adamw_moments``) to bfloat16, which holds them exactly.
        ``out`` (8-bit states): two bfloat16 buffers of 256 entries per block
        of 256 elements, which receive the values and are returned instead; tensor j
        starts at 256 times the blocks of the tensors before it, and entries
        between tensors are left as they are."""
        if self._closed:
            raise ValueError("the optimizer is closed")
        if self.state_bits == 32:
            if out is not None:
                raise ValueError("out is for 8-bit states: 32-bit ones are returned themselves")
            return tuple([s[k].view(p.shape) for s, p in zip(self.states, self.params)] for k in ("m", "v"))
        stream = _check_current(self.device, "the optimizer's tensors")
        # Before a first step any type of gradient will do.
        self._plan(self._grad_dtype or self._dtype)
        total = _abi.PR_ADAMW_BLOCK * sum(self._blocks)
        given = out is not None
        if not given:
            out = tuple(torch.zeros(total, dtype=torch.bfloat16, device=self.device) for _ in range(2))
        for t in out:
            self._check(t, "out", torch.bfloat16, total)
        _abi.check("pr_adamw_moments", _abi.lib().pr_adamw_moments(self._h, _ptr(out[0]), _ptr(out[1]), stream))
        if given:
            return out
        lists = ([], [])
        at = 0
        for p, size, blocks in zip(self.params, self._sizes, self._blocks):
            for flat, views in zip(out, lists):
                views.append(flat[at:at + size].view(p.shape))
            at += _abi.PR_ADAMW_BLOCK * blocks
        return lists

    def _destroy(self):
        if self._h:
            _abi.lib().pr_adamw_destroy(self._h)
            self._h = C.c_void_p()

    def close(self) -> None:
        self._closed = True
        self._destroy()

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass
