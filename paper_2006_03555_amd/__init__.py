"""FAVOR attention (arXiv 2006.03555) on AMD MI355X: Python binding of libfavor.

Every function here only marshals arguments for the C ABI declared in
``include/favor.h`` (device pointers, sizes, the current HIP stream); all
arithmetic runs in the library's HIP kernels. PyTorch provides device memory
and streams. If ``libfavor.so`` has not been built the calls raise
``FavorLibraryMissing``; there is no fallback.

Tensors: Q, K, V [B, H, L, d] (bfloat16 or float32, contiguous, on the GPU);
W [H, M, d] float32 and b [H, M] float32 from ``orf_draw``.

Keyword options of the feature and attention calls: kernel (KERNEL_SOFTMAX, the
Gaussian-kernel features of softmax attention, or KERNEL_RELU, generalized
attention with ReLU features), renormalize (False returns Q' K'^T V without the
division by D-hat) and kernel_eps (added to every ReLU feature). The attention
calls take row_scale (a [B, H, L] float32 tensor) to save each row's
1 / (D-hat + eps) for the backward calls, which then skip recomputing it.
"""
import ctypes
import functools
import operator
import os

from ._lib import (  # noqa: F401
    BF16, F32, RF_IID, RF_ORTHO_CHI, RF_ORTHO_FIXED, RF_HADAMARD, RF_GIVENS, OP_BIDIR, OP_BOTH, OP_CAUSAL, OP_FEATURE_MAP,
    OP_BIDIR_BACKWARD, OP_CAUSAL_BACKWARD, OP_BOTH_BACKWARD, KERNEL_RELU, KERNEL_SOFTMAX, backward_workspace_size,
    FavorDesc, FavorError, FavorLibraryMissing, lib, lib_path, make_desc, status_string,
    validate_desc, workspace_size, last_error, timing_enable, timing_reset, timing_read,
    FavorDecayDesc, decay_workspace_size, make_decay_desc, validate_decay_desc,
    FavorBeamDesc, FavorBeamPool, FavorConvDesc, FavorScanDesc, beam_workspace_size,
    conv_workspace_size, make_beam_desc, make_conv_desc, make_scan_desc, scan_workspace_size,
    validate_beam_desc, validate_conv_desc, validate_scan_desc,
)

__all__ = [
    "orf_draw", "feature_map", "attn_bidir", "attn_causal", "attn_both", "workspace_size",
    "attn_bidir_backward", "attn_causal_backward", "attn_both_backward",
    "backward_workspace_size", "make_desc",
    "attn_both_noalloc", "noalloc_scratch_bytes",
    "attn_decay", "attn_decay_backward", "attn_decay_step", "decay_workspace_size",
    "make_decay_desc", "validate_decay_desc", "dropout", "dropout_backward",
    "causal_conv", "causal_conv_backward", "causal_conv_step", "conv_workspace_size",
    "make_conv_desc", "validate_conv_desc",
    "selective_scan", "selective_scan_backward", "selective_scan_step", "scan_workspace_size",
    "make_scan_desc", "validate_scan_desc",
    "beam_select", "beam_reorder", "beam_workspace_size", "make_beam_desc",
    "validate_beam_desc",
    "validate_desc", "FavorError", "FavorLibraryMissing", "lib", "lib_path",
]


_torch_module = None


def _torch():
    global _torch_module
    if _torch_module is None:
        import torch
        _torch_module = torch
    return _torch_module


def _dtype_code(t):
    torch = _torch()
    if t == torch.bfloat16:
        return BF16
    if t == torch.float32:
        return F32
    raise FavorError(1, f"unsupported tensor dtype {t}; use bfloat16 or float32")


def _torch_dtype(code):
    torch = _torch()
    return torch.bfloat16 if code == BF16 else torch.float32


def _stream(stream):
    """HIP stream handle of `stream`, or of the current device's current stream (the
    raw handle where torch offers it: building a Stream object costs microseconds
    of every call)."""
    if stream is not None:
        return stream.cuda_stream
    torch = _torch()
    raw = getattr(torch._C, "_cuda_getCurrentRawStream", None)
    if raw is None:
        return torch.cuda.current_stream().cuda_stream
    return raw(torch.cuda.current_device())


def _on_stream(fn):
    """Run fn with the caller's stream (keyword `stream`) as torch's current
    stream, so that the outputs and the temporary workspace fn allocates belong
    to the stream the kernels run on: the caching allocator then hands a freed
    workspace block only to later work on that same stream, never to another
    stream while the kernels may still use it."""
    @functools.wraps(fn)
    def wrapper(*args, stream=None, **kw):
        # entering a stream context costs microseconds of host time per call:
        # skip it when the caller's stream already is the current one
        if stream is None:
            return fn(*args, **kw)
        if stream == _torch().cuda.current_stream():
            return fn(*args, stream=stream, **kw)
        with _torch().cuda.stream(stream):
            return fn(*args, stream=stream, **kw)
    return wrapper


def _ptr(t):
    """Address of a tensor, NULL for None (the ctypes signatures take both)."""
    return None if t is None else t.data_ptr()


def _check(status):
    if status != 0:
        raise FavorError(status, last_error())


def _require_cuda(*ts):
    for t in ts:
        if t is not None and not (t.is_cuda and t.is_contiguous()):
            raise FavorError(1, "tensors must be contiguous GPU tensors")


@_on_stream
def orf_draw(seed, n_heads, M, d=64, kind=RF_ORTHO_CHI, W=None, b=None, stream=None):
    """Draw W [n_heads, M, d] and b [n_heads, M] on the GPU (favor_orf_draw)."""
    torch = _torch()
    if W is None or b is None:
        dev = torch.device("cuda", torch.cuda.current_device())
    if W is None:
        W = torch.empty((n_heads, M, d), dtype=torch.float32, device=dev)
    if b is None:
        b = torch.empty((n_heads, M), dtype=torch.float32, device=dev)
    _require_features(W, b, n_heads, M, d)
    _require_cuda(W, b)
    _check(lib().favor_orf_draw(ctypes.c_uint64(seed), n_heads, M, d, kind, _ptr(W), _ptr(b),
                                _stream(stream)))
    return W, b


def _require_like(t, shape, dtype, name):
    """A caller-supplied tensor must have exactly the shape and dtype the call
    writes or reads (the kernels trust the descriptor, not the tensor)."""
    if t is None:
        return
    if t.shape != shape or t.dtype != dtype:   # torch.Size compares as a tuple
        raise FavorError(1, f"{name} must be {tuple(shape)} {dtype}, got {tuple(t.shape)} "
                            f"{t.dtype}")


def _require_features(W, b, H, M, d):
    torch = _torch()
    _require_like(W, (H, M, d), torch.float32, "W")
    _require_like(b, (H, M), torch.float32, "b")


class _Call:
    """A descriptor with its by-reference argument and the workspace sizes asked
    for so far. Held by value (see _call_for), read-only once built."""
    __slots__ = ("g", "ref", "B", "H", "L", "d", "M", "out_code", "sizes")

    def __init__(self, g):
        self.g = g
        self.ref = ctypes.byref(g)
        self.B, self.H, self.L, self.d, self.M = g.B, g.H, g.L, g.d, g.M
        self.out_code = g.out_dtype
        self.sizes = {}

    def workspace(self, op):
        n = self.sizes.get(op)
        if n is None:
            n = self.sizes[op] = workspace_size(self.g, op)
        return n

    def backward_workspace(self, op):
        n = self.sizes.get(("backward", op))
        if n is None:
            n = self.sizes[("backward", op)] = backward_workspace_size(self.g, op)
        return n


@functools.lru_cache(maxsize=256)
def _call_for(B, H, L, d, M, in_code, out_code, input_scale, denom_eps, segment, kernel,
              renormalize, kernel_eps, chunk):
    """The _Call of these values. Building the descriptor and asking the library for
    the workspace size cost several microseconds of every call of a program that
    makes the same one again; every argument is a plain number, so an entry depends
    on nothing else."""
    return _Call(make_desc(B, H, L, d, M, in_code, out_code, input_scale, denom_eps, segment,
                           kernel=kernel, renormalize=renormalize, kernel_eps=kernel_eps,
                           chunk=chunk))


def _desc_for(X, W, input_scale, out_dtype, denom_eps=0.0, segment=0, others=(),
              kernel=KERNEL_SOFTMAX, renormalize=True, kernel_eps=1e-3, chunk=0):
    """_Call for inputs X [B, H, L, d] (and tensors `others` of the same shape
    and dtype) with features W [H, M, d], b [H, M]."""
    if X.dim() != 4:
        raise FavorError(1, f"inputs must be [B, H, L, d], got {tuple(X.shape)}")
    shape, dtype = X.shape, X.dtype
    B, H, L, d = shape
    for name, t in others:
        _require_like(t, shape, dtype, name)
    if W.dim() != 3:
        raise FavorError(1, f"W must be [H, M, d], got {tuple(W.shape)}")
    in_code = _dtype_code(dtype)
    out_code = in_code if out_dtype is None else _dtype_code(out_dtype)
    return _call_for(B, H, L, d, W.shape[1], in_code, out_code, float(input_scale),
                     float(denom_eps), operator.index(segment), int(kernel), bool(renormalize),
                     float(kernel_eps), operator.index(chunk))


def _out_dtype(out_dtype, out, X):
    """Output dtype: as given, else that of a supplied output tensor, else X's."""
    if out_dtype is not None:
        return out_dtype
    return out.dtype if out is not None else X.dtype


@_on_stream
def feature_map(X, W, b, input_scale, out_dtype=None, out=None, stream=None,
                kernel=KERNEL_SOFTMAX, kernel_eps=1e-3):
    """X' [B, H, L, M] (favor_feature_map): D_X X-hat, or the ReLU features."""
    torch = _torch()
    g = _desc_for(X, W, input_scale, _out_dtype(out_dtype, out, X),
                  kernel=kernel, kernel_eps=kernel_eps)
    _require_features(W, b, g.H, g.M, g.d)
    shape = (g.B, g.H, g.L, g.M)
    if out is None:
        out = torch.empty(shape, dtype=_torch_dtype(g.out_code), device=X.device)
    _require_like(out, shape, _torch_dtype(g.out_code), "out")
    _require_cuda(X, W, b, out)
    _check(lib().favor_feature_map(g.ref, _ptr(X), _ptr(W), _ptr(b), _ptr(out),
                                   _stream(stream)))
    return out


def _workspace(g, causal, workspace):
    return _workspace_of(g.workspace(causal), workspace)


def _workspace_of(n, workspace):
    torch = _torch()
    if workspace is not None:
        return workspace, workspace.numel() * workspace.element_size()
    n = max(n, 1)
    return torch.empty(n, dtype=torch.uint8,
                       device=torch.device("cuda", torch.cuda.current_device())), n


def _require_row_scale(t, g, name):
    torch = _torch()
    _require_like(t, (g.B, g.H, g.L), torch.float32, name)


@_on_stream
def attn_bidir(Q, K, V, W, b, input_scale, denom_eps=0.0, out_dtype=None, out=None,
               workspace=None, stream=None, kernel=KERNEL_SOFTMAX, renormalize=True,
               kernel_eps=1e-3, row_scale=None):
    """Bidirectional FAVOR, Algorithm 1 (favor_attn_bidir). Returns out [B, H, L, d]."""
    torch = _torch()
    g = _desc_for(Q, W, input_scale, _out_dtype(out_dtype, out, Q), denom_eps,
                  others=(("K", K), ("V", V)), kernel=kernel, renormalize=renormalize,
                  kernel_eps=kernel_eps)
    _require_features(W, b, g.H, g.M, g.d)
    if out is None:
        out = torch.empty(Q.shape, dtype=_torch_dtype(g.out_code), device=Q.device)
    _require_like(out, Q.shape, _torch_dtype(g.out_code), "out")
    _require_row_scale(row_scale, g, "row_scale")
    _require_cuda(Q, K, V, W, b, out, row_scale)
    ws, nbytes = _workspace(g, 0, workspace)
    if row_scale is None:
        _check(lib().favor_attn_bidir(g.ref, _ptr(Q), _ptr(K), _ptr(V), _ptr(W),
                                      _ptr(b), _ptr(out), _ptr(ws), nbytes,
                                      _stream(stream)))
    else:
        _check(lib().favor_attn_bidir_save(g.ref, _ptr(Q), _ptr(K), _ptr(V), _ptr(W),
                                           _ptr(b), _ptr(out), _ptr(row_scale), _ptr(ws),
                                           nbytes, _stream(stream)))
    return out


@_on_stream
def attn_causal(Q, K, V, W, b, input_scale, denom_eps=0.0, state_in=None, return_state=False,
                segment=0, out_dtype=None, out=None, state_out=None, workspace=None, stream=None,
                kernel=KERNEL_SOFTMAX, renormalize=True, kernel_eps=1e-3, row_scale=None,
                chunk=0):
    """Unidirectional FAVOR by prefix sums (favor_attn_causal; favor_attn_causal_save
    when row_scale is given). segment: rows per causal segment (0 = library default);
    chunk: tokens per step of the scan (64; bf16 inputs also take 32; 0 = the library's
    choice).

    Returns out, or (out, state_out [B, H, M, d+1]) when return_state is true.
    """
    torch = _torch()
    g = _desc_for(Q, W, input_scale, _out_dtype(out_dtype, out, Q), denom_eps, segment,
                  others=(("K", K), ("V", V)),
                  kernel=kernel, renormalize=renormalize, kernel_eps=kernel_eps, chunk=chunk)
    _require_features(W, b, g.H, g.M, g.d)
    sshape = (g.B, g.H, g.M, g.d + 1)
    if out is None:
        out = torch.empty(Q.shape, dtype=_torch_dtype(g.out_code), device=Q.device)
    if return_state and state_out is None:
        state_out = torch.empty(sshape, dtype=torch.float32, device=Q.device)
    _require_like(out, Q.shape, _torch_dtype(g.out_code), "out")
    _require_like(state_in, sshape, torch.float32, "state_in")
    _require_like(state_out, sshape, torch.float32, "state_out")
    _require_row_scale(row_scale, g, "row_scale")
    _require_cuda(Q, K, V, W, b, out, state_in, state_out, row_scale)
    ws, nbytes = _workspace(g, 1, workspace)
    if row_scale is None:
        _check(lib().favor_attn_causal(g.ref, _ptr(Q), _ptr(K), _ptr(V), _ptr(W),
                                       _ptr(b), _ptr(out), _ptr(state_in), _ptr(state_out),
                                       _ptr(ws), nbytes, _stream(stream)))
    else:
        _check(lib().favor_attn_causal_save(g.ref, _ptr(Q), _ptr(K), _ptr(V), _ptr(W),
                                            _ptr(b), _ptr(out), _ptr(state_in), _ptr(state_out),
                                            _ptr(row_scale), _ptr(ws), nbytes,
                                            _stream(stream)))
    return (out, state_out) if return_state else out


@_on_stream
def attn_both(Q, K, V, W, b, input_scale, denom_eps=0.0, state_in=None, return_state=False,
              segment=0, out_dtype=None, out_bidir=None, out_causal=None, state_out=None,
              workspace=None, stream=None, kernel=KERNEL_SOFTMAX, renormalize=True,
              kernel_eps=1e-3, row_scale_bidir=None, row_scale_causal=None, chunk=0):
    """Both directions over the same inputs with one key pass (favor_attn_both);
    segment and chunk as for attn_causal.

    Returns (out_bidir, out_causal) or (out_bidir, out_causal, state_out).
    """
    torch = _torch()
    g = _desc_for(Q, W, input_scale, _out_dtype(out_dtype, out_bidir, Q), denom_eps, segment,
                  others=(("K", K), ("V", V)),
                  kernel=kernel, renormalize=renormalize, kernel_eps=kernel_eps, chunk=chunk)
    _require_features(W, b, g.H, g.M, g.d)
    odt = _torch_dtype(g.out_code)
    sshape = (g.B, g.H, g.M, g.d + 1)
    if out_bidir is None:
        out_bidir = torch.empty(Q.shape, dtype=odt, device=Q.device)
    if out_causal is None:
        out_causal = torch.empty(Q.shape, dtype=odt, device=Q.device)
    if return_state and state_out is None:
        state_out = torch.empty(sshape, dtype=torch.float32, device=Q.device)
    _require_like(out_bidir, Q.shape, odt, "out_bidir")
    _require_like(out_causal, Q.shape, odt, "out_causal")
    _require_like(state_in, sshape, torch.float32, "state_in")
    _require_like(state_out, sshape, torch.float32, "state_out")
    _require_row_scale(row_scale_bidir, g, "row_scale_bidir")
    _require_row_scale(row_scale_causal, g, "row_scale_causal")
    _require_cuda(Q, K, V, W, b, out_bidir, out_causal, state_in, state_out, row_scale_bidir,
                  row_scale_causal)
    ws, nbytes = _workspace(g, 2, workspace)
    _check(lib().favor_attn_both(g.ref, _ptr(Q), _ptr(K), _ptr(V), _ptr(W), _ptr(b),
                                 _ptr(out_bidir), _ptr(out_causal), _ptr(state_in),
                                 _ptr(state_out), _ptr(row_scale_bidir), _ptr(row_scale_causal),
                                 _ptr(ws), nbytes, _stream(stream)))
    if return_state:
        return out_bidir, out_causal, state_out
    return out_bidir, out_causal


@_on_stream
def attn_both_noalloc(Q, K, V, W, b, input_scale, denom_eps=0.0, state_in=None,
                      segment=0, out_bidir=None, out_causal=None, state_out=None, stream=None,
                      kernel=KERNEL_SOFTMAX, renormalize=True, kernel_eps=1e-3,
                      row_scale_bidir=None, row_scale_causal=None, chunk=0):
    """attn_both with the library's static scratch as workspace
    (favor_attn_both_noalloc): nothing is allocated when the outputs are given.
    Returns (out_bidir, out_causal)."""
    torch = _torch()
    odt = out_bidir.dtype if out_bidir is not None else Q.dtype
    g = _desc_for(Q, W, input_scale, odt, denom_eps, segment,
                  others=(("K", K), ("V", V)),
                  kernel=kernel, renormalize=renormalize, kernel_eps=kernel_eps, chunk=chunk)
    _require_features(W, b, g.H, g.M, g.d)
    tdt = _torch_dtype(g.out_code)
    sshape = (g.B, g.H, g.M, g.d + 1)
    if out_bidir is None:
        out_bidir = torch.empty(Q.shape, dtype=tdt, device=Q.device)
    if out_causal is None:
        out_causal = torch.empty(Q.shape, dtype=tdt, device=Q.device)
    _require_like(out_bidir, Q.shape, tdt, "out_bidir")
    _require_like(out_causal, Q.shape, tdt, "out_causal")
    _require_like(state_in, sshape, torch.float32, "state_in")
    _require_like(state_out, sshape, torch.float32, "state_out")
    _require_row_scale(row_scale_bidir, g, "row_scale_bidir")
    _require_row_scale(row_scale_causal, g, "row_scale_causal")
    _require_cuda(Q, K, V, W, b, out_bidir, out_causal, state_in, state_out, row_scale_bidir,
                  row_scale_causal)
    _check(lib().favor_attn_both_noalloc(
        g.ref, _ptr(Q), _ptr(K), _ptr(V), _ptr(W), _ptr(b), _ptr(out_bidir),
        _ptr(out_causal), _ptr(state_in), _ptr(state_out), _ptr(row_scale_bidir),
        _ptr(row_scale_causal), _stream(stream)))
    return out_bidir, out_causal


def noalloc_scratch_bytes():
    """Size of the static scratch array attn_both_noalloc uses (per GPU)."""
    return lib().favor_noalloc_scratch_bytes()


def _bwd_workspace(g, causal, workspace):
    return _workspace_of(g.backward_workspace(causal), workspace)


def _bwd_grads(Q, dQ, dK, dV):
    torch = _torch()
    out = []
    for name, t in (("dQ", dQ), ("dK", dK), ("dV", dV)):
        if t is None:
            t = torch.empty_like(Q)
        _require_like(t, Q.shape, Q.dtype, name)
        out.append(t)
    return out


_FWD_OPS = {"bidir": OP_BIDIR, "causal": OP_CAUSAL, "both": OP_BOTH}


def _forward_ws(forward_workspace, forward_call, allowed):
    """(pointer, op code) of a forward call's workspace offered to a backward call."""
    if forward_workspace is None:
        if forward_call is not None:
            raise FavorError(1, "forward_call without forward_workspace")
        return None, 0
    if forward_call not in allowed:
        raise FavorError(1, f"forward_call must be one of {sorted(allowed)}, got {forward_call!r}")
    _require_cuda(forward_workspace)
    return _ptr(forward_workspace), _FWD_OPS[forward_call]


def _saved(out, row_scale, g, Q):
    if (out is None) != (row_scale is None):
        raise FavorError(1, "pass the forward call's out and row_scale together")
    if out is not None:
        _require_like(out, Q.shape, Q.dtype, "out")
        _require_row_scale(row_scale, g, "row_scale")


@_on_stream
def attn_bidir_backward(Q, K, V, W, b, input_scale, dout, denom_eps=0.0, dQ=None, dK=None,
                        dV=None, workspace=None, stream=None, kernel=KERNEL_SOFTMAX,
                        renormalize=True, kernel_eps=1e-3, out=None, row_scale=None,
                        forward_workspace=None, forward_call=None):
    """Gradients (dQ, dK, dV) of attn_bidir for the upstream gradient dout
    (favor_attn_bidir_backward). out and row_scale, from the forward call with
    row_scale, spare recomputing them; forward_workspace, the workspace of the
    forward call forward_call ("bidir" or "both") with the same descriptor and
    inputs, spares recomputing Buf1."""
    g = _desc_for(Q, W, input_scale, Q.dtype, denom_eps,
                  others=(("K", K), ("V", V), ("dout", dout)),
                  kernel=kernel, renormalize=renormalize,
                  kernel_eps=kernel_eps)
    _require_features(W, b, g.H, g.M, g.d)
    dQ, dK, dV = _bwd_grads(Q, dQ, dK, dV)
    _saved(out, row_scale, g, Q)
    _require_cuda(Q, K, V, W, b, dout, dQ, dK, dV, out, row_scale)
    fptr, fop = _forward_ws(forward_workspace, forward_call, ("bidir", "both"))
    ws, nbytes = _bwd_workspace(g, False, workspace)
    _check(lib().favor_attn_bidir_backward(g.ref, _ptr(Q), _ptr(K), _ptr(V), _ptr(W),
                                           _ptr(b), _ptr(dout), _ptr(out), _ptr(row_scale),
                                           fptr, fop, _ptr(dQ), _ptr(dK), _ptr(dV), _ptr(ws),
                                           nbytes, _stream(stream)))
    return dQ, dK, dV


@_on_stream
def attn_causal_backward(Q, K, V, W, b, input_scale, dout, denom_eps=0.0, state_in=None,
                         dstate_out=None, return_state_grad=False, dQ=None, dK=None, dV=None,
                         dstate_in=None, workspace=None, stream=None, kernel=KERNEL_SOFTMAX,
                         renormalize=True, kernel_eps=1e-3, out=None, row_scale=None,
                         forward_workspace=None, forward_call=None, chunk=0):
    """Gradients of attn_causal (favor_attn_causal_backward). Returns (dQ, dK, dV), plus
    dstate_in [B, H, M, d+1] when return_state_grad is true. out and row_scale as for
    attn_bidir_backward; forward_workspace of the forward call forward_call ("causal"
    or "both", same descriptor, inputs and state_in) spares recomputing the segment
    prefixes. chunk: the scan's chunk length for the forward quantities the call
    recomputes (as for attn_causal)."""
    torch = _torch()
    g = _desc_for(Q, W, input_scale, Q.dtype, denom_eps,
                  others=(("K", K), ("V", V), ("dout", dout)),
                  kernel=kernel, renormalize=renormalize, kernel_eps=kernel_eps, chunk=chunk)
    _require_features(W, b, g.H, g.M, g.d)
    dQ, dK, dV = _bwd_grads(Q, dQ, dK, dV)
    sshape = (g.B, g.H, g.M, g.d + 1)
    if return_state_grad and dstate_in is None:
        dstate_in = torch.empty(sshape, dtype=torch.float32, device=Q.device)
    for name, t in (("state_in", state_in), ("dstate_out", dstate_out), ("dstate_in", dstate_in)):
        _require_like(t, sshape, torch.float32, name)
    _saved(out, row_scale, g, Q)
    _require_cuda(Q, K, V, W, b, dout, dQ, dK, dV, state_in, dstate_out, dstate_in, out,
                  row_scale)
    fptr, fop = _forward_ws(forward_workspace, forward_call, ("causal", "both"))
    ws, nbytes = _bwd_workspace(g, True, workspace)
    _check(lib().favor_attn_causal_backward(
        g.ref, _ptr(Q), _ptr(K), _ptr(V), _ptr(W), _ptr(b), _ptr(state_in), _ptr(dout),
        _ptr(out), _ptr(row_scale), fptr, fop, _ptr(dstate_out), _ptr(dQ), _ptr(dK), _ptr(dV),
        _ptr(dstate_in), _ptr(ws), nbytes, _stream(stream)))
    return (dQ, dK, dV, dstate_in) if return_state_grad else (dQ, dK, dV)


def attn_both_backward(Q, K, V, W, b, input_scale, dout_bidir, dout_causal, denom_eps=0.0,
                       state_in=None, dstate_out=None, return_state_grad=False, dQ=None,
                       dK=None, dV=None, dstate_in=None, workspace=None, stream=None,
                       kernel=KERNEL_SOFTMAX, renormalize=True, kernel_eps=1e-3,
                       out_bidir=None, row_scale_bidir=None, out_causal=None,
                       row_scale_causal=None, forward_workspace=None, forward_call=None,
                       chunk=0, segment=0):
    """Gradients of attn_both (favor_attn_both_backward): of a loss of both outputs,
    given dout_bidir and dout_causal. Returns (dQ, dK, dV), the sums over the two
    directions, plus the causal state gradient dstate_in when return_state_grad is
    true. out_* and row_scale_* as the forward call saved them (each pair or
    neither); forward_workspace of an attn_both call (forward_call "both", same
    descriptor, inputs and state_in) spares recomputing Buf1 and the segment
    prefixes."""
    torch = _torch()
    g = _desc_for(Q, W, input_scale, Q.dtype, denom_eps, segment,
                  others=(("K", K), ("V", V), ("dout_bidir", dout_bidir),
                          ("dout_causal", dout_causal)),
                  kernel=kernel, renormalize=renormalize, kernel_eps=kernel_eps, chunk=chunk)
    _require_features(W, b, g.H, g.M, g.d)
    dQ, dK, dV = _bwd_grads(Q, dQ, dK, dV)
    sshape = (g.B, g.H, g.M, g.d + 1)
    if return_state_grad and dstate_in is None:
        dstate_in = torch.empty(sshape, dtype=torch.float32, device=Q.device)
    for name, t in (("state_in", state_in), ("dstate_out", dstate_out), ("dstate_in", dstate_in)):
        _require_like(t, sshape, torch.float32, name)
    _saved(out_bidir, row_scale_bidir, g, Q)
    _saved(out_causal, row_scale_causal, g, Q)
    _require_cuda(Q, K, V, W, b, dout_bidir, dout_causal, dQ, dK, dV, state_in, dstate_out,
                  dstate_in, out_bidir, row_scale_bidir, out_causal, row_scale_causal)
    fptr, fop = _forward_ws(forward_workspace, forward_call, ("both",))
    ws, nbytes = _bwd_workspace(g, 2, workspace)
    _check(lib().favor_attn_both_backward(
        g.ref, _ptr(Q), _ptr(K), _ptr(V), _ptr(W), _ptr(b), _ptr(state_in),
        _ptr(dout_bidir), _ptr(dout_causal), _ptr(out_bidir), _ptr(row_scale_bidir),
        _ptr(out_causal), _ptr(row_scale_causal), fptr, fop, _ptr(dstate_out), _ptr(dQ),
        _ptr(dK), _ptr(dV), _ptr(dstate_in), _ptr(ws), nbytes,
        _stream(stream)))
    return (dQ, dK, dV, dstate_in) if return_state_grad else (dQ, dK, dV)


def library_loaded_from():
    """Absolute path of the libfavor.so this process uses."""
    return os.path.realpath(lib_path())


# ------------------------------------------------- linear attention with a decay per head
def _require_here(*ts):
    """The kernels run on the current device and read raw addresses there. Returns that
    device's number (-1 without a tensor)."""
    here = -1
    for t in ts:
        if t is None:
            continue
        dev = t.get_device()
        if dev < 0:
            raise FavorError(1, "tensors must be GPU tensors")
        if here < 0:
            here = _torch().cuda.current_device()
        if dev != here:
            raise FavorError(1, f"a tensor is on device {dev}, the current device is {here}")
    return here


def _require_whole(*ts):
    for t in ts:
        if t is not None and not t.is_contiguous():
            raise FavorError(1, "states, decays, lengths and slots must be contiguous")


def _like(t):
    """What a call's plan depends on of one tensor."""
    return None if t is None else (t.shape, t.dtype, t.stride())


def _row_strides(shape, s, name):
    """(batch, head, token) strides of [B, H, L, d] rows (token: any for [B, H, d]) of a
    tensor with strides s. Dimensions of one element have no stride; d stands in for it,
    since three zeros mean the contiguous layout."""
    d = shape[-1]
    if d > 1 and s[-1] != 1:
        raise FavorError(1, f"rows of {name} must be contiguous")
    got = tuple(s[i] if shape[i] > 1 else d for i in range(len(shape) - 1))
    if len(got) == 2:
        got += (d,)
    if not any(got):
        raise FavorError(1, f"{name} is one row broadcast to all")
    return got


class _DecayCall:
    """A decay descriptor with its by-reference argument and workspace size."""
    __slots__ = ("g", "ref", "workspace")

    def __init__(self, g, backward=None):
        self.g = g
        self.ref = ctypes.byref(g)
        self.workspace = 0 if backward is None else decay_workspace_size(g, backward)


def _require_shape(like, shape, dtype, name):
    if like is not None and (like[0] != shape or like[1] != dtype):
        raise FavorError(1, f"{name} must be {tuple(shape)} {dtype}, got {tuple(like[0])} "
                            f"{like[1]}")


@functools.lru_cache(maxsize=256)
def _decay_plan(backward, q, k, v, rows, log_decay, lengths, states, scale):
    """The _DecayCall of a forward (False), backward (True) or single-token (None) call, its
    tensors' shapes and types checked. Every argument is made of _like()'s plain values, so
    a program that makes the same call again pays for one look into the cache.

    rows: (name, descriptor field, which of "qkv" it is shaped like, _like()) of the others.
    """
    torch = _torch()
    dims = 3 if backward is None else 4
    if len(q[0]) != dims or len(v[0]) != dims:
        want = "[B, H, d]" if dims == 3 else "[B, H, L, d]"
        raise FavorError(1, f"inputs must be {want}, got {tuple(q[0])} and {tuple(v[0])}")
    B, H = q[0][:2]
    L = 1 if backward is None else q[0][2]
    dk, dv = q[0][-1], v[0][-1]
    if dk == 0 or dv == 0:
        raise FavorError(1, "dk and dv must be positive")
    dtype = q[1]
    _require_shape(k, q[0], dtype, "K")
    _require_shape(v, q[0][:-1] + (dv,), dtype, "V")
    _require_shape(log_decay, (H,), torch.float32, "log_decay")
    _require_shape(lengths, (B,), torch.int32, "slots" if backward is None else "lengths")
    strides = {n: _row_strides(t[0], t[2], n.upper()) for n, t in (("q", q), ("k", k), ("v", v))}
    like = {"q": q, "k": k, "v": v}
    for name, field, of, t in rows:
        _require_shape(t, like[of][0], dtype, name)
        if t is not None:
            strides[field] = _row_strides(t[0], t[2], name)
    for name, t in states:
        if t is not None:
            n = t[0][0] if backward is None and len(t[0]) == 4 else B
            _require_shape(t, (n, H, dk, dv), torch.float32, name)
    return _DecayCall(make_decay_desc(B, H, L, dk, dv, _dtype_code(dtype), scale, **strides),
                      backward)


def _decay_workspace(n, workspace):
    if workspace is not None:
        _require_here(workspace)
        _require_whole(workspace)
    elif n == 0:
        return None, 0
    return _workspace_of(n, workspace)


def _stream_on(device, stream):
    """As _stream, where the current device is already known (-1: it is not)."""
    if stream is None and device >= 0:
        raw = getattr(_torch()._C, "_cuda_getCurrentRawStream", None)
        if raw is not None:
            return raw(device)
    return _stream(stream)


@_on_stream
def attn_decay(Q, K, V, log_decay, scale=1.0, lengths=None, state_in=None, return_state=False,
               out=None, state_out=None, workspace=None, stream=None):
    """Linear attention with a decay per head (favor_attn_decay):
    out_i = scale (sum_{j <= i} a^(i - j) (q_i . k_j) v_j + a^(i + 1) q_i state_in) with
    a = exp(log_decay[h]).

    Q, K [B, H, L, dk], V [B, H, L, dv]: bfloat16 or float32, rows contiguous, any other
    strides (a transposed [B, L, H, d], slices of a projection, expanded tensors); dk and
    dv multiples of 8 up to 256. lengths [B] int32: tokens of each right-padded sequence.
    State tensors [B, H, dk, dv] float32. Returns out [B, H, L, dv] (in V's layout unless
    given), or (out, state_out) when return_state is true.
    """
    torch = _torch()
    if out is None:
        out = torch.empty_like(V)
    c = _decay_plan(False, _like(Q), _like(K), _like(V), (("out", "out", "v", _like(out)),),
                    _like(log_decay), _like(lengths),
                    (("state_in", _like(state_in)), ("state_out", _like(state_out))),
                    float(scale))
    if return_state and state_out is None:
        g = c.g
        state_out = torch.empty((g.B, g.H, g.dk, g.dv), dtype=torch.float32, device=Q.device)
    here = _require_here(Q, K, V, log_decay, lengths, out, state_in, state_out)
    _require_whole(log_decay, lengths, state_in, state_out)
    ws, nbytes = _decay_workspace(c.workspace, workspace)
    _check(lib().favor_attn_decay(c.ref, _ptr(Q), _ptr(K), _ptr(V), _ptr(log_decay),
                                  _ptr(lengths), _ptr(out), _ptr(state_in), _ptr(state_out),
                                  _ptr(ws), nbytes, _stream_on(here, stream)))
    return (out, state_out) if return_state else out


@_on_stream
def attn_decay_backward(Q, K, V, log_decay, dout, scale=1.0, lengths=None, state_in=None,
                        dstate_out=None, return_state_grad=False, dQ=None, dK=None, dV=None,
                        dstate_in=None, workspace=None, stream=None):
    """Gradients of attn_decay (favor_attn_decay_backward). dout: the gradient of out, and
    dstate_out (default zeros) of state_out. log_decay receives none; an expanded input's
    gradients come for every head and batch entry.

    Returns (dQ, dK, dV), or (dQ, dK, dV, dstate_in) when return_state_grad is true.
    """
    torch = _torch()
    dQ, dK, dV = (torch.empty_like(x) if t is None else t
                  for t, x in ((dQ, Q), (dK, K), (dV, V)))
    c = _decay_plan(True, _like(Q), _like(K), _like(V),
                    (("dout", "grad_out", "v", _like(dout)), ("dQ", "grad_q", "q", _like(dQ)),
                     ("dK", "grad_k", "k", _like(dK)), ("dV", "grad_v", "v", _like(dV))),
                    _like(log_decay), _like(lengths),
                    (("state_in", _like(state_in)), ("dstate_out", _like(dstate_out)),
                     ("dstate_in", _like(dstate_in))), float(scale))
    if return_state_grad and dstate_in is None:
        g = c.g
        dstate_in = torch.empty((g.B, g.H, g.dk, g.dv), dtype=torch.float32, device=Q.device)
    here = _require_here(Q, K, V, log_decay, lengths, dout, dQ, dK, dV, state_in, dstate_out,
                         dstate_in)
    _require_whole(log_decay, lengths, state_in, dstate_out, dstate_in)
    ws, nbytes = _decay_workspace(c.workspace, workspace)
    _check(lib().favor_attn_decay_backward(
        c.ref, _ptr(Q), _ptr(K), _ptr(V), _ptr(log_decay), _ptr(lengths), _ptr(state_in),
        _ptr(dout), _ptr(dstate_out), _ptr(dQ), _ptr(dK), _ptr(dV), _ptr(dstate_in), _ptr(ws),
        nbytes, _stream_on(here, stream)))
    return (dQ, dK, dV, dstate_in) if return_state_grad else (dQ, dK, dV)


@_on_stream
def attn_decay_step(q, k, v, log_decay, state, scale=1.0, slots=None, out=None, stream=None):
    """The next token of B sequences (favor_attn_decay_step): state <- a state + k v^T in
    place, out = scale q state.

    q, k [B, H, dk], v [B, H, dv] (rows contiguous, any other strides); state
    [n, H, dk, dv] float32. slots [B] int32: the place of each sequence's state (default:
    its own index); one outside 0 .. n - 1 is padding and gives out = 0. Returns out
    [B, H, dv].
    """
    if out is None:
        out = _torch().empty_like(v, memory_format=_torch().contiguous_format)
    c = _decay_plan(None, _like(q), _like(k), _like(v), (("out", "out", "v", _like(out)),),
                    _like(log_decay), _like(slots), (("state", _like(state)),), float(scale))
    here = _require_here(q, k, v, log_decay, state, slots, out)
    _require_whole(log_decay, state, slots)
    _check(lib().favor_attn_decay_step(c.ref, q.data_ptr(), k.data_ptr(), v.data_ptr(),
                                       log_decay.data_ptr(), _ptr(slots), state.shape[0],
                                       state.data_ptr(), out.data_ptr(),
                                       _stream_on(here, stream)))
    return out


# ------------------------------------------------------------------------------- dropout
@_on_stream
def dropout(x, p, seed=0, offset=0, residual=None, out=None, rng=None, stream=None):
    """residual + x with a share p of its elements dropped and the others divided by
    1 - p (favor_dropout; p to 16 bits). The mask is Philox4x32-10's at (seed, offset) and
    is not stored: advance offset from call to call, and give dropout_backward the same.
    rng: a device tensor of two int64 words {seed, offset} read in their place when the
    kernel runs (for captured graphs). out may be x or residual.
    """
    torch = _torch()
    if out is None:
        out = torch.empty_like(x, memory_format=torch.contiguous_format)
    _require_like(residual, x.shape, x.dtype, "residual")
    _require_like(out, x.shape, x.dtype, "out")
    if rng is not None and (rng.shape != (2,) or rng.dtype not in (torch.int64, torch.uint64)):
        raise FavorError(1, f"rng must be two 64-bit words, got {tuple(rng.shape)} {rng.dtype}")
    here = _require_here(x, residual, out, rng)
    _require_cuda(x, residual, out, rng)
    if not (0 <= operator.index(seed) < 1 << 64 and 0 <= operator.index(offset) < 1 << 64):
        raise FavorError(1, f"seed and offset are 64-bit unsigned numbers, got {seed}, {offset}")
    _check(lib().favor_dropout(_ptr(x), _ptr(residual), _ptr(out), x.numel(),
                               _dtype_code(x.dtype), float(p), seed, offset, _ptr(rng),
                               _stream_on(here, stream)))
    return out


def dropout_backward(dout, p, seed=0, offset=0, dx=None, rng=None, stream=None):
    """The gradient of dropout's x (its residual's is dout): the same mask on dout."""
    return dropout(dout, p, seed, offset, out=dx, rng=rng, stream=stream)


# ------------------------------------------------- short convolution and selective scan
class _Planned:
    """A descriptor with its by-reference argument and workspace size."""
    __slots__ = ("g", "ref", "workspace")

    def __init__(self, g, workspace):
        self.g = g
        self.ref = ctypes.byref(g)
        self.workspace = workspace


def _token_rows(like, name):
    """(batch, unused, token) strides of [B, L, D] (or [B, D]) rows; see _row_strides."""
    return _row_strides((like[0][0], 1) + tuple(like[0][1:]),
                        (like[2][0], 0) + tuple(like[2][1:]), name)


def _group_rows(like, name):
    """(batch, group, token) strides of [B, L, G, N] (or [B, G, N]) rows."""
    shape, s = like[0], like[2]
    if len(shape) == 3:
        return _row_strides(shape, s, name)
    return _row_strides((shape[0], shape[2], shape[1], shape[3]), (s[0], s[2], s[1], s[3]), name)


def _require_dims(like, dims, want, name):
    if len(like[0]) != dims:
        raise FavorError(1, f"{name} must be {want}, got {tuple(like[0])}")


def _require_state(name, like, shape, dtype, pool):
    """A state of every sequence; pool: of any number of places."""
    if like is not None:
        _require_dims(like, len(shape), f"of {len(shape)} dimensions", name)
        _require_shape(like, (like[0][0],) + shape[1:] if pool else shape, dtype, name)


@functools.lru_cache(maxsize=256)
def _conv_plan(op, x, weight, bias, lengths, rows, states, silu):
    """The _Planned call of a forward (0), backward (1) or single-token (2) convolution, its tensors'
    shapes and types checked; every argument is made of _like()'s plain values."""
    torch = _torch()
    _require_dims(x, 2 if op == 2 else 3, "[B, D]" if op == 2 else "[B, L, D]", "x")
    _require_dims(weight, 2, "[D, width]", "weight")
    B, D, L = x[0][0], x[0][-1], 1 if op == 2 else x[0][1]
    width = weight[0][1]
    _require_shape(weight, (D, width), torch.float32, "weight")
    _require_shape(bias, (D,), torch.float32, "bias")
    _require_shape(lengths, (B,), torch.int32, "slots" if op == 2 else "lengths")
    strides = {"x": _token_rows(x, "x")}
    for name, field, t in rows:
        if field is None:
            _require_shape(t, (D, width) if name == "dweight" else (D,), torch.float32, name)
        else:
            _require_shape(t, x[0], x[1], name)
            strides[field] = _token_rows(t, name)
    for name, t in states:
        _require_state(name, t, (B, width - 1, D), x[1], op == 2)
    g = make_conv_desc(B, L, D, width, _dtype_code(x[1]), silu, **strides)
    _check(validate_conv_desc(g, op))
    return _Planned(g, conv_workspace_size(g) if op == 1 else 0)


@_on_stream
def causal_conv(x, weight, bias=None, silu=False, lengths=None, state_in=None,
                return_state=False, out=None, state_out=None, stream=None):
    """Short causal convolution, one filter per channel (favor_conv):
    y_t = act(bias + sum_j weight[:, j] x_{t - width + 1 + j}).

    x [B, L, D]: bfloat16 or float32, rows contiguous, any other strides (a half of a
    projection); D a multiple of 8. weight [D, width] (2 to 8 taps) and bias [D] float32;
    silu: y = u sigmoid(u). lengths [B] int32: tokens of each right-padded sequence. States
    [B, width - 1, D] in x's type: the last inputs. Returns y [B, L, D] (contiguous unless
    given), or (y, state_out) when return_state is true.
    """
    torch = _torch()
    if out is None:
        out = torch.empty_like(x, memory_format=torch.contiguous_format)
    c = _conv_plan(0, _like(x), _like(weight), _like(bias), _like(lengths),
                   (("out", "y", _like(out)),),
                   (("state_in", _like(state_in)), ("state_out", _like(state_out))), bool(silu))
    if return_state and state_out is None:
        g = c.g
        state_out = torch.empty((g.B, g.width - 1, g.D), dtype=x.dtype, device=x.device)
    here = _require_here(x, weight, bias, lengths, out, state_in, state_out)
    _require_whole(weight, bias, lengths, state_in, state_out)
    _check(lib().favor_conv(c.ref, _ptr(x), _ptr(weight), _ptr(bias), _ptr(lengths), _ptr(out),
                            _ptr(state_in), _ptr(state_out), _stream_on(here, stream)))
    return (out, state_out) if return_state else out


@_on_stream
def causal_conv_backward(x, weight, dout, bias=None, silu=False, lengths=None, state_in=None,
                         dstate_out=None, return_state_grad=False, dx=None, dweight=None,
                         dbias=None, dstate_in=None, workspace=None, stream=None):
    """Gradients of causal_conv (favor_conv_backward) from dout and dstate_out (default zeros).

    Returns (dx, dweight, dbias), or (dx, dweight, dbias, dstate_in) when return_state_grad is
    true; dbias is None without a bias.
    """
    torch = _torch()
    if dx is None:
        dx = torch.empty_like(x, memory_format=torch.contiguous_format)
    if dweight is None:
        dweight = torch.empty_like(weight)
    if bias is None:
        dbias = None
    elif dbias is None:
        dbias = torch.empty_like(bias)
    c = _conv_plan(1, _like(x), _like(weight), _like(bias), _like(lengths),
                   (("dout", "grad_y", _like(dout)), ("dx", "grad_x", _like(dx)),
                    ("dweight", None, _like(dweight)), ("dbias", None, _like(dbias))),
                   (("state_in", _like(state_in)), ("dstate_out", _like(dstate_out)),
                    ("dstate_in", _like(dstate_in))), bool(silu))
    if return_state_grad and dstate_in is None:
        g = c.g
        dstate_in = torch.empty((g.B, g.width - 1, g.D), dtype=x.dtype, device=x.device)
    here = _require_here(x, weight, bias, lengths, dout, dx, dweight, dbias, state_in, dstate_out,
                         dstate_in)
    _require_whole(weight, bias, lengths, dweight, dbias, state_in, dstate_out, dstate_in)
    ws, nbytes = _decay_workspace(c.workspace, workspace)
    _check(lib().favor_conv_backward(
        c.ref, _ptr(x), _ptr(weight), _ptr(bias), _ptr(lengths), _ptr(state_in), _ptr(dout),
        _ptr(dstate_out), _ptr(dx), _ptr(dweight), _ptr(dbias), _ptr(dstate_in), _ptr(ws), nbytes,
        _stream_on(here, stream)))
    return (dx, dweight, dbias, dstate_in) if return_state_grad else (dx, dweight, dbias)


@_on_stream
def causal_conv_step(x, weight, state, bias=None, silu=False, slots=None, out=None, stream=None):
    """The next token of B sequences (favor_conv_step): x [B, D], state [n, width - 1, D] (the
    last inputs) updated in place. slots [B] int32: the place of each sequence's state
    (default: its own index); one outside 0 .. n - 1 is padding and gives y = 0. Returns
    y [B, D].
    """
    if out is None:
        out = _torch().empty_like(x, memory_format=_torch().contiguous_format)
    c = _conv_plan(2, _like(x), _like(weight), _like(bias), _like(slots),
                   (("out", "y", _like(out)),), (("state", _like(state)),), bool(silu))
    here = _require_here(x, weight, bias, state, slots, out)
    _require_whole(weight, bias, state, slots)
    _check(lib().favor_conv_step(c.ref, x.data_ptr(), weight.data_ptr(), _ptr(bias), _ptr(slots),
                                 state.shape[0], state.data_ptr(), out.data_ptr(),
                                 _stream_on(here, stream)))
    return out


@functools.lru_cache(maxsize=256)
def _scan_plan(op, x, A, params, b, c, rows, lengths, states, softplus):
    """As _conv_plan, of a selective scan. params: (name, _like()) of [D] ones; rows: (name,
    field, which of "x" and "b" it is shaped like, _like())."""
    torch = _torch()
    _require_dims(x, 2 if op == 2 else 3, "[B, D]" if op == 2 else "[B, L, D]", "x")
    _require_dims(A, 2, "[D, N]", "A")
    lead, D, N = x[0][:-1], x[0][-1], A[0][1]
    if op == 2:
        _require_dims(b, 3, "[B, groups, N]", "B")
    else:
        _require_dims(b, 4, "[B, L, groups, N]", "B")
    groups = b[0][-2]
    _require_shape(A, (D, N), torch.float32, "A")
    for name, t in params:
        _require_shape(t, (D, N) if name == "dA" else (D,), torch.float32, name)
    _require_shape(b, lead + (groups, N), x[1], "B")
    _require_shape(c, b[0], x[1], "C")
    _require_shape(lengths, lead[:1], torch.int32, "slots" if op == 2 else "lengths")
    strides = {"x": _token_rows(x, "x"), "b": _group_rows(b, "B"), "c": _group_rows(c, "C")}
    for name, field, of, t in rows:
        if t is None:
            continue
        _require_shape(t, x[0] if of == "x" else b[0], x[1], name)
        strides[field] = _token_rows(t, name) if of == "x" else _group_rows(t, name)
    for name, t in states:
        _require_state(name, t, (lead[0], D, N), torch.float32, op == 2)
    g = make_scan_desc(lead[0], 1 if op == 2 else lead[1], D, N, _dtype_code(x[1]), groups,
                       softplus, **strides)
    _check(validate_scan_desc(g, op))
    return _Planned(g, 0 if op == 2 else scan_workspace_size(g, op == 1))


@_on_stream
def selective_scan(x, dt, A, B, C, D=None, z=None, dt_bias=None, softplus=True, lengths=None,
                   state_in=None, return_state=False, out=None, state_out=None, workspace=None,
                   stream=None):
    """Selective state space scan (favor_selective_scan): with s = softplus(dt + dt_bias),
    h_t = exp(s_t A) h_{t-1} + s_t x_t B_t and y_t = (C_t h_t + D x_t) silu(z_t).

    x, dt, z [B, L, D]: bfloat16 or float32, rows contiguous, any other strides; B, C
    [B, L, groups, N] of the same type (channel d reads group d / (D / groups)), N up to 256;
    D / groups a multiple of 8. A [D, N], D and dt_bias [D] float32; D, z and dt_bias may be
    left out, softplus=False takes s = dt + dt_bias. lengths [B] int32: tokens of each
    right-padded sequence. States [B, D, N] float32. Returns y [B, L, D] (contiguous unless
    given), or (y, state_out) when return_state is true.
    """
    torch = _torch()
    if out is None:
        out = torch.empty_like(x, memory_format=torch.contiguous_format)
    c = _scan_plan(0, _like(x), _like(A), (("D", _like(D)), ("dt_bias", _like(dt_bias))),
                   _like(B), _like(C),
                   (("dt", "dt", "x", _like(dt)), ("z", "z", "x", _like(z)),
                    ("out", "y", "x", _like(out))), _like(lengths),
                   (("state_in", _like(state_in)), ("state_out", _like(state_out))),
                   bool(softplus))
    if return_state and state_out is None:
        g = c.g
        state_out = torch.empty((g.B, g.D, g.N), dtype=torch.float32, device=x.device)
    here = _require_here(x, dt, A, B, C, D, z, dt_bias, lengths, out, state_in, state_out)
    _require_whole(A, D, dt_bias, lengths, state_in, state_out)
    ws, nbytes = _decay_workspace(c.workspace, workspace)
    _check(lib().favor_selective_scan(
        c.ref, _ptr(x), _ptr(dt), _ptr(A), _ptr(B), _ptr(C), _ptr(D), _ptr(z), _ptr(dt_bias),
        _ptr(lengths), _ptr(out), _ptr(state_in), _ptr(state_out), _ptr(ws), nbytes,
        _stream_on(here, stream)))
    return (out, state_out) if return_state else out


@_on_stream
def selective_scan_backward(x, dt, A, B, C, dout, D=None, z=None, dt_bias=None, softplus=True,
                            lengths=None, state_in=None, dstate_out=None,
                            return_state_grad=False, dx=None, ddt=None, dA=None, dB=None, dC=None,
                            dD=None, dz=None, ddt_bias=None, dstate_in=None, workspace=None,
                            stream=None):
    """Gradients of selective_scan (favor_selective_scan_backward) from dout and dstate_out
    (default zeros).

    Returns (dx, ddt, dA, dB, dC, dD, dz, ddt_bias), followed by dstate_in when
    return_state_grad is true; dD, dz and ddt_bias are None where D, z and dt_bias are.
    """
    torch = _torch()
    whole = torch.contiguous_format
    dx, ddt, dB, dC = (torch.empty_like(like, memory_format=whole) if t is None else t
                       for t, like in ((dx, x), (ddt, dt), (dB, B), (dC, C)))
    dA = torch.empty_like(A) if dA is None else dA
    dD, dz, ddt_bias = (None if like is None else
                        torch.empty_like(like, memory_format=whole) if t is None else t
                        for t, like in ((dD, D), (dz, z), (ddt_bias, dt_bias)))
    c = _scan_plan(1, _like(x), _like(A),
                   (("D", _like(D)), ("dt_bias", _like(dt_bias)), ("dA", _like(dA)),
                    ("dD", _like(dD)), ("ddt_bias", _like(ddt_bias))), _like(B), _like(C),
                   (("dt", "dt", "x", _like(dt)), ("z", "z", "x", _like(z)),
                    ("dout", "grad_y", "x", _like(dout)), ("dx", "grad_x", "x", _like(dx)),
                    ("ddt", "grad_dt", "x", _like(ddt)), ("dz", "grad_z", "x", _like(dz)),
                    ("dB", "grad_b", "b", _like(dB)), ("dC", "grad_c", "b", _like(dC))),
                   _like(lengths),
                   (("state_in", _like(state_in)), ("dstate_out", _like(dstate_out)),
                    ("dstate_in", _like(dstate_in))), bool(softplus))
    if return_state_grad and dstate_in is None:
        g = c.g
        dstate_in = torch.empty((g.B, g.D, g.N), dtype=torch.float32, device=x.device)
    here = _require_here(x, dt, A, B, C, D, z, dt_bias, lengths, state_in, dout, dstate_out, dx,
                         ddt, dA, dB, dC, dD, dz, ddt_bias, dstate_in)
    _require_whole(A, D, dt_bias, lengths, state_in, dstate_out, dA, dD, ddt_bias, dstate_in)
    ws, nbytes = _decay_workspace(c.workspace, workspace)
    _check(lib().favor_selective_scan_backward(
        c.ref, _ptr(x), _ptr(dt), _ptr(A), _ptr(B), _ptr(C), _ptr(D), _ptr(z), _ptr(dt_bias),
        _ptr(lengths), _ptr(state_in), _ptr(dout), _ptr(dstate_out), _ptr(dx), _ptr(ddt), _ptr(dA),
        _ptr(dB), _ptr(dC), _ptr(dD), _ptr(dz), _ptr(ddt_bias), _ptr(dstate_in), _ptr(ws), nbytes,
        _stream_on(here, stream)))
    grads = (dx, ddt, dA, dB, dC, dD, dz, ddt_bias)
    return grads + (dstate_in,) if return_state_grad else grads


@_on_stream
def selective_scan_step(x, dt, A, B, C, state, D=None, z=None, dt_bias=None, softplus=True,
                        slots=None, out=None, stream=None):
    """The next token of B sequences (favor_selective_scan_step): x, dt, z [B, D], B, C
    [B, groups, N], state [n, D, N] float32 updated in place; slots as for causal_conv_step.
    Returns y [B, D].
    """
    if out is None:
        out = _torch().empty_like(x, memory_format=_torch().contiguous_format)
    c = _scan_plan(2, _like(x), _like(A), (("D", _like(D)), ("dt_bias", _like(dt_bias))),
                   _like(B), _like(C),
                   (("dt", "dt", "x", _like(dt)), ("z", "z", "x", _like(z)),
                    ("out", "y", "x", _like(out))), _like(slots), (("state", _like(state)),),
                   bool(softplus))
    here = _require_here(x, dt, A, B, C, D, z, dt_bias, state, slots, out)
    _require_whole(A, D, dt_bias, state, slots)
    _check(lib().favor_selective_scan_step(
        c.ref, x.data_ptr(), dt.data_ptr(), A.data_ptr(), B.data_ptr(), C.data_ptr(), _ptr(D),
        _ptr(z), _ptr(dt_bias), _ptr(slots), state.shape[0], state.data_ptr(), out.data_ptr(),
        _stream_on(here, stream)))
    return out


# ----------------------------------------------------------------------------- beam search
@functools.lru_cache(maxsize=256)
def _beam_plan(logits, scores, ended, outs, n, end_token):
    torch = _torch()
    _require_dims(logits, 3, "[B, K, V]", "logits")
    B, K, V = logits[0]
    if V > 1 and logits[2][2] != 1:
        raise FavorError(1, "rows of logits must be contiguous")
    _require_shape(scores, (B, K), torch.float32, "scores")
    if ended is not None and (ended[0] != (B, K) or ended[1] not in (torch.bool, torch.uint8)):
        raise FavorError(1, f"ended must be {(B, K)} bool or uint8, got {tuple(ended[0])} "
                            f"{ended[1]}")
    for (name, t), dtype in zip(outs, (torch.float32, torch.int32, torch.int32)):
        _require_shape(t, (B, n), dtype, name)
    batch, beam = (logits[2][i] if logits[0][i] > 1 else V for i in range(2))
    if batch == 0 and beam == 0:
        raise FavorError(1, "logits is one row broadcast to all")
    g = make_beam_desc(B, K, V, n, _dtype_code(logits[1]), batch, beam, end_token)
    _check(validate_beam_desc(g))
    return _Planned(g, beam_workspace_size(g))


@_on_stream
def beam_select(logits, scores, n=None, ended=None, end_token=-1, out_scores=None, parent=None,
                token=None, workspace=None, stream=None):
    """The best n (default K) continuations of each entry's K beams (favor_beam_select) by
    scores[b, k] + log_softmax(logits[b, k])[v].

    logits [B, K, V] (bfloat16 or float32, V contiguous, any other strides and alignment),
    scores [B, K] float32. ended [B, K] (bool or uint8): beams that stay as they are, with
    end_token. Ties go to the lower beam and token. Returns (scores [B, n] float32 in falling
    order, parent [B, n] int32, token [B, n] int32); where fewer can be chosen the rest has
    the score -inf, parent 0 and end_token (0 without one).
    """
    torch = _torch()
    if n is None:
        n = logits.shape[1] if logits.dim() == 3 else 1
    n = operator.index(n)
    if logits.dim() == 3:
        shape, dev = (logits.shape[0], max(n, 0)), logits.device
        if out_scores is None:
            out_scores = torch.empty(shape, dtype=torch.float32, device=dev)
        if parent is None:
            parent = torch.empty(shape, dtype=torch.int32, device=dev)
        if token is None:
            token = torch.empty(shape, dtype=torch.int32, device=dev)
    c = _beam_plan(_like(logits), _like(scores), _like(ended),
                   (("out_scores", _like(out_scores)), ("parent", _like(parent)),
                    ("token", _like(token))), n, operator.index(end_token))
    here = _require_here(logits, scores, ended, out_scores, parent, token)
    _require_whole(scores, ended, out_scores, parent, token)
    ws, nbytes = _decay_workspace(c.workspace, workspace)
    _check(lib().favor_beam_select(c.ref, _ptr(logits), _ptr(scores), _ptr(ended),
                                   _ptr(out_scores), _ptr(parent), _ptr(token), _ptr(ws), nbytes,
                                   _stream_on(here, stream)))
    return out_scores, parent, token


@_on_stream
def beam_reorder(parent, slots, pools, new_slots=None, stream=None):
    """Moves the states of pools behind chosen beams, in place (favor_beam_reorder): beam j of
    entry b continues beam parent[b, j], whose state is at slots[b, parent[b, j]] of every pool
    (slots None: b K + the beam). A beam's first child keeps its place, the others get copies
    in the places of beams without children.

    parent, slots [B, K] int32 (the valid places all different), pools: contiguous tensors
    [n, ...] whose entries are multiples of 16 bytes, such as the states of attn_decay_step,
    causal_conv_step and selective_scan_step. Returns the new slots [B, K].
    """
    torch = _torch()
    if parent.dim() != 2:
        raise FavorError(1, f"parent must be [B, K], got {tuple(parent.shape)}")
    if new_slots is None:
        new_slots = torch.empty_like(parent, memory_format=torch.contiguous_format)
    for name, t in (("parent", parent), ("slots", slots), ("new_slots", new_slots)):
        _require_like(t, parent.shape, torch.int32, name)
    here = _require_here(parent, slots, new_slots, *pools)
    _require_whole(parent, slots, new_slots)
    table = (FavorBeamPool * len(pools))()
    for row, p in zip(table, pools):
        if p.dim() < 1 or not p.is_contiguous():
            raise FavorError(1, "pools must be contiguous tensors [n, ...]")
        n = p.shape[0]
        row.data, row.n_slots = p.data_ptr(), n
        row.bytes_per_slot = p.numel() // n * p.element_size() if n else 0
    _check(lib().favor_beam_reorder(parent.shape[0], parent.shape[1], _ptr(parent), _ptr(slots),
                                    _ptr(new_slots), table, len(pools), _stream_on(here, stream)))
    return new_slots
