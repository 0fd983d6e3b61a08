"""Torch-facing binding of librocs: argument marshalling only.

Each function checks shapes, dtypes and devices, allocates outputs (and the
linear's workspace) with torch when the caller does not pass them, and calls
the C entry point of the same name on the current HIP stream. Every step of
the computation runs in the library's kernels; there is no Python or CPU
fallback, and a missing library raises.

The extension module _binding does the same marshalling natively for the calls
that pass these checks (1 to 2 us instead of 14 to 19 us a call); it returns
None for all others, and the code here then raises the error or makes the call.
Where the module is missing or was built for another torch, the code here makes
every call, on the same kernels.
"""

import ctypes
import warnings

import torch

from . import _lib

__all__ = [
    "load_library", "ikbo_linear", "ikbo_linear_mapped", "glm_linear", "ikbo_linear_combined",
    "linear_workspace_size", "pad_dims",
    "dca_attention", "dca_attention_mapped", "dca_attention_mapped_workspace_size",
    "dca_request_attention", "glm_interaction",
    "ikbo_lcb", "ikbo_lcb_mapped", "ikbo_mlp2", "mlp2_workspace_size", "glm_fm_linear",
    "fm_linear_workspace_size", "request_ids",
    "validate_offsets", "RocsError",
    "history_attention", "paged_attention", "history_workspace_size", "cache_pool", "cache_reserve",
    "cache_write", "cache_fork", "cache_free", "cache_compact", "cache_copy", "cache_check",
    "cache_workspace_size",
    "adapter_linear", "adapter_workspace_size", "rotate", "cache_append", "cache_pool_fp4",
    "fp4_row_bytes", "cache_read_fp4", "paged_attention_fp4", "paged_fp4_workspace_size",
]

RocsError = _lib.RocsError
_ACT = {"none": _lib.ACT_NONE, None: _lib.ACT_NONE, "relu": _lib.ACT_RELU}


def load_library():
    return _lib.load()


_binding = None


class _PythonPath:
    """In the place of the _binding module: takes no call."""

    def _none(*args):
        return None

    linear = glm_linear = mlp2 = fm_linear = lcb = plan = attention = _none
    history = paged = cache_reserve = cache_write = cache_fork = cache_free = cache_compact = _none
    adapter = append = paged_fp4 = rotate = read_fp4 = _none


def _native():
    """The _binding module, loaded (with librocs) on first use."""
    global _binding
    if _binding is None:
        _lib.load()
        try:
            from . import _binding as mod
        except ImportError as e:
            warnings.warn("the native call path (_binding.so) is missing or does not load: calls "
                          "cost 12 to 17 us more on the host; build it with `python -c 'import "
                          f"__graft_entry__ as g; g.build()'`: {e}", RuntimeWarning, stacklevel=3)
            mod = _PythonPath()
        _binding = mod
    return _binding


def _dtype_code(t):
    if t.dtype == torch.bfloat16:
        return _lib.DTYPE_BF16
    if t.dtype == torch.float32:
        return _lib.DTYPE_F32
    raise TypeError(f"unsupported dtype {t.dtype} (bfloat16 or float32)")


def _ptr(t):
    return None if t is None else ctypes.c_void_p(t.data_ptr())


def _stream(stream):
    s = torch.cuda.current_stream() if stream is None else stream
    return ctypes.c_void_p(s.cuda_stream)


def _need(cond, msg):
    if not cond:
        raise ValueError(msg)


def _new(shape, dtype, device, stream, scratch=False):
    """A tensor for a call on `stream`. The allocator hands freed memory on in
    the order of the stream that it was allocated under, so for a call on
    another stream than the current one it comes from that stream's memory: the
    kernels run after its earlier uses, and a workspace (scratch) goes back
    after them. An output is also marked as used on the current stream, where
    its owner may read and free it."""
    if stream is not None and device.type == "cuda":
        current = torch.cuda.current_stream(device)
        if stream.cuda_stream != current.cuda_stream:
            if not isinstance(stream, torch.cuda.Stream):
                stream = (torch.cuda.ExternalStream(stream.cuda_stream, device)
                          if stream.cuda_stream else torch.cuda.default_stream(device))
            with torch.cuda.stream(stream):
                t = torch.empty(shape, dtype=dtype, device=device)
            if not scratch:
                t.record_stream(current)
            return t
    return torch.empty(shape, dtype=dtype, device=device)


def _on_gpu(*ts):
    dev = None
    for t in ts:
        if t is None:
            continue
        _need(t.is_cuda, "all tensors must be on the GPU")
        dev = t.device if dev is None else dev
        _need(t.device == dev, "all tensors must be on the same GPU")


def _offsets(off, n_req):
    _need(off.dtype == torch.int32 and off.dim() == 1 and off.is_contiguous(),
          "offsets must be a contiguous 1-D int32 tensor")
    _need(off.numel() == n_req + 1, f"offsets need {n_req + 1} entries, got {off.numel()}")


def _request_map(ids, n_cand):
    _need(ids.dtype == torch.int32 and ids.dim() == 1 and ids.is_contiguous(),
          "cand_request_ids must be a contiguous 1-D int32 tensor")
    _need(ids.numel() == n_cand, f"cand_request_ids needs {n_cand} entries, got {ids.numel()}")


def linear_workspace_size(num_requests, num_cand, d_out, k_req):
    return int(_lib.load().rocs_ikbo_linear_workspace_size(num_requests, num_cand, d_out, k_req))


def ikbo_linear(x_cand, w_cand, *, x_req=None, w_req=None, cand_offsets=None, bias=None,
                activation="none", x_cand_add=None, out=None, workspace=None, stream=None):
    """out[n] = act(w_cand @ xc[n] + w_req @ x_req[m_n] + bias), xc = x_cand (+ x_cand_add).

    x_cand [N, K_c], w_cand [D, K_c], x_req [R, K_r], w_req [D, K_r] (paper's [out, in]
    orientation), cand_offsets [R + 1] int32, bias [D] float32.
    """
    done = (_binding or _native()).linear(x_cand, w_cand, x_req, w_req, cand_offsets, False, bias,
                                          activation, x_cand_add, out, workspace, stream)
    if done is not None:
        return done
    return _linear(x_cand, w_cand, x_req, w_req, cand_offsets, None, None, bias, activation,
                   x_cand_add, out, workspace, stream)


def ikbo_linear_mapped(x_cand, w_cand, *, x_req=None, w_req=None, cand_request_ids=None,
                       bias=None, activation="none", x_cand_add=None, out=None,
                       workspace=None, stream=None):
    """rocs_ikbo_linear_mapped: as ikbo_linear, with m given per candidate
    (cand_request_ids int32 [N], each in [0, R) with R = x_req.shape[0])."""
    done = (_binding or _native()).linear(x_cand, w_cand, x_req, w_req, cand_request_ids, True,
                                          bias, activation, x_cand_add, out, workspace, stream)
    if done is not None:
        return done
    return _linear(x_cand, w_cand, x_req, w_req, None, cand_request_ids, True, bias,
                   activation, x_cand_add, out, workspace, stream)


def pad_dims(x, w, multiple=64):
    """The memory-alignment transform (Section 4.2.4): zero-pad the reduction
    width K of an activation x [rows, K] and of its weight w [D, K] up to a
    multiple of `multiple`. The added columns are zero on both sides, so
    x @ w.T is unchanged; the padded shapes reach the aligned kernels (K a
    multiple of 64 for the streaming candidate GEMM, 8 for the request GEMM).
    Layout only: returns (x, w) unchanged when K is already a multiple, else
    zero-padded copies (pad weights once, ahead of the calls that use them)."""
    _need(x.dim() == 2 and w.dim() == 2 and x.shape[1] == w.shape[1],
          "x [rows, K] and w [D, K] expected")
    _need(multiple >= 1, "multiple must be positive")
    k = x.shape[1]
    pad = (-k) % multiple
    if pad == 0:
        return x, w
    xp = torch.zeros((x.shape[0], k + pad), dtype=x.dtype, device=x.device)
    wp = torch.zeros((w.shape[0], k + pad), dtype=w.dtype, device=w.device)
    xp[:, :k] = x
    wp[:, :k] = w
    return xp, wp


def ikbo_linear_combined(x_req, x_cand, w_cr, w_cc, cand_offsets, *, w_rr=None, b_req=None,
                         b_cand=None, activation="none", x_cand_add=None, y_req=None,
                         y_cand=None, workspace=None, stream=None):
    """rocs_ikbo_linear_combined: the request-side GEMM and the candidate GEMM in
    one launch (Section 4.2.3). Returns (y_req or None, y_cand); y_req =
    act(W_RR x^R + b^R) when w_rr is given. Results equal glm_linear /
    ikbo_linear bit for bit."""
    lib = _lib.load()
    _need(x_req is not None and x_req.dim() == 2, "x_req must be [R, k_req]")
    n_req, k_req = x_req.shape
    side = None
    if w_rr is not None:
        _need(w_rr.dim() == 2 and w_rr.shape[1] == k_req, "w_rr must be [d_req, k_req]")
        d_req = w_rr.shape[0]
        _need(w_rr.dtype == x_req.dtype and w_rr.is_contiguous(), "w_rr must match x_req")
        if b_req is not None:
            _need(b_req.dtype == torch.float32 and b_req.shape == (d_req,) and
                  b_req.is_contiguous(), "b_req must be contiguous float32 [d_req]")
        if y_req is None:
            y_req = _new((n_req, d_req), x_req.dtype, x_req.device, stream)
        _need(y_req.shape == (n_req, d_req) and y_req.dtype == x_req.dtype and
              y_req.is_contiguous(), "y_req must be a contiguous [R, d_req] tensor")
        _on_gpu(w_rr, b_req, y_req)
        side = (w_rr, b_req, y_req, d_req, lib)
    y_cand = _linear(x_cand, w_cc, x_req, w_cr, cand_offsets, None, None, b_cand, activation,
                     x_cand_add, y_cand, workspace, stream, request_side=side, combined=True)
    return y_req, y_cand


def glm_linear(x_req, x_cand, w_rr, w_cr, w_cc, cand_offsets, *, b_req=None, b_cand=None,
               activation="none", x_cand_add=None, y_req=None, y_cand=None, workspace=None,
               stream=None):
    """Both outputs of a two-group GLM linear (Eq. glm-linear): returns
    (y_req [R, d_req] = act(W_RR x^R + b^R), y_cand [N, d_cand] = act(W_CR x^R_m + W_CC x^C + b^C))."""
    done = (_binding or _native()).glm_linear(x_req, x_cand, w_rr, w_cr, w_cc, cand_offsets, b_req,
                                              b_cand, activation, x_cand_add, y_req, y_cand,
                                              workspace, stream)
    if done is not None:
        return done
    lib = _lib.load()
    _need(x_req is not None and x_req.dim() == 2, "x_req must be [R, k_req]")
    n_req, k_req = x_req.shape
    _need(w_rr.dim() == 2 and w_rr.shape[1] == k_req, "w_rr must be [d_req, k_req]")
    d_req = w_rr.shape[0]
    _need(w_rr.dtype == x_req.dtype and w_rr.is_contiguous(), "w_rr must match x_req")
    if b_req is not None:
        _need(b_req.dtype == torch.float32 and b_req.shape == (d_req,) and b_req.is_contiguous(),
              "b_req must be contiguous float32 [d_req]")
    if y_req is None:
        y_req = _new((n_req, d_req), x_req.dtype, x_req.device, stream)
    _need(y_req.shape == (n_req, d_req) and y_req.dtype == x_req.dtype and y_req.is_contiguous(),
          "y_req must be a contiguous [R, d_req] tensor")
    _on_gpu(x_req, w_rr, b_req, y_req)
    y_cand = _linear(x_cand, w_cc, x_req, w_cr, cand_offsets, None, None, b_cand, activation,
                     x_cand_add, y_cand, workspace, stream,
                     request_side=(w_rr, b_req, y_req, d_req, lib))
    return y_req, y_cand


def _linear(x_cand, w_cand, x_req, w_req, cand_offsets, cand_ids, mapped, bias, activation,
            x_cand_add, out, workspace, stream, request_side=None, combined=False):
    lib = _lib.load()
    _need(x_cand.dim() == 2 and w_cand.dim() == 2, "x_cand and w_cand must be 2-D")
    n_cand, k_cand = x_cand.shape
    d_out = w_cand.shape[0]
    _need(w_cand.shape[1] == k_cand, "w_cand must be [d_out, k_cand]")
    code = _dtype_code(x_cand)
    for t in (w_cand, x_req, w_req, x_cand_add):
        _need(t is None or t.dtype == x_cand.dtype, "inputs must share one dtype")
    index = cand_ids if mapped else cand_offsets
    if x_req is not None:
        _need(w_req is not None and index is not None,
              "x_req needs w_req and " + ("cand_request_ids" if mapped else "cand_offsets"))
        _need(x_req.dim() == 2 and w_req.dim() == 2, "x_req and w_req must be 2-D")
        n_req, k_req = x_req.shape
        _need(w_req.shape == (d_out, k_req), "w_req must be [d_out, k_req]")
    else:
        k_req = 0
        n_req = 0 if mapped or cand_offsets is None else cand_offsets.numel() - 1
    if mapped:
        if cand_ids is not None:
            _request_map(cand_ids, n_cand)
    elif cand_offsets is not None:
        _offsets(cand_offsets, n_req)
    if x_cand_add is not None:
        _need(x_cand_add.shape == x_cand.shape, "x_cand_add must match x_cand")
    if bias is not None:
        _need(bias.dtype == torch.float32 and bias.shape == (d_out,), "bias must be float32 [d_out]")
    for t in (x_cand, w_cand, x_req, w_req, x_cand_add, bias):
        _need(t is None or t.is_contiguous(), "tensors must be contiguous")
    if out is None:
        out = _new((n_cand, d_out), x_cand.dtype, x_cand.device, stream)
    _need(out.shape == (n_cand, d_out) and out.dtype == x_cand.dtype and out.is_contiguous(),
          "out must be a contiguous [N, d_out] tensor of the input dtype")
    need = int(lib.rocs_ikbo_linear_workspace_size(n_req, n_cand, d_out, k_req))
    if workspace is None and need > 0:
        workspace = _new(need, torch.uint8, x_cand.device, stream, scratch=True)
    _on_gpu(x_cand, w_cand, x_req, w_req, index, bias, x_cand_add, out, workspace)
    _need(activation in _ACT, f"activation must be one of {sorted(k for k in _ACT if k)}")
    ws_bytes = 0 if workspace is None else workspace.numel() * workspace.element_size()
    if combined:
        w_rr, b_req, y_req, d_req = (request_side or (None, None, None, 0, None))[:4]
        _lib.check(lib.rocs_ikbo_linear_combined(
            _ptr(x_req), k_req, _ptr(x_cand), _ptr(x_cand_add), k_cand, _ptr(w_rr), _ptr(w_req),
            _ptr(w_cand), _ptr(b_req), _ptr(bias), _ptr(cand_offsets), n_req, n_cand, d_req,
            d_out, code, _ACT[activation], _ptr(y_req), _ptr(out), _ptr(workspace), ws_bytes,
            _stream(stream)), "rocs_ikbo_linear_combined")
        return out
    if request_side is not None:
        w_rr, b_req, y_req, d_req, _ = request_side
        _lib.check(lib.rocs_glm_linear(
            _ptr(x_req), k_req, _ptr(x_cand), _ptr(x_cand_add), k_cand, _ptr(w_rr), _ptr(w_req),
            _ptr(w_cand), _ptr(b_req), _ptr(bias), _ptr(cand_offsets), n_req, n_cand, d_req,
            d_out, code, _ACT[activation], _ptr(y_req), _ptr(out), _ptr(workspace), ws_bytes,
            _stream(stream)), "rocs_glm_linear")
        return out
    fn, name = ((lib.rocs_ikbo_linear_mapped, "rocs_ikbo_linear_mapped") if mapped
                else (lib.rocs_ikbo_linear, "rocs_ikbo_linear"))
    _lib.check(fn(
        _ptr(x_req), k_req, _ptr(x_cand), _ptr(x_cand_add), k_cand, _ptr(w_req), _ptr(w_cand),
        _ptr(bias), _ptr(index), n_req, n_cand, d_out, code, _ACT[activation],
        _ptr(out), _ptr(workspace), ws_bytes, _stream(stream)), name)
    return out


def mlp2_workspace_size(num_requests, num_cand, k_req, k_cand, d_hidden, d_out, dtype):
    code = _lib.DTYPE_BF16 if dtype == torch.bfloat16 else _lib.DTYPE_F32
    return int(_lib.load().rocs_ikbo_mlp2_workspace_size(num_requests, num_cand, k_req, k_cand,
                                                          d_hidden, d_out, code))


def ikbo_mlp2(x_cand, w1_cand, w2, *, x_req=None, w1_req=None, cand_offsets=None, b1=None,
              b2=None, activation1="relu", activation2="none", out=None, workspace=None,
              stream=None):
    """rocs_ikbo_mlp2: out[n] = act2(w2 @ H[n] + b2), H[n] = act1(w1_cand @ x_cand[n] +
    w1_req @ x_req[m_n] + b1) rounded to the input dtype; H stays on chip on the fused path.

    x_cand [N, K_c], w1_cand [D_h, K_c], w2 [D_o, D_h], x_req [R, K_r], w1_req [D_h, K_r],
    cand_offsets [R + 1] int32, b1 [D_h] and b2 [D_o] float32.
    """
    done = (_binding or _native()).mlp2(x_cand, w1_cand, w2, x_req, w1_req, cand_offsets, b1, b2,
                                        activation1, activation2, out, workspace, stream)
    if done is not None:
        return done
    lib = _lib.load()
    _need(x_cand.dim() == 2 and w1_cand.dim() == 2 and w2.dim() == 2, "2-D operands expected")
    n_cand, k_cand = x_cand.shape
    d_hidden = w1_cand.shape[0]
    _need(w1_cand.shape[1] == k_cand, "w1_cand must be [d_hidden, k_cand]")
    _need(w2.shape[1] == d_hidden, "w2 must be [d_out, d_hidden]")
    d_out = w2.shape[0]
    code = _dtype_code(x_cand)
    for t in (w1_cand, w2, x_req, w1_req):
        _need(t is None or t.dtype == x_cand.dtype, "inputs must share one dtype")
    if x_req is not None:
        _need(w1_req is not None and cand_offsets is not None,
              "x_req needs w1_req and cand_offsets")
        _need(x_req.dim() == 2 and w1_req.dim() == 2, "x_req and w1_req must be 2-D")
        n_req, k_req = x_req.shape
        _need(w1_req.shape == (d_hidden, k_req), "w1_req must be [d_hidden, k_req]")
        _offsets(cand_offsets, n_req)
    else:
        n_req, k_req = 0, 0
    for b, n, name in ((b1, d_hidden, "b1"), (b2, d_out, "b2")):
        if b is not None:
            _need(b.dtype == torch.float32 and b.shape == (n,), f"{name} must be float32 [{n}]")
    for t in (x_cand, w1_cand, w2, x_req, w1_req, b1, b2):
        _need(t is None or t.is_contiguous(), "tensors must be contiguous")
    if out is None:
        out = _new((n_cand, d_out), x_cand.dtype, x_cand.device, stream)
    _need(out.shape == (n_cand, d_out) and out.dtype == x_cand.dtype and out.is_contiguous(),
          "out must be a contiguous [N, d_out] tensor of the input dtype")
    need = int(lib.rocs_ikbo_mlp2_workspace_size(n_req, n_cand, k_req, k_cand, d_hidden, d_out,
                                                 code))
    if workspace is None and need > 0:
        workspace = _new(need, torch.uint8, x_cand.device, stream, scratch=True)
    _on_gpu(x_cand, w1_cand, w2, x_req, w1_req, cand_offsets, b1, b2, out, workspace)
    for a in (activation1, activation2):
        _need(a in _ACT, f"activation must be one of {sorted(k for k in _ACT if k)}")
    ws_bytes = 0 if workspace is None else workspace.numel() * workspace.element_size()
    _lib.check(lib.rocs_ikbo_mlp2(
        _ptr(x_req), k_req, _ptr(x_cand), k_cand, _ptr(w1_req), _ptr(w1_cand), _ptr(b1), _ptr(w2),
        _ptr(b2), _ptr(cand_offsets), n_req, n_cand, d_hidden, d_out, code, _ACT[activation1],
        _ACT[activation2], _ptr(out), _ptr(workspace), ws_bytes, _stream(stream)),
        "rocs_ikbo_mlp2")
    return out


def fm_linear_workspace_size(num_requests, num_cand, f_req, f_cand, emb_dim, d_out, dtype):
    code = _lib.DTYPE_BF16 if dtype == torch.bfloat16 else _lib.DTYPE_F32
    return int(_lib.load().rocs_glm_fm_linear_workspace_size(num_requests, num_cand, f_req,
                                                              f_cand, emb_dim, d_out, code))


def glm_fm_linear(x_req, x_cand, cand_offsets, w_req, w_cand, *, bias=None, activation="relu",
                  out=None, workspace=None, stream=None):
    """rocs_glm_fm_linear: out[n] = act(w_req @ vec(Y^R[m_n]) + w_cand @ vec(Y^C[n]) + bias)
    with Y^R, Y^C the GLM FM interaction of x_req [R, F_r, E] and x_cand [N, F_c, E].
    w_req [D, F_r^2], w_cand [D, F_c (F_r + F_c)], bias [D] float32. Returns out [N, D];
    the workspace then holds Y^R at its start."""
    done = (_binding or _native()).fm_linear(x_req, x_cand, cand_offsets, w_req, w_cand, bias,
                                             activation, out, workspace, stream)
    if done is not None:
        return done
    lib = _lib.load()
    _need(x_req.dim() == 3 and x_cand.dim() == 3 and x_req.shape[2] == x_cand.shape[2],
          "x_req [R, F_r, E] and x_cand [N, F_c, E] expected")
    n_req, f_req, emb = x_req.shape
    n_cand, f_cand = x_cand.shape[0], x_cand.shape[1]
    _offsets(cand_offsets, n_req)
    d_out = w_cand.shape[0]
    _need(w_req.shape == (d_out, f_req * f_req), "w_req must be [d_out, f_req^2]")
    _need(w_cand.shape == (d_out, f_cand * (f_req + f_cand)),
          "w_cand must be [d_out, f_cand (f_req + f_cand)]")
    code = _dtype_code(x_cand)
    for t in (x_req, w_req, w_cand):
        _need(t.dtype == x_cand.dtype, "inputs must share one dtype")
    if bias is not None:
        _need(bias.dtype == torch.float32 and bias.shape == (d_out,), "bias must be float32 [d_out]")
    for t in (x_req, x_cand, w_req, w_cand, bias):
        _need(t is None or t.is_contiguous(), "tensors must be contiguous")
    if out is None:
        out = _new((n_cand, d_out), x_cand.dtype, x_cand.device, stream)
    _need(out.shape == (n_cand, d_out) and out.dtype == x_cand.dtype and out.is_contiguous(),
          "out must be a contiguous [N, d_out] tensor of the input dtype")
    need = int(lib.rocs_glm_fm_linear_workspace_size(n_req, n_cand, f_req, f_cand, emb, d_out,
                                                     code))
    if workspace is None and need > 0:
        workspace = _new(need, torch.uint8, x_cand.device, stream, scratch=True)
    _on_gpu(x_req, x_cand, cand_offsets, w_req, w_cand, bias, out, workspace)
    _need(activation in _ACT, f"activation must be one of {sorted(k for k in _ACT if k)}")
    ws_bytes = 0 if workspace is None else workspace.numel() * workspace.element_size()
    _lib.check(lib.rocs_glm_fm_linear(
        _ptr(x_req), _ptr(x_cand), _ptr(cand_offsets), n_req, n_cand, f_req, f_cand, emb,
        _ptr(w_req), _ptr(w_cand), _ptr(bias), d_out, code, _ACT[activation], _ptr(out),
        _ptr(workspace), ws_bytes, _stream(stream)), "rocs_glm_fm_linear")
    return out


def dca_attention(q, k, v, cand_offsets, kv_offsets, *, scale=None, out=None, stream=None):
    """Candidate-side DCA: q [N, T, H, d]; k, v [L_total, H, d] (rows may be strided,
    e.g. column slices of one [L, 2 H d] projection); offsets int32 [R + 1]."""
    return _attention(q, k, v, cand_offsets, None, kv_offsets, scale, out, stream)


def dca_attention_residual(q, k, v, cand_offsets, kv_offsets, residual, *, scale=None, out=None,
                           out_sum=None, stream=None):
    """dca_attention plus the stacked-DCA residual: returns (out, out_sum) with
    out_sum = round(out + residual) formed in the kernel's epilogue; residual has
    q's shape [N, T, H, d]."""
    return _attention(q, k, v, cand_offsets, None, kv_offsets, scale, out, stream,
                      residual=residual, out_sum=out_sum)


def dca_attention_plan_size(num_requests):
    return int(_lib.load().rocs_dca_attention_plan_size(num_requests))


def dca_attention_plan(cand_offsets, kv_offsets, *, num_cand, heads, q_len=1, plan=None,
                       stream=None):
    """rocs_dca_attention_plan: the tiled attention's tile order for these offsets
    (longest history first), into `plan` (uint8 device tensor, allocated here when
    not given). One plan serves every attention call over the same offsets."""
    done = (_binding or _native()).plan(cand_offsets, kv_offsets, num_cand, heads, q_len, plan,
                                        stream)
    if done is not None:
        return done
    lib = _lib.load()
    n_req = kv_offsets.numel() - 1
    _offsets(kv_offsets, n_req)
    _offsets(cand_offsets, n_req)
    need = dca_attention_plan_size(n_req)
    if plan is None:
        plan = _new(need, torch.uint8, kv_offsets.device, stream)
    _need(plan.dtype == torch.uint8 and plan.is_contiguous() and plan.numel() >= need,
          f"plan must be a contiguous uint8 tensor of at least {need} bytes")
    _on_gpu(cand_offsets, kv_offsets, plan)
    _lib.check(lib.rocs_dca_attention_plan(_ptr(cand_offsets), _ptr(kv_offsets), n_req,
                                           num_cand, q_len, heads, _ptr(plan), plan.numel(),
                                           _stream(stream)), "rocs_dca_attention_plan")
    return plan


def dca_attention_ex(q, k, v, cand_offsets, kv_offsets, *, w_q=None, heads=None, plan=None,
                     residual=None, scale=None, out=None, out_sum=None, stream=None):
    """rocs_dca_attention_ex. Without w_q, q is the query [N, T, H, d]; with w_q
    [heads * d, d_in], q holds x [N, T, d_in] and the kernel projects it
    (q = x @ w_q^T viewed as [N, T, heads, d]). `plan` (from dca_attention_plan)
    orders the tiles. Returns out, or (out, out_sum) when `residual` is given
    (out_sum = round(out + residual))."""
    done = (_binding or _native()).attention(q, w_q, heads, k, v, cand_offsets, None, kv_offsets,
                                             plan, residual, scale, out, out_sum, None, stream,
                                             True)
    if done is not None:
        return done
    lib = _lib.load()
    if w_q is None:
        _need(q.dim() == 4 and q.is_contiguous(), "q must be a contiguous [N, T, H, d] tensor")
        n_cand, q_len, heads, dim = q.shape
        d_in = 0
    else:
        _need(q.dim() == 3 and q.is_contiguous(), "x must be a contiguous [N, T, d_in] tensor")
        _need(heads is not None, "heads is required with w_q")
        n_cand, q_len, d_in = q.shape
        _need(w_q.dim() == 2 and w_q.is_contiguous() and w_q.shape[1] == d_in
              and w_q.shape[0] % heads == 0, "w_q must be a contiguous [heads * d, d_in] tensor")
        _need(w_q.dtype == q.dtype, "x and w_q must share one dtype")
        dim = w_q.shape[0] // heads
    _need(k.dim() == 3 and v.dim() == 3 and k.shape == v.shape and k.shape[1:] == (heads, dim),
          "k and v must be [L, heads, d]")
    _need(k.stride(2) == 1 and k.stride(1) == dim and v.stride(2) == 1 and v.stride(1) == dim,
          "k/v rows must be dense [H, d] blocks")
    _need(k.stride(0) == v.stride(0), "k and v must share a row stride")
    for t in (k, v):
        _need(t.dtype == q.dtype, "q (or x), k, v must share one dtype")
    n_req = kv_offsets.numel() - 1
    _offsets(kv_offsets, n_req)
    _offsets(cand_offsets, n_req)
    shape = (n_cand, q_len, heads, dim)
    if out is None:
        out = _new(shape, q.dtype, q.device, stream)
    _need(tuple(out.shape) == shape and out.dtype == q.dtype and out.is_contiguous(),
          "out must be [N, T, heads, d] of q's dtype")
    if residual is not None:
        _need(tuple(residual.shape) == shape and residual.dtype == q.dtype and
              residual.is_contiguous(), "residual must be a contiguous [N, T, heads, d] tensor")
        if out_sum is None:
            out_sum = _new(shape, q.dtype, q.device, stream)
        _need(out_sum.shape == out.shape and out_sum.dtype == out.dtype and
              out_sum.is_contiguous(), "out_sum must match out")
    if plan is not None:
        _need(plan.dtype == torch.uint8 and plan.is_contiguous(), "plan must be a uint8 tensor")
    _on_gpu(q, w_q, k, v, cand_offsets, kv_offsets, out, residual, out_sum, plan)
    stride = k.stride(0) if k.shape[0] > 1 else heads * dim
    _lib.check(lib.rocs_dca_attention_ex(
        _ptr(q), d_in, _ptr(w_q), _ptr(k), _ptr(v), _ptr(cand_offsets), _ptr(kv_offsets),
        _ptr(plan), plan.numel() if plan is not None else 0, n_req, n_cand, q_len, heads, dim,
        stride, float(scale or 0.0), _dtype_code(q), _ptr(residual), _ptr(out),
        _ptr(out_sum) if residual is not None else None, _stream(stream)),
        "rocs_dca_attention_ex")
    return (out, out_sum) if residual is not None else out


def dca_attention_proj(x, w_q, k, v, cand_offsets, kv_offsets, *, heads, residual=None,
                       plan=None, scale=None, out=None, out_sum=None, stream=None):
    """DCA with the candidate queries projected in the kernel: q = x @ w_q^T viewed as
    [N, T, heads, d] (x [N, T, d_in], w_q [heads * d, d_in]). Returns out, or
    (out, out_sum) when `residual` is given (out_sum = round(out + residual))."""
    _need(w_q is not None, "w_q is required")
    return dca_attention_ex(x, k, v, cand_offsets, kv_offsets, w_q=w_q, heads=heads, plan=plan,
                            residual=residual, scale=scale, out=out, out_sum=out_sum,
                            stream=stream)


def dca_attention_mapped_workspace_size(num_requests, num_cand):
    return int(_lib.load().rocs_dca_attention_mapped_workspace_size(num_requests, num_cand))


def dca_attention_mapped(q, k, v, cand_request_ids, kv_offsets, *, scale=None, out=None,
                         workspace=None, stream=None):
    """rocs_dca_attention_mapped: as dca_attention, with m given per candidate
    (cand_request_ids int32 [N], each in [0, R) with R = kv_offsets.numel() - 1).
    The workspace (allocated here when not given) receives the grouping of the
    candidates by request: grp_off [R + 1] int32 at offset 0, then order [N]
    int32 at the next 256-byte boundary."""
    return _attention(q, k, v, None, cand_request_ids, kv_offsets, scale, out, stream,
                      workspace=workspace)


def dca_request_attention(q_req, k, v, kv_offsets, *, scale=None, out=None, stream=None):
    """Request-side cross attention A^R = Attn(Q^R, K, V) (Eq. dca-attention): request r's
    queries q_req[r] [T, H, d] attend over r's own history. The identity map (request r is
    its own single "candidate") on rocs_dca_attention; the offsets are built on the device."""
    _need(q_req.dim() == 4, "q_req must be [R, T, H, d]")
    n_req = q_req.shape[0]
    _need(kv_offsets.numel() == n_req + 1, "kv_offsets needs R + 1 entries")
    return _attention(q_req, k, v, _identity_offsets(n_req, q_req.device, stream), None, kv_offsets,
                      scale, out, stream)


_IDENTITY = {}       # (power of two, device): [0, 1, ..]
_IDENTITY_VIEWS = {}  # (R, device): its first R + 1 entries; a slice costs 1 us


def _identity_offsets(n_req, device, stream):
    """[0, 1, ..., R] int32 on the device: the front of an array built once per
    (power of two, device), complete before any stream reads it. Under capture
    an array that is not there yet becomes part of the graph instead, which
    fills it on every replay."""
    view = _IDENTITY_VIEWS.get((n_req, device))
    if view is not None:
        return view
    key = (1 << max(n_req + 1, 1024).bit_length(), device)
    if key not in _IDENTITY:
        if device.type == "cuda" and torch.cuda.is_current_stream_capturing():
            t = _new(n_req + 1, torch.int32, device, stream, scratch=True)
            with torch.cuda.stream(stream):
                return torch.arange(n_req + 1, dtype=torch.int32, device=device, out=t)
        t = torch.arange(key[0], dtype=torch.int32, device=device)
        if t.is_cuda:
            torch.cuda.current_stream(device).synchronize()
        _IDENTITY[key] = t
    if len(_IDENTITY_VIEWS) >= 1024:
        _IDENTITY_VIEWS.clear()
    view = _IDENTITY_VIEWS[n_req, device] = _IDENTITY[key][:n_req + 1]
    return view


def _attention(q, k, v, cand_offsets, cand_ids, kv_offsets, scale, out, stream, workspace=None,
               residual=None, out_sum=None):
    done = (_binding or _native()).attention(q, None, None, k, v, cand_offsets, cand_ids,
                                             kv_offsets, None, residual, scale, out, out_sum,
                                             workspace, stream, False)
    if done is not None:
        return done
    lib = _lib.load()
    mapped = cand_ids is not None
    _need(q.dim() == 4 and q.is_contiguous(), "q must be a contiguous [N, T, H, d] tensor")
    n_cand, q_len, heads, dim = q.shape
    _need(k.dim() == 3 and v.dim() == 3 and k.shape == v.shape, "k and v must be [L, H, d]")
    _need(k.shape[1:] == (heads, dim), "k/v heads and head_dim must match q")
    _need(k.stride(2) == 1 and k.stride(1) == dim and v.stride(2) == 1 and v.stride(1) == dim,
          "k/v rows must be dense [H, d] blocks")
    _need(k.stride(0) == v.stride(0), "k and v must share a row stride")
    for t in (k, v):
        _need(t.dtype == q.dtype, "q, k, v must share one dtype")
    n_req = kv_offsets.numel() - 1
    _offsets(kv_offsets, n_req)
    if mapped:
        _request_map(cand_ids, n_cand)
    else:
        _offsets(cand_offsets, n_req)
    if out is None:
        out = _new(q.shape, q.dtype, q.device, stream)
    _need(out.shape == q.shape and out.dtype == q.dtype and out.is_contiguous(),
          "out must match q")
    _on_gpu(q, k, v, cand_offsets, cand_ids, kv_offsets, out)
    stride = k.stride(0) if k.shape[0] > 1 else heads * dim
    if residual is not None:
        _need(residual.shape == q.shape and residual.dtype == q.dtype and
              residual.is_contiguous(), "residual must be a contiguous tensor shaped like q")
        if out_sum is None:
            out_sum = _new(q.shape, q.dtype, q.device, stream)
        _need(out_sum.shape == q.shape and out_sum.dtype == q.dtype and out_sum.is_contiguous(),
              "out_sum must match q")
        _on_gpu(residual, out_sum)
        _lib.check(lib.rocs_dca_attention_residual(
            _ptr(q), _ptr(k), _ptr(v), _ptr(cand_offsets), _ptr(kv_offsets), n_req, n_cand,
            q_len, heads, dim, stride, float(scale or 0.0), _dtype_code(q), _ptr(residual),
            _ptr(out), _ptr(out_sum), _stream(stream)), "rocs_dca_attention_residual")
        return out, out_sum
    if mapped:
        need = int(lib.rocs_dca_attention_mapped_workspace_size(n_req, n_cand))
        if workspace is None and need > 0:
            workspace = _new(need, torch.uint8, q.device, stream, scratch=True)
        _on_gpu(workspace)
        ws_bytes = 0 if workspace is None else workspace.numel() * workspace.element_size()
        _lib.check(lib.rocs_dca_attention_mapped(
            _ptr(q), _ptr(k), _ptr(v), _ptr(cand_ids), _ptr(kv_offsets), n_req, n_cand, q_len,
            heads, dim, stride, float(scale or 0.0), _dtype_code(q), _ptr(out), _ptr(workspace),
            ws_bytes, _stream(stream)), "rocs_dca_attention_mapped")
        return out
    _lib.check(lib.rocs_dca_attention(
        _ptr(q), _ptr(k), _ptr(v), _ptr(cand_offsets), _ptr(kv_offsets), n_req, n_cand, q_len,
        heads, dim, stride, float(scale or 0.0), _dtype_code(q), _ptr(out), _stream(stream)),
        "rocs_dca_attention")
    return out


def glm_interaction(x_req, x_cand, cand_offsets, *, request_side=True, candidate_side=True,
                    y_req=None, y_cand=None, stream=None):
    """GLM FM: returns (y_req [R, F_r^2] or None, y_cand [N, F_c (F_r + F_c)] or None)."""
    lib = _lib.load()
    _need(x_req.dim() == 3 and x_cand.dim() == 3, "x_req / x_cand must be [rows, fields, emb]")
    n_req, f_req, emb = x_req.shape
    n_cand, f_cand, emb_c = x_cand.shape
    _need(emb == emb_c, "embedding widths differ")
    _need(x_req.dtype == x_cand.dtype, "x_req and x_cand must share one dtype")
    _need(x_req.is_contiguous() and x_cand.is_contiguous(), "inputs must be contiguous")
    _offsets(cand_offsets, n_req)
    if request_side and y_req is None:
        y_req = _new((n_req, f_req * f_req), x_req.dtype, x_req.device, stream)
    if candidate_side and y_cand is None:
        y_cand = _new((n_cand, f_cand * (f_req + f_cand)), x_req.dtype, x_req.device, stream)
    for t, shape in ((y_req, (n_req, f_req * f_req)),
                     (y_cand, (n_cand, f_cand * (f_req + f_cand)))):
        _need(t is None or (t.shape == shape and t.dtype == x_req.dtype and t.is_contiguous()),
              "output shape / dtype mismatch")
    _on_gpu(x_req, x_cand, cand_offsets, y_req, y_cand)
    _lib.check(lib.rocs_glm_interaction(
        _ptr(x_req), _ptr(x_cand), _ptr(cand_offsets), n_req, n_cand, f_req, f_cand, emb,
        _dtype_code(x_req), _ptr(y_req if request_side else None),
        _ptr(y_cand if candidate_side else None), _stream(stream)), "rocs_glm_interaction")
    return (y_req if request_side else None), (y_cand if candidate_side else None)


def ikbo_lcb(x_req, x_cand, w_cr, w_cc, cand_offsets, *, w_rr=None, y_req=None, y_cand=None,
             workspace=None, stream=None):
    """Two-group GLM LCB (Eq. glm-lcb-two-groups): returns (y_req [R, O_r, E] or None,
    y_cand [N, O_c, E]); y_req = W_RR X^R when w_rr is given, y_cand = W_CR X^R_m + W_CC X^C.
    x_req [R, F_r, E], x_cand [N, F_c, E], w_rr [O_r, F_r], w_cr [O_c, F_r], w_cc [O_c, F_c]."""
    return _lcb(x_req, x_cand, w_rr, w_cr, w_cc, cand_offsets, None, y_req, y_cand, workspace,
                stream)


def ikbo_lcb_mapped(x_req, x_cand, w_cr, w_cc, cand_request_ids, *, w_rr=None, y_req=None,
                    y_cand=None, workspace=None, stream=None):
    """rocs_ikbo_lcb_mapped: ikbo_lcb with m given per candidate (int32 [N] in [0, R))."""
    return _lcb(x_req, x_cand, w_rr, w_cr, w_cc, None, cand_request_ids, y_req, y_cand,
                workspace, stream)


def _lcb(x_req, x_cand, w_rr, w_cr, w_cc, cand_offsets, cand_ids, y_req, y_cand, workspace,
         stream):
    mapped = cand_ids is not None
    done = (_binding or _native()).lcb(x_req, x_cand, w_rr, w_cr, w_cc,
                                       cand_ids if mapped else cand_offsets, mapped, y_req, y_cand,
                                       workspace, stream)
    if done is not None:
        return done
    lib = _lib.load()
    _need(x_req.dim() == 3 and x_cand.dim() == 3, "x_req / x_cand must be [rows, fields, emb]")
    n_req, f_req, emb = x_req.shape
    n_cand, f_cand, emb_c = x_cand.shape
    _need(emb == emb_c, "embedding widths differ")
    o_cand = w_cc.shape[0]
    _need(w_cc.shape == (o_cand, f_cand) and w_cr.shape == (o_cand, f_req),
          "w_cc must be [O_c, F_c] and w_cr [O_c, F_r]")
    o_req = 0 if w_rr is None else w_rr.shape[0]
    _need(w_rr is None or w_rr.shape == (o_req, f_req), "w_rr must be [O_r, F_r]")
    for t in (x_cand, w_rr, w_cr, w_cc):
        _need(t is None or t.dtype == x_req.dtype, "inputs must share one dtype")
    for t in (x_req, x_cand, w_rr, w_cr, w_cc):
        _need(t is None or t.is_contiguous(), "tensors must be contiguous")
    if mapped:
        _request_map(cand_ids, n_cand)
    else:
        _offsets(cand_offsets, n_req)
    if o_req > 0 and y_req is None:
        y_req = _new((n_req, o_req, emb), x_req.dtype, x_req.device, stream)
    if y_cand is None:
        y_cand = _new((n_cand, o_cand, emb), x_req.dtype, x_req.device, stream)
    _need(y_cand.shape == (n_cand, o_cand, emb) and y_cand.dtype == x_req.dtype and
          y_cand.is_contiguous(), "y_cand must be a contiguous [N, O_c, E] tensor")
    _need(y_req is None or (y_req.shape == (n_req, o_req, emb) and y_req.dtype == x_req.dtype
                            and y_req.is_contiguous()), "y_req must be [R, O_r, E]")
    need = int(lib.rocs_ikbo_lcb_workspace_size(n_req, o_cand, emb))
    if workspace is None:
        workspace = _new(max(need, 1), torch.uint8, x_req.device, stream, scratch=True)
    _on_gpu(x_req, x_cand, w_rr, w_cr, w_cc, cand_offsets, cand_ids, y_req, y_cand, workspace)
    fn, name = ((lib.rocs_ikbo_lcb_mapped, "rocs_ikbo_lcb_mapped") if mapped
                else (lib.rocs_ikbo_lcb, "rocs_ikbo_lcb"))
    _lib.check(fn(
        _ptr(x_req), _ptr(x_cand), _ptr(w_rr), _ptr(w_cr), _ptr(w_cc),
        _ptr(cand_ids if mapped else cand_offsets), n_req, n_cand, f_req, f_cand, o_req, o_cand,
        emb, _dtype_code(x_req), _ptr(y_req), _ptr(y_cand), _ptr(workspace),
        workspace.numel() * workspace.element_size(), _stream(stream)), name)
    return y_req, y_cand


def request_ids(cand_offsets, num_cand, *, stream=None):
    """m_n for every candidate, computed on the device (int32 [N])."""
    lib = _lib.load()
    n_req = cand_offsets.numel() - 1
    _offsets(cand_offsets, n_req)
    out = _new(num_cand, torch.int32, cand_offsets.device, stream)
    _on_gpu(cand_offsets, out)
    _lib.check(lib.rocs_request_ids(_ptr(cand_offsets), n_req, num_cand, _ptr(out),
                                    _stream(stream)), "rocs_request_ids")
    return out


def validate_offsets(offsets, total, *, stream=None):
    """Host-side check of device offsets (synchronises the stream)."""
    lib = _lib.load()
    _lib.check(lib.rocs_validate_offsets(_ptr(offsets), offsets.numel(), total,
                                         _stream(stream)), "rocs_validate_offsets")


# ---------------------------------------------------------------------------
# Attention of a request's own rows over its history, and the cache's pages
# ---------------------------------------------------------------------------

def _launch(device, stream, name, *args):
    """The C entry point `name` on the tensors' device, on `stream` or that device's current
    stream."""
    fn = getattr(_lib.load(), name)
    if device.index != torch.cuda.current_device():
        with torch.cuda.device(device):
            s = torch.cuda.current_stream() if stream is None else stream
            _lib.check(fn(*args, ctypes.c_void_p(s.cuda_stream)), name)
        return
    _lib.check(fn(*args, _stream(stream)), name)


def history_workspace_size(num_requests, num_rows, heads, kv_heads, head_dim, max_kv_len, dtype):
    """Bytes of workspace of one history_attention call over at most max_kv_len keys a request, or
    of a paged_attention call (there at most table width * page size keys). A smaller call may
    need more: include/rocs_history.h has a bound for one workspace under calls of many sizes."""
    code = _lib.DTYPE_BF16 if dtype == torch.bfloat16 else _lib.DTYPE_F32
    return int(_lib.load().rocs_history_workspace_size(num_requests, num_rows, heads, kv_heads,
                                                       head_dim, max_kv_len, code))


def _rows_of(t, name):
    """Row stride of [rows, heads, d] (or pages of such rows) whose rows are dense; 0: one row."""
    h, d = t.shape[-2:]
    _need((d == 1 or t.stride(-1) == 1) and (h == 1 or t.stride(-2) == d),
          f"{name} rows must be dense [heads, d] blocks")
    if t.shape[-3] <= 1:
        return 0
    _need(t.stride(-3) >= h * d, f"{name} rows must not overlap")
    return t.stride(-3)


def _int_vector(t, n, name):
    _need(t is None or (t.dtype == torch.int32 and t.dim() == 1 and t.is_contiguous()
                        and t.numel() == n),
          f"{name} must be a contiguous int32 tensor of {n} entries")


def _score_rules(q, k, v, heads_of, prefix_lens, q_offsets, slopes, cap, causal, max_kv_len, out):
    """The checks that both attentions share; returns (out's shape, cap, max_kv_len)."""
    _need(q.dim() == 3, "q must be [N, heads, d]")
    n, h, d = q.shape
    hk = heads_of.shape[-2]
    _need(heads_of.shape[-1] == d and hk >= 1 and h % hk == 0,
          "k and v must have q's head_dim, and heads that divide q's")
    _dtype_code(q)
    _need(k.dtype == q.dtype and v.dtype == q.dtype, "q, k, v must share one dtype")
    _need(q_offsets.numel() >= 1, "q_offsets needs R + 1 entries")
    r = q_offsets.numel() - 1
    _offsets(q_offsets, r)
    _int_vector(prefix_lens, r, "prefix_lens")
    _need(slopes is None or (slopes.dtype == torch.float32 and slopes.shape == (h,)
                             and slopes.is_contiguous()),
          "slopes must be contiguous float32 [heads]")
    _need(causal in (True, False), "causal must be True or False")
    cap = float(cap or 0.0)
    _need(cap == 0.0 or 1e-30 <= cap < 3.4e38, "cap must be 0, or finite and at least 1e-30")
    _need(max_kv_len is None or max_kv_len >= 0, "max_kv_len must not be negative")
    _need(out is None or (out.shape == q.shape and out.dtype == q.dtype and out.is_contiguous()),
          "out must be a contiguous [N, heads, d] tensor of q's dtype")
    return r, cap, int(max_kv_len or 0)


def _history_scratch(workspace, need, device, stream):
    if workspace is None and need > 0:
        workspace = _new(need, torch.uint8, device, stream, scratch=True)
    _on_gpu(workspace)
    _need(workspace is None or workspace.is_contiguous(), "workspace must be contiguous")
    return workspace, 0 if workspace is None else workspace.numel() * workspace.element_size()


def history_attention(q, k, v, q_offsets, kv_offsets, *, causal=True, prefix_lens=None,
                      q_docs=None, kv_docs=None, slopes=None, cap=0.0, max_kv_len=None, scale=None,
                      out=None, workspace=None, stream=None):
    """rocs_history_attention: each request's query rows (the last rows of its history) attend
    over the history's keys.

    q [N, H, d], k and v [L_total, H_kv, d] with H_kv dividing H (rows may be strided: column
    slices of one projection), q_offsets and kv_offsets int32 [R + 1]. `causal` hides the keys
    after a row, but for the first prefix_lens[r] (int32 [R]); q_docs [N] and kv_docs [L_total]
    (int32) keep a row to its own document; `cap` > 0 caps scores to cap * tanh(s / cap);
    `slopes` (float32 [H]) takes slopes[h] * distance off them. A row that sees no key is zero.
    max_kv_len: a bound on the histories' lengths, if the host knows one."""
    done = (_binding or _native()).history(q, k, v, q_offsets, kv_offsets, causal, prefix_lens,
                                           q_docs, kv_docs, slopes, cap, max_kv_len, scale, out,
                                           workspace, stream)
    if done is not None:
        return done
    _need(k.dim() == 3 and v.dim() == 3 and k.shape == v.shape, "k and v must be [L, kv_heads, d]")
    r, cap, most = _score_rules(q, k, v, k, prefix_lens, q_offsets, slopes, cap, causal,
                                max_kv_len, out)
    n, h, d = q.shape
    rows, hk = k.shape[0], k.shape[1]
    _offsets(kv_offsets, r)
    _need((q_docs is None) == (kv_docs is None), "q_docs and kv_docs go together")
    _int_vector(q_docs, n, "q_docs")
    _int_vector(kv_docs, rows, "kv_docs")
    q_stride, k_stride = _rows_of(q, "q"), _rows_of(k, "k")
    _need(_rows_of(v, "v") == k_stride, "k and v must share a row stride")
    _on_gpu(q, k, v, q_offsets, kv_offsets, prefix_lens, q_docs, kv_docs, slopes, out)
    if out is None:
        out = _new(q.shape, q.dtype, q.device, stream)
    need = history_workspace_size(r, n, h, hk, d, most or rows, q.dtype)
    workspace, ws_bytes = _history_scratch(workspace, need, q.device, stream)
    _on_gpu(q, workspace)
    _launch(q.device, stream, "rocs_history_attention", _ptr(q), q_stride, _ptr(k), _ptr(v),
            k_stride, _ptr(q_offsets), _ptr(kv_offsets), _ptr(prefix_lens), _ptr(q_docs),
            _ptr(kv_docs), _ptr(slopes), r, n, rows, h, hk, d, float(scale or 0.0), cap,
            int(causal), most, _dtype_code(q), _ptr(out), _ptr(workspace), ws_bytes)
    return out


def paged_attention(q, k_pages, v_pages, page_table, kv_lens, q_offsets, *, slots=None,
                    causal=True, prefix_lens=None, slopes=None, cap=0.0, max_kv_len=None,
                    scale=None, out=None, workspace=None, stream=None):
    """rocs_paged_attention: history_attention over histories kept in pages.

    k_pages, v_pages [P, page_size, H_kv, d] (views of one cache: pages and rows may be strided),
    page_table int32 [S, W], kv_lens int32 [S], slots int32 [R] (None: request r is slot r),
    q [N, H, d] with q_offsets int32 [R + 1]: the last rows of each history, whose K/V are in
    the cache already, or with causal=False any rows (candidates) that attend over it."""
    done = (_binding or _native()).paged(q, k_pages, v_pages, page_table, kv_lens, q_offsets,
                                         slots, causal, prefix_lens, slopes, cap, max_kv_len,
                                         scale, out, workspace, stream)
    if done is not None:
        return done
    _need(k_pages.dim() == 4 and v_pages.dim() == 4 and k_pages.shape == v_pages.shape,
          "k_pages and v_pages must be [pages, page_size, kv_heads, d]")
    r, cap, most = _score_rules(q, k_pages, v_pages, k_pages, prefix_lens, q_offsets, slopes, cap,
                                causal, max_kv_len, out)
    n, h, d = q.shape
    pages, page, hk = k_pages.shape[:3]
    _need(pages >= 1 and page >= 1, "the cache needs at least one page and one row a page")
    _need(page_table.dtype == torch.int32 and page_table.dim() == 2 and page_table.is_contiguous()
          and page_table.shape[1] >= 1, "page_table must be a contiguous int32 [slots, width]")
    n_slots, width = page_table.shape
    _int_vector(kv_lens, n_slots, "kv_lens")
    _int_vector(slots, r, "slots")
    _need(slots is not None or r <= n_slots, "without slots, request r is slot r: R <= slots")
    q_stride, k_stride = _rows_of(q, "q"), _rows_of(k_pages, "k_pages")
    _need(_rows_of(v_pages, "v_pages") == k_stride, "k_pages and v_pages must share strides")
    page_stride = 0
    if pages > 1:
        page_stride = k_pages.stride(0)
        _need(v_pages.stride(0) == page_stride, "k_pages and v_pages must share strides")
        _need(page_stride >= (page - 1) * k_stride + hk * d, "pages must not overlap")
    _on_gpu(q, k_pages, v_pages, page_table, kv_lens, q_offsets, slots, prefix_lens, slopes, out)
    if out is None:
        out = _new(q.shape, q.dtype, q.device, stream)
    bound = min(most or width * page, width * page)
    need = history_workspace_size(r, n, h, hk, d, bound, q.dtype)
    workspace, ws_bytes = _history_scratch(workspace, need, q.device, stream)
    _on_gpu(q, workspace)
    _launch(q.device, stream, "rocs_paged_attention", _ptr(q), q_stride, _ptr(k_pages),
            _ptr(v_pages), page_stride, k_stride, _ptr(page_table), width, _ptr(kv_lens),
            _ptr(slots), n_slots, _ptr(q_offsets), _ptr(prefix_lens), _ptr(slopes), r, n, pages,
            page, h, hk, d, float(scale or 0.0), cap, int(causal), most, _dtype_code(q), _ptr(out),
            _ptr(workspace), ws_bytes)
    return out


def cache_workspace_size(entries, num_pages):
    return int(_lib.load().rocs_cache_workspace_size(entries, num_pages))


def cache_pool(layers, pages, page_size, kv_heads, head_dim, *, slots, table_width,
               dtype=torch.bfloat16, device="cuda"):
    """An empty cache: (pool [layers, pages, page_size, 2, kv_heads, head_dim], page_table
    int32 [slots, table_width], lens int32 [slots], refs int32 [pages]). A row holds K, then V, as
    a stacked K/V projection writes it; layer l's pages for paged_attention are
    pool[l, :, :, 0] and pool[l, :, :, 1]."""
    pool = torch.zeros((layers, pages, page_size, 2, kv_heads, head_dim), dtype=dtype,
                       device=device)
    table = torch.full((slots, table_width), -1, dtype=torch.int32, device=device)
    return (pool, table, torch.zeros(slots, dtype=torch.int32, device=device),
            torch.zeros(pages, dtype=torch.int32, device=device))


def _cache_state(page_table, lens, refs):
    _need(page_table.dtype == torch.int32 and page_table.dim() == 2
          and page_table.is_contiguous() and page_table.shape[0] >= 1
          and page_table.shape[1] >= 1, "page_table must be a contiguous int32 [slots, width]")
    if lens is not None:
        _int_vector(lens, page_table.shape[0], "lens")
    _need(refs.dtype == torch.int32 and refs.dim() == 1 and refs.is_contiguous()
          and refs.numel() >= 1, "refs must be a contiguous int32 [pages]")
    return page_table.shape[0], page_table.shape[1], refs.numel()


def _cache_layers(pool, pages=None):
    """(layers, page_size, bytes of a row) of a pool [layers, pages, page_size, ...]."""
    _need(pool.dim() >= 4 and pool.is_contiguous() and pages in (None, pool.shape[1])
          and pool.numel() > 0, "pool must be a contiguous [layers, pages, page_size, ...] tensor")
    layers, pages, page = pool.shape[:3]
    return layers, page, pool.numel() // (layers * pages * page) * pool.element_size()


def _cache_status(status, device, stream):
    if status is None:
        return _new(2, torch.int32, device, stream)
    _int_vector(status, 2, "status")
    return status


def cache_reserve(slots, row_offsets, num_rows, page_table, lens, refs, page_size, *, rows=None,
                  status=None, workspace=None, stream=None):
    """rocs_cache_reserve: entry i adds row_offsets[i + 1] - row_offsets[i] rows to slot slots[i]
    (int32 [n], [n + 1]; num_rows >= row_offsets[n]); lens, page_table and refs follow in place.
    Returns (rows int32 [num_rows]: the pool row of each new row, for cache_write, -1 past
    row_offsets[n]; status int32 [2], see cache_check). All or nothing: a call that cannot be done
    leaves the cache unchanged, and its rows are -1."""
    done = (_binding or _native()).cache_reserve(slots, row_offsets, num_rows, page_table, lens,
                                                 refs, page_size, rows, status, workspace, stream)
    if done is not None:
        return done
    n_slots, width, pages = _cache_state(page_table, lens, refs)
    n = slots.numel()
    _int_vector(slots, n, "slots")
    _offsets(row_offsets, n)
    _need(num_rows >= 0 and (n > 0 or num_rows == 0) and page_size >= 1,
          "num_rows must not be negative (or without entries), page_size at least 1")
    _on_gpu(slots, row_offsets, page_table, lens, refs, rows, status)
    if rows is None:
        rows = _new(num_rows, torch.int32, slots.device, stream)
    _int_vector(rows, num_rows, "rows")
    status = _cache_status(status, slots.device, stream)
    workspace, ws_bytes = _history_scratch(workspace, cache_workspace_size(n, pages), slots.device,
                                           stream)
    _on_gpu(slots, workspace)
    _launch(slots.device, stream, "rocs_cache_reserve", _ptr(slots), _ptr(row_offsets), n, num_rows,
            _ptr(page_table), width, _ptr(lens), n_slots, _ptr(refs), pages, page_size, _ptr(rows),
            _ptr(status), _ptr(workspace), ws_bytes)
    return rows, status


def cache_write(x, rows, pool, *, stream=None):
    """rocs_cache_write: row m of x [M, ...] into pool row rows[m] (from cache_reserve) of one
    layer's pool [pages, page_size, ...]. x's rows may be strided; rows that are -1 are passed
    over; a pool row that is named twice holds any mix of the two."""
    if (_binding or _native()).cache_write(x, rows, pool, stream) is not None:
        return pool
    _need(pool.dim() >= 3 and pool.is_contiguous() and pool.numel() > 0,
          "pool must be a contiguous [pages, page_size, ...] tensor")
    _need(x.dtype == pool.dtype, "x and pool must share one dtype")
    pool_rows = pool.shape[0] * pool.shape[1]
    width = pool.numel() // pool_rows
    _need(x.dim() >= 2 and x.numel() == x.shape[0] * width, "x must hold rows of the pool's width")
    _int_vector(rows, x.shape[0], "rows")
    m = x.shape[0]
    if m == 0:
        return pool
    _need(x[0].is_contiguous() and (m == 1 or x.stride(0) >= width), "x's rows must be dense")
    _on_gpu(x, rows, pool)
    size = x.element_size()
    _launch(x.device, stream, "rocs_cache_write", _ptr(x), (x.stride(0) if m > 1 else width) * size,
            _ptr(rows), m, _ptr(pool), pool_rows, width * size)
    return pool


def cache_fork(parents, children, page_table, lens, refs, pool, *, status=None, workspace=None,
               stream=None):
    """rocs_cache_fork: the empty slot children[i] becomes a copy of slot parents[i] (int32 [n]):
    full pages are shared, the rows of a page that is not full are copied in every layer of pool
    [layers, pages, page_size, ...]. Returns status (see cache_check)."""
    done = (_binding or _native()).cache_fork(parents, children, page_table, lens, refs, pool,
                                              status, workspace, stream)
    if done is not None:
        return done
    n_slots, width, pages = _cache_state(page_table, lens, refs)
    layers, page, row_bytes = _cache_layers(pool, pages)
    n = parents.numel()
    _int_vector(parents, n, "parents")
    _int_vector(children, n, "children")
    _on_gpu(parents, children, page_table, lens, refs, pool, status)
    status = _cache_status(status, pool.device, stream)
    workspace, ws_bytes = _history_scratch(workspace, cache_workspace_size(n, pages), pool.device,
                                           stream)
    _on_gpu(pool, workspace)
    _launch(pool.device, stream, "rocs_cache_fork", _ptr(parents), _ptr(children), n,
            _ptr(page_table), width, _ptr(lens), n_slots, _ptr(refs), pages, page, _ptr(pool),
            layers, row_bytes, _ptr(status), _ptr(workspace), ws_bytes)
    return status


def cache_free(slots, page_table, lens, refs, page_size, *, stream=None):
    """rocs_cache_free: the pages of these slots (int32 [n]) back to the cache; the slots are
    empty then."""
    if (_binding or _native()).cache_free(slots, page_table, lens, refs, page_size,
                                          stream) is not None:
        return
    n_slots, width, pages = _cache_state(page_table, lens, refs)
    _int_vector(slots, slots.numel(), "slots")
    _need(page_size >= 1, "page_size must be at least 1")
    _on_gpu(slots, page_table, lens, refs)
    _launch(refs.device, stream, "rocs_cache_free", _ptr(slots), slots.numel(), _ptr(page_table),
            width, _ptr(lens), n_slots, _ptr(refs), pages, page_size)


def cache_compact(page_table, lens, refs, pool, *, status=None, workspace=None, stream=None):
    """rocs_cache_compact: the live pages moved together to the cache's front, in every layer of
    pool; page_table and refs follow. Returns status int32 [2]: {0, number of live pages}."""
    done = (_binding or _native()).cache_compact(page_table, lens, refs, pool, status, workspace,
                                                 stream)
    if done is not None:
        return done
    n_slots, width, pages = _cache_state(page_table, lens, refs)
    layers, page, row_bytes = _cache_layers(pool, pages)
    _on_gpu(page_table, lens, refs, pool, status)
    status = _cache_status(status, pool.device, stream)
    workspace, ws_bytes = _history_scratch(workspace, cache_workspace_size(0, pages), pool.device,
                                           stream)
    _on_gpu(pool, workspace)
    _launch(pool.device, stream, "rocs_cache_compact", _ptr(page_table), width, n_slots, _ptr(refs),
            pages, page, _ptr(pool), layers, row_bytes, _ptr(status), _ptr(workspace), ws_bytes)
    return status


def cache_copy(src_pages, dst_pages, src_pool, dst_pool=None, *, stream=None):
    """rocs_cache_copy: page src_pages[i] of src_pool into page dst_pages[i] of dst_pool (None: the
    same pool), in every layer of [layers, pages, page_size, ...]. A page that is written twice in
    one call, or read and written, leaves any mix of the contents (of each layer its own)."""
    dst_pool = src_pool if dst_pool is None else dst_pool
    layers, page, row_bytes = _cache_layers(src_pool)
    _need(_cache_layers(dst_pool) == (layers, page, row_bytes),
          "the pools must have the same layers and pages of the same size")
    _need(src_pool.dtype == dst_pool.dtype, "the pools must share one dtype")
    n = src_pages.numel()
    _int_vector(src_pages, n, "src_pages")
    _int_vector(dst_pages, n, "dst_pages")
    _on_gpu(src_pages, dst_pages, src_pool, dst_pool)
    _launch(src_pool.device, stream, "rocs_cache_copy", _ptr(src_pages), _ptr(dst_pages), n,
            _ptr(src_pool), src_pool.shape[1], _ptr(dst_pool), dst_pool.shape[1], layers,
            page * row_bytes)
    return dst_pool


def cache_check(status):
    """Raises RocsError if a page operator could not be done. Reads status on the host (waits for
    the current stream). Returns status[1]."""
    code, detail = status.tolist()
    if code != 0:
        why = {_lib.CACHE_NO_PAGES: f"{detail} pages are missing",
               _lib.CACHE_TABLE_FULL: "a slot would need more pages than its table row has",
               _lib.CACHE_BAD_SLOT: "a slot is out of range, named twice or (a child) not empty"}
        raise RocsError(_lib.INVALID_ARGUMENT,
                        f"the cache is unchanged: {why.get(code, f'status {code}')}")
    return detail


# --- adapters beside a projection, rotated rows, a cache in 4 bits -----------

def adapter_workspace_size(num_requests, num_rows, k, d_out, rank, dtype):
    code = _lib.DTYPE_BF16 if dtype == torch.bfloat16 else _lib.DTYPE_F32
    return int(_lib.load().rocs_adapter_workspace_size(num_requests, num_rows, k, d_out, rank, code))


def adapter_linear(x, w, a, b, offsets, adapter_ids, *, scales=None, bias=None, activation="none",
                   out=None, workspace=None, stream=None):
    """rocs_adapter_linear: out[n] = act(W x[n] + bias + s B (A x[n])) with the low-rank adapter
    (A, B, s) of the request that owns row n, beside the projection that all rows share.

    x [N, K] (rows may be strided), w [D, K], a [adapters, rank, K], b [adapters, D, rank], offsets
    int32 [R + 1], adapter_ids int32 [R] (an id outside [0, adapters): no adapter), scales float32
    [adapters], bias float32 [D]. Rows past offsets[R] stay as they are in `out`. Adapters of a
    smaller rank than the array's are the caller's to pad with zeros; in bfloat16 pad the rank to a
    multiple of 8 as well, since others run a general kernel, 27 times slower on large calls."""
    done = (_binding or _native()).adapter(x, w, a, b, offsets, adapter_ids, scales, bias, activation,
                                           out, workspace, stream)
    if done is not None:
        return done
    _need(x.dim() == 2 and w.dim() == 2 and x.shape[1] == w.shape[1] and w.shape[0] >= 1
          and w.shape[1] >= 1, "x must be [N, K] and w [D, K]")
    n, k = x.shape
    d = w.shape[0]
    _need(a.dim() == 3 and b.dim() == 3 and a.shape[0] == b.shape[0] and a.shape[2] == k
          and b.shape[1] == d and a.shape[1] == b.shape[2] and a.shape[1] >= 1,
          "a must be [adapters, rank, K] and b [adapters, D, rank]")
    count, rank = a.shape[:2]
    code = _dtype_code(x)
    _need(w.dtype == x.dtype and a.dtype == x.dtype and b.dtype == x.dtype,
          "x, w, a and b must share one dtype")
    _need(w.is_contiguous() and a.is_contiguous() and b.is_contiguous(),
          "w, a and b must be contiguous")
    _need((k == 1 or x.stride(1) == 1) and (n <= 1 or x.stride(0) >= k), "x's rows must be dense")
    _need(offsets.numel() >= 1, "offsets needs R + 1 entries")
    r = offsets.numel() - 1
    _offsets(offsets, r)
    _int_vector(adapter_ids, r, "adapter_ids")
    _need(scales is None or (scales.dtype == torch.float32 and scales.shape == (count,)
                             and scales.is_contiguous()), "scales must be contiguous float32 [adapters]")
    _need(bias is None or (bias.dtype == torch.float32 and bias.shape == (d,) and bias.is_contiguous()),
          "bias must be contiguous float32 [D]")
    _need(activation in _ACT, f"activation must be one of {sorted(k for k in _ACT if k)}")
    _need(out is None or (out.shape == (n, d) and out.dtype == x.dtype and out.is_contiguous()),
          "out must be a contiguous [N, D] tensor of x's dtype")
    _on_gpu(x, w, a, b, offsets, adapter_ids, scales, bias, out)
    if out is None:
        out = _new((n, d), x.dtype, x.device, stream)
    workspace, ws_bytes = _history_scratch(
        workspace, adapter_workspace_size(r, n, k, d, rank, x.dtype), x.device, stream)
    _on_gpu(x, workspace)
    _launch(x.device, stream, "rocs_adapter_linear", _ptr(x), x.stride(0) if n > 1 else 0, _ptr(w),
            _ptr(a), _ptr(b), _ptr(scales), _ptr(bias), _ptr(offsets), _ptr(adapter_ids), r, n, k, d,
            rank, count, code, _ACT[activation], _ptr(out), _ptr(workspace), ws_bytes)
    return out


def _turn(m, d, freqs, positions, offsets, slots, lens, interleaved):
    """The checks of a rotation's arguments: (rot_dim, R, num_slots)."""
    rot = 0
    if freqs is not None:
        _need(freqs.dtype == torch.float32 and freqs.dim() == 1 and freqs.is_contiguous()
              and 2 * freqs.numel() <= d, "freqs must be contiguous float32 [rot_dim / 2], rot_dim <= d")
        rot = 2 * freqs.numel()
    _int_vector(positions, m, "positions")
    _need(interleaved in (True, False), "interleaved must be True or False")
    if offsets is None:
        _need(slots is None and lens is None, "slots and lens need offsets")
        _need(positions is not None or rot == 0, "a rotation needs positions, or offsets and lens")
        return rot, 0, 0
    _need(offsets.numel() >= 1, "offsets needs R + 1 entries")
    r = offsets.numel() - 1
    _offsets(offsets, r)
    _int_vector(slots, r, "slots")
    n_slots = 0
    if lens is not None:
        n_slots = lens.numel()
        _int_vector(lens, n_slots, "lens")
        _need(slots is not None or r <= n_slots, "without slots, request r is slot r: R <= slots")
    _need(lens is not None or positions is not None or rot == 0,
          "a rotation needs positions, or offsets and lens")
    return rot, r, n_slots


def rotate(x, freqs, *, positions=None, offsets=None, slots=None, lens=None, interleaved=False,
           out=None, stream=None):
    """rocs_rotate: the position rotation of x [M, heads, d] (rows may be strided). Pair i of a head's
    first 2 * len(freqs) dims, dims (i, i + len(freqs)) or with `interleaved` (2 i, 2 i + 1), turns by
    position * freqs[i] (float32, radians). Positions are `positions` (int32 [M]), or those of the
    last rows of each request's history: offsets int32 [R + 1], slots int32 [R] (None: request r is
    slot r), lens int32 [slots], as paged_attention takes them."""
    done = (_binding or _native()).rotate(x, freqs, positions, offsets, slots, lens, interleaved, out,
                                          stream)
    if done is not None:
        return done
    _need(x.dim() == 3 and x.shape[1] >= 1 and x.shape[2] >= 1, "x must be [M, heads, d]")
    m, h, d = x.shape
    code = _dtype_code(x)
    rot, r, n_slots = _turn(m, d, freqs, positions, offsets, slots, lens, interleaved)
    stride = _rows_of(x, "x")
    _need(out is None or (out.shape == x.shape and out.dtype == x.dtype and out.is_contiguous()),
          "out must be a contiguous [M, heads, d] tensor of x's dtype")
    _on_gpu(x, freqs, positions, offsets, slots, lens, out)
    if out is None:
        out = _new(x.shape, x.dtype, x.device, stream)
    _launch(x.device, stream, "rocs_rotate", _ptr(x), stride, _ptr(freqs), rot, int(interleaved),
            _ptr(positions), _ptr(offsets), _ptr(slots), _ptr(lens), r, n_slots, m, h, d, code,
            _ptr(out))
    return out


def fp4_row_bytes(kv_heads, head_dim):
    """Bytes of a row (K and V of all heads) of a 4-bit cache; head_dim a multiple of 32."""
    n = int(_lib.load().rocs_fp4_row_bytes(kv_heads, head_dim))
    _need(n > 0, "a cache in 4 bits needs a head_dim that is a multiple of 32, up to 256")
    return n


def cache_pool_fp4(layers, pages, page_size, kv_heads, head_dim, *, slots, table_width,
                   device="cuda"):
    """An empty cache in 4 bits: cache_pool's tuple with a pool of bytes [layers, pages, page_size,
    fp4_row_bytes(kv_heads, head_dim)]. cache_append writes its rows, paged_attention_fp4 and
    cache_read_fp4 read them; cache_reserve, _fork, _free, _compact and _copy keep its pages as
    they do another pool's."""
    pool = torch.zeros((layers, pages, page_size, fp4_row_bytes(kv_heads, head_dim)),
                       dtype=torch.uint8, device=device)
    table = torch.full((slots, table_width), -1, dtype=torch.int32, device=device)
    return (pool, table, torch.zeros(slots, dtype=torch.int32, device=device),
            torch.zeros(pages, dtype=torch.int32, device=device))


def _pool_rows_fp4(pool, kv_heads, head_dim):
    """Rows of one layer's 4-bit pool [pages, page_size, row bytes]."""
    row = fp4_row_bytes(kv_heads, head_dim)
    _need(pool.dtype == torch.uint8 and pool.dim() == 3 and pool.is_contiguous()
          and pool.shape[2] == row and pool.shape[0] >= 1 and pool.shape[1] >= 1,
          f"a pool in 4 bits must be contiguous uint8 [pages, page_size, {row}]")
    return pool.shape[0] * pool.shape[1]


def cache_append(k, v, rows, pool, freqs=None, *, q=None, positions=None, offsets=None, slots=None,
                 lens=None, interleaved=False, q_out=None, stream=None):
    """rocs_cache_append: row m of k and v [M, kv_heads, d] (column slices of one projection) into
    pool row rows[m] (from cache_reserve) of one layer's pool, k turned by its position as rotate()
    does; with q [M, heads, d] the same rows' queries are turned too and returned (q_out). The pool
    is [pages, page_size, 2, kv_heads, d] of k's dtype, or a 4-bit layer's bytes [pages, page_size,
    fp4_row_bytes]. Rows that are -1 are passed over; without freqs nothing is turned."""
    done = (_binding or _native()).append(k, v, rows, pool, freqs, q, positions, offsets, slots, lens,
                                          interleaved, q_out, stream)
    if done is not None:
        return None if q is None else done
    _need(k.dim() == 3 and k.shape == v.shape and k.shape[1] >= 1 and k.shape[2] >= 1,
          "k and v must be [M, kv_heads, d]")
    m, hk, d = k.shape
    code = _dtype_code(k)
    _need(v.dtype == k.dtype, "k and v must share one dtype")
    stride = _rows_of(k, "k")
    _need(_rows_of(v, "v") == stride, "k and v must share a row stride")
    _int_vector(rows, m, "rows")
    rot, r, n_slots = _turn(m, d, freqs, positions, offsets, slots, lens, interleaved)
    if pool.dtype == torch.uint8:
        form, pool_rows = _lib.POOL_FP4, _pool_rows_fp4(pool, hk, d)
    else:
        form = _lib.POOL_ROWS
        _need(pool.dtype == k.dtype and pool.dim() == 5 and pool.is_contiguous()
              and tuple(pool.shape[2:]) == (2, hk, d) and pool.shape[0] >= 1 and pool.shape[1] >= 1,
              "pool must be contiguous [pages, page_size, 2, kv_heads, d] of k's dtype, or 4-bit rows")
        pool_rows = pool.shape[0] * pool.shape[1]
    h, q_stride = 0, 0
    _need(q is not None or q_out is None, "q_out needs q")
    if q is not None:
        _need(q.dim() == 3 and q.shape[0] == m and q.shape[1] >= 1 and q.shape[2] == d
              and q.dtype == k.dtype, "q must be [M, heads, d] of k's dtype")
        h, q_stride = q.shape[1], _rows_of(q, "q")
        _need(q_out is None or (q_out.shape == q.shape and q_out.dtype == q.dtype
                                and q_out.is_contiguous()),
              "q_out must be a contiguous [M, heads, d] tensor of q's dtype")
    _on_gpu(k, v, rows, pool, freqs, q, positions, offsets, slots, lens, q_out)
    if q is not None and q_out is None:
        q_out = _new(q.shape, q.dtype, q.device, stream)
    _launch(k.device, stream, "rocs_cache_append", _ptr(q), q_stride, _ptr(k), _ptr(v), stride,
            _ptr(rows), _ptr(freqs), rot, int(interleaved), _ptr(positions), _ptr(offsets),
            _ptr(slots), _ptr(lens), r, n_slots, m, h, hk, d, code, _ptr(pool), pool_rows, form,
            _ptr(q_out))
    return q_out


def cache_read_fp4(rows, pool, kv_heads, head_dim, *, dtype=torch.bfloat16, out=None, stream=None):
    """rocs_cache_read_fp4: rows rows[m] (int32 [M]) of one layer's 4-bit pool as values [M, 2,
    kv_heads, head_dim] (K, then V) in bfloat16 (exactly) or float32; a row outside the pool is
    zero."""
    done = (_binding or _native()).read_fp4(rows, pool, kv_heads, head_dim, dtype == torch.bfloat16, out,
                                            stream) if dtype in (torch.bfloat16, torch.float32) else None
    if done is not None:
        return done
    _need(dtype in (torch.bfloat16, torch.float32), "dtype must be bfloat16 or float32")
    pool_rows = _pool_rows_fp4(pool, kv_heads, head_dim)
    m = rows.numel()
    _int_vector(rows, m, "rows")
    shape = (m, 2, kv_heads, head_dim)
    _need(out is None or (out.shape == shape and out.dtype == dtype and out.is_contiguous()),
          "out must be a contiguous [M, 2, kv_heads, head_dim] tensor of dtype")
    _on_gpu(rows, pool, out)
    if out is None:
        out = _new(shape, dtype, pool.device, stream)
    _launch(pool.device, stream, "rocs_cache_read_fp4", _ptr(rows), m, _ptr(pool), pool_rows, kv_heads,
            head_dim, _dtype_code(out), _ptr(out))
    return out


def paged_fp4_workspace_size(num_requests, num_rows, heads, kv_heads, head_dim, max_kv_len, dtype):
    """Bytes of workspace of one paged_attention_fp4 call over at most max_kv_len keys a request (at
    most table width * page size)."""
    code = _lib.DTYPE_BF16 if dtype == torch.bfloat16 else _lib.DTYPE_F32
    return int(_lib.load().rocs_paged_fp4_workspace_size(num_requests, num_rows, heads, kv_heads,
                                                         head_dim, max_kv_len, code))


def paged_attention_fp4(q, pages, page_table, kv_lens, q_offsets, *, kv_heads, slots=None,
                        causal=True, prefix_lens=None, slopes=None, cap=0.0, max_kv_len=None,
                        scale=None, out=None, workspace=None, stream=None):
    """rocs_paged_attention_fp4: paged_attention over one layer's pages in 4 bits, uint8 [pages,
    page_size, fp4_row_bytes(kv_heads, d)]; q [N, H, d] with d a multiple of 32. The other
    arguments, the masks and the result are paged_attention's."""
    done = (_binding or _native()).paged_fp4(q, pages, page_table, kv_lens, q_offsets, kv_heads, slots,
                                             causal, prefix_lens, slopes, cap, max_kv_len, scale, out,
                                             workspace, stream)
    if done is not None:
        return done
    _need(q.dim() == 3, "q must be [N, heads, d]")
    n, h, d = q.shape
    _need(kv_heads >= 1 and h >= 1 and h % kv_heads == 0, "kv_heads must divide q's heads")
    _pool_rows_fp4(pages, kv_heads, d)
    n_pages, page = pages.shape[:2]
    # The rules that every attention checks, with q in the place of K and V.
    own = q[:, :kv_heads]
    r, cap, most = _score_rules(q, own, own, own, prefix_lens, q_offsets, slopes, cap, causal,
                                max_kv_len, out)
    _need(page_table.dtype == torch.int32 and page_table.dim() == 2 and page_table.is_contiguous()
          and page_table.shape[1] >= 1, "page_table must be a contiguous int32 [slots, width]")
    n_slots, width = page_table.shape
    _int_vector(kv_lens, n_slots, "kv_lens")
    _int_vector(slots, r, "slots")
    _need(slots is not None or r <= n_slots, "without slots, request r is slot r: R <= slots")
    q_stride = _rows_of(q, "q")
    _on_gpu(q, pages, page_table, kv_lens, q_offsets, slots, prefix_lens, slopes, out)
    if out is None:
        out = _new(q.shape, q.dtype, q.device, stream)
    bound = min(most or width * page, width * page)
    need = paged_fp4_workspace_size(r, n, h, kv_heads, d, bound, q.dtype)
    workspace, ws_bytes = _history_scratch(workspace, need, q.device, stream)
    _on_gpu(q, workspace)
    _launch(q.device, stream, "rocs_paged_attention_fp4", _ptr(q), q_stride, _ptr(pages),
            _ptr(page_table), width, _ptr(kv_lens), _ptr(slots), n_slots, _ptr(q_offsets),
            _ptr(prefix_lens), _ptr(slopes), r, n, n_pages, page, h, kv_heads, d, float(scale or 0.0),
            cap, int(causal), most, _dtype_code(q), _ptr(out), _ptr(workspace), ws_bytes)
    return out
