"""Operators around the network, on torch tensors: thin callers of the C ABI (include/lp.h), which defines them.

Every call enqueues its work on the current stream of the tensors' device and returns; outputs and workspaces come from
torch's allocator on that stream, so calls on several streams, and calls captured into HIP graphs, do not share any.  As with
any torch operator, a tensor that another stream produced has to be waited for by the caller.

Nothing here records a graph: the gradients are a call of their own (linear_ce_backward), and the update works in place.  So tensors
that require a gradient are refused unless autograd is off (torch.no_grad), as their results would be cut off from them unseen.
"""
import contextlib
import functools
import math

import torch

from . import binding as B

_DTYPES = {torch.float32: B.LP_F32, torch.bfloat16: B.LP_BF16}
_INT_MAX = 2 ** 31 - 1          # sizes are ints of the C ABI, which would take a larger one for another


def _device(*tensors):
    if torch.is_grad_enabled() and any(t.requires_grad for t in tensors if isinstance(t, torch.Tensor)):
        raise ValueError("a tensor requires a gradient, and no graph is recorded here: call under torch.no_grad()")
    dev = None
    for t in tensors:
        if t is None:
            continue
        if not isinstance(t, torch.Tensor) or not t.is_cuda:
            raise ValueError("expected tensors on the GPU (there is no CPU fallback)")
        if dev is None:
            dev = t.device
        elif t.device != dev:
            raise ValueError(f"tensors on {dev} and on {t.device}")
    return dev


def _on(dev):
    """The device's own context where it is not the current one (changing to the same costs as much as a launch)."""
    return contextlib.nullcontext() if torch.cuda.current_device() == dev.index else torch.cuda.device(dev)


def _stream(dev):
    """The current stream of the device (without the object around it, which takes as long to make as a launch)."""
    return torch._C._cuda_getCurrentRawStream(dev.index)


@functools.lru_cache(maxsize=1024)
def _ce_workspace(rows, channels, classes, dtype, ld_features, ld_weight, backward):
    return B.lp_linear_ce_workspace_bytes(B.lp_linear_ce_desc(rows, channels, classes, dtype, ld_features, ld_weight, 0), backward)


def _rows(t):
    """A matrix whose rows lie as the library reads them: consecutive elements, any row stride, 16-byte aligned."""
    if t.shape[0] and t.shape[1] and (t.data_ptr() % 16 or (t.shape[1] > 1 and t.stride(1) != 1) or (t.shape[0] > 1 and t.stride(0) < t.shape[1])):
        return t.clone(memory_format=torch.contiguous_format)
    return t


def _ld(t):
    return t.stride(0) if t.shape[0] > 1 else t.shape[1]


def _ce_args(features, weight, labels, bias, lse=None):
    dev = _device(features, weight, labels, bias, lse)
    if features.dtype not in _DTYPES or weight.dtype != features.dtype:
        raise ValueError(f"features {features.dtype} and weight {weight.dtype}: both float32 or both bfloat16")
    if features.dim() != 2 or weight.dim() != 2:
        raise ValueError(f"features {tuple(features.shape)} and weight {tuple(weight.shape)}: expected matrices")
    n, c = features.shape
    v = weight.shape[0]
    if max(n, c, v) > _INT_MAX:
        raise ValueError(f"features {tuple(features.shape)} and weight {tuple(weight.shape)}: more rows or columns than an int holds")
    if weight.shape[1] != c:
        raise ValueError(f"features {tuple(features.shape)} and weight {tuple(weight.shape)} do not fit")
    if labels.shape != (n,) or labels.dtype != torch.int32:
        raise ValueError(f"labels: expected int32 [{n}], got {labels.dtype} {tuple(labels.shape)}")
    if bias is not None and (bias.shape != (v,) or bias.dtype != torch.float32):
        raise ValueError(f"bias: expected float32 [{v}], got {bias.dtype} {tuple(bias.shape)}")
    features, weight = _rows(features), _rows(weight)
    d = B.lp_linear_ce_desc(n, c, v, _DTYPES[features.dtype], _ld(features), _ld(weight), 0)
    return dev, d, features, weight, labels.contiguous(), None if bias is None else bias.contiguous()


def _ptr(t):
    return None if t is None else t.data_ptr()


def linear_ce_forward(features, weight, labels, bias=None):
    """Softmax cross-entropy of the classifier features @ weight.T + bias, without its logits (lp_linear_ce_forward).

    features [N, C] and weight [V, C] (both float32 or both bfloat16, any row stride), labels int32 [N], bias float32 [V].
    Rows whose label is outside [0, V) are left out.  Returns (loss [1], row_loss [N], lse [N]), float32: the mean over
    the rows that count, the loss of every row, and the log of every row's sum of exponentials."""
    dev, d, features, weight, labels, bias = _ce_args(features, weight, labels, bias)
    with _on(dev):
        out = torch.empty(1 + 2 * d.rows, dtype=torch.float32, device=dev)
        loss, row_loss, lse = out[:1], out[1:1 + d.rows], out[1 + d.rows:]
        size = _ce_workspace(d.rows, d.channels, d.classes, d.dtype, d.ld_features, d.ld_weight, False)
        ws = torch.empty(size, dtype=torch.uint8, device=dev)
        B.lp_linear_ce_forward(d, _stream(dev), features.data_ptr(), weight.data_ptr(), _ptr(bias), labels.data_ptr(),
                               loss.data_ptr(), row_loss.data_ptr(), lse.data_ptr(), ws.data_ptr(), size)
    return loss, row_loss, lse


def linear_ce_backward(features, weight, labels, lse, bias=None, scale=1.0):
    """Gradients of scale * loss (lp_linear_ce_backward), from lse as linear_ce_forward returned it for the same operands:
    (dfeatures [N, C] in the type of features, dweight [V, C] float32, dbias [V] float32 or None without a bias)."""
    dev, d, features, weight, labels, bias = _ce_args(features, weight, labels, bias, lse)
    if lse.shape != (d.rows,) or lse.dtype != torch.float32:
        raise ValueError(f"lse: expected float32 [{d.rows}], got {lse.dtype} {tuple(lse.shape)}")
    lse = lse.contiguous()
    with _on(dev):
        dx = torch.empty((d.rows, d.channels), dtype=features.dtype, device=dev)
        dw = torch.empty((d.classes, d.channels), dtype=torch.float32, device=dev)
        db = None if bias is None else torch.empty(d.classes, dtype=torch.float32, device=dev)
        size = _ce_workspace(d.rows, d.channels, d.classes, d.dtype, d.ld_features, d.ld_weight, True)
        ws = torch.empty(size, dtype=torch.uint8, device=dev)
        B.lp_linear_ce_backward(d, _stream(dev), features.data_ptr(), weight.data_ptr(), _ptr(bias), labels.data_ptr(),
                                lse.data_ptr(), scale, dx.data_ptr(), dw.data_ptr(), _ptr(db), ws.data_ptr(), size)
    return dx, dw, db


def orthogonalize(matrices, steps=5, out_dtype=None):
    """The matrices with their singular values taken towards one by Newton-Schulz products (lp_orthogonalize): a list of new
    tensors, each of its matrix's type (or `out_dtype`).  float32 or bfloat16, any sizes and row strides, all in the same launches (whose tiles are chosen for the
    list as a whole: a large matrix beside others may differ from itself alone within its error)."""
    matrices = list(matrices)
    dev = _device(*matrices)
    mats = (B.lp_matrix * len(matrices))()
    outs, keep = [], []
    for i, m in enumerate(matrices):
        o = out_dtype or m.dtype
        if m.dim() != 2 or m.dtype not in _DTYPES or o not in _DTYPES or max(m.shape) > _INT_MAX:
            raise ValueError(f"matrix {i}: expected a float32 or bfloat16 matrix of at most 2^20 rows and columns, got {m.dtype} {tuple(m.shape)}, result {o}")
        if m.numel() and ((m.shape[1] > 1 and m.stride(1) != 1) or (m.shape[0] > 1 and m.stride(0) < m.shape[1])):
            m = m.clone(memory_format=torch.contiguous_format)
            keep.append(m)
        out = torch.empty(m.shape, dtype=o, device=dev)
        outs.append(out)
        mats[i] = B.lp_matrix(m.shape[0], m.shape[1], _DTYPES[m.dtype], _DTYPES[o], m.data_ptr(), out.data_ptr(), _ld(m), 0)
    if dev is None:
        return outs
    with _on(dev):
        size = B.lp_orthogonalize_workspace_bytes(mats)
        ws = torch.empty(size, dtype=torch.uint8, device=dev)
        B.lp_orthogonalize(_stream(dev), mats, steps, ws.data_ptr(), size)
    return outs


@functools.lru_cache(maxsize=64)
def _muon_table(table):
    """(tensors of a packed set as the library reads them, workspace they need, bytes of the parameters and of the fp32 buffers)"""
    arr = (B.lp_muon_tensor * len(table))()
    end = gend = 0
    for i, (shape, dtype, orthogonal, offset, grad_offset) in enumerate(table):
        n = math.prod(shape)
        rows = shape[0] if len(shape) > 1 else 1
        if dtype not in ("f32", "bf16") or n < 1 or max(rows, n // rows) > _INT_MAX:
            raise ValueError(f"tensor {i}: {dtype} {shape}")
        if offset < 0 or grad_offset < 0:
            raise ValueError(f"tensor {i}: offset {offset} or {grad_offset} in front of its buffer")
        arr[i] = B.lp_muon_tensor(rows, n // rows, B.LP_BF16 if dtype == "bf16" else B.LP_F32, int(orthogonal), offset, grad_offset)
        end, gend = max(end, offset + n * (2 if dtype == "bf16" else 4)), max(gend, grad_offset + 4 * n)
    return arr, B.lp_muon_step_workspace_bytes(arr), end, gend


def muon_update(table, params, grads, velocity, master=None, *, lr, momentum=0.95, nesterov=True, weight_decay=0.0, rest_lr=None, steps=5):
    """Parameter update by orthogonalised momentum of a packed set of tensors, in place (lp_muon_step).

    table: a tuple of (shape, "f32" or "bf16", orthogonal, byte offset in params, byte offset in the fp32 buffers), the layout
    lp_net_tensor_info describes; a tensor of several dimensions is read as a matrix of shape[0] rows.  params: uint8; grads,
    velocity, master: float32, one-dimensional, contiguous.  No two tensors may share elements.  rest_lr (default lr): learning rate of the tensors that are not
    orthogonalised."""
    arr, size, end, gend = _muon_table(tuple(table))
    dev = _device(params, grads, velocity, master)
    if params.dtype != torch.uint8 or not params.is_contiguous() or params.numel() < end:
        raise ValueError(f"params: expected {end} bytes (uint8, contiguous), got {params.dtype} {tuple(params.shape)}")
    for name, t in (("grads", grads), ("velocity", velocity), ("master", master)):
        if t is not None and (t.dtype != torch.float32 or not t.is_contiguous() or 4 * t.numel() < gend):
            raise ValueError(f"{name}: expected {gend // 4} float32, contiguous, got {t.dtype} {tuple(t.shape)}")
    opts = B.lp_muon_opts(lr, momentum, weight_decay, lr if rest_lr is None else rest_lr, int(nesterov), steps)
    with _on(dev):
        ws = torch.empty(size, dtype=torch.uint8, device=dev)
        B.lp_muon_step(_stream(dev), arr, params.data_ptr(), grads.data_ptr(), velocity.data_ptr(), _ptr(master),
                       opts, ws.data_ptr(), size)
