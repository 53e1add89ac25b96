"""Operators around the network, on torch tensors: thin callers of the C ABI (include/lp.h), which defines them.

Every call enqueues its work on the current stream of the tensors' device and returns; outputs and workspaces come from
torch's allocator on that stream, so calls on several streams, and calls captured into HIP graphs, do not share any.  As with
any torch operator, a tensor that another stream produced has to be waited for by the caller.
"""
import torch

from . import binding as B

_DTYPES = {torch.float32: B.LP_F32, torch.bfloat16: B.LP_BF16}


def _device(*tensors):
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


def _rows(t, name):
    """A matrix whose rows lie as the library reads them: consecutive elements, any row stride, 16-byte aligned."""
    if t.dim() != 2:
        raise ValueError(f"{name}: expected a matrix, got {tuple(t.shape)}")
    if t.shape[0] and t.shape[1] and (t.data_ptr() % 16 or (t.shape[1] > 1 and t.stride(1) != 1) or (t.shape[0] > 1 and t.stride(0) < t.shape[1])):
        return t.clone(memory_format=torch.contiguous_format)
    return t


def _ld(t):
    return t.stride(0) if t.shape[0] > 1 else t.shape[1]


def _ce_args(features, weight, labels, bias):
    dev = _device(features, weight, labels, bias)
    if features.dtype not in _DTYPES or weight.dtype != features.dtype:
        raise ValueError(f"features {features.dtype} and weight {weight.dtype}: both float32 or both bfloat16")
    features, weight = _rows(features, "features"), _rows(weight, "weight")
    n, c = features.shape
    v = weight.shape[0]
    if weight.shape[1] != c:
        raise ValueError(f"features {tuple(features.shape)} and weight {tuple(weight.shape)} do not fit")
    if labels.shape != (n,) or labels.dtype != torch.int32:
        raise ValueError(f"labels: expected int32 [{n}], got {labels.dtype} {tuple(labels.shape)}")
    if bias is not None and (bias.shape != (v,) or bias.dtype != torch.float32):
        raise ValueError(f"bias: expected float32 [{v}], got {bias.dtype} {tuple(bias.shape)}")
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
    with torch.cuda.device(dev):
        out = torch.empty(1 + 2 * d.rows, dtype=torch.float32, device=dev)
        loss, row_loss, lse = out[:1], out[1:1 + d.rows], out[1 + d.rows:]
        size = B.lp_linear_ce_workspace_bytes(d, False)
        ws = torch.empty(size, dtype=torch.uint8, device=dev)
        B.lp_linear_ce_forward(d, torch.cuda.current_stream().cuda_stream, features.data_ptr(), weight.data_ptr(), _ptr(bias), labels.data_ptr(),
                               loss.data_ptr(), row_loss.data_ptr(), lse.data_ptr(), ws.data_ptr(), size)
    return loss, row_loss, lse


def linear_ce_backward(features, weight, labels, lse, bias=None, scale=1.0):
    """Gradients of scale * loss (lp_linear_ce_backward), from lse as linear_ce_forward returned it for the same operands:
    (dfeatures [N, C] in the type of features, dweight [V, C] float32, dbias [V] float32 or None without a bias)."""
    dev, d, features, weight, labels, bias = _ce_args(features, weight, labels, bias)
    _device(features, lse)
    if lse.shape != (d.rows,) or lse.dtype != torch.float32:
        raise ValueError(f"lse: expected float32 [{d.rows}], got {lse.dtype} {tuple(lse.shape)}")
    lse = lse.contiguous()
    with torch.cuda.device(dev):
        dx = torch.empty((d.rows, d.channels), dtype=features.dtype, device=dev)
        dw = torch.empty((d.classes, d.channels), dtype=torch.float32, device=dev)
        db = None if bias is None else torch.empty(d.classes, dtype=torch.float32, device=dev)
        size = B.lp_linear_ce_workspace_bytes(d, True)
        ws = torch.empty(size, dtype=torch.uint8, device=dev)
        B.lp_linear_ce_backward(d, torch.cuda.current_stream().cuda_stream, features.data_ptr(), weight.data_ptr(), _ptr(bias), labels.data_ptr(),
                                lse.data_ptr(), scale, dx.data_ptr(), dw.data_ptr(), _ptr(db), ws.data_ptr(), size)
    return dx, dw, db
