"""Operators of language models on torch tensors: matrices held in microscaled 8- or 4-bit numbers and their products, the
root-mean-square norm that feeds them, and log probabilities of given tokens.

What the activation codec does for feature maps these do for the layers of a transformer: what a linear layer keeps for its
backward pass is the quantised form of its input, 8.25 or 4.25 bits a number, and the products take that form as it is.

    q = mx_quantize(w, "e2m1")                        # weights, laid out once
    y = mx_matmul(mx_quantize(x, "e2m1"), q, x.dtype) # inference
    y = mx_linear(x, w)                               # training: gradients of x and w from quantised operands
    y, h = rms_norm(x, g, residual)                   # h = x + residual, y = its norm; gradients
    q, h = rms_norm_mx(x, g, residual)                # inference: y in 8 bits, what mx_matmul takes
    logprobs, entropy, top, indices = token_logprobs(logits, targets, top=5)

`DivisionLinear`, `DivisionRMSNorm` and `DivisionNormLinear` are the modules; `to_division_layers` puts them in place of torch's.

Glue only, as in `autograd`: every step, of backward passes too, runs in the CUDA library through the C ABI (include/division.h says what it
computes), on the current stream of the inputs' device.  Inputs are CUDA tensors of dtype float32, bfloat16 or float16; leading
dimensions are folded into rows.  Rows that are runs of neighbours are read where they are, whatever their stride.  The calls may
be captured into CUDA graphs; a backward pass only while no eager graph of the same leaves is alive, as with any operator of
torch (its accumulation nodes tie the eager stream to the capture, which torch refuses).
"""
from __future__ import annotations

from typing import NamedTuple

import torch

from . import binding

_native = None


def _load():
    global _native
    _native = binding.native()
    return _native


class MxTensor:
    """A matrix in microscaled numbers: rows x cols, blocks of 32 neighbours along a row with one scale each."""
    __slots__ = ("blob", "rows", "cols", "fmt")

    def __init__(self, blob, rows: int, cols: int, fmt: str):
        self.blob, self.rows, self.cols, self.fmt = blob, rows, cols, fmt

    @property
    def shape(self):
        return torch.Size((self.rows, self.cols))

    @property
    def device(self):
        return self.blob.device

    @property
    def nbytes(self) -> int:
        """Bytes of the codes and scales themselves (the blob is a little larger: whole tiles)."""
        return int(binding.div_mx_bytes(self.rows, self.cols, self.fmt).closed_form_bytes) if self.rows else 0

    def dequantize(self, dtype=torch.bfloat16):
        """The numbers it stands for (exact in bfloat16 and float32)."""
        return (_native or _load()).mx_dequantize(self.blob, self.rows, self.cols, self.fmt, dtype)

    def __repr__(self):
        return f"MxTensor({self.rows} x {self.cols}, {self.fmt}, {self.blob.device})"


def mx_quantize(x, fmt: str = "e4m3") -> MxTensor:
    """x (leading dimensions folded) quantised by rows: blocks along the last dimension.  No gradient passes."""
    blob, _, rows, cols = (_native or _load()).mx_quantize(x, fmt, True, False)
    return MxTensor(blob, rows, cols, fmt)


def mx_quantize_both(x, fmt: str = "e4m3"):
    """(x by rows, its transpose by rows) from one reading: what the forward product takes, and what the gradient of the
    weights takes, whose sum runs over the rows of x.  No gradient passes."""
    by_rows, by_columns, rows, cols = (_native or _load()).mx_quantize(x, fmt, True, True)
    return MxTensor(by_rows, rows, cols, fmt), MxTensor(by_columns, cols, rows, fmt)


def mx_quantize_columns(x, fmt: str = "e4m3") -> MxTensor:
    """The transpose of x quantised by rows."""
    _, blob, rows, cols = (_native or _load()).mx_quantize(x, fmt, False, True)
    return MxTensor(blob, cols, rows, fmt)


def mx_matmul(a: MxTensor, b: MxTensor, dtype=torch.bfloat16):
    """a @ b.T of two matrices with rows of equal length and one format; sums in 32 bits, rounded to dtype once."""
    if not isinstance(a, MxTensor) or not isinstance(b, MxTensor):
        raise ValueError("mx_matmul takes two MxTensors")
    if a.fmt != b.fmt or a.cols != b.cols:
        raise ValueError(f"operands differ in format or length of rows: {a!r}, {b!r}")
    return (_native or _load()).mx_matmul(a.blob, a.rows, b.blob, b.rows, a.cols, a.fmt, dtype)


def mx_linear(x, w, fmt: str = "e4m3"):
    """x @ w.T with both operands quantised, blocks of 32 along the features; the gradients of x and w come from quantised
    operands too, their blocks along what each product sums over (straight through the rounding): dx = Q(dy) Q(w^T)^T,
    dw = Q(dy^T) Q(x^T)^T.  Kept for them: x and w by columns, as far as they are wanted.  The result has x's dtype."""
    return (_native or _load()).mx_linear(x, w, fmt)


def rms_norm(x, weight, residual=None, eps: float = 1e-6):
    """(y, h): h = x + residual rounded to x's dtype (x itself without a residual), y = h / sqrt(mean(h^2) + eps) * weight over the last
    dimension.  weight: x's dtype or float32.  Differentiable in x, residual and weight."""
    return (_native or _load()).rms_norm(x, residual, weight, eps)


def rms_norm_mx(x, weight, residual=None, eps: float = 1e-6, fmt: str = "e4m3"):
    """(q, h): as rms_norm, with y handed on as an MxTensor (rows folded), quantised from its 32-bit values.  No gradient passes."""
    blob, rows, cols, h = (_native or _load()).rms_norm_mx(x, residual, weight, eps, fmt)
    return MxTensor(blob, rows, cols, fmt), h


def mx_norm_linear(x, norm_weight, w, residual=None, eps: float = 1e-6, fmt: str = "e4m3"):
    """(out, h): the norm and the linear layer behind it.  The norm's output goes into the product in few bits, quantised from its 32-bit
    values, and is not kept: the backward pass makes it again from h, rounded to x's dtype, for the gradient of w.  Gradients as of
    rms_norm and, at its result, of mx_linear."""
    return (_native or _load()).mx_norm_linear(x, residual, norm_weight, w, eps, fmt)


class TokenLogprobs(NamedTuple):
    logprobs: torch.Tensor
    entropy: torch.Tensor
    top_logprobs: torch.Tensor
    top_indices: torch.Tensor


def token_logprobs(logits, targets, top: int = 0) -> TokenLogprobs:
    """Log probabilities of `targets` (int64, one a row; negative: none, 0) under softmax(logits), the entropies, and the `top` (at most
    32) most probable tokens with theirs, equal ones by index.  logits: ... x vocabulary.  Results in float32.  The logits are all that
    is kept for the backward pass, beside four numbers a row; log probabilities and entropies are differentiable, the alternatives
    are not."""
    return TokenLogprobs(*(_native or _load()).token_logprobs(logits, targets, top))


# ------------------------------------------------------------------------------------------------------------
# modules
# ------------------------------------------------------------------------------------------------------------
def _known(fmt):
    if fmt not in binding.MX_FORMATS:
        raise ValueError(f"fmt must be one of {tuple(binding.MX_FORMATS)}, not {fmt!r}")
    return fmt


class DivisionLinear(torch.nn.Linear):
    """nn.Linear whose products take quantised operands; what it keeps of its input has 8 or 4 bits a number.  For training: the weight is quantised
    at every call.  To answer with it, lay the weight out once (mx_quantize) and call mx_matmul."""

    def __init__(self, in_features, out_features, bias=True, fmt: str = "e4m3", device=None, dtype=None):
        super().__init__(in_features, out_features, bias, device, dtype)
        self.fmt = _known(fmt)

    def forward(self, x):
        y = mx_linear(x, self.weight, self.fmt)
        return y if self.bias is None else y + self.bias.to(y.dtype)


class DivisionRMSNorm(torch.nn.Module):
    """rms_norm with its weight; with a residual it returns (y, h).  What it keeps of its input has the input's shape and type, and is what
    `autograd.DivisionCache` compresses, where that takes maps of the kind."""

    def __init__(self, features, eps: float = 1e-6, device=None, dtype=None):
        super().__init__()
        self.weight, self.eps = torch.nn.Parameter(torch.ones(features, device=device, dtype=dtype)), eps

    def forward(self, x, residual=None):
        y, h = rms_norm(x, self.weight, residual, self.eps)
        return y if residual is None else (y, h)


class DivisionNormLinear(torch.nn.Module):
    """A norm and the linear layer behind it, without a bias; with a residual it returns (out, h)."""

    def __init__(self, in_features, out_features, eps: float = 1e-6, fmt: str = "e4m3", device=None, dtype=None):
        super().__init__()
        self.fmt = _known(fmt)
        self.norm_weight = torch.nn.Parameter(torch.ones(in_features, device=device, dtype=dtype))
        self.weight = torch.nn.Parameter(torch.empty(out_features, in_features, device=device, dtype=dtype))
        torch.nn.init.kaiming_uniform_(self.weight, a=5 ** 0.5)
        self.eps = eps

    def forward(self, x, residual=None):
        out, h = mx_norm_linear(x, self.norm_weight, self.weight, residual, self.eps, self.fmt)
        return out if residual is None else (out, h)


def to_division_layers(module: torch.nn.Module, fmt: str = "e4m3") -> torch.nn.Module:
    """Replace every nn.Linear below `module` by DivisionLinear and every nn.RMSNorm over one dimension by DivisionRMSNorm, with their
    parameters (in place; returns the module).  A layer that is used in several places is replaced by one in all of them; hooks of a
    replaced layer are not carried over."""
    made = {}                                       # what has been seen -> what stands in its place

    def replaced(child):
        if child in made:
            return made[child]
        new = child
        if type(child) is torch.nn.Linear:
            new = DivisionLinear(child.in_features, child.out_features, child.bias is not None, fmt, device="meta")
            new.weight, new.bias = child.weight, child.bias
        elif type(child) is torch.nn.RMSNorm and len(child.normalized_shape) == 1 and child.weight is not None:
            # (torch's default: the epsilon of the type that it computes in, float32 for the 16-bit types)
            eps = torch.finfo(torch.float32).eps if child.eps is None else child.eps
            new = DivisionRMSNorm(child.normalized_shape[0], eps, device="meta")
            new.weight = child.weight
        made[child] = new.train(child.training) if new is not child else child
        if new is child:
            below(child)
        return made[child]

    def below(parent):
        # (named_children names a child once, however often it is used)
        for name, child in list(parent._modules.items()):
            if child is not None and replaced(child) is not child:
                setattr(parent, name, made[child])

    below(module)
    return module
