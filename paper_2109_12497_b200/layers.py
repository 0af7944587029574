"""A layer whose gradients go into a worker's row of the gradients that ``Quantizer`` aggregates.

``NormLinear`` is layer norm followed by a linear map without a bias, the products in microscaled 4-bit arithmetic.  Its
parameters lie in one flat binary32 vector, ``[gamma | beta | weight]``, and its backward pass writes their gradients to the
same places of one worker's row of ``g``; the step's update (``Quantizer.aggregate_decode_update``) then moves the vector.

Activations y and weights W are rounded to the nearest 4-bit value, Q; the gradient dy stochastically.  So the weight's gradient
is unbiased for dy^T Q(y) and the input's (in front of layer norm) for dy Q(W), as the quantizers that follow are for what they
are given; they are not for dy^T y and dy W.  Nor is the backward pass the derivative of the forward pass: that one uses y and W
with blocks along d_in, this one the same matrices with blocks along the tokens and along d_out, which are other roundings.

The class holds buffers and makes the calls of the C ABI; it holds no arithmetic.
"""
from __future__ import annotations

from typing import Optional

import torch

from . import binding as B


class NormLinear:
    """out = layer_norm(x) weight^T for x [tokens, d_in]; weight [d_out, d_in]."""

    def __init__(self, tokens: int, d_in: int, d_out: int, dtype: torch.dtype = torch.bfloat16, eps: float = 1e-5,
                 device: str | torch.device = "cuda"):
        if tokens < 1 or d_in < 1 or d_out < 1:
            raise ValueError("uq: a layer has at least one token, one input and one output")
        if dtype not in (torch.float32, torch.bfloat16):
            raise ValueError("uq: activations are float32 or bfloat16")
        B.lib()                                     # fail now if the CUDA library is not built
        self.tokens, self.d_in, self.d_out, self.dtype, self.eps = tokens, d_in, d_out, dtype, eps
        empty = lambda *shape, dt=dtype: torch.empty(shape, dtype=dt, device=device)
        mx = lambda rows, cols: B.MxMatrix(rows, cols, device=device)
        self.status = torch.zeros(1, dtype=torch.int32, device=device)
        # kept between the forward and the backward pass
        self.y, self.mean, self.rstd = empty(tokens, d_in), empty(tokens, dt=torch.float32), empty(tokens, dt=torch.float32)
        self.yq, self.yt = mx(tokens, d_in), mx(d_in, tokens)
        self.wq, self.wt = mx(d_out, d_in), mx(d_in, d_out)
        self.out = empty(tokens, d_out)
        self.dyq, self.dyt = mx(tokens, d_out), mx(d_out, tokens)
        self.dx_in, self.dx = empty(tokens, d_in), empty(tokens, d_in)
        self.workspace = empty(max(16, B.uq_layer_norm_workspace_bytes(tokens, d_in)), dt=torch.uint8)
        self.gamma: Optional[torch.Tensor] = None
        self.beta: Optional[torch.Tensor] = None

    @property
    def size(self) -> int:
        """Parameters of the layer, and places that its gradients take in a worker's row."""
        return 2 * self.d_in + self.d_out * self.d_in

    def segments(self):
        """Offsets of the layer's three tensors: the segment table of a Quantizer over this layer alone."""
        return [0, self.d_in, 2 * self.d_in, self.size]

    def _split(self, flat: torch.Tensor, what: str):
        if flat.dim() != 1 or flat.shape[0] < self.size or not flat.is_contiguous():
            raise ValueError(f"uq: {what} must be a contiguous 1-D tensor with >= {self.size} elements")
        d = self.d_in
        return flat[:d], flat[d:2 * d], flat[2 * d:self.size].view(self.d_out, d)

    def load(self, theta: torch.Tensor) -> None:
        """Takes the parameters from their place in theta (binary32): quantizes the weight for both passes.  To be called
        after every update; gamma and beta are read where they lie."""
        if theta.dtype is not torch.float32:
            raise ValueError("uq: theta must be float32")
        self.gamma, self.beta, weight = self._split(theta, "theta")
        B.uq_mx_quantize(weight, 0, 0, self.wq, self.wt, self.status)

    def _loaded(self) -> None:
        if self.gamma is None:
            raise RuntimeError("uq: the layer has no parameters yet (load)")

    def forward(self, x: torch.Tensor) -> torch.Tensor:
        """The training pass: keeps what backward needs.  The result is this object's own buffer."""
        self._loaded()
        B.uq_layer_norm(x, self.gamma, self.beta, self.eps, self.y, self.mean, self.rstd)
        B.uq_mx_quantize(self.y, 0, 0, self.yq, self.yt, self.status)
        B.uq_mx_product(self.yq, self.wq, self.out, None, self.status)
        return self.out

    def infer(self, x: torch.Tensor, out: Optional[torch.Tensor] = None) -> torch.Tensor:
        """The forward pass for any number of rows of up to ``tokens`` (new tokens in serving), in two kernels: the normalised
        rows leave layer norm quantized.  Its binary32 sums may have another order than ``forward``'s (and another one for
        another number of rows), and a value of y that this takes across a border gets the neighbouring code (float32, 20 x 300
        x 4096: 4 of 12 million bytes of codes).  Without ``out`` the result is a part of the buffer that ``forward`` returns."""
        self._loaded()
        n = x.shape[0]
        if not 1 <= n <= self.tokens:
            raise ValueError(f"uq: x must have 1 to {self.tokens} rows")
        q = B.MxMatrix(n, self.d_in, self.yq.codes[:n], self.yq.scales)
        out = self.out[:n] if out is None else out
        B.uq_layer_norm(x, self.gamma, self.beta, self.eps, None, None, None, q, self.status)
        B.uq_mx_product(q, self.wq, out, None, self.status)
        return out

    def backward(self, x: torch.Tensor, dy: torch.Tensor, grad: torch.Tensor, seed: int) -> torch.Tensor:
        """From dy [tokens, d_out] and the x of the last forward: the parameters' gradients into ``grad`` (this layer's place
        in a worker's row of g, float32 or bfloat16), and the input's gradient, this object's own buffer.  ``seed`` keys the
        draws; every worker and every step needs its own."""
        self._loaded()
        dgamma, dbeta, dweight = self._split(grad, "grad")
        B.uq_mx_quantize(dy, seed, 16, self.dyq, self.dyt, self.status)
        B.uq_mx_product(self.dyq, self.wt, self.dx_in, None, self.status)
        B.uq_mx_product(self.dyt, self.yt, dweight, None, self.status)
        B.uq_layer_norm_backward(self.dx_in, x, self.gamma, self.mean, self.rstd, self.dx, dgamma, dbeta, self.workspace)
        return self.dx

    def status_bits(self) -> int:
        """Synchronizes and returns the device status word (0 = clean)."""
        return int(self.status.item())
