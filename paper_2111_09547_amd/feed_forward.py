"""A pre-norm gated feed-forward block on 8-bit floats, for the dense layers around a quantized network:

    s = x + residual        h = act(n.gate') * (n.up'),  n = norm(s)        y = h.down'

Only the calls are put together here; the arithmetic is in the kernels.  Between them activations are in 8-bit floats: a forward
pass is three calls, four launches at most.  For training the block keeps what its backward pass wants."""
from __future__ import annotations

import torch

from . import fp8 as F


def _plain(w: torch.Tensor) -> torch.Tensor:
    return w.detach() if w.requires_grad else w


def _packed(w: torch.Tensor, old: F.Fp8 | None, columns: bool = False) -> F.Fp8:
    rows, cols = reversed(w.shape) if columns else w.shape
    if old is not None and (old.rows, old.cols, old.device) != (rows, cols, w.get_device()):
        old = None
    return F.qgtc_fp8_quantize(_plain(w), columns=columns, out=old)


class GatedFeedForward:
    """norm_weight [D], gate and up [H, D], down [D, H]: float32, float16 or bfloat16 on one device, quantized once by pack().
    training: forward() keeps its intermediate results until backward(), which returns the gradients: parameters may be given, and
    keep theirs to the caller."""

    def __init__(self, norm_weight: torch.Tensor, gate: torch.Tensor, up: torch.Tensor, down: torch.Tensor, eps: float = 1e-6,
                 act: str = "silu", training: bool = False):
        if gate.shape != up.shape or down.shape != (gate.shape[1], gate.shape[0]) or norm_weight.shape != (gate.shape[1],):
            raise ValueError("gate and up: H x D, down: D x H, norm_weight: D")
        self.norm_weight, self.gate, self.up, self.down = norm_weight, gate, up, down
        self.eps, self.act, self.training = eps, act, training
        self._kept = None
        self.gate_q = self.up_q = self.down_q = self.down_t = self.gate_up_t = None
        self.pack()

    def pack(self):
        """Weights into 8-bit floats; to be called again when any of them has changed, or when training has been set on a block that
        was made without.  For training also along the other axis, as the backward pass contracts over it: once a block has those,
        every call brings them up to date, whether it is training then or not.  Weights of the sizes and the device of before go
        where those were, since a recorded pass reads them there: passes on other streams have to be done with them.  What a forward
        pass has kept for backward() is of the weights before, and is let go."""
        self._kept = None
        self.gate_q, self.up_q = _packed(self.gate, self.gate_q), _packed(self.up, self.up_q)
        self.down_q = _packed(self.down, self.down_q)
        if self.training or self.down_t is not None:
            self.down_t = _packed(self.down, self.down_t, columns=True)
            self.gate_up_t = _packed(torch.cat([_plain(self.gate), _plain(self.up)]), self.gate_up_t, columns=True)

    def forward(self, x: torch.Tensor, residual: torch.Tensor | None = None):
        """(y, s) of x [T, D]: the block's result, which the next norm adds to s."""
        n = F.qgtc_rms_norm(x, _plain(self.norm_weight), self.eps, residual=residual, y=self.training, rstd=self.training)
        h = torch.empty((x.shape[0], self.gate.shape[0]), dtype=x.dtype, device=x.device) if self.training else None
        hq = F.qgtc_fp8_gated(n.fp8, self.gate_q, self.up_q, self.act, h=h)
        self._kept = (n, h) if self.training else None
        return F.qgtc_fp8_product(hq, self.down_q, x.dtype), n.sum

    def backward(self, dy: torch.Tensor, dsum: torch.Tensor | None = None) -> dict:
        """Gradients of the last forward() from that of y and, unless None, that of s: of x and of the residual ("x", one for both)
        and of the weights ("norm_weight", "gate", "up", "down": float32).  Quantization counts as the identity.  Until then x (where
        there was no residual) and norm_weight hold what they did: they are read again."""
        if self._kept is None:
            raise RuntimeError("backward() follows a forward() of a block that is training")
        if self.down_t is None:
            raise RuntimeError("the block was packed for forward passes alone: pack() once more")
        n, h = self._kept
        hidden, f32 = self.gate.shape[0], torch.float32
        down = F.qgtc_fp8_product(F.qgtc_fp8_quantize(dy, columns=True), F.qgtc_fp8_quantize(h, columns=True), f32)
        dh = F.qgtc_fp8_product(F.qgtc_fp8_quantize(dy), self.down_t, dy.dtype)
        d = F.qgtc_fp8_gated_backward(n.fp8, self.gate_q, self.up_q, dh, self.act)
        gate_up = F.qgtc_fp8_product(F.qgtc_fp8_quantize(d, columns=True), F.qgtc_fp8_quantize(n.y, columns=True), f32)
        dn = F.qgtc_fp8_product(F.qgtc_fp8_quantize(d), self.gate_up_t, dy.dtype)
        dx, dw = F.qgtc_rms_norm_backward(dn, n.sum, _plain(self.norm_weight), n.rstd, dsum=dsum)
        self._kept = None                                # (a gradient that was refused can be given again)
        return {"x": dx, "norm_weight": dw, "gate": gate_up[:hidden], "up": gate_up[hidden:], "down": down}

    def capture(self, x: torch.Tensor, residual: torch.Tensor | None = None):
        """(graph, y, s): one forward pass on these tensors as a HIP graph; a replay reads what x and residual hold then.
        The graph keeps what it reads."""
        if self.training:
            raise RuntimeError("a block that is training is not recorded")
        stream = torch.cuda.Stream(x.device)
        stream.wait_stream(torch.cuda.current_stream(x.device))
        with torch.cuda.stream(stream):                  # what is done once per kernel is done outside the recording
            self.forward(x, residual)
        torch.cuda.current_stream(x.device).wait_stream(stream)
        with torch.cuda.device(x.device):                # (a recording is on the current device's stream otherwise)
            graph = torch.cuda.CUDAGraph()
            with torch.cuda.graph(graph, stream=stream):
                y, s = self.forward(x, residual)
        graph.reads = (x, residual, self.norm_weight, self.gate_q, self.up_q, self.down_q)
        return graph, y, s
