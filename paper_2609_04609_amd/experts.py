"""A layer of experts over weights that the codec has brought up to date.

    y[t] = sum_s w[t, s] W[e[t, s]] x[t]        W[e]: n_out x n_in

with the experts e[t, :] and weights w[t, :] of a router's logits and every
product in 8 bits (e4m3 with a power-of-two scale per block of 128). The layer
owns its buffers and runs the operators of the C ABI in turn; it allocates
nothing after its construction, so load(), forward() and backward() may be
captured into a graph. One call at a time: forward() leaves in the buffers
what backward() reads, and every call writes the same outputs again.

  load(w)      W, and its transpose for backward(), to 8 bits by blocks of
               128 x 128: weights change once a step and are read for every token
  forward()    choose experts, sort the (token, slot) pairs by expert, put each
               token's 8-bit row where its pairs are, multiply, and sum a token's
               rows with its weights
  backward()   the rows' and the weights' gradients; the rows' in 8 bits times the
               transposed weights, summed over a token's slots, is x's gradient; the
               products over an expert's tokens are W's; the weights' gradient
               through the choice's scores is the logits'

Rounding to 8 bits counts as the identity in backward(), and the choice as fixed.
"""
from __future__ import annotations

import torch

from . import ciera


def _shape(t, name, *shape):
    if t.shape != shape:
        raise ValueError(f"{name} has shape {tuple(t.shape)}, not {shape}")


def _inputs(*args):
    """Check (tensor, name, types, shape) of rows that may be apart, so that a
    call refuses them before its first operator runs."""
    for t, name, _, shape in args:
        _shape(t, name, *shape)
    dev = ciera._device(args[0][0], args[0][1])
    if not all(ciera._strided(t, dev, types, shape)
               for t, _, types, shape in args):
        ciera._refuse(dev, *(a + (ciera._strided,) for a in args))


class ExpertLayer:
    """``top_k`` of ``n_experts`` experts of [n_out, n_in] weights for
    ``n_tokens`` tokens of ``dtype``; ``choice`` are the keywords of
    ciera.route_t (sigmoid, normalize, scale, groups, ...). With ``train`` there
    are buffers for backward() too; ``grad_dtype`` is the weights' gradients'
    type, the layer's if None."""

    def __init__(self, n_tokens, top_k, n_experts, n_out, n_in,
                 dtype=torch.bfloat16, device="cuda", train=True,
                 grad_dtype=None, **choice):
        T, k, E, N, C = n_tokens, top_k, n_experts, n_out, n_in
        if min(T, k, E, N, C) < 1:
            raise ValueError("a layer needs tokens, experts and values")
        if dtype not in ciera._WIDE:
            raise ValueError(f"dtype is {dtype}")
        if grad_dtype is None:
            grad_dtype = dtype
        elif grad_dtype not in ciera._WIDE:
            raise ValueError(f"grad_dtype is {grad_dtype}")
        P = T * k
        self.T, self.k, self.E, self.N, self.C = T, k, E, N, C
        self.train, self.choice = train, choice

        def new(*shape, dtype=dtype):
            return torch.empty(shape, dtype=dtype, device=device)

        def eight(*shape):
            return new(*shape, dtype=torch.float8_e4m3fn)

        def scales(*shape):
            return new(*shape, dtype=torch.uint8)

        i32, f32 = torch.int32, torch.float32
        self.ws = ciera.PlanWorkspace(T, k, E, device)
        self.ids, self.weights = new(T, k, dtype=i32), new(T, k, dtype=f32)
        self.offsets = new(E + 1, dtype=i32)
        self.source, self.position = new(P, dtype=i32), new(T, k, dtype=i32)
        (_, Cq), (_, Cs) = ciera.quantized_shapes(P, C)
        (_, Nq), (_, Ns) = ciera.quantized_shapes(P, N)
        nb, cb = Nq // 128, Cq // 128
        self.w, self.w_scales = eight(E, N, Cq), scales(E, nb, Cs)
        self.w_t = self.w_t_scales = None
        self.x, self.x_scales = eight(P, Cq), scales(P, Cs)
        self.rows, self.out = new(P, N), new(T, N)
        if not train:
            return
        self.w_t, self.w_t_scales = eight(E, C, Nq), scales(E, cb, Ns)
        self.d_rows, self.d_weights = new(P, N), new(T, k, dtype=f32)
        self.dy, self.dy_scales = eight(P, Nq), scales(P, Ns)
        self.d_x_rows, self.d_x = new(P, C), new(T, C)
        L = ciera.ciera_columns_length(P, E)
        (_, _), (_, Ls) = ciera.quantized_shapes(1, L)
        self.dy_t, self.dy_t_scales = eight(N, L), scales(N, Ls)
        self.x_t, self.x_t_scales = eight(C, L), scales(C, Ls)
        self.d_w = new(E, N, C, dtype=grad_dtype)
        # the logits' gradient has their type, which need not be the tokens'
        room = new(T * E, dtype=f32)
        self._d_logits = {t: room.view(t)[:T * E].view(T, E)
                          for t in (torch.bfloat16, torch.float16, f32)}
        self.d_logits = self._d_logits[dtype]

    def load(self, w):
        """Take the weights ``w`` [n_experts, n_out, n_in]."""
        _shape(w, "w", self.E, self.N, self.C)
        ciera.quantize_blocks_t(w, self.w, self.w_scales, self.w_t,
                                self.w_t_scales)

    def forward(self, x, logits, bias=None):
        """``x`` [n_tokens, n_in] and the router's ``logits`` [n_tokens,
        n_experts], each of any wide type -> the layer's output, [n_tokens,
        n_out]."""
        _inputs((x, "x", ciera._WIDE, (self.T, self.C)),
                (logits, "logits", ciera._WIDE, (self.T, self.E)))
        ciera.route_t(logits, self.ids, self.weights, bias, **self.choice)
        ciera.route_plan_t(self.ids, self.E, self.offsets, self.source,
                           self.position, self.ws)
        ciera.quantize_rows_t(x, self.x, self.x_scales, self.position)
        ciera.expert_matmul_t(self.x, self.x_scales, self.w, self.w_scales,
                              self.offsets, self.rows)
        ciera.combine_t(self.rows, self.position, self.out, self.weights)
        return self.out

    def backward(self, d_out, x, logits):
        """Gradient of the output that forward() gave for ``x`` and ``logits``
        -> gradients of x (of the layer's type), of the weights (of grad_dtype) and
        of the logits (of their type)."""
        if not self.train:
            raise ValueError("a layer without train has no backward")
        _inputs((d_out, "d_out", (self.out.dtype,), (self.T, self.N)),
                (x, "x", ciera._WIDE, (self.T, self.C)),
                (logits, "logits", ciera._WIDE, (self.T, self.E)))
        self.d_logits = self._d_logits[logits.dtype]
        ciera.combine_backward_t(d_out, self.rows, self.weights,
                                 self.position, self.d_rows, self.d_weights)
        ciera.quantize_rows_t(self.d_rows, self.dy, self.dy_scales)
        ciera.expert_matmul_t(self.dy, self.dy_scales, self.w_t,
                              self.w_t_scales, self.offsets, self.d_x_rows)
        ciera.combine_t(self.d_x_rows, self.position, self.d_x)
        ciera.quantize_columns_t(self.d_rows, self.offsets, self.dy_t,
                                 self.dy_t_scales)
        ciera.quantize_columns_t(x, self.offsets, self.x_t, self.x_t_scales,
                                 self.source, self.k)
        ciera.expert_weight_grad_t(self.dy_t, self.dy_t_scales, self.x_t,
                                   self.x_t_scales, self.offsets, self.d_w)
        own = {key: self.choice[key]
               for key in ("sigmoid", "normalize", "scale")
               if key in self.choice}
        ciera.route_backward_t(logits, self.ids, self.d_weights,
                               self.d_logits, **own)
        return self.d_x, self.d_w, self.d_logits
