"""The end of a denoising forward: tokens and confidences of the masked positions.

Only the positions that are still masked need logits.  ``TokenHead`` lists them on the GPU
(``reflex_select_rows``), rounds their hidden states to 8 bits (``reflex_quantize_fp8``, with
integer weights ``reflex_quantize_int8``), multiplies them with the 8-bit head weights
(``reflex_matmul_fp8``, ``reflex_matmul_int8``) and draws a token and its
confidence from each row of logits (``reflex_sample_tokens``).  The host never learns how many
rows there are: nothing is copied back and the launches can be captured.
"""
from __future__ import annotations

from typing import Callable

import torch

from . import _lib
from .layer import quantize_weight


class TokenHead:
    """Buffers and 8-bit weights of a head for T positions.

    weight: bf16 [V, d], rounded to 8 bits here, or a pair of codes and scales as
    ``quantize_weight`` or ``quantize_weight_int8`` gives them.  tokens int32 [T] and conf float32 [T] hold the last
    prediction at every position: -1 and 0 until there is one, and from the forward that
    commits a position on what that forward predicted.  logits: [T, V], the masked positions'
    rows in front (room for all of them: 4.3 GB for 8192 positions of 131072 tokens in fp32)."""

    def __init__(self, T: int, weight, temperature: float = 0.0, top_k: int = 0, top_p: float = 1.0,
                 min_p: float = 0.0, logits_dtype=torch.float32):
        self.w, self.w_scale = weight if isinstance(weight, (tuple, list)) else quantize_weight(weight)
        V, d = self.w.shape
        self.T, self.d, self.V = int(T), d, V
        self.params = _lib.SampleParamsC(temperature, top_k, top_p, min_p)
        dev = self.w.device
        self.rows = torch.empty(T, dtype=torch.int32, device=dev)
        self.n_rows = torch.zeros(1, dtype=torch.int32, device=dev)
        self.integers = self.w.dtype == torch.int8
        if self.integers:
            self.q = torch.empty((T, d), dtype=torch.int8, device=dev)
            self.scale = torch.empty(T, dtype=torch.float32, device=dev)
        else:
            self.q = torch.empty((T, d), dtype=torch.float8_e4m3fn, device=dev)
            self.scale = torch.empty(_lib.fp8_scale_shape(T, d), dtype=torch.uint8, device=dev)
        self.logits = torch.empty((T, V), dtype=logits_dtype, device=dev)
        self.tokens = torch.full((T,), -1, dtype=torch.int32, device=dev)
        self.conf = torch.zeros(T, dtype=torch.float32, device=dev)
        nbytes = max(_lib.reflex_select_rows_workspace_size(T), _lib.reflex_sample_workspace_size(T, V), 256)
        self.ws = torch.empty(nbytes, dtype=torch.uint8, device=dev)

    def forward(self, x: torch.Tensor, masked: torch.Tensor, u: torch.Tensor, stream=None):
        """x: hidden states bf16 [T, d]; masked: uint8 or bool [T]; u: float32 [T] in [0, 1).
        Updates and returns (tokens, conf)."""
        if tuple(x.shape) != (self.T, self.d) or masked.shape[0] != self.T:
            raise ValueError(f"TokenHead: x {tuple(x.shape)} and masked {tuple(masked.shape)} "
                             f"for {self.T} positions of {self.d}")
        _lib.reflex_select_rows(masked, self.rows, self.n_rows, ws=self.ws, stream=stream)
        quantize = _lib.reflex_quantize_int8 if self.integers else _lib.reflex_quantize_fp8
        multiply = _lib.reflex_matmul_int8 if self.integers else _lib.reflex_matmul_fp8
        quantize(x, self.q, self.scale, self.rows, self.n_rows, stream=stream)
        multiply(self.q, self.scale, self.w, self.w_scale, self.logits, self.n_rows, stream=stream)
        _lib.reflex_sample_tokens(self.logits, u, self.params, self.tokens, self.conf, self.rows, self.n_rows,
                                  ws=self.ws, stream=stream)
        return self.tokens, self.conf

    def confidence(self, x: torch.Tensor, masked: torch.Tensor,
                   uniform: Callable[[int], torch.Tensor]) -> Callable[[int], torch.Tensor]:
        """For ``run_trajectory``: forward t's confidences from the hidden states x (the layer's
        output buffer) and the uniform numbers uniform(t)."""
        return lambda t: self.forward(x, masked, uniform(t))[1]
