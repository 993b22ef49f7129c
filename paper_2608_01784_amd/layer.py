"""The fused variable-K MoE layer (``reflex_moe_forward``) from torch tensors.

This module only allocates device buffers with torch and fills the C argument
struct; every step of the layer runs in the HIP kernels of libreflex.
"""
from __future__ import annotations

from dataclasses import dataclass
from typing import Optional

import torch

from . import _lib


@dataclass
class TokenState:
    """Per-token decoding state of one denoising forward (device tensors).

    block_idx int32 [T] (prompt = 0), masked uint8 [T], hist_len int8 [T],
    conf_prev1 / conf_prev2 float32 [T], seq_offsets int32 [B+1], active_block int32 [B].
    """
    block_idx: torch.Tensor
    masked: torch.Tensor
    hist_len: torch.Tensor
    conf_prev1: torch.Tensor
    conf_prev2: torch.Tensor
    seq_offsets: torch.Tensor
    active_block: torch.Tensor


@dataclass
class ExpertWeights:
    """bf16 expert weights: w_gate, w_up [E, f, d]; w_down [E, d, f]; router fp32 [E, d];
    optional shared expert (ws_gate, ws_up [fs, d], ws_down [d, fs])."""
    w_gate: torch.Tensor
    w_up: torch.Tensor
    w_down: torch.Tensor
    w_router: torch.Tensor
    router_bias: Optional[torch.Tensor] = None
    ws_gate: Optional[torch.Tensor] = None
    ws_up: Optional[torch.Tensor] = None
    ws_down: Optional[torch.Tensor] = None

    @property
    def E(self):
        return self.w_router.shape[0]

    @property
    def f(self):
        return self.w_gate.shape[1]

    @property
    def f_shared(self):
        return 0 if self.ws_gate is None else self.ws_gate.shape[0]


class MoELayer:
    """Holds the workspace and output buffers for repeated fused forwards of one shape."""

    def __init__(self, T: int, d: int, weights: ExpertWeights, params, uniform_k: int = 0,
                 norm_topk: int = 1, k_rule: int = 0, k_threshold: float = 0.0, device="cuda"):
        """k_rule: 0 = REFLEX budget; 1 = Top-p, 2 = Expert-Threshold with k_threshold
        (counts bounded by params.k_min, params.k_max)."""
        self.T, self.d, self.w = T, d, weights
        self.params = params
        self.uniform_k = int(uniform_k)
        self.norm_topk = int(norm_topk)
        self.k_rule, self.k_threshold = int(k_rule), float(k_threshold)
        self.kcap = self.uniform_k if self.uniform_k > 0 else int(params.k_max)
        nbytes = self._workspace_bytes()
        if nbytes == 0 and T > 0:
            raise ValueError("unsupported layer shape")
        self.ws = torch.empty(max(nbytes, 256), dtype=torch.uint8, device=device)
        self.out = torch.empty((T, d), dtype=torch.bfloat16, device=device)
        self.k = torch.empty(T, dtype=torch.int32, device=device)
        self.pairs = torch.empty(1, dtype=torch.int32, device=device)
        self.logits = torch.empty((T, weights.E), dtype=torch.float32, device=device)

    def _workspace_bytes(self) -> int:
        w = self.w
        return _lib.reflex_workspace_size(self.T, w.E, self.d, w.f, w.f_shared, self.kcap)

    def args(self, h: torch.Tensor, state: Optional[TokenState] = None,
             k_in: Optional[torch.Tensor] = None, residual_a=None, residual_b=None,
             out: Optional[torch.Tensor] = None) -> _lib.MoeArgsC:
        w = self.w
        a = _lib.MoeArgsC()
        a.T, a.d, a.E, a.f, a.f_shared = self.T, self.d, w.E, w.f, w.f_shared
        a.norm_topk, a.uniform_k = self.norm_topk, self.uniform_k
        a.k_rule, a.k_threshold = self.k_rule, self.k_threshold
        P = _lib.ptr
        a.h, a.w_gate, a.w_up, a.w_down = P(h), P(w.w_gate), P(w.w_up), P(w.w_down)
        a.ws_gate, a.ws_up, a.ws_down = P(w.ws_gate), P(w.ws_up), P(w.ws_down)
        a.w_router, a.router_bias = P(w.w_router), P(w.router_bias)
        if state is not None:
            a.B = state.active_block.shape[0]
            a.block_idx, a.seq_offsets, a.active_block = (P(state.block_idx), P(state.seq_offsets),
                                                          P(state.active_block))
            a.masked, a.hist_len = P(state.masked), P(state.hist_len)
            a.conf_prev1, a.conf_prev2 = P(state.conf_prev1), P(state.conf_prev2)
        a.k_in = P(k_in)
        a.residual_a, a.residual_b = P(residual_a), P(residual_b)
        a.params = _lib.alloc_params(self.params)
        a.out = P(self.out if out is None else out)
        a.k_out, a.pairs_out, a.logits_out = P(self.k), P(self.pairs), P(self.logits)
        return a

    def forward(self, h, state=None, k_in=None, residual_a=None, residual_b=None, out=None,
                stream=None) -> torch.Tensor:
        args = self.args(h, state, k_in, residual_a, residual_b, out)
        _lib.reflex_moe_forward(args, self.ws, stream)
        return self.out if out is None else out


# The forward as written above: a caller that does without the method (because it has made the
# arguments already) compares with this, so that a wrapped or replaced one is still called.
PLAIN_FORWARD = MoELayer.forward


def quantize_weight(w: torch.Tensor, stream=None):
    """Codes and scales of bf16 weights [N, K] or [E, N, K] (``reflex_quantize_fp8_weight``)."""
    q = torch.empty(w.shape, dtype=torch.float8_e4m3fn, device=w.device)
    scale = torch.empty(_lib.fp8_weight_scale_shape(*w.shape), dtype=torch.uint8, device=w.device)
    _lib.reflex_quantize_fp8_weight(w, q, scale, stream=stream)
    return q, scale


@dataclass
class ExpertWeights8:
    """8-bit expert weights, shapes as in ExpertWeights: codes (float8_e4m3fn or uint8) and their
    scales (uint8, ``fp8_weight_scale_shape``); the router stays fp32."""
    w_gate: torch.Tensor
    w_up: torch.Tensor
    w_down: torch.Tensor
    s_gate: torch.Tensor
    s_up: torch.Tensor
    s_down: torch.Tensor
    w_router: torch.Tensor
    router_bias: Optional[torch.Tensor] = None
    ws_gate: Optional[torch.Tensor] = None
    ws_up: Optional[torch.Tensor] = None
    ws_down: Optional[torch.Tensor] = None
    ss_gate: Optional[torch.Tensor] = None
    ss_up: Optional[torch.Tensor] = None
    ss_down: Optional[torch.Tensor] = None

    E = ExpertWeights.E
    f = ExpertWeights.f
    f_shared = ExpertWeights.f_shared

    @classmethod
    def quantize(cls, w: ExpertWeights, stream=None) -> "ExpertWeights8":
        """The bf16 weights rounded to 8 bits (the router is shared, not copied)."""
        made = {"w_router": w.w_router, "router_bias": w.router_bias}
        for name in ("gate", "up", "down"):
            made["w_" + name], made["s_" + name] = quantize_weight(getattr(w, "w_" + name), stream)
            shared = getattr(w, "ws_" + name)
            if shared is not None:
                made["ws_" + name], made["ss_" + name] = quantize_weight(shared, stream)
        return cls(**made)

    def check(self, d: int):
        """Shapes, types, density and device of all weights (the C call sees addresses alone)."""
        where, E, f, fs = "ExpertWeights8", self.E, self.f, self.f_shared
        sets = [("w_", "s_", (E, f, d), (E, d, f))]
        if fs:
            sets.append(("ws_", "ss_", (fs, d), (d, fs)))
        for codes, scales, wide, back in sets:
            for name, shape in (("gate", wide), ("up", wide), ("down", back)):
                w, s = getattr(self, codes + name), getattr(self, scales + name)
                if w is None or s is None:
                    raise ValueError(f"{where}: {codes + name} without all of its tensors")
                _lib.want(where, codes + name, w, _lib.code_types(), shape)
                _lib.want(where, scales + name, s, torch.uint8, _lib.fp8_weight_scale_shape(*shape))
                if w.device != self.w_router.device or s.device != self.w_router.device:
                    raise ValueError(f"{where}: {codes + name} on {w.device}, the router on {self.w_router.device}")
        _lib.want(where, "w_router", self.w_router, torch.float32, (E, d))
        if self.router_bias is not None:
            _lib.want(where, "router_bias", self.router_bias, torch.float32, (E,))
            if self.router_bias.device != self.w_router.device:
                raise ValueError(f"{where}: router_bias on {self.router_bias.device}, the router on "
                                 f"{self.w_router.device}")

    def tensors(self):
        """All tensors, the 8-bit ones in the order of ``reflex_fp8_experts``, and their addresses."""
        all_ = (self.w_gate, self.w_up, self.w_down, self.s_gate, self.s_up, self.s_down, self.ws_gate, self.ws_up,
                self.ws_down, self.ss_gate, self.ss_up, self.ss_down, self.w_router, self.router_bias)
        return all_, tuple(_lib.ptr(t) for t in all_)


class MoELayer8(MoELayer):
    """MoELayer with the experts in 8 bits (``reflex_moe_forward_fp8``): hidden states come in and go
    out in bf16, router, counts, TopK and combine are the same.

    A forward reads the tensors that ``w`` holds then, so weights can be replaced (by ones of the same
    shapes) between forwards.  It checks types, shapes, density and device of all tensors (the C call sees
    addresses alone) and runs on the layer's device, that of the weights."""

    def __init__(self, T: int, d: int, weights: ExpertWeights8, params, uniform_k: int = 0, norm_topk: int = 1,
                 k_rule: int = 0, k_threshold: float = 0.0, device=None):
        weights.check(d)
        at = weights.w_router.device
        if device is not None and torch.empty(0, device=device).device != at:
            raise ValueError(f"MoELayer8: device {device}, but weights on {at}")
        super().__init__(T, d, weights, params, uniform_k, norm_topk, k_rule, k_threshold, at)
        self._sizes = (weights.E, weights.f, weights.f_shared)
        self._set_experts(*weights.tensors())

    def _set_experts(self, tensors, addresses):
        self._checked, self._addresses = tensors, addresses
        self.experts = _lib.Fp8ExpertsC(*addresses[:12])

    def _workspace_bytes(self) -> int:
        w = self.w
        return _lib.reflex_workspace_fp8_size(self.T, w.E, self.d, w.f, w.f_shared, self.kcap)

    def _check(self, h, state, k_in, residual_a, residual_b, out):
        w, where, T = self.w, "MoELayer8", self.T
        tensors, addresses = w.tensors()
        # replaced: other tensors, or the same ones with other memory
        if addresses != self._addresses or any(a is not b for a, b in zip(tensors, self._checked)):
            w.check(self.d)
            if (w.E, w.f, w.f_shared) != self._sizes:
                raise ValueError(f"{where}: weights of (E, f, f_shared) = {(w.E, w.f, w.f_shared)} in a layer made "
                                 f"for {self._sizes}")
            self._set_experts(tensors, addresses)
        at = self.ws.get_device()
        if w.w_router.get_device() != at:
            raise ValueError(f"{where}: weights on {w.w_router.device}, the layer on {self.ws.device}")

        def check(name, t, types, n, width=None):      # (positions may be spread over several dimensions)
            if t.dtype not in types:
                raise TypeError(f"{where}: {name} has element type {t.dtype}, not {types}")
            if t.numel() != n or (width is not None and t.shape[-1] != width):
                of = "" if width is None else f" in rows of {width}"
                raise ValueError(f"{where}: {name} has shape {tuple(t.shape)}, not {n} elements{of}")
            if not t.is_contiguous():
                raise ValueError(f"{where}: {name} is not contiguous")
            if t.get_device() != at:
                raise ValueError(f"{where}: {name} on {t.device}, the layer on {self.ws.device}")
        for name, t in (("h", h), ("residual_a", residual_a), ("residual_b", residual_b), ("out", out)):
            if t is not None or name == "h":
                check(name, t, (torch.bfloat16,), T * self.d, self.d)
        if k_in is not None:
            check("k_in", k_in, (torch.int32,), T)
        if state is not None:
            B = state.active_block.shape[0]
            check("active_block", state.active_block, (torch.int32,), B)
            check("seq_offsets", state.seq_offsets, (torch.int32,), B + 1)
            check("block_idx", state.block_idx, (torch.int32,), T)
            check("masked", state.masked, (torch.uint8, torch.int8, torch.bool), T)
            check("hist_len", state.hist_len, (torch.int8, torch.uint8), T)
            check("conf_prev1", state.conf_prev1, (torch.float32,), T)
            check("conf_prev2", state.conf_prev2, (torch.float32,), T)

    def args(self, h, state=None, k_in=None, residual_a=None, residual_b=None, out=None) -> _lib.MoeArgsC:
        self._check(h, state, k_in, residual_a, residual_b, out)
        a = super().args(h, state, k_in, residual_a, residual_b, out)
        a.w_gate = a.w_up = a.w_down = a.ws_gate = a.ws_up = a.ws_down = None      # (bf16 weights: not read)
        return a

    def forward(self, h, state=None, k_in=None, residual_a=None, residual_b=None, out=None,
                stream=None) -> torch.Tensor:
        args = self.args(h, state, k_in, residual_a, residual_b, out)
        if self.T > 0:      # (empty tensors have no address)
            _lib.reflex_moe_forward_fp8(args, self.experts, self.ws, stream)
        else:               # (the call enqueues nothing)
            self.pairs.zero_()
        return self.out if out is None else out
