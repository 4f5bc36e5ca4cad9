"""Device buffers for one MoE layer and the call sequence of one step.

Torch provides device memory and the stream; every computation is a call
into libmoe.so through :mod:`paper_2609_36070_amd.binding`.
"""
from __future__ import annotations

import numpy as np
import torch

from . import binding as B
from .workloads import Workload


def _empty(shape, dtype, device):
    """Uninitialised tensor whose data pointer is valid even when it has no elements."""
    n = int(np.prod(shape))
    return torch.empty((max(n, 1),), dtype=dtype, device=device)[:n].view(*shape)


def _dev_bf16(a, device):
    if a is None:
        return None
    a = np.ascontiguousarray(a, np.float32)
    out = _empty(a.shape, torch.bfloat16, device)
    if a.size:
        out.copy_(torch.from_numpy(a).to(torch.bfloat16))
    return out


class DeviceLayer:
    """All tensors of one layer instance on the GPU, laid out as the C ABI expects."""

    def __init__(self, w: Workload, inputs: dict, device="cuda", with_backward=None, mx=False,
                 ring_rows=None, mx_wgrad=False, routing=None, int8=False, few=False):
        """ring_rows: run forward/backward in bounded memory, with the per-route
        activations in a ring of that many rows (None: room for all T*k routes).
        mx_wgrad: the MXFP8 backward computes its weight gradients in MXFP8.
        routing: route by scores (a MoeRouting), with inputs["balance"] if given.
        int8: the experts in 8-bit integers too (forward_int, step_int).
        few: up to 16 tokens in two launches too (step_few); for inference, without a
        backward."""
        self.w = w
        self.mx = mx
        self.routing = routing
        self.int8 = int8
        self.mx_wgrad = bool(mx_wgrad)
        self.ring_rows = ring_rows
        self.device = torch.device(device)
        self.with_backward = w.backward if with_backward is None else with_backward
        T, d, E, k, f, fs = w.T, w.d, w.E, w.k, w.f, w.f_s
        dev = self.device
        self.shape = B.make_shape(T, d, E, k, f, fs)
        self.X = _dev_bf16(inputs["X"], dev)
        self.W_r = _dev_bf16(inputs["W_r"], dev)
        self.bias = None if inputs.get("bias") is None else \
            torch.from_numpy(np.asarray(inputs["bias"], np.float32)).to(dev)
        self.balance = None if inputs.get("balance") is None else \
            torch.from_numpy(np.asarray(inputs["balance"], np.float32)).to(dev)
        if routing is None and self.balance is not None:
            raise ValueError("a balance belongs to routing by scores")
        self.W_gate = _dev_bf16(inputs["W_gate"], dev)
        self.W_up = _dev_bf16(inputs["W_up"], dev)
        self.W_down = _dev_bf16(inputs["W_down"], dev)
        self.Wg_s = _dev_bf16(inputs.get("Wg_s"), dev)
        self.Wu_s = _dev_bf16(inputs.get("Wu_s"), dev)
        self.Wd_s = _dev_bf16(inputs.get("Wd_s"), dev)
        self.dY = _dev_bf16(inputs.get("dY"), dev) if self.with_backward else None

        i32, f32, bf = torch.int32, torch.float32, torch.bfloat16
        R = T * k
        self.logits = _empty((T, E), f32, dev)
        self.topk_idx = _empty((T, k), i32, dev)
        self.topk_w = _empty((T, k), f32, dev)
        self.counts = _empty((E,), i32, dev)
        self.offsets = _empty((E + 1,), i32, dev)
        self.perm = _empty((R,), i32, dev)
        self.route_pos = _empty((R,), i32, dev)
        self.Y = _empty((T, d), bf, dev)
        if ring_rows is None:
            nbytes = B.moe_workspace_bytes(self.shape, self.with_backward)
        else:
            if mx:
                raise ValueError("the MXFP8 forward has no bounded-memory variant")
            nbytes = B.moe_ring_workspace_bytes(self.shape, ring_rows, self.with_backward)
        if nbytes == 0:
            raise ValueError(f"unsupported shape {w}")
        if mx:
            mx_bytes = B.moe_mx_workspace_bytes(
                self.shape, (2 if self.mx_wgrad else 1) if self.with_backward else 0)
            if mx_bytes == 0:
                raise ValueError(f"shape unsupported in MXFP8 {w}")
            nbytes = max(nbytes, mx_bytes)
        if int8:
            if ring_rows is not None:
                raise ValueError("the int8 forward has no bounded-memory variant")
            int_bytes = B.moe_int_workspace_bytes(self.shape)
            if int_bytes == 0:
                raise ValueError(f"shape unsupported in int8 {w}")
            nbytes = max(nbytes, int_bytes)
        if few:
            self._no_backward()
            few_bytes = B.moe_few_workspace_bytes(self.shape)
            if few_bytes == 0:
                raise ValueError(f"not a shape of a few tokens {w}")
            nbytes = max(nbytes, few_bytes)
        self.ws = torch.empty((nbytes,), dtype=torch.uint8, device=dev)
        self.weights = B.weights_struct(self.W_gate, self.W_up, self.W_down,
                                        self.Wg_s, self.Wu_s, self.Wd_s)
        self.plan_bufs = B.plan_bufs(self.counts, self.offsets, self.perm, self.route_pos)
        if self.with_backward:
            self.dX = _empty((T, d), bf, dev)
            self.dW_gate = torch.empty((E, d, f), dtype=f32, device=dev)
            self.dW_up = torch.empty((E, d, f), dtype=f32, device=dev)
            self.dW_down = torch.empty((E, f, d), dtype=f32, device=dev)
            self.dW_r = torch.empty((d, E), dtype=f32, device=dev)
            self.dZ = _empty((T, E), f32, dev)
            if fs:
                self.dWg_s = torch.empty((d, fs), dtype=f32, device=dev)
                self.dWu_s = torch.empty((d, fs), dtype=f32, device=dev)
                self.dWd_s = torch.empty((fs, d), dtype=f32, device=dev)
            else:
                self.dWg_s = self.dWu_s = self.dWd_s = None
            self.grads = B.grads_struct(self.dW_gate, self.dW_up, self.dW_down, self.dW_r, self.dZ,
                                        self.dWg_s, self.dWu_s, self.dWd_s)

        if mx:
            u8 = torch.uint8
            self.Wg_q = torch.empty((E, f, d), dtype=u8, device=dev)
            self.Wu_q = torch.empty((E, f, d), dtype=u8, device=dev)
            self.Wd_q = torch.empty((E, d, f), dtype=u8, device=dev)
            self.Wg_sc = torch.empty((E, f, d // 32), dtype=u8, device=dev)
            self.Wu_sc = torch.empty((E, f, d // 32), dtype=u8, device=dev)
            self.Wd_sc = torch.empty((E, d, f // 32), dtype=u8, device=dev)
            self.mx_weights = B.mx_weights_struct(self.Wg_q, self.Wu_q, self.Wd_q, self.Wg_sc,
                                                  self.Wu_sc, self.Wd_sc)
            if self.with_backward:
                # backward layouts: each weight row quantised along its own axis
                self.Wg_qb = torch.empty((E, d, f), dtype=u8, device=dev)
                self.Wu_qb = torch.empty((E, d, f), dtype=u8, device=dev)
                self.Wd_qb = torch.empty((E, f, d), dtype=u8, device=dev)
                self.Wg_scb = torch.empty((E, d, f // 32), dtype=u8, device=dev)
                self.Wu_scb = torch.empty((E, d, f // 32), dtype=u8, device=dev)
                self.Wd_scb = torch.empty((E, f, d // 32), dtype=u8, device=dev)
                self.mx_bwd_weights = B.mx_bwd_weights_struct(self.Wg_qb, self.Wu_qb, self.Wd_qb,
                                                              self.Wg_scb, self.Wu_scb, self.Wd_scb)
            self.quantize_mx()

        if int8:
            def codes(*size):
                return torch.empty(size, dtype=torch.int8, device=dev)

            def scales(*size):
                return torch.empty(size, dtype=torch.float32, device=dev)

            self.int_bufs = [codes(E, f, d), codes(E, f, d), codes(E, d, f),
                             scales(E, f), scales(E, f), scales(E, d)]
            if fs:
                self.int_bufs += [codes(fs, d), codes(fs, d), codes(d, fs), scales(fs), scales(fs), scales(d)]
            self.int_weights = B.int_weights_struct(*self.int_bufs)
            self.quantize_int()

    # -- the four calls of the path --------------------------------------
    def route(self, stream=None):
        if self.routing is not None:
            B.moe_route_scored(self.shape, self.routing, self.X, self.W_r, self.bias, self.balance,
                               self.logits, self.topk_idx, self.topk_w, self.ws, stream=stream)
            return
        B.moe_route(self.shape, self.X, self.W_r, self.bias, self.logits, self.topk_idx,
                    self.topk_w, self.ws, stream=stream)

    def plan(self, stream=None):
        B.moe_plan(self.shape, self.topk_idx, self.plan_bufs, self.ws, stream=stream)

    def forward(self, save_for_backward=None, stream=None, events=None):
        save = self.with_backward if save_for_backward is None else save_for_backward
        if self.ring_rows is not None:
            if events is not None:
                raise ValueError("stage events are not recorded in bounded-memory execution")
            B.moe_forward_ring(self.shape, self.X, self.weights, self.topk_idx, self.topk_w,
                               self.plan_bufs, self.Y, self.ring_rows, save, self.ws,
                               stream=stream)
            return
        B.moe_forward(self.shape, self.X, self.weights, self.topk_idx, self.topk_w,
                      self.plan_bufs, self.Y, save, self.ws, stream=stream, events=events)

    def forward_fused(self, save_for_backward=None, stream=None):
        """The forward as one persistent launch (same results as forward())."""
        if self.ring_rows is not None:
            raise ValueError("the fused forward has no bounded-memory variant")
        save = self.with_backward if save_for_backward is None else save_for_backward
        B.moe_forward_fused(self.shape, self.X, self.weights, self.topk_idx, self.topk_w,
                            self.plan_bufs, self.Y, save, self.ws, stream=stream)

    def backward(self, stream=None, events=None):
        if self.ring_rows is not None:
            if events is not None:
                raise ValueError("stage events are not recorded in bounded-memory execution")
            if self.routing is not None:
                B.moe_backward_ring_scored(self.shape, self.routing, self.logits, self.balance, self.dY,
                                           self.X, self.W_r, self.weights, self.topk_idx, self.topk_w,
                                           self.plan_bufs, self.dX, self.grads, self.ring_rows, self.ws,
                                           stream=stream)
                return
            B.moe_backward_ring(self.shape, self.dY, self.X, self.W_r, self.weights,
                                self.topk_idx, self.topk_w, self.plan_bufs, self.dX, self.grads,
                                self.ring_rows, self.ws, stream=stream)
            return
        if self.routing is not None:
            B.moe_backward_scored(self.shape, self.routing, self.logits, self.balance, self.dY, self.X,
                                  self.W_r, self.weights, self.topk_idx, self.topk_w, self.plan_bufs,
                                  self.dX, self.grads, self.ws, stream=stream, events=events)
            return
        B.moe_backward(self.shape, self.dY, self.X, self.W_r, self.weights, self.topk_idx,
                       self.topk_w, self.plan_bufs, self.dX, self.grads, self.ws, stream=stream,
                       events=events)

    def quantize_mx(self, stream=None):
        """Pre-quantise the routed weights to MXFP8 (once per weight update)."""
        B.moe_mx_quantize_weights(self.shape, self.weights, self.mx_weights, stream=stream)
        if self.with_backward:
            B.moe_mx_quantize_weights_bwd(self.shape, self.weights, self.mx_bwd_weights,
                                          stream=stream)

    def forward_mx(self, stream=None, events=None, save_for_backward=None):
        save = self.with_backward if save_for_backward is None else save_for_backward
        B.moe_forward_mx(self.shape, self.X, self.weights, self.mx_weights, self.topk_idx,
                         self.topk_w, self.plan_bufs, self.Y, self.ws, stream=stream,
                         events=events, save_for_backward=save)

    def backward_mx(self, stream=None):
        if self.routing is not None:
            B.moe_backward_mx_scored(self.shape, self.routing, self.logits, self.balance, self.dY, self.X,
                                     self.W_r, self.weights, self.mx_bwd_weights, self.topk_idx,
                                     self.topk_w, self.plan_bufs, self.dX, self.grads, self.ws,
                                     stream=stream, wgrad_mxfp8=self.mx_wgrad)
            return
        B.moe_backward_mx(self.shape, self.dY, self.X, self.W_r, self.weights, self.mx_bwd_weights,
                          self.topk_idx, self.topk_w, self.plan_bufs, self.dX, self.grads, self.ws,
                          stream=stream, wgrad_mxfp8=self.mx_wgrad)

    def quantize_int(self, stream=None):
        """Quantise the routed and shared weights to int8 (once per weight update)."""
        B.moe_int_quantize_weights(self.shape, self.weights, self.int_weights, stream=stream)

    def forward_int(self, stream=None, events=None):
        B.moe_forward_int(self.shape, self.X, self.int_weights, self.topk_idx, self.topk_w,
                          self.plan_bufs, self.Y, self.ws, stream=stream, events=events)

    def _no_backward(self):
        if self.with_backward:
            raise ValueError("the few-token path leaves nothing for a backward: the layer has to be without one")

    def step_few(self, stream=None):
        """Route, plan and forward of up to 16 tokens in two launches (inference: no plan and no activations
        are left, and the workspace is written over)."""
        self._no_backward()
        B.moe_forward_few(self.shape, B.routing() if self.routing is None else self.routing, self.X, self.W_r,
                          self.bias, self.balance, self.weights, self.logits, self.topk_idx, self.topk_w,
                          self.Y, self.ws, stream=stream)

    def step_int(self, stream=None, fwd_events=None):
        """Route, plan and the int8 forward."""
        self.route(stream)
        self.plan(stream)
        self.forward_int(stream=stream, events=fwd_events)

    def step_mx(self, stream=None, fwd_events=None):
        """Route, plan, the MXFP8 forward (and the MXFP8 backward)."""
        self.route(stream)
        self.plan(stream)
        self.forward_mx(stream=stream, events=fwd_events)
        if self.with_backward:
            self.backward_mx(stream)

    def step(self, stream=None, fwd_events=None, bwd_events=None):
        """One pass of the whole path: route, plan, forward (and backward)."""
        self.route(stream)
        self.plan(stream)
        self.forward(stream=stream, events=fwd_events)
        if self.with_backward:
            self.backward(stream, events=bwd_events)

    # -- inspection -------------------------------------------------------
    def ws_tensor(self, which, dtype, shape):
        if self.ring_rows is not None and which != B.WS_ERROR:
            raise ValueError("named regions describe the one-pass layout only")
        off, nbytes = B.moe_workspace_region(self.shape, self.with_backward, which)
        return self.ws[off:off + nbytes].view(dtype).view(*shape)

    def mx_ws_tensor(self, which, dtype, shape):
        off, nbytes = B.moe_mx_workspace_region(self.shape, which)
        return self.ws[off:off + nbytes].view(dtype).view(*shape)

    def error_word(self) -> int:
        return int(self.ws_tensor(B.WS_ERROR, torch.int32, (1,)).item())


class DeviceBlock:
    """A layer between the norms of a residual block, on the GPU:

        h0 = N(x), y = layer(h0), r = x + scale gate token_gate dropout(N_y(y)), h = N_r(r)

    r goes on as the stream and h into the next block.  The layer's inputs["X"] is
    the stream x; params holds numpy arrays: in_weight and in_bias of the first
    norm, and those of the join (binding.JOIN_PARAMS), each optional.  With up
    to 16 tokens, no backward and no ring_rows the layer runs as step_few.
    layer_options are DeviceLayer's; the experts run in bf16, and mx, mx_wgrad and
    int8 are refused."""

    def __init__(self, w: Workload, inputs: dict, params: dict | None = None, stream="bf16", in_norm="rms",
                 y_norm="none", r_norm="rms", eps=1e-6, scale=1.0, drop=0.0, seed=0, device="cuda",
                 with_backward=None, **layer_options):
        params = params or {}
        unknown = sorted(set(params) - {"in_weight", "in_bias", *B.JOIN_PARAMS})
        if unknown:
            raise ValueError(f"no parameters of a block: {unknown}")
        other = sorted(n for n in ("mx", "mx_wgrad", "int8") if layer_options.get(n))
        if other:
            raise ValueError(f"a block's experts are in bf16: {other}")
        backward = w.backward if with_backward is None else with_backward
        self.few = not backward and 0 < w.T <= 16 and layer_options.get("ring_rows") is None
        self.layer = L = DeviceLayer(w, inputs, device, with_backward=backward, few=self.few, **layer_options)
        dev, T, d = L.device, w.T, w.d
        kind = torch.float32 if stream == "f32" else torch.bfloat16
        up = {n: None if v is None else torch.from_numpy(np.ascontiguousarray(v, np.float32)).to(dev)
              for n, v in params.items()}
        self.x = _empty((T, d), kind, dev)
        if T:
            self.x.copy_(torch.from_numpy(np.ascontiguousarray(inputs["X"], np.float32)).to(kind))
        self.first = B.join(T, d, stream, "none", in_norm, r_eps=eps)
        self.first_tensors = dict(r_weight=up.get("in_weight"), r_bias=up.get("in_bias"))
        self.join = B.join(T, d, stream, y_norm, r_norm, eps, eps, scale, drop)
        self.tensors = {n: up.get(n) for n in B.JOIN_PARAMS}
        self.first_params = B.join_params(**self.first_tensors)
        self.params = B.join_params(**self.tensors)
        # seed and offset; a program moves the offset on from step to step
        self.rng = torch.tensor([seed, 0], dtype=torch.int64, device=dev) if self.join.drop >= 2.0 ** -17 else None
        self.r, self.h = _empty((T, d), kind, dev), _empty((T, d), torch.bfloat16, dev)
        self.first_stats = self.stats = None
        if backward:
            self.first_stats, self.stats = (_empty((T, 4), torch.float32, dev) for _ in range(2))
            self.dr, self.dx = _empty((T, d), kind, dev), _empty((T, d), kind, dev)
            self.dh, L.dY = (_empty((T, d), torch.bfloat16, dev) for _ in range(2))
            self.first_grads, self.grads = ({n: torch.empty_like(v) for n, v in t.items() if v is not None}
                                            for t in (self.first_tensors, self.tensors))
            self.first_grads_struct = B.join_grads(**self.first_grads)
            self.grads_struct = B.join_grads(**self.grads)
            nbytes = max(B.moe_join_workspace_bytes(j) for j in (self.first, self.join))
            self.ws = torch.empty((nbytes,), dtype=torch.uint8, device=dev)

    def forward(self, stream=None):
        L = self.layer
        B.moe_join_forward(self.first, self.x, None, self.first_params, None, None, L.X, self.first_stats,
                           stream=stream)
        if self.few:
            L.step_few(stream)
        else:
            L.route(stream)
            L.plan(stream)
            L.forward(stream=stream)
        B.moe_join_forward(self.join, self.x, L.Y, self.params, self.rng, self.r, self.h, self.stats,
                           stream=stream)

    def backward(self, stream=None):
        """From dr and dh to dx (the gradient of x, through the stream and the layer), the layer's gradients
        and those of the norms and gates (grads, first_grads)."""
        L = self.layer
        B.moe_join_backward(self.join, L.Y, self.r, self.stats, self.params, self.rng, self.dr, self.dh,
                            self.dx, L.dY, self.grads_struct, self.ws, stream=stream)
        L.backward(stream)
        B.moe_join_backward(self.first, None, self.x, self.first_stats, self.first_params, None, self.dx, L.dX,
                            self.dx, None, self.first_grads_struct, self.ws, stream=stream)
