"""Device buffers of a workload, the workers' local gradients and the call of the
fused step on them.

Allocation and argument conversion only: the step and the gradients run in the
HIP library through its Python binding (but for the layer's input gradient, a
plain matrix product).
"""
from __future__ import annotations

import torch

import paper_2507_07114_amd as ll

from . import (ADAM, BERNOULLI, MOMENTUM, SGD, Workload, draw_grads, draw_layer_inputs,
               draw_theta0, initial_replicas, torch_dtype)

def loss_spec(w: Workload) -> "ll.LossSpec":
    l = w.loss
    if l["kind"] == BERNOULLI:
        return ll.bernoulli(l["p"], seed=w.seed)
    return ll.gilbert_elliott(l["p_gb"], l["p_bg"], l["loss_good"], l["loss_bad"], seed=w.seed)


def opt_spec(w: Workload, lam: float = 0.0) -> "ll.OptSpec":
    o = w.opt
    if o["kind"] == SGD:
        return ll.sgd(o["lr"], lam)
    if o["kind"] == MOMENTUM:
        return ll.sgd_momentum(o["lr"], o["momentum"], lam)
    return ll.adam(o["lr"], o["beta1"], o["beta2"], o["eps"], lam)


class DeviceState:
    """All device buffers of one workload (rows padded to `ld`)."""

    def __init__(self, w: Workload, device="cuda", pad: int = 0, draw_grads_now=True):
        self.w = w
        self.ld = w.ld(pad)
        self.theta = draw_theta0(w, device)
        self.m = torch.zeros(w.d, dtype=torch.float32, device=device) \
            if w.opt["kind"] in (MOMENTUM, ADAM) else None
        self.v = torch.zeros(w.d, dtype=torch.float32, device=device) \
            if w.opt["kind"] == ADAM else None
        self.replicas = initial_replicas(self.theta, w, ld=self.ld)
        self.grads = torch.zeros((w.n, self.ld), dtype=torch_dtype(w.gdtype), device=device)
        if w.layer:
            self._layer_buffers(device)
        if draw_grads_now:
            if w.layer:
                self.local_gradients(0)
            else:
                draw_grads(w, 0, device=device, ld=self.ld, out=self.grads)
        P = w.num_packets
        self.arrived_g = torch.zeros((w.n, P), dtype=torch.uint8, device=device)
        self.arrived_b = torch.zeros((w.n, P), dtype=torch.uint8, device=device)
        self.counts = torch.zeros(P, dtype=torch.int32, device=device)
        self.ge_g = torch.zeros(w.n, dtype=torch.uint8, device=device)
        self.ge_b = torch.zeros(w.n, dtype=torch.uint8, device=device)
        self.workspace = torch.zeros(max(ll.ll_workspace_bytes(w.n, w.d, w.packet), 256),
                                     dtype=torch.uint8, device=device)
        self.drift = ll.drift_buffer(device)

    def _layer_buffers(self, device):
        w, l = self.w, self.w.layer
        if (l["vocab"] + l["o"]) * l["h"] != w.d:
            raise ValueError(f"{w.name}: a shard of {w.d} elements does not hold its layer")
        dt = torch_dtype(w.gdtype)
        rows, h = (w.n, l["t"]), l["h"]
        self.x = torch.empty((*rows, h), dtype=dt, device=device)
        self.dx = torch.empty_like(self.x)
        self.codes = torch.empty((*rows, h), dtype=torch.uint8, device=device)
        self.scales = torch.empty((*rows, -(-h // ll.LL_ACT_GROUP)), dtype=torch.uint8,
                                  device=device)
        need = max(ll.ll_embed_grad_workspace_bytes(w.n, l["t"], h, l["vocab"]),
                   ll.ll_act_wgrad_workspace_bytes(w.n, l["t"], l["o"], h), 256)
        self.layer_ws = torch.empty(need, dtype=torch.uint8, device=device)

    def local_gradients(self, step: int, inputs=None):
        """Every worker's gradient of its batch on its own replica, into its
        gradient row: the embedding's output is looked up and kept as an 8-bit
        checkpoint; given the layer's output gradient, the layer's weight
        gradient is taken from the checkpoint and the embedding's from the
        layer's input gradient.  inputs: (tokens, dy), drawn for `step` if
        None."""
        w, l = self.w, self.w.layer
        tokens, dy = draw_layer_inputs(w, step, self.theta.device) if inputs is None else inputs
        weight = l["vocab"] * l["h"]  # offset of the layer's weight
        ll.ll_embed(tokens, self.replicas, self.x, v=l["vocab"])
        ll.ll_act_pack(self.x, self.codes, self.scales)
        ll.ll_act_wgrad(dy, self.codes, self.scales, self.grads, offset=weight,
                        workspace=self.layer_ws)
        for i in range(w.n):
            torch.mm(dy[i], self.replicas[i, weight:w.d].view(l["o"], l["h"]), out=self.dx[i])
        ll.ll_embed_grad(tokens, self.dx, self.grads, v=l["vocab"], workspace=self.layer_ws)

    def fused(self, step: int, drift=True, lam: float = 0.0, masks_out=True, ext=None):
        w = self.w
        spec = loss_spec(w)
        ll.lossy_step_fused(
            d=w.d, packet=w.packet, step=step, loss_g=spec, loss_b=spec, grads=self.grads,
            opt=opt_spec(w, lam), theta=self.theta, replicas=self.replicas, m=self.m, v=self.v,
            ge_state_g=self.ge_g, ge_state_b=self.ge_b,
            arrived_g=self.arrived_g if masks_out else None,
            arrived_b=self.arrived_b if masks_out else None,
            counts=self.counts if masks_out else None, workspace=self.workspace,
            drift=self.drift if drift else None, ext=ext)
