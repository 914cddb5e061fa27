"""Device buffers and calls for one MoE layer through the C ABI.

PyTorch provides the device memory and the stream; every step runs in
libec2moe.so.  Used by the tests, ``bench.py`` and ``__graft_entry__``.
"""

from __future__ import annotations

from typing import Dict, Optional

import torch

from . import ec2moe as C
from .synth import LayerConfig


def desc_for(cfg: LayerConfig, T: Optional[int] = None) -> C.LayerDesc:
    return C.make_desc(T=cfg.T if T is None else T, d=cfg.d, E=cfg.E, d_ff=cfg.d_ff, k=cfg.k,
                       n_groups=cfg.n_groups, act=cfg.act, dtype=cfg.dtype, r=cfg.r, n_shared=cfg.n_shared,
                       d_ff_shared=cfg.d_ff_shared, renorm_topk=cfg.renorm_topk, top_groups=cfg.top_groups)


def weights_for(inp: Dict[str, Optional[torch.Tensor]]) -> C.LayerWeights:
    return C.make_weights(W_local=inp["W_local"], b_local=inp["b_local"], W_global=inp.get("W_global"),
                          b_global=inp.get("b_global"), W1=inp.get("W1"), W3=inp.get("W3"), W2=inp.get("W2"),
                          W1s=inp.get("W1s"), W3s=inp.get("W3s"), W2s=inp.get("W2s"), V_enc=inp.get("V_enc"),
                          V_dec=inp.get("V_dec"))


class LayerRun:
    """Output and workspace buffers of one layer shape on one device."""

    def __init__(self, cfg: LayerConfig, inp: Dict[str, Optional[torch.Tensor]], device="cuda"):
        self.cfg = cfg
        self.inp = inp
        self.desc = desc_for(cfg)
        self.weights = weights_for(inp)
        self.mask = C.host_mask(inp["mask"].to("cpu"))
        dt = cfg.torch_dtype
        T = cfg.T
        self.Y = torch.empty(T, cfg.d, dtype=dt, device=device)
        self.topk_idx = torch.empty(T, cfg.k, dtype=torch.int32, device=device)
        self.topk_w = torch.empty(T, cfg.k, dtype=torch.float32, device=device)
        self.counts = torch.empty(cfg.E, dtype=torch.int32, device=device)
        self.Z = torch.empty(T, cfg.r, dtype=dt, device=device) if cfg.r > 0 else None
        self.ws_bytes = C.ec2moe_workspace_size(self.desc)
        self.workspace = torch.empty(max(self.ws_bytes, 16), dtype=torch.uint8, device=device)

    def forward_pipelined(self, n_micro: int, stream_end=None, stream_cloud=None,
                          X: Optional[torch.Tensor] = None) -> torch.Tensor:
        """The end/cloud pipelined layer call (two streams, n_micro micro-batches)."""
        need = C.ec2moe_pipelined_workspace_size(self.desc, n_micro)
        if getattr(self, "pws", None) is None or self.pws.numel() < need:
            self.pws = torch.empty(max(need, 16), dtype=torch.uint8, device=self.Y.device)
        C.ec2moe_layer_forward_pipelined(self.desc, self.weights, self.inp["X"] if X is None else X, self.mask,
                                         self.Y, self.topk_idx, self.topk_w, self.counts, self.Z, self.pws,
                                         self.pws.numel(), n_micro, stream_end, stream_cloud)
        return self.Y

    def forward(self, X: Optional[torch.Tensor] = None, stream=None) -> torch.Tensor:
        C.ec2moe_layer_forward(self.desc, self.weights, self.inp["X"] if X is None else X, self.mask, self.Y,
                               self.topk_idx, self.topk_w, self.counts, self.Z, self.workspace, self.ws_bytes,
                               stream)
        return self.Y


class Fp8LayerRun:
    """The same layer with its routed experts in 8-bit floating point, and the
    balance of its gate.

    The weights are quantised once, here.  ``forward`` composes the layer from the
    single entry points: gate, routing, codec, activations quantised straight into
    expert order, 8-bit experts, shared experts (in the layer's own type), combine.
    ``balance`` then gives the loss, the counts and the gradients of the gate on
    the same batch, whose biases ``rebalance`` moves.
    """

    def __init__(self, cfg: LayerConfig, inp: Dict[str, Optional[torch.Tensor]], device="cuda"):
        self.cfg = cfg
        self.inp = dict(inp)
        self.desc = desc_for(cfg)
        self.mask = C.host_mask(inp["mask"].to("cpu"))
        T, d, E, k, n = cfg.T, cfg.d, cfg.E, cfg.k, cfg.T * cfg.k
        dt = cfg.torch_dtype

        def empty(*shape, dtype=torch.float32):
            return torch.empty(*shape, dtype=dtype, device=device)

        def blocks(x):
            return -(-x // C.FP8_BLOCK)

        self.quantised = {}
        for i, (rows, cols) in {"1": (cfg.d_ff, d), "3": (cfg.d_ff, d), "2": (d, cfg.d_ff)}.items():
            w = inp.get("W" + i)
            if w is None:
                continue
            q, s = empty(E, rows, cols, dtype=torch.float8_e4m3fn), empty(E, blocks(rows), blocks(cols))
            C.ec2moe_fp8_quantize(cfg.dtype, E, rows, cols, cols, w, C.FP8_BLOCK, None, 0, q, s)
            self.quantised["W" + i], self.quantised["S" + i] = q, s
        self.weights = C.make_fp8_weights(**self.quantised)
        # calls may run on any stream, and nothing orders those behind this one
        torch.cuda.current_stream().synchronize()

        self.Y, self.slot = empty(T, d, dtype=dt), empty(n, d, dtype=dt)
        self.topk_idx, self.topk_w = empty(T, k, dtype=torch.int32), empty(T, k)
        self.counts, self.offsets = empty(E, dtype=torch.int32), empty(E + 1, dtype=torch.int32)
        self.perm, self.inv_perm = empty(n, dtype=torch.int32), empty(n, dtype=torch.int32)
        self.Xq, self.Xs = empty(n, d, dtype=torch.float8_e4m3fn), empty(n, blocks(d))
        self.Z = empty(T, cfg.r, dtype=dt) if cfg.r else None
        self.X_hat = empty(T, d, dtype=dt) if cfg.r else None
        self.shared = empty(cfg.n_shared * T, d, dtype=dt) if cfg.n_shared else None
        O = E + (cfg.n_groups if cfg.n_groups > 1 else 0)
        self.logits, self.d_logits, self.d_bias = empty(T, O), empty(T, O), empty(O)
        self.loss = empty(1)
        need = [C.ec2moe_route_workspace_size(self.desc), C.ec2moe_experts_fp8_workspace_size(self.desc),
                C.ec2moe_gate_logits_workspace_size(self.desc), C.ec2moe_balance_loss_workspace_size(self.desc, 1)]
        if cfg.n_shared:
            need.append(C.ec2moe_experts_workspace_size(self.desc))
        self.workspace = empty(max(16, *need), dtype=torch.uint8)

    def forward(self, X: Optional[torch.Tensor] = None, stream=None) -> torch.Tensor:
        t, cfg, desc = self.inp, self.cfg, self.desc
        ws, n_ws = self.workspace, self.workspace.numel()
        X = t["X"] if X is None else X
        C.ec2moe_gate(desc, X, t["W_local"], t["b_local"], t["W_global"], t["b_global"], self.mask, self.topk_idx,
                      self.topk_w, stream)
        C.ec2moe_route(desc, self.topk_idx, self.counts, self.offsets, self.perm, self.inv_perm, None, 0, None, ws, n_ws,
                       stream)
        x = X
        if cfg.r:
            C.ec2moe_lr_encode(desc, X, t["V_enc"], self.Z, stream)
            C.ec2moe_lr_decode(desc, self.Z, t["V_dec"], self.X_hat, stream)
            x = self.X_hat
        C.ec2moe_fp8_quantize(cfg.dtype, 1, cfg.T, cfg.d, cfg.d, x, 1, self.inv_perm, cfg.k, self.Xq, self.Xs, stream)
        C.ec2moe_experts_fp8(desc, self.Xq, self.Xs, self.offsets, self.weights, self.topk_w, self.perm, self.slot, ws, n_ws,
                             stream)
        if cfg.n_shared:
            C.ec2moe_shared_experts(desc, x, t["W1s"], t["W3s"], t["W2s"], self.shared, ws, n_ws, stream)
        C.ec2moe_combine(desc, self.slot, self.shared, self.Y, stream)
        return self.Y

    def balance(self, X: Optional[torch.Tensor] = None, coef: float = 1.0, stream=None) -> torch.Tensor:
        """The balance loss of the gate on the batch that ``forward`` routed; counts, d_logits and d_bias with it."""
        t, ws = self.inp, self.workspace
        X = t["X"] if X is None else X
        C.ec2moe_gate_logits(self.desc, X, t["W_local"], t["b_local"], t["W_global"], t["b_global"], self.logits, ws,
                             ws.numel(), stream)
        C.ec2moe_balance_loss(self.desc, self.logits, self.logits.shape[1], self.mask, self.topk_idx, None, None, 1, coef,
                              None, self.loss, self.counts, self.d_logits, self.d_bias, ws, ws.numel(), stream)
        return self.loss

    def rebalance(self, steps: int, rate: float) -> list:
        """`steps` gradient steps of the gate's biases towards even loads on this batch; the losses before each.

        A device's mask takes experts away from a gate that was trained with all of
        them; its biases are E + K numbers that can follow the mask."""
        E = self.cfg.E
        self.inp["b_local"] = self.inp["b_local"].clone()
        if self.cfg.n_groups > 1:
            self.inp["b_global"] = self.inp["b_global"].clone()
        losses = []
        for _ in range(steps):
            self.forward()
            losses.append(float(self.balance()))
            self.inp["b_local"] -= rate * self.d_bias[:E]
            if self.cfg.n_groups > 1:
                self.inp["b_global"] -= rate * self.d_bias[E:]
        return losses


def main(argv=None) -> int:
    """Runs `--calls` eager layer calls of a preset shape (for profilers such as
    ncu, which want a short program with a known launch sequence).  With `--fp8`
    the routed experts are 8-bit, and the balance of the gate is printed too."""
    import argparse

    from . import build as B
    from . import synth as S

    ap = argparse.ArgumentParser(description="run a preset MoE layer shape through the C ABI")
    ap.add_argument("--workload", default="mixtral_bf16")
    ap.add_argument("--calls", type=int, default=2)
    ap.add_argument("--fp8", action="store_true", help="8-bit experts, and the balance of the gate")
    for key in ("T", "E", "n_allowed", "k", "r", "d_ff", "n_groups", "seed"):
        ap.add_argument(f"--{key}", type=int, default=None)
    args = ap.parse_args(argv)
    over = {k: getattr(args, k) for k in ("T", "E", "n_allowed", "k", "r", "d_ff", "n_groups", "seed")
            if getattr(args, k) is not None}
    cfg = S.preset(args.workload, **over)
    B.build()
    C.load()
    inp = S.make_inputs(cfg, device="cuda")
    run = LayerRun(cfg, inp, device="cuda")
    if args.fp8:
        exact = run.forward().float()
        run = Fp8LayerRun(cfg, inp, device="cuda")
    for _ in range(args.calls):
        run.forward()
    if args.fp8:
        loss = float(run.balance())
        off = float((run.Y.float() - exact).norm() / exact.norm())
        print(f"8-bit experts: {off:.3f} of the layer's norm from the {cfg.torch_dtype} layer; "
              f"balance loss {loss:.4f} (1 = even loads), rows per expert {run.counts.tolist()}")
    status = C.ec2moe_last_device_error()
    torch.cuda.synchronize()
    print(f"{cfg}: {args.calls} calls, {C.ec2moe_last_launch_count()} launches per call, "
          f"status {C.status_string(status)}")
    return 0 if status == C.OK else 1


if __name__ == "__main__":
    raise SystemExit(main())
