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


def _check_norm_weight(cfg: LayerConfig, device, w: torch.Tensor) -> None:
    if w.dtype != torch.float32 or w.numel() != cfg.d or not w.is_contiguous() or w.device.type != torch.device(device).type:
        raise ValueError(f"a norm's weight is dense fp32 [{cfg.d}] on {device}, not {w.dtype} {tuple(w.shape)} of strides "
                         f"{w.stride()} on {w.device}")


def _check_rows(cfg: LayerConfig, device: torch.device, **rows: Optional[torch.Tensor]) -> None:
    """The kernels are given addresses alone: rows of another type, number, order or device would be read as if they were
    dense ones (an expanded gradient beyond its end)."""
    for name, t in rows.items():
        if t is not None and (t.dtype != cfg.torch_dtype or t.numel() != cfg.T * cfg.d or not t.is_contiguous()
                              or t.device != device):
            raise ValueError(f"{name} is dense {cfg.torch_dtype} [{cfg.T}, {cfg.d}] on {device}, not {t.dtype} "
                             f"{tuple(t.shape)} of strides {t.stride()} on {t.device}")


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

    With ``norm_weight`` the layer has a root-mean-square norm in front, of X plus the
    ``residual`` that ``forward`` is given (the sum stays in ``H``).  Without a codec its
    shared experts are then 8-bit too and read the rows that the norm quantised.
    """

    def __init__(self, cfg: LayerConfig, inp: Dict[str, Optional[torch.Tensor]], device="cuda",
                 norm_weight: Optional[torch.Tensor] = None, eps: float = 1e-5):
        if norm_weight is not None:
            _check_norm_weight(cfg, device, norm_weight)
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

        def quantised(tail, n, ff):
            out = {}
            for i, (rows, cols) in {"1": (ff, d), "3": (ff, d), "2": (d, ff)}.items():
                w = inp.get("W" + i + tail)
                if w is None:
                    continue
                q, s = empty(n, rows, cols, dtype=torch.float8_e4m3fn), empty(n, blocks(rows), blocks(cols))
                C.ec2moe_fp8_quantize(cfg.dtype, n, rows, cols, cols, w, C.FP8_BLOCK, None, 0, q, s)
                out["W" + i], out["S" + i] = q, s
            return out

        self.quantised = quantised("", E, cfg.d_ff)
        self.weights = C.make_fp8_weights(**self.quantised)
        self.norm_weight, self.eps = norm_weight, eps
        self.shared8 = []
        if norm_weight is not None:
            self.H, self.Xn = empty(T, d, dtype=dt), empty(T, d, dtype=dt)
            if cfg.n_shared and not cfg.r:
                # each shared expert as a layer of one expert that every token goes to
                self.shared_quantised = quantised("s", cfg.n_shared, cfg.d_ff_shared)
                self.shared_desc = C.make_desc(T=T, d=d, E=1, d_ff=cfg.d_ff_shared, k=1, act=cfg.act, dtype=cfg.dtype)
                self.shared8 = [C.make_fp8_weights(**{n: w[j] for n, w in self.shared_quantised.items()})
                                for j in range(cfg.n_shared)]
                self.Xn8, self.Xn8_s = empty(T, d, dtype=torch.float8_e4m3fn), empty(T, blocks(d))
                self.every = (torch.tensor([0, T], dtype=torch.int32, device=device),
                              torch.arange(T, dtype=torch.int32, device=device), torch.ones(T, device=device))
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
        if self.shared8:
            need.append(C.ec2moe_experts_fp8_workspace_size(self.shared_desc))
        elif cfg.n_shared:
            need.append(C.ec2moe_experts_workspace_size(self.desc))
        self.workspace = empty(max(16, *need), dtype=torch.uint8)

    def forward(self, X: Optional[torch.Tensor] = None, stream=None,
                residual: Optional[torch.Tensor] = None) -> torch.Tensor:
        if residual is not None and self.norm_weight is None:
            raise ValueError("a residual is added in front of a norm, and this layer has none")
        t, cfg, desc = self.inp, self.cfg, self.desc
        ws, n_ws = self.workspace, self.workspace.numel()
        X = t["X"] if X is None else X
        if self.norm_weight is not None:
            _check_rows(cfg, self.Y.device, X=X, residual=residual)
            q, s = (self.Xn8, self.Xn8_s) if self.shared8 else (None, None)
            C.ec2moe_rmsnorm(cfg.dtype, cfg.dtype, cfg.T, cfg.d, cfg.d, X, residual, self.norm_weight, self.eps, self.H, None,
                             self.Xn, q, s, stream)
            X = self.Xn
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
        for j, w in enumerate(self.shared8):
            offsets, perm, ones = self.every
            C.ec2moe_experts_fp8(self.shared_desc, self.Xn8, self.Xn8_s, offsets, w, ones, perm,
                                 self.shared[j * cfg.T:(j + 1) * cfg.T], ws, n_ws, stream)
        if cfg.n_shared and not self.shared8:
            C.ec2moe_shared_experts(desc, x, t["W1s"], t["W3s"], t["W2s"], self.shared, ws, n_ws, stream)
        C.ec2moe_combine(desc, self.slot, self.shared, self.Y, stream)
        return self.Y

    def balance(self, X: Optional[torch.Tensor] = None, coef: float = 1.0, stream=None) -> torch.Tensor:
        """The balance loss of the gate on the batch that ``forward`` routed; counts, d_logits and d_bias with it.

        X is what the gate read of that batch; with a norm those are the rows that ``forward`` normed, and no X is taken."""
        if X is not None and self.norm_weight is not None:
            raise ValueError("the gate of a normed layer read the rows that forward normed, not X")
        t, ws = self.inp, self.workspace
        X = self.Xn if self.norm_weight is not None else t["X"] if X is None else X
        C.ec2moe_gate_logits(self.desc, X, t["W_local"], t["b_local"], t["W_global"], t["b_global"], self.logits, ws,
                             ws.numel(), stream)
        C.ec2moe_balance_loss(self.desc, self.logits, self.logits.shape[1], self.mask, self.topk_idx, None, None, 1, coef,
                              None, self.loss, self.counts, self.d_logits, self.d_bias, ws, ws.numel(), stream)
        return self.loss

    def rebalance(self, steps: int, rate: float, X: Optional[torch.Tensor] = None,
                  residual: Optional[torch.Tensor] = None) -> list:
        """`steps` gradient steps of the gate's biases towards even loads on this batch (``forward``'s X and residual); the
        losses before each.

        A device's mask takes experts away from a gate that was trained with all of
        them; its biases are E + K numbers that can follow the mask."""
        E = self.cfg.E
        self.inp["b_local"] = self.inp["b_local"].clone()
        if self.cfg.n_groups > 1:
            self.inp["b_global"] = self.inp["b_global"].clone()
        losses = []
        for _ in range(steps):
            self.forward(X, residual=residual)
            losses.append(float(self.balance(X if self.norm_weight is None else None)))
            self.inp["b_local"] -= rate * self.d_bias[:E]
            if self.cfg.n_groups > 1:
                self.inp["b_global"] -= rate * self.d_bias[E:]
        return losses


class TrainBlockRun:
    """A training step of one residual block around a bf16 layer.

    ``forward`` adds X to the residual stream, norms the sum, and composes the layer from
    the single entry points, keeping what the gradients need: gate, routing, codec, the up
    products of W1 and W3 as one (their rows joined), the activation with the gate's
    weights, the down product into the tokens' slots, combine.  Its results are the
    residual stream ``H`` and the layer's output ``Y``; the next block's are its own norm's
    residual and X.

    ``backward`` takes the gradients that arrive at both and gives those of X and the
    residual (one sum, ``dX``), of the norm's weight, of the experts', shared experts'
    and codec's weights (fp32, ``grads``; ``accumulate`` adds to them), and of the gate
    weights of Top-k (``d_topk_w``, where the gate's own gradient starts: it is not carried
    on into the gate rows and X here, so ``dX`` is without the gate's path).  ``params`` has the
    tensors that the gradients are of.
    """

    def __init__(self, cfg: LayerConfig, inp: Dict[str, Optional[torch.Tensor]], norm_weight: torch.Tensor,
                 eps: float = 1e-5, device="cuda"):
        if cfg.dtype != C.BF16:
            raise ValueError("the grouped products take bf16 operands")
        _check_norm_weight(cfg, device, norm_weight)
        self.cfg, self.inp, self.norm_weight, self.eps = cfg, dict(inp), norm_weight, eps
        self.desc = desc_for(cfg)
        self.mask = C.host_mask(inp["mask"].to("cpu"))
        T, d, E, k, n, f = cfg.T, cfg.d, cfg.E, cfg.k, cfg.T * cfg.k, cfg.d_ff
        bf = torch.bfloat16

        def empty(*shape, dtype=bf):
            return torch.empty(*shape, dtype=dtype, device=device)

        def joined(a, b):
            return a.contiguous() if b is None else torch.cat([a, b], 1)

        self.up = joined(inp["W1"], inp.get("W3"))                      # [E, F, d], F = d_ff or 2 d_ff
        self.F = self.up.shape[1]
        self.H, self.rstd, self.Xn = empty(T, d), empty(T, dtype=torch.float32), empty(T, d)
        self.topk_idx, self.topk_w = empty(T, k, dtype=torch.int32), empty(T, k, dtype=torch.float32)
        self.counts, self.offsets = empty(E, dtype=torch.int32), empty(E + 1, dtype=torch.int32)
        self.perm, self.inv_perm = empty(n, dtype=torch.int32), empty(n, dtype=torch.int32)
        self.Z, self.X_hat = (empty(T, cfg.r), empty(T, d)) if cfg.r else (None, None)
        self.Xp, self.UV, self.Hid, self.slot, self.Y = empty(n, d), empty(n, self.F), empty(n, f), empty(n, d), empty(T, d)
        # gradients
        self.dYp, self.dHid, self.dUV, self.dslot = empty(n, d), empty(n, f), empty(n, self.F), empty(n, d)
        self.dXe, self.dX = empty(T, d), empty(T, d)
        self.dXn, self.dZ = (empty(T, d), empty(T, cfg.r)) if cfg.r else (self.dXe, None)
        self.d_topk_w = empty(T, k, dtype=torch.float32)
        f32 = dict(dtype=torch.float32)
        self.grads = {"norm": empty(d, **f32), "up": empty(*self.up.shape, **f32), "W2": empty(E, d, f, **f32)}
        sizes = [(E, n, self.F, d), (E, n, d, f)]
        if cfg.n_shared:
            fs = cfg.d_ff_shared
            self.ups = joined(inp["W1s"], inp.get("W3s"))
            self.Fs = self.ups.shape[1]
            self.UVs, self.Hids, self.shared = empty(cfg.n_shared, T, self.Fs), empty(cfg.n_shared, T, fs), empty(cfg.n_shared * T, d)
            self.dHids, self.dUVs, self.dshared = empty(T, fs), empty(T, self.Fs), empty(cfg.n_shared * T, d)
            self.grads["ups"], self.grads["W2s"] = empty(*self.ups.shape, **f32), empty(cfg.n_shared, d, fs, **f32)
            sizes += [(1, T, self.Fs, d), (1, T, d, fs)]
        else:
            self.shared = self.dshared = None
        if cfg.r:
            self.grads["V_enc"], self.grads["V_dec"] = empty(cfg.r, d, **f32), empty(d, cfg.r, **f32)
            sizes += [(1, T, d, cfg.r), (1, T, cfg.r, d)]
        need = [C.ec2moe_route_workspace_size(self.desc), C.ec2moe_rmsnorm_backward_workspace_size(T, d)]
        need += [C.ec2moe_grouped_gemm_workspace_size(*s) for s in sizes]
        self.workspace = empty(max(16, *need), dtype=torch.uint8)
        # the joined rows: calls may run on any stream, and nothing orders those behind this one
        torch.cuda.current_stream().synchronize()

    @property
    def params(self) -> Dict[str, torch.Tensor]:
        """The tensors that every call reads, under the names of ``grads``: an optimiser updates these, in place.

        They are the tensors that the constructor was given but for ``up`` and ``ups`` of SwiGLU, which hold W1's rows with
        W3's behind them: copies, so a later change of W1 or W3 is not seen."""
        p = {"norm": self.norm_weight, "up": self.up, "W2": self.inp["W2"]}
        if self.cfg.n_shared:
            p["ups"], p["W2s"] = self.ups, self.inp["W2s"]
        if self.cfg.r:
            p["V_enc"], p["V_dec"] = self.inp["V_enc"], self.inp["V_dec"]
        return p

    # the three products of rows X [rows, K] and weights B [G, N, K], their gradients' names as in the header
    def _product(self, G, X, offsets, B, perm, out, stream):
        ws, (rows, K), N = self.workspace, X.shape, B.shape[-2]
        C.ec2moe_grouped_gemm(G, rows, N, K, X, K, offsets, B, perm, C.BF16, out, N, ws, ws.numel(), stream)

    def _dgrad(self, G, dY, offsets, B, perm, out, stream):
        ws, (rows, N), K = self.workspace, dY.shape, B.shape[-1]
        C.ec2moe_grouped_gemm_dgrad(G, rows, N, K, dY, N, offsets, B, perm, C.BF16, out, K, ws, ws.numel(), stream)

    def _wgrad(self, G, dY, X, offsets, accumulate, out, stream):
        ws, (rows, N), K = self.workspace, dY.shape, X.shape[1]
        C.ec2moe_grouped_gemm_wgrad(G, rows, N, K, dY, N, X, K, offsets, C.F32, accumulate, out, ws, ws.numel(), stream)

    def _activation(self, f, UV, perm, scale, out, stream):
        glu = self.cfg.act == C.SWIGLU
        C.ec2moe_activation(C.BF16, self.cfg.act, UV.shape[0], f, UV.shape[1], UV, UV[:, f:] if glu else None, perm, scale, out,
                            stream)

    def _activation_backward(self, f, UV, perm, scale, dH, dUV, H, d_scale, stream):
        glu = self.cfg.act == C.SWIGLU
        C.ec2moe_activation_backward(C.BF16, self.cfg.act, UV.shape[0], f, UV.shape[1], UV, UV[:, f:] if glu else None, perm,
                                     scale, dH, dUV, dUV[:, f:] if glu else None, H, d_scale, stream)

    def forward(self, X: Optional[torch.Tensor] = None, residual: Optional[torch.Tensor] = None, stream=None):
        """(H, Y): the residual stream behind X's addition, and the layer's output on its norm."""
        t, cfg, desc, ws = self.inp, self.cfg, self.desc, self.workspace
        X = t["X"] if X is None else X
        _check_rows(cfg, self.Y.device, X=X, residual=residual)
        C.ec2moe_rmsnorm(C.BF16, C.BF16, cfg.T, cfg.d, cfg.d, X, residual, self.norm_weight, self.eps, self.H, self.rstd, self.Xn,
                         None, None, stream)
        C.ec2moe_gate(desc, self.Xn, t["W_local"], t["b_local"], t["W_global"], t["b_global"], self.mask, self.topk_idx,
                      self.topk_w, stream)
        x = self.Xn
        if cfg.r:
            C.ec2moe_lr_encode(desc, x, t["V_enc"], self.Z, stream)
            C.ec2moe_lr_decode(desc, self.Z, t["V_dec"], self.X_hat, stream)
            x = self.X_hat
        self.x = x
        C.ec2moe_route(desc, self.topk_idx, self.counts, self.offsets, self.perm, self.inv_perm, x, cfg.d, self.Xp, ws, ws.numel(),
                       stream)
        self._product(cfg.E, self.Xp, self.offsets, self.up, None, self.UV, stream)
        self._activation(cfg.d_ff, self.UV, self.perm, self.topk_w, self.Hid, stream)
        self._product(cfg.E, self.Hid, self.offsets, t["W2"], self.perm, self.slot, stream)
        for j in range(cfg.n_shared):
            self._product(1, x, None, self.ups[j], None, self.UVs[j], stream)
            self._activation(cfg.d_ff_shared, self.UVs[j], None, None, self.Hids[j], stream)
            self._product(1, self.Hids[j], None, t["W2s"][j], None, self.shared[j * cfg.T:], stream)
        C.ec2moe_combine(desc, self.slot, self.shared, self.Y, stream)
        return self.H, self.Y

    def backward(self, dY: torch.Tensor, dH: Optional[torch.Tensor] = None, accumulate: int = 0, stream=None) -> torch.Tensor:
        """dX (without the gate's path) from the gradients that arrive at Y and (the blocks behind) at H; call it after
        ``forward``."""
        t, cfg, desc, ws, g = self.inp, self.cfg, self.desc, self.workspace, self.grads
        _check_rows(cfg, self.Y.device, dY=dY, dH=dH)
        # the combine's: every slot of a token gets the token's row, here in expert order
        C.ec2moe_route(desc, self.topk_idx, self.counts, self.offsets, self.perm, self.inv_perm, dY, cfg.d, self.dYp, ws,
                       ws.numel(), stream)
        self._dgrad(cfg.E, self.dYp, self.offsets, t["W2"], None, self.dHid, stream)
        self._activation_backward(cfg.d_ff, self.UV, self.perm, self.topk_w, self.dHid, self.dUV, self.Hid, self.d_topk_w, stream)
        self._wgrad(cfg.E, self.dYp, self.Hid, self.offsets, accumulate, g["W2"], stream)
        self._wgrad(cfg.E, self.dUV, self.Xp, self.offsets, accumulate, g["up"], stream)
        self._dgrad(cfg.E, self.dUV, self.offsets, self.up, self.perm, self.dslot, stream)
        for j in range(cfg.n_shared):
            self._dgrad(1, dY, None, t["W2s"][j], None, self.dHids, stream)
            self._wgrad(1, dY, self.Hids[j], None, accumulate, g["W2s"][j], stream)
            self._activation_backward(cfg.d_ff_shared, self.UVs[j], None, None, self.dHids, self.dUVs, None, None, stream)
            self._wgrad(1, self.dUVs, self.x, None, accumulate, g["ups"][j], stream)
            self._dgrad(1, self.dUVs, None, self.ups[j], None, self.dshared[j * cfg.T:], stream)
        C.ec2moe_combine(desc, self.dslot, self.dshared, self.dXe, stream)
        if cfg.r:
            self._wgrad(1, self.dXe, self.Z, None, accumulate, g["V_dec"], stream)
            self._dgrad(1, self.dXe, None, t["V_dec"], None, self.dZ, stream)
            self._wgrad(1, self.dZ, self.Xn, None, accumulate, g["V_enc"], stream)
            self._dgrad(1, self.dZ, None, t["V_enc"], None, self.dXn, stream)
        C.ec2moe_rmsnorm_backward(C.BF16, C.BF16, cfg.T, cfg.d, cfg.d, self.dXn, self.H, self.rstd, self.norm_weight, dH, self.dX,
                                  g["norm"], ws, ws.numel(), stream, accumulate)
        return self.dX


def main(argv=None) -> int:
    """Runs `--calls` eager layer calls of a preset shape (for profilers such as
    ncu, which want a short program with a known launch sequence).  With `--fp8`
    the routed experts are 8-bit, and the balance of the gate is printed too; with
    `--train` a call is a training step of the block around the layer."""
    import argparse

    from . import build as B
    from . import synth as S

    ap = argparse.ArgumentParser(description="run a preset MoE layer shape through the C ABI")
    ap.add_argument("--workload", default="mixtral_bf16")
    ap.add_argument("--calls", type=int, default=2)
    ap.add_argument("--fp8", action="store_true", help="8-bit experts, and the balance of the gate")
    ap.add_argument("--train", action="store_true", help="forward and backward of the block: norm, layer, residual")
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
    if args.fp8 and not args.train:
        exact = run.forward().float()
        run = Fp8LayerRun(cfg, inp, device="cuda")
    if args.train:
        run = TrainBlockRun(cfg, inp, torch.ones(cfg.d, device="cuda"))
        dY = torch.randn(cfg.T, cfg.d, device="cuda").to(cfg.torch_dtype)
    for _ in range(args.calls):
        run.forward()
        if args.train:
            run.backward(dY, dY)
    if args.train:
        print("gradients, root mean square:", {n: float(f"{float(v.square().mean().sqrt()):.3g}") for n, v in run.grads.items()})
    elif args.fp8:
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
