"""The 8-bit expert products and the gate's balance loss, as cases to measure.

Operators (a case's "op"):

  quantize  rows or weight matrices to 8-bit floating point (e4m3) with one fp32
            scale for each block of 128 columns (of a row, or of 128 rows); rows
            optionally placed into expert order on the way
  gemm      the grouped product of two such operands, bf16 or fp32 results
  experts   the routed experts' FFN on 8-bit rows and weights: up projection,
            activation, its result quantised again, down projection, gate weight
            and scatter to the token's slot
  logits    the gate's logits (local and global rows) in fp32
  balance   per-expert counts, the balance loss of the gate and its gradients in
            the logits and the biases, over ragged segments with padding tokens

on the layer shapes this library is built for: Mixtral-shaped (d = 4096, 8 SwiGLU
experts of 14336, Top-2), fine-grained (d = 2048, 64 SwiGLU experts of 1408, Top-6
over 8 groups, Zipf popularity) and Switch-Transformer-base ones (d = 768, GELU
experts of four times that, Top-1).

Inputs: activations N(0, 1) with a few channels an order of magnitude larger (what
a residual stream looks like), weights N(0, 1 / fan_in), logits N(0, 1) with a
Zipf bias.
"""

from __future__ import annotations

import math

import torch

own = False

MIXTRAL = dict(d=4096, E=8, d_ff=14336, k=2, groups=2, act="swiglu", zipf=0.0)
FINE = dict(d=2048, E=64, d_ff=1408, k=6, groups=8, act="swiglu", zipf=1.2)
SWITCH = dict(d=768, E=16, d_ff=3072, k=1, groups=1, act="gelu", zipf=0.0)
TINY = dict(d=512, E=8, d_ff=1024, k=2, groups=2, act="gelu", zipf=0.0)

BLOCK = 128
TOP = 448.0          # the largest e4m3 value
FLOOR = 2.0 ** -96   # the least magnitude a block's scale is taken from
E4M3 = torch.float8_e4m3fn


# ----------------------------------------------------------------- cases
def _quantize(rows, cols, dtype="bf16", mats=1, block_rows=1, k=0):
    return dict(op="quantize", rows=rows, cols=cols, dtype=dtype, mats=mats, block_rows=block_rows, k=k)


def _gemm(rows, N, K, G=1, dtype="bf16", zipf=0.0):
    return dict(op="gemm", rows=rows, N=N, K=K, G=G, dtype=dtype, zipf=zipf)


def _experts(family, T, allowed, dtype="bf16"):
    return dict(family, op="experts", T=T, allowed=allowed, dtype=dtype)


def _logits(family, T, dtype="bf16"):
    return dict(op="logits", T=T, d=family["d"], E=family["E"], groups=family["groups"], dtype=dtype)


def _balance(family, T, allowed, segments, padded, top_groups=0):
    return dict(op="balance", T=T, E=family["E"], groups=family["groups"], k=family["k"], zipf=family["zipf"],
                allowed=allowed, segments=segments, padded=padded, top_groups=top_groups)


def listed():
    named = [
        # A decode step's activations (64 tokens), each placed for its two experts: latency.
        ("quantize_decode_64", _quantize(64, 4096, k=2)),
        # A fine-grained prefill batch's activations, each placed for its six experts.
        ("quantize_place_16384", _quantize(16384, 2048, k=6)),
        # One expert's product on a ragged chunk of a prefill, no routing.
        ("gemm_dense_777", _gemm(777, 4096, 4096)),
        # A decode step of 16 tokens, Top-2: every expert's weights once, a few rows each.
        ("gemm_decode_32", _gemm(32, 14336, 4096, G=8)),
        # The up projection of the largest prefill batch.
        ("gemm_prefill_16384", _gemm(16384, 14336, 4096, G=8)),
        # One token of a Mixtral-shaped decoder: two experts' weights.
        ("experts_decode_1", _experts(MIXTRAL, 1, 8)),
        # A ragged fine-grained batch under a device mask: 32 experts, Zipf popularity, odd row counts.
        ("experts_fine_2001", _experts(FINE, 2001, 32)),
        # The largest prefill batch, 6 of 8 experts on the device.
        ("experts_mixtral_8192", _experts(MIXTRAL, 8192, 6)),
        # The gate of a small Switch batch (4 x 256 tokens), 64 experts.
        ("logits_switch_1024", dict(_logits(SWITCH, 1024), E=64)),
        # The gate of a fine-grained prefill batch.
        ("logits_fine_16384", _logits(FINE, 16384)),
        # Balance of one small batch with padding tokens, 12 of 16 experts allowed.
        ("balance_switch_1021", _balance(SWITCH, 1021, 12, 1, 0.1)),
        # A training step's worth of fine-grained routing: 64 ragged sequences, padding.
        ("balance_fine_262144", _balance(FINE, 262144, 32, 64, 0.05)),
    ]
    return [dict(c, name=n) for n, c in named]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["quantize", "gemm", "gemm", "experts", "experts", "logits", "balance"])
    if op == "quantize":
        family = rng.choice([MIXTRAL, FINE, SWITCH])
        kind = rng.choice(["rows", "placed", "weights"])
        if kind == "weights":
            return _quantize(rng.choice([family["d_ff"], family["d"], 200]), family["d"], mats=rng.choice([1, 3, 8]),
                             block_rows=BLOCK)
        return _quantize(_log_int(rng, 1, 16384), rng.choice([family["d"], family["d"] - 16 * rng.randint(1, 7)]),
                         dtype=rng.choice(["bf16", "bf16", "fp32"]), k=rng.randint(1, 6) if kind == "placed" else 0)
    if op == "gemm":
        G = rng.choice([1, 8, 8, 64])
        N, K = rng.choice([(4096, 4096), (14336, 4096), (4096, 14336)] if G < 64 else [(1408, 2048), (2048, 1408)])
        if rng.random() < 0.3:
            N, K = N - 16 * rng.randint(1, 40), K - 16 * rng.randint(1, 40)
        return _gemm(_log_int(rng, 1, 16384), N, K, G=G, dtype=rng.choice(["bf16", "bf16", "fp32"]),
                     zipf=rng.choice([0.0, 1.2]))
    if op == "experts":
        family = rng.choice([MIXTRAL, FINE, SWITCH, TINY])
        E = family["E"]
        return _experts(family, _log_int(rng, 1, 8192), rng.choice([E // 2, 3 * E // 4, E]),
                        dtype=rng.choice(["bf16", "bf16", "fp32"]))
    if op == "logits":
        family = rng.choice([MIXTRAL, FINE, SWITCH, TINY])
        c = _logits(family, _log_int(rng, 1, 16384), dtype=rng.choice(["bf16", "bf16", "fp32"]))
        if family is SWITCH:
            c["E"] = rng.choice([16, 32, 64])
        return c
    family = rng.choice([MIXTRAL, FINE, FINE, SWITCH])
    E = family["E"]
    T = _log_int(rng, 1, 262144)
    return _balance(family, T, rng.choice([E // 2, 3 * E // 4, E]), rng.choice([1, 2, _log_int(rng, 3, 64)]),
                    rng.choice([0.0, 0.05, 0.3]), top_groups=4 if family is FINE and rng.random() < 0.5 else 0)


# ----------------------------------------------------------------- inputs
def _gen(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return g


def _dtype(case):
    return torch.float32 if case["dtype"] == "fp32" else torch.bfloat16


def _normal(g, *shape, fan_in=1):
    return torch.randn(*shape, generator=g, device="cuda") * (1.0 / math.sqrt(fan_in))


def _activations(g, rows, cols):
    x = torch.randn(rows, cols, generator=g, device="cuda")
    big = torch.randint(0, cols, (max(1, cols // 256),), generator=g, device="cuda")
    x[:, big] *= 12.0
    return x


def _cdiv(a, b):
    return -(-a // b)


def _blocks(x, block_rows):
    """x [mats, rows, cols] padded with zeros and cut into blocks: [mats, row blocks, block_rows, column blocks, 128]."""
    m, r, c = x.shape
    x = torch.nn.functional.pad(x, (0, -c % BLOCK, 0, -r % block_rows))
    return x.view(m, _cdiv(r, block_rows), block_rows, _cdiv(c, BLOCK), BLOCK)


def _to_fp8(x, block_rows):
    """(e4m3 [mats, rows, cols], fp32 scales [mats, row blocks, column blocks]) of x [mats, rows, cols]."""
    m, r, c = x.shape
    b = _blocks(x.float(), block_rows)
    a = b.abs().amax((2, 4)).clamp_min(FLOOR)
    q = (b * (TOP / a)[:, :, None, :, None]).clamp(-TOP, TOP).to(E4M3)
    return q.view(m, b.shape[1] * block_rows, -1)[:, :r, :c].contiguous(), a / TOP


def _weights(g, mats, rows, cols):
    return _to_fp8(_normal(g, mats, rows, cols, fan_in=cols), BLOCK)


def _popularity(g, n, zipf):
    rank = torch.randperm(n, generator=g, device="cuda")
    return -zipf * torch.log(rank + 1.0)


def _perm(topk_idx, E):
    """counts, offsets, perm and inv_perm of Top-k expert ids [T, k], rows of one expert in (t, s) order."""
    flat = topk_idx.reshape(-1).long()
    perm = torch.argsort(flat, stable=True)
    inv = torch.empty_like(perm)
    inv[perm] = torch.arange(flat.numel(), device="cuda")
    counts = torch.bincount(flat, minlength=E)
    offsets = torch.nn.functional.pad(counts.cumsum(0), (1, 0))
    return counts, offsets.int(), perm.int(), inv.int()


def _allowed(case, g):
    """The device mask: as many allowed experts in each group."""
    E, K, a = case["E"], case["groups"], case["allowed"]
    mask = torch.zeros(E, dtype=torch.bool, device="cuda")
    for j in range(K):
        n = a * (j + 1) // K - a * j // K
        mask[j * (E // K) + torch.randperm(E // K, generator=g, device="cuda")[:n]] = True
    return mask


def _inputs(case, seed):
    g = _gen(seed)
    op = case["op"]
    if op == "quantize":
        m, r, c = case["mats"], case["rows"], case["cols"]
        x = _activations(g, r, c)[None] if case["block_rows"] == 1 else _normal(g, m, r, c, fan_in=c)
        t = {"X": x.to(_dtype(case)), "inv_perm": None}
        if case["k"]:
            t["inv_perm"] = torch.randperm(r * case["k"], generator=g, device="cuda").int()
        return t
    if op == "gemm":
        a, sa = _to_fp8(_activations(g, case["rows"], case["K"])[:, None], 1)
        b, sb = _weights(g, case["G"], case["N"], case["K"])
        t = {"A": a[:, 0], "SA": sa[:, 0].contiguous(), "B": b, "SB": sb}
        group = torch.multinomial(torch.softmax(_popularity(g, case["G"], case["zipf"]), 0), case["rows"],
                                  replacement=True, generator=g)
        t["counts"], t["offsets"], _, _ = _perm(group, case["G"])
        return t
    if op == "experts":
        T, d, E, f, k = (case[n] for n in ("T", "d", "E", "d_ff", "k"))
        score = _popularity(g, E, case["zipf"]) + _normal(g, T, E)
        score = score.masked_fill(~_allowed(case, g), float("-inf"))
        w, idx = torch.topk(torch.softmax(score, 1), k, dim=1)
        t = {"topk_w": w.contiguous()}
        t["counts"], t["offsets"], t["perm"], _ = _perm(idx, E)
        x, sx = _to_fp8(_activations(g, T, d).to(torch.bfloat16)[:, None], 1)
        rows = t["perm"].long() // k
        t["X"], t["SX"] = x[:, 0].view(torch.uint8)[rows].view(E4M3), sx[:, 0][rows].contiguous()
        t["W1"], t["S1"] = _weights(g, E, f, d)
        t["W3"], t["S3"] = _weights(g, E, f, d) if case["act"] == "swiglu" else (None, None)
        t["W2"], t["S2"] = _weights(g, E, d, f)
        return t
    K = case["groups"]
    if op == "logits":
        T, d, E = case["T"], case["d"], case["E"]
        return {"X": _activations(g, T, d).to(_dtype(case)), "W_local": _normal(g, E, d, fan_in=d),
                "b_local": 0.3 * _normal(g, E), "W_global": _normal(g, K, d, fan_in=d) if K > 1 else None,
                "b_global": 0.3 * _normal(g, K) if K > 1 else None}
    T, E, k, S = case["T"], case["E"], case["k"], case["segments"]
    allowed = _allowed(case, g)
    logits = _normal(g, T, E + (K if K > 1 else 0))
    logits[:, :E] += _popularity(g, E, case["zipf"])
    p = _gate_probabilities(case, logits.double(), allowed)
    t = {"logits": logits, "allowed": allowed, "topk_idx": torch.topk(p, k, dim=1).indices.int().contiguous()}
    t["valid"] = (torch.rand(T, generator=g, device="cuda") >= case["padded"]).to(torch.uint8) if case["padded"] else None
    cuts = torch.sort(torch.randint(0, T + 1, (S - 1,), generator=g, device="cuda")).values
    ends = torch.tensor([0, T], device="cuda")
    t["segments"] = torch.cat([ends[:1], cuts, ends[1:]]).int() if S > 1 else None
    t["d_loss"] = torch.full((1,), 0.5, device="cuda")
    return t


def _gate_probabilities(case, logits, allowed):
    """The gate's g [T, E] from its logits, as the input generator needs it to choose the experts."""
    T, E, K = logits.shape[0], case["E"], case["groups"]
    neg = float("-inf")
    z = logits[:, :E].masked_fill(~allowed, neg).view(T, K, E // K)
    local = torch.softmax(z, 2).nan_to_num(0.0)
    if K == 1:
        return local.view(T, E)
    m = logits[:, E:].masked_fill(~allowed.view(K, -1).any(1), neg)
    if case["top_groups"]:
        least = m.topk(case["top_groups"], 1).values[:, -1:]
        m = m.masked_fill(m < least, neg)
    return (local * torch.softmax(m, 1)[:, :, None]).view(T, E)


def prepare(case, seed):
    st = dict(case, t=_inputs(case, seed))
    t, op = st["t"], case["op"]
    if op in ("gemm", "experts"):
        st["most"] = int(t["counts"].max())
    if own:
        _plan(st)
    return st


# ----------------------------------------------------------------- the framework's calls
def _plan(st):
    """The outputs, workspaces and descriptions that a program keeps from call to call."""
    from paper_2508_06024_gb300 import ec2moe as C

    t, op = st["t"], st["op"]

    def empty(*shape, dtype=torch.float32):
        return torch.empty(*shape, dtype=dtype, device="cuda")

    def space(n):
        return empty(max(16, n), dtype=torch.uint8)

    def desc():
        return C.make_desc(T=st["T"], d=st.get("d", 8), E=st["E"], d_ff=st.get("d_ff", 0), k=st.get("k", 1),
                           n_groups=st["groups"], act=C.SWIGLU if st.get("act") == "swiglu" else C.GELU,
                           dtype=C.F32 if st.get("dtype") == "fp32" else C.BF16, top_groups=st.get("top_groups", 0))

    st["C"] = C
    if op == "quantize":
        rows = st["mats"] * st["rows"] * max(1, st["k"])
        per = st["mats"] * _cdiv(st["rows"], BLOCK) if st["block_rows"] == BLOCK else rows
        st["Q"], st["S"] = empty(rows, st["cols"], dtype=E4M3), empty(per, _cdiv(st["cols"], BLOCK))
    elif op == "gemm":
        st["Y"] = empty(st["rows"], st["N"], dtype=_dtype(st))
        st["ws"] = space(C.ec2moe_fp8_gemm_workspace_size(st["G"], st["rows"], st["N"], st["K"]))
    elif op == "experts":
        st["desc"] = desc()
        st["weights"] = C.make_fp8_weights(**{n: t[n] for n in ("W1", "S1", "W3", "S3", "W2", "S2")})
        st["Y"] = empty(st["T"] * st["k"], st["d"], dtype=_dtype(st))
        st["ws"] = space(C.ec2moe_experts_fp8_workspace_size(st["desc"]))
    elif op == "logits":
        st["desc"] = desc()
        st["Y"] = empty(st["T"], st["E"] + (st["groups"] if st["groups"] > 1 else 0))
        st["ws"] = space(C.ec2moe_gate_logits_workspace_size(st["desc"]))
    else:
        st["desc"] = desc()
        st["mask"] = C.host_mask(t["allowed"].to(torch.uint8).cpu())
        st["loss"], st["counts"] = empty(1), empty(st["segments"], st["E"], dtype=torch.int32)
        st["d_logits"], st["d_bias"] = empty(*t["logits"].shape), empty(t["logits"].shape[1])
        st["ws"] = space(C.ec2moe_balance_loss_workspace_size(st["desc"], st["segments"]))


def _run_own(st):
    C, t, op = st["C"], st["t"], st["op"]
    if op == "quantize":
        C.ec2moe_fp8_quantize(C.F32 if st["dtype"] == "fp32" else C.BF16, st["mats"], st["rows"], st["cols"], st["cols"],
                              t["X"], st["block_rows"], t["inv_perm"], st["k"], st["Q"], st["S"])
        return {"Q": st["Q"], "S": st["S"]}
    ws = st["ws"]
    if op == "gemm":
        C.ec2moe_fp8_gemm(st["G"], st["rows"], st["N"], st["K"], t["A"], t["SA"], t["offsets"], t["B"], t["SB"],
                          C.F32 if st["dtype"] == "fp32" else C.BF16, st["Y"], st["N"], ws, ws.numel())
        return st["Y"]
    if op == "experts":
        C.ec2moe_experts_fp8(st["desc"], t["X"], t["SX"], t["offsets"], st["weights"], t["topk_w"], t["perm"], st["Y"],
                             ws, ws.numel())
        return st["Y"]
    if op == "logits":
        C.ec2moe_gate_logits(st["desc"], t["X"], t["W_local"], t["b_local"], t["W_global"], t["b_global"], st["Y"], ws,
                             ws.numel())
        return st["Y"]
    C.ec2moe_balance_loss(st["desc"], t["logits"], t["logits"].shape[1], st["mask"], t["topk_idx"], t["valid"],
                          t["segments"], st["segments"], 0.01, t["d_loss"], st["loss"], st["counts"], st["d_logits"],
                          st["d_bias"], ws, ws.numel())
    return {n: st[n] for n in ("loss", "counts", "d_logits", "d_bias")}


# ----------------------------------------------------------------- the plain forms
def _wide(q, s, block_rows):
    """e4m3 [mats, rows, cols] times its scales, fp32."""
    m, r, c = q.shape
    s = s.view(m, -1, s.shape[-1])
    s = s.repeat_interleave(block_rows, 1)[:, :r].repeat_interleave(BLOCK, 2)[:, :, :c]
    return q.float() * s


def _padded(rows, offsets, most):
    """Rows [n, c] as [groups, most, c], with the truth values of the places that hold one."""
    at = offsets[:-1, None] + torch.arange(most, device="cuda")
    held = at < offsets[1:, None]
    return rows[torch.where(held, at, 0).long()] * held[:, :, None], held


def _run_plain(st):
    t, op = st["t"], st["op"]
    if op == "quantize":
        q, s = _to_fp8(t["X"], st["block_rows"])
        q, s = q.view(-1, st["cols"]), s.view(-1, s.shape[-1])
        if t["inv_perm"] is not None:
            src = torch.argsort(t["inv_perm"]) // st["k"]
            q, s = q.view(torch.uint8)[src].view(E4M3), s[src]
        return {"Q": q, "S": s}
    if op == "gemm":
        a, held = _padded(_wide(t["A"][None], t["SA"], 1)[0], t["offsets"], st["most"])
        return torch.bmm(a, _wide(t["B"], t["SB"], BLOCK).transpose(1, 2))[held].to(_dtype(st))
    if op == "experts":
        x, held = _padded(_wide(t["X"][None], t["SX"], 1)[0], t["offsets"], st["most"])
        h = torch.bmm(x, _wide(t["W1"], t["S1"], BLOCK).transpose(1, 2))
        if t["W3"] is not None:
            h = h / (1.0 + torch.exp(-h)) * torch.bmm(x, _wide(t["W3"], t["S3"], BLOCK).transpose(1, 2))
        else:
            h = 0.5 * h * (1.0 + torch.erf(h * math.sqrt(0.5)))
        q, s = _to_fp8(h, 1)
        y = torch.bmm(_wide(q, s, 1), _wide(t["W2"], t["S2"], BLOCK).transpose(1, 2))[held]
        out = torch.empty_like(y)
        perm = t["perm"].long()
        out[perm] = y * t["topk_w"].view(-1, 1)[perm]
        return out.to(_dtype(st))
    if op == "logits":
        w, b = t["W_local"], t["b_local"]
        if t["W_global"] is not None:
            w, b = torch.cat([w, t["W_global"]]), torch.cat([b, t["b_global"]])
        return t["X"].float() @ w.T + b
    return _balance_plain(st)


def _balance_plain(st):
    t, E, K, k, S = st["t"], st["E"], st["groups"], st["k"], st["segments"]
    logits = t["logits"]
    T = logits.shape[0]
    zero = torch.zeros((), device="cuda")
    valid = torch.ones(T, device="cuda") if t["valid"] is None else t["valid"].float()
    # per-segment counts
    at = torch.arange(T, device="cuda")
    seg = torch.zeros_like(at) if t["segments"] is None else (torch.searchsorted(t["segments"], at, right=True) - 1)
    n = torch.zeros(S, device="cuda").index_add_(0, seg, valid)
    cell = (seg[:, None] * E + t["topk_idx"]).view(-1)
    counts = torch.zeros(S * E, dtype=torch.int32, device="cuda")
    counts.index_add_(0, cell, valid.int().repeat_interleave(k))
    counts = counts.view(S, E)
    # the gate's probabilities
    allowed = t["allowed"].view(K, E // K)
    z = logits[:, :E].view(T, K, E // K)
    top = torch.where(allowed, z, -torch.inf).amax(2, keepdim=True)
    e = torch.where(allowed, torch.exp(z - torch.where(allowed.any(1)[:, None], top, zero)), zero)
    p_local = e / e.sum(2, keepdim=True).clamp_min(1e-30)
    if K > 1:
        m = torch.where(allowed.any(1), logits[:, E:], -torch.inf)
        if st["top_groups"]:
            order = torch.argsort(m, dim=1, descending=True, stable=True)
            place = torch.argsort(order, dim=1)
            m = torch.where(place < st["top_groups"], m, -torch.inf)
        e = torch.exp(m - m.amax(1, keepdim=True))
        p_group = e / e.sum(1, keepdim=True)
    else:
        p_group = torch.ones(T, 1, device="cuda")
    # the loss, and its gradient through the two softmaxes
    c = 0.01 * t["allowed"].sum() / (n > 0).sum().clamp_min(1)
    f = counts / (k * n.clamp_min(1))[:, None]
    w = (c * f / n.clamp_min(1)[:, None])[seg].view(T, K, E // K) * valid[:, None, None]
    mean = (p_local * w).sum(2)
    loss = (p_group * mean).sum().view(1)
    d_z = p_group[:, :, None] * p_local * (w - mean[:, :, None])
    d = d_z.view(T, E)
    if K > 1:
        d = torch.cat([d, p_group * (mean - (p_group * mean).sum(1, keepdim=True))], 1)
    d = d * t["d_loss"]
    return {"loss": loss, "counts": counts, "d_logits": d, "d_bias": d.sum(0)}


def run(state):
    """One pass through the case's operator."""
    return _run_own(state) if own else _run_plain(state)


# ----------------------------------------------------------------- floors
def work(case):
    op = case["op"]
    if op == "quantize":
        n = case["mats"] * case["rows"]
        es = 4 if case["dtype"] == "fp32" else 2
        copies = max(1, case["k"])
        blocks = _cdiv(case["cols"], BLOCK)
        scales = n * blocks * copies if case["block_rows"] == 1 else case["mats"] * _cdiv(case["rows"], BLOCK) * blocks
        return {"bytes": n * case["cols"] * (es + copies) + 4.0 * scales + 4.0 * n * case["k"], "flops": 2.0 * n * case["cols"]}
    if op == "gemm":
        r, N, K, G = case["rows"], case["N"], case["K"], case["G"]
        touched = G * (1.0 - (1.0 - 1.0 / G) ** r)
        return {"bytes": r * K * (1 + 4.0 / BLOCK) + touched * N * K + r * N * (4 if case["dtype"] == "fp32" else 2) + 4.0 * G,
                "flops": 2.0 * r * N * K}
    if op == "experts":
        T, d, f, k, a = (case[n] for n in ("T", "d", "d_ff", "k", "allowed"))
        mats = 3 if case["act"] == "swiglu" else 2
        touched = a * (1.0 - (1.0 - k / a) ** T)
        n = T * k
        return {"bytes": touched * mats * d * f + n * d * (1 + 4.0 / BLOCK + (4 if case["dtype"] == "fp32" else 2)) + 8.0 * n,
                "flops": 2.0 * mats * n * d * f}
    O = case["E"] + (case["groups"] if case["groups"] > 1 else 0)
    T = case["T"]
    if op == "logits":
        es = 4 if case["dtype"] == "fp32" else 2
        return {"bytes": T * case["d"] * es + 4.0 * O * case["d"] + 4.0 * T * O, "flops": 2.0 * T * case["d"] * O}
    return {"bytes": 8.0 * T * O + 4.0 * T * case["k"] + (T if case["padded"] else 0) + 4.0 * case["segments"] * case["E"],
            "flops": 12.0 * T * O}


# ----------------------------------------------------------------- the same in 64 bits
def _e4m3_64(x):
    """x rounded to the nearest e4m3 value (ties to even), in 64 bits: 3 mantissa bits down to 2^-6, steps of 2^-9 below."""
    exponent = torch.frexp(x).exponent.clamp_min(-5) - 4
    step = torch.ldexp(torch.ones_like(x), exponent)
    return (torch.round(x / step) * step).clamp(-448.0, 448.0)


def _requantized_64(h):
    """Rows rounded to e4m3 per 128 columns and scaled back, in 64 bits."""
    parts = []
    for c in range(0, h.shape[1], BLOCK):
        x = h[:, c:c + BLOCK]
        s = x.abs().amax(1, keepdim=True).clamp_min(2.0 ** -96) / 448.0
        parts.append(_e4m3_64(x / s) * s)
    return torch.cat(parts, 1)


def _scaled_64(q, s, block_rows):
    """One matrix [rows, cols] of e4m3 values times its scales, in 64 bits."""
    x = q.to(torch.float32).double()
    r = torch.arange(x.shape[0], device="cuda") // block_rows
    c = torch.arange(x.shape[1], device="cuda") // BLOCK
    return x * s.double()[r][:, c]


def exact(case, seed):
    t = _inputs(case, seed)
    op = case["op"]
    if op == "quantize":
        x, br = t["X"].double(), case["block_rows"]
        m, r, c = x.shape
        row, col = torch.arange(r, device="cuda") // br, torch.arange(c, device="cuda") // BLOCK
        rb, cb = int(row[-1]) + 1, int(col[-1]) + 1
        most = torch.zeros(m, rb * cb, dtype=torch.float64, device="cuda")
        cell = (row[:, None] * cb + col[None, :]).reshape(-1)
        most.scatter_reduce_(1, cell.expand(m, -1), x.abs().reshape(m, -1), "amax")
        s = most.clamp_min(2.0 ** -96) / 448.0
        q = _e4m3_64(x.reshape(m, -1) / s[:, cell]).reshape(m * r, c)
        s = s.reshape(m * rb, cb)
        if t["inv_perm"] is not None:
            placed = torch.empty(r * case["k"], dtype=torch.long, device="cuda")
            placed[t["inv_perm"].long()] = torch.arange(r * case["k"], device="cuda")
            q, s = q[placed // case["k"]], s[placed // case["k"]]
        return {"Q": q, "S": s}
    if op == "gemm":
        at = t["offsets"].tolist()
        parts = []
        for g in range(case["G"]):
            if at[g + 1] > at[g]:
                a = _scaled_64(t["A"][at[g]:at[g + 1]], t["SA"][at[g]:at[g + 1]], 1)
                parts.append(a @ _scaled_64(t["B"][g], t["SB"][g], BLOCK).T)
        return torch.cat(parts)
    if op == "experts":
        at = t["offsets"].tolist()
        out = torch.zeros(case["T"] * case["k"], case["d"], dtype=torch.float64, device="cuda")
        for g in range(case["E"]):
            lo, hi = at[g], at[g + 1]
            if hi == lo:
                continue
            x = _scaled_64(t["X"][lo:hi], t["SX"][lo:hi], 1)
            u = x @ _scaled_64(t["W1"][g], t["S1"][g], BLOCK).T
            if t["W3"] is not None:
                h = torch.nn.functional.silu(u) * (x @ _scaled_64(t["W3"][g], t["S3"][g], BLOCK).T)
            else:
                h = torch.nn.functional.gelu(u)
            slots = t["perm"][lo:hi].long()
            y = _requantized_64(h) @ _scaled_64(t["W2"][g], t["S2"][g], BLOCK).T
            out[slots] = y * t["topk_w"].double().reshape(-1)[slots, None]
        return out
    if op == "logits":
        x = t["X"].double()
        y = torch.nn.functional.linear(x, t["W_local"].double(), t["b_local"].double())
        if t["W_global"] is not None:
            y = torch.cat([y, torch.nn.functional.linear(x, t["W_global"].double(), t["b_global"].double())], 1)
        return y
    # balance: the definition, differentiated by autograd
    T, E, S, k = case["T"], case["E"], case["segments"], case["k"]
    logits = t["logits"].double().requires_grad_()
    g = _gate_probabilities(case, logits, t["allowed"])
    valid = torch.ones(T, dtype=torch.bool, device="cuda") if t["valid"] is None else t["valid"].bool()
    at = [0, T] if t["segments"] is None else t["segments"].tolist()
    terms = []
    for s in range(S):
        v = valid[at[s]:at[s + 1]]
        if bool(v.any()):
            f = torch.nn.functional.one_hot(t["topk_idx"][at[s]:at[s + 1]][v].long(), E).sum(1).double().mean(0) / k
            terms.append((f * g[at[s]:at[s + 1]][v].mean(0)).sum() * int(t["allowed"].sum()))
    zero = logits.sum() * 0.0
    loss = 0.01 * (torch.stack(terms).mean() if terms else zero)
    d, = torch.autograd.grad(loss * 0.5, logits)
    return {"loss": loss.detach().view(1), "counts": None, "d_logits": d, "d_bias": d.sum(0)}
