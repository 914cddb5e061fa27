"""The gate's logits and its balance loss on the GPU against the 64-bit oracle.

Tolerances, from fp32 arithmetic:
* logits: products of the exact terms are added in ranges of at most 512 columns
  (32 tensor-core steps, each truncating by at most 2^-23 of the sum of
  magnitudes), their sums and the bias in fp32: |error| <= (32 + d / 512 + 8)
  2^-23 (sum |x| |w| + |b|);
* gradients: with |z| differences up to 20, the exponent's argument and the
  exponential are off by 2^-24 * 20 + 2^-22, about 1.5e-6 relative; sums of up to
  128 terms and a dozen further roundings stay below 1e-5 of g_i max_i |w_i - mean|;
* loss and bias gradients: the same relative to the sum of magnitudes.
"""
import numpy as np
import pytest
import torch

from oracle import fp8_balance_oracle as orc
from paper_2508_06024_gb300 import build as B
from paper_2508_06024_gb300 import ec2moe as C

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def lib():
    B.build()
    return C.load()


def cuda(a):
    return torch.from_numpy(np.ascontiguousarray(a)).cuda()


def run(z, mask, idx, K, coef=0.5, valid=None, seg=None, top_groups=0, d_loss=None, ld=None, k=None, want_d=True):
    T, O = z.shape
    E = len(mask)
    S = 1 if seg is None else len(seg) - 1
    k = idx.shape[1] if k is None else k
    desc = C.make_desc(T=T, d=8, E=E, d_ff=0, k=k, n_groups=K, top_groups=top_groups)
    wsb = C.ec2moe_balance_loss_workspace_size(desc, S)
    ws = torch.randint(0, 255, (wsb,), dtype=torch.uint8, device="cuda")
    loss = torch.full((2,), 7.0, device="cuda")
    counts = torch.full((S + 1, E), -7, dtype=torch.int32, device="cuda")
    d = torch.full((T + 1, O), 7.0, device="cuda") if want_d else None
    db = torch.full((O + 1,), 7.0, device="cuda") if want_d else None
    zz = np.full((T, O if ld is None else ld), np.nan, np.float32)
    zz[:, :O] = z
    C.ec2moe_balance_loss(desc, cuda(zz), zz.shape[1], np.asarray(mask, np.uint8), cuda(idx.astype(np.int32)),
                          None if valid is None else cuda(np.asarray(valid, np.uint8)),
                          None if seg is None else cuda(np.array(seg, np.int32)), S, coef,
                          None if d_loss is None else cuda(np.array([d_loss], np.float32)), loss, counts, d, db, ws, wsb)
    status = C.ec2moe_last_device_error()
    assert loss[1] == 7.0 and (counts[-1] == -7).all()
    if want_d:
        assert (d[-1] == 7.0).all() and db[-1] == 7.0
        d, db = d[:-1].double().cpu().numpy(), db[:-1].double().cpu().numpy()
    return float(loss[0]), counts[:-1].cpu().numpy(), d, db, status


def check(z, mask, idx, K, coef=0.5, valid=None, seg=None, top_groups=0, d_loss=None, ld=None):
    T, O = z.shape
    E = len(mask)
    got = run(z, mask, idx, K, coef, valid, seg, top_groups, d_loss, ld)
    clean = np.where(np.isfinite(z), z, 0.0)  # what is masked is not used
    want = orc.balance(clean, mask, idx, K, coef, valid, seg, top_groups, 1.0 if d_loss is None else d_loss)
    assert got[4] == C.OK
    assert np.array_equal(got[1], want[1])
    assert abs(got[0] - want[0]) <= 1e-5 * abs(want[0]) + 1e-30
    # per token: g_i times the largest weight difference
    g = orc.gate_probabilities(clean, mask, K, top_groups)
    S = len(want[1])
    bounds = [0, T] if seg is None else list(seg)
    spread = np.zeros(T)
    ok = np.ones(T, bool) if valid is None else np.asarray(valid, bool)
    live = sum(ok[bounds[s]:bounds[s + 1]].any() for s in range(S))
    for s in range(S):
        n = ok[bounds[s]:bounds[s + 1]].sum()
        if n:
            c = want[1][s].astype(float)
            unit = coef * sum(mask) / (live * idx.shape[1] * n * n)
            spread[bounds[s]:bounds[s + 1]] = unit * np.abs(c - c.sum() / sum(mask)).max()
    spread *= ok * abs(1.0 if d_loss is None else d_loss)
    pg = g.reshape(T, K, -1).sum(2)
    mag = np.concatenate([g, pg] if K > 1 else [g], 1) * (spread[:, None] + 1e-30)
    assert (np.abs(got[2] - want[2]) <= 1e-5 * mag).all(), np.max(np.abs(got[2] - want[2]) / np.maximum(mag, 1e-300))
    assert (np.abs(got[3] - want[3]) <= 1e-5 * mag.sum(0) + 1e-30).all()
    return got


def case(rng, T, E, K, k, n_allowed, top_groups=0, scale=1.0):
    z = (rng.normal(size=(T, E + (K if K > 1 else 0))) * scale).astype(np.float32)
    mask = np.zeros(E, int)
    for j in range(K):  # as many in each group
        n = n_allowed * (j + 1) // K - n_allowed * j // K
        mask[j * (E // K) + rng.permutation(E // K)[:n]] = 1
    g = orc.gate_probabilities(z, mask, K, top_groups)
    return z, mask, np.argsort(-g, 1, kind="stable")[:, :k]


@pytest.mark.parametrize("T,E,K,k,n_allowed,top_groups", [
    (1, 8, 1, 1, 8, 0), (1, 8, 2, 2, 4, 0), (2, 1, 1, 1, 1, 0), (127, 16, 1, 1, 12, 0), (128, 24, 3, 3, 11, 0),
    (129, 64, 8, 6, 32, 0), (300, 64, 8, 6, 32, 4), (257, 128, 16, 8, 100, 2), (1025, 128, 1, 8, 128, 0),
    (3000, 8, 2, 2, 6, 1)])
def test_one_segment(T, E, K, k, n_allowed, top_groups):
    check(*case(np.random.default_rng(T + E), T, E, K, k, n_allowed, top_groups), K, top_groups=top_groups)


# Batches beyond the one-launch size, on every arrangement of the logits: lanes of 8
# and of 4 logits, aligned to 16 bytes or not, and rows in shared memory.
@pytest.mark.parametrize("T,E,K,k,n_allowed,top_groups", [
    (4000, 64, 8, 6, 32, 0), (3100, 64, 8, 6, 40, 3), (9000, 8, 2, 2, 6, 0), (20001, 16, 1, 1, 12, 0), (2500, 128, 16, 8, 70, 5),
    (5600, 12, 3, 3, 9, 0), (3500, 48, 12, 5, 30, 4), (2800, 96, 12, 6, 60, 0), (2800, 96, 1, 6, 60, 0), (9000, 16, 4, 2, 12, 2)])
def test_long_batches(T, E, K, k, n_allowed, top_groups):
    rng = np.random.default_rng(T)
    seg = [0, 100, 100, T // 2 + 1, T]
    check(*case(rng, T, E, K, k, n_allowed, top_groups), K, top_groups=top_groups, valid=rng.random(T) > 0.1, seg=seg)


def test_many_short_segments():
    T = 3000
    seg = sorted(np.random.default_rng(5).integers(0, T, 900).tolist())
    check(*case(np.random.default_rng(6), T, 64, 8, 6, 32), 8, seg=[0] + seg + [T])


def test_rows_with_a_pitch():
    for T in (300, 4000):
        check(*case(np.random.default_rng(T), T, 64, 8, 6, 32), 8, ld=77)


@pytest.mark.parametrize("seg", [[0, 700], [0, 1, 700], [0, 0, 350, 350, 699, 700, 700], [0, 100, 101, 400, 650],
                                 list(range(0, 701, 7))])
@pytest.mark.parametrize("padded", [0.0, 0.4])
def test_segments_and_padding(seg, padded):
    rng = np.random.default_rng(len(seg))
    z, mask, idx = case(rng, 700, 32, 4, 3, 20)
    valid = rng.random(700) >= padded if padded else None
    if seg[-1] < 700:  # tokens of no segment
        got = run(z, mask, idx, 4, valid=valid, seg=seg)
        assert not got[2][seg[-1]:].any()
        v = np.ones(700, bool) if valid is None else valid.copy()
        v[seg[-1]:] = False
        want = orc.balance(z, mask, idx, 4, 0.5, v, seg[:-1] + [700])
        assert abs(got[0] - want[0]) <= 1e-5 * want[0] and np.array_equal(got[1], want[1])
        return
    check(z, mask, idx, 4, valid=valid, seg=seg, d_loss=-3.0)


def test_no_token_counts():
    z, mask, idx = case(np.random.default_rng(1), 50, 8, 2, 2, 6)
    loss, counts, d, db, status = run(z, mask, idx, 2, valid=np.zeros(50))
    assert status == C.OK and loss == 0.0 and not counts.any() and not d.any() and not db.any()


def test_no_tokens():
    z, mask, idx = np.zeros((0, 10), np.float32), np.ones(8, int), np.zeros((0, 2), int)
    loss, counts, d, db, status = run(z, mask, idx, 2, k=2, seg=[0, 0, 0])
    assert status == C.OK and loss == 0.0 and not counts.any() and not db.any()


def test_masked_places_hold_anything():
    rng = np.random.default_rng(2)
    z, mask, idx = case(rng, 200, 16, 4, 2, 12)
    mask[4:8] = 0                                   # a group without an allowed expert
    idx = np.argsort(-orc.gate_probabilities(z, mask, 4), 1, kind="stable")[:, :2]
    z[:, 16 + 1] = np.nan                           # its global logit
    z[::3, np.flatnonzero(mask == 0)] = np.nan
    z[1::3, np.flatnonzero(mask == 0)] = np.inf
    z[2::3, np.flatnonzero(mask == 0)] = np.finfo(np.float32).min
    check(z, mask, idx, 4, ld=25)


def test_large_logits():
    z, mask, idx = case(np.random.default_rng(3), 300, 16, 2, 2, 16, scale=3.0)
    z += 1000.0
    check(z, mask, idx, 2)
    z[:, 3] = np.finfo(np.float32).min  # an allowed expert that no token can choose
    check(z, mask, np.where(idx == 3, 0, idx), 2)


def test_even_counts_give_no_gradient():
    """Even counts make the weights equal: the gradient is 0, not a rounding error."""
    T, E = 256, 8
    z = np.random.default_rng(4).normal(size=(T, E)).astype(np.float32)
    idx = (np.arange(T)[:, None] * 2 + np.arange(2)) % E
    loss, counts, d, db, _ = run(z, np.ones(E, int), idx, 1, coef=0.25)
    assert (counts == T * 2 // E).all() and not d.any() and abs(loss - 0.25) < 1e-6


def test_gradient_is_the_loss_difference():
    """Along a direction v: the loss is smooth, so (L(z + e v) - L(z - e v)) / 2e is the gradient's product with v
    up to e^2 (4e-4 of it) and 2^-22 of the loss over e."""
    rng = np.random.default_rng(6)
    z, mask, idx = case(rng, 16, 8, 2, 2, 7)
    idx = np.zeros_like(idx) + np.array([0, 1]) if mask[0] and mask[1] else idx
    _, _, d, _, _ = run(z, mask, idx, 2, coef=1.0)
    v = np.sign(d)
    e = 0.02
    hi = run((z + e * v).astype(np.float32), mask, idx, 2, coef=1.0)[0]
    lo = run((z - e * v).astype(np.float32), mask, idx, 2, coef=1.0)[0]
    want = np.abs(d).sum()
    assert want > 0.1
    assert abs((hi - lo) / (2 * e) - want) <= 5e-3 * want + 2.0 ** -22 * 8 / e


def test_ids_out_of_range_are_skipped():
    z, mask, idx = case(np.random.default_rng(7), 40, 8, 2, 2, 8)
    idx = idx.copy()
    idx[3, 1], idx[9, 0] = 8, -1
    loss, counts, _, _, status = run(z, mask, idx, 2)
    assert status == C.ERR_INVALID_ARG and counts.sum() == 78
    assert C.ec2moe_last_device_error() == C.OK


@pytest.mark.parametrize("T", [40, 9000])
@pytest.mark.parametrize("seg", [[0, 50, 20, 40], [-3, 10, 40], [0, 10, 9999]])
def test_bad_segments_are_reported(seg, T):
    z, mask, idx = case(np.random.default_rng(7), T, 8, 2, 2, 8)
    loss, counts, d, _, status = run(z, mask, idx, 2, seg=seg)
    assert status == C.ERR_INVALID_ARG and np.isfinite(loss) and np.isfinite(d).all()
    assert C.ec2moe_last_device_error() == C.OK


def test_outputs_that_are_not_wanted_and_repeats():
    z, mask, idx = case(np.random.default_rng(11), 5000, 64, 8, 6, 32)
    one = run(z, mask, idx, 8)
    none = run(z, mask, idx, 8, want_d=False)
    again = run(z, mask, idx, 8)
    assert one[0] == none[0] == again[0] and np.array_equal(one[2], again[2]) and np.array_equal(one[3], again[3])


# ----------------------------------------------------------------- logits
@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("T,d,E,K", [(1, 8, 1, 1), (1, 512, 8, 2), (5, 264, 10, 5), (130, 768, 64, 1), (257, 2048, 64, 8),
                                     (100, 1032, 128, 16), (300, 4096, 8, 2), (64, 520, 24, 3),
                                     (20000, 64, 8, 1), (5000, 264, 40, 5), (2000, 136, 16, 1), (400, 200, 112, 16)])
def test_gate_logits(dtype, T, d, E, K):
    rng = np.random.default_rng(T + d)
    dt = torch.bfloat16 if dtype == "bf16" else torch.float32
    X = cuda(rng.normal(size=(T, d)).astype(np.float32) * np.exp(rng.normal(size=(T, 1)))).to(dt)
    Wl, bl = (rng.normal(size=(E, d)) / np.sqrt(d)).astype(np.float32), rng.normal(size=E).astype(np.float32)
    Wg, bg = (rng.normal(size=(K, d)) / np.sqrt(d)).astype(np.float32), rng.normal(size=K).astype(np.float32)
    desc = C.make_desc(T=T, d=d, E=E, d_ff=0, k=1, n_groups=K, dtype=C.BF16 if dtype == "bf16" else C.F32)
    wsb = C.ec2moe_gate_logits_workspace_size(desc)
    ws = torch.randint(0, 255, (wsb,), dtype=torch.uint8, device="cuda")
    O = E + (K if K > 1 else 0)
    out = torch.full((T + 1, O), 7.0, device="cuda")
    C.ec2moe_gate_logits(desc, X, cuda(Wl), cuda(bl), cuda(Wg) if K > 1 else None, cuda(bg) if K > 1 else None, out, ws, wsb)
    assert C.ec2moe_last_device_error() == C.OK and (out[-1] == 7.0).all()
    W, b = (np.concatenate([Wl, Wg]), np.concatenate([bl, bg])) if K > 1 else (Wl, bl)
    x = X.double().cpu().numpy()
    want, mag = x @ W.T.astype(float) + b, np.abs(x) @ np.abs(W.T.astype(float)) + np.abs(b)
    err = np.abs(out[:-1].double().cpu().numpy() - want)
    assert (err <= (32 + d / 512 + 8) * 2.0 ** -23 * mag).all(), np.max(err / mag)


def test_gate_logits_zero_wait_budget_times_out_and_recovers():
    T, d, E, K = 20000, 2048, 64, 8
    g = torch.Generator(device="cuda")
    g.manual_seed(3)
    X = torch.randn(T, d, generator=g, device="cuda").to(torch.bfloat16)
    W = [torch.randn(n, d, generator=g, device="cuda") for n in (E, K)]
    b = [torch.zeros(n, device="cuda") for n in (E, K)]
    desc = C.make_desc(T=T, d=d, E=E, d_ff=0, k=1, n_groups=K)
    wsb = C.ec2moe_gate_logits_workspace_size(desc)
    ws = torch.empty(wsb, dtype=torch.uint8, device="cuda")

    def call():
        out = torch.zeros(T, E + K, device="cuda")
        C.ec2moe_gate_logits(desc, X, W[0], b[0], W[1], b[1], out, ws, wsb)
        return out, C.ec2moe_last_device_error()

    ref, status = call()
    assert status == C.OK
    old = C.ec2moe_get_wait_budget()
    try:
        C.ec2moe_set_wait_budget(0)
        status = call()[1]
    finally:
        C.ec2moe_set_wait_budget(old)
    assert status == C.ERR_TIMEOUT
    again, status = call()
    assert status == C.OK and torch.equal(again, ref)
