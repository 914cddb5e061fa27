"""The grouped bf16 products and their gradients against 64 bits, element by element.

Error of one element, with S the sum of its terms' magnitudes.  A tensor core's step
adds 16 products to the fp32 accumulator; each of its 17 addends is cut below 2^-23 of the
largest (at most S): 17 2^-23 S.  fp32 results hand a segment of 32 steps over: 544 2^-23 S at
most over all segments together (each segment's bound is of its own S), and the segments'
sums are added with 2^-24 S each.  bf16 results take segments of 512 steps, and are rounded by
2^-8 of themselves.
"""
import pytest
import torch

from paper_2508_06024_gb300 import build as B
from paper_2508_06024_gb300 import ec2moe as C
from tests import train_reference as ref

pytestmark = pytest.mark.gpu
BF = torch.bfloat16
SENTINEL = 7.0


@pytest.fixture(scope="module", autouse=True)
def lib():
    B.build()
    C.load()


def tolerance(value, mag, out, length):
    per_segment, steps = (32, length // 16 + 1) if out == C.F32 else (512, length // 16 + 1)
    segments = steps // per_segment + 17  # and the ranges of a split sum, which has fp32 segments
    bound = (17 * min(per_segment, steps) * 2.0 ** -23 + segments * 2.0 ** -24) * mag
    return bound if out == C.F32 else bound + 2.0 ** -8 * value.abs()


def operands(form, rows, N, K, G, seed=0, pad=0):
    g = torch.Generator(device="cuda").manual_seed(seed)

    def rand(*shape):
        return torch.randn(*shape, generator=g, device="cuda").to(BF)

    if form == "fwd":
        return rand(rows, K + pad), rand(G, N, K)
    if form == "dgrad":
        return rand(rows, N + pad), rand(G, N, K)
    return rand(rows, N + pad), rand(rows, K + pad)


def call(form, X, W, offsets, G, rows, N, K, out_type=C.BF16, perm=None, ldo=None, accumulate=0, into=None, stream=None,
         ws=None):
    offs = None if offsets is None else torch.tensor(offsets, dtype=torch.int32, device="cuda")
    if ws is None:
        ws = torch.empty(max(16, C.ec2moe_grouped_gemm_workspace_size(G, rows, N, K)), dtype=torch.uint8, device="cuda")
    t = torch.float32 if out_type == C.F32 else BF
    if form == "wgrad":
        out = torch.full((G, N, K), SENTINEL, dtype=t, device="cuda") if into is None else into
        C.ec2moe_grouped_gemm_wgrad(G, rows, N, K, X, X.stride(0), W, W.stride(0), offs, out_type, accumulate, out, ws,
                                    ws.numel(), stream)
        return out
    cols = N if form == "fwd" else K
    ldo = ldo or cols
    out = torch.full((rows, ldo), SENTINEL, dtype=t, device="cuda") if into is None else into
    fn = C.ec2moe_grouped_gemm if form == "fwd" else C.ec2moe_grouped_gemm_dgrad
    fn(G, rows, N, K, X, X.stride(0), offs, W, perm, out_type, out, ldo, ws, ws.numel(), stream)
    return out


def check(form, X, W, offsets, G, rows, N, K, out, out_type, perm=None, error=C.OK):
    assert C.ec2moe_last_device_error() == error
    owned = ref.groups([0, rows] if offsets is None else offsets, rows)
    depth = {"fwd": K, "dgrad": N}.get(form)
    x = X[:, :K if form == "fwd" else N]
    value, mag = ref.grouped(form, x, W if form != "wgrad" else W[:, :K], owned)
    if form == "wgrad":
        for g, (a, n) in enumerate(owned):
            err = (out[g].double() - value[g]).abs()
            assert bool((err <= tolerance(value[g], mag[g], out_type, n)).all()), (g, float(err.max()))
        return
    cols = value.shape[1]
    dest = torch.arange(rows, device="cuda") if perm is None else perm.long()
    held = ~torch.isnan(value).any(1)
    got = out[dest][held].double()
    err = (got[:, :cols] - value[held]).abs()
    assert bool((err <= tolerance(value[held], mag[held], out_type, depth)).all()), float(err.max())
    left = torch.ones(rows, dtype=torch.bool, device="cuda")
    left[dest[held]] = False
    assert bool((out[left] == SENTINEL).all()) and bool((out[:, cols:] == SENTINEL).all())


FORMS = ["fwd", "dgrad", "wgrad"]
TABLES = {
    "one": [0, 1],
    "one_of_many": [0, 0, 0, 1, 1],
    "ragged": [0, 3, 3, 20, 149, 150, 406, 663],
    "tails": [0, 16, 33, 65, 129, 193, 320, 321, 400],
    "gaps": [5, 40, 40, 100, 357],       # rows before the first and behind the last group
}


@pytest.mark.parametrize("form", FORMS)
@pytest.mark.parametrize("N,K", [(8, 8), (72, 64), (136, 520), (512, 256), (1000, 776)])
@pytest.mark.parametrize("table", list(TABLES))
def test_small(form, N, K, table):
    offsets = TABLES[table]
    G, rows = len(offsets) - 1, offsets[-1] + (9 if table == "gaps" else 0)
    X, W = operands(form, rows, N, K, G)
    for out_type in (C.BF16, C.F32):
        out = call(form, X, W, offsets, G, rows, N, K, out_type)
        check(form, X, W, offsets, G, rows, N, K, out, out_type)


@pytest.mark.parametrize("form", FORMS)
@pytest.mark.parametrize("rows,N,K", [(1, 4096, 1024), (300, 512, 4096), (5000, 264, 1408), (1027, 3000, 2056), (20001, 4104, 2560),
                                      (2500, 2560, 10248), (2500, 10248, 2560)])
@pytest.mark.parametrize("out_type", [C.BF16, C.F32])
def test_one_group(form, rows, N, K, out_type):
    X, W = operands(form, rows, N, K, 1, seed=1)
    out = call(form, X, W, None, 1, rows, N, K, out_type)
    check(form, X, W, None, 1, rows, N, K, out, out_type)


@pytest.mark.parametrize("form", FORMS)
@pytest.mark.parametrize("rows", [1, 31, 700, 6000])
def test_many_groups(form, rows):
    """64 and 128 groups, most of them with few rows or none."""
    for G in (64, 128):
        g = torch.Generator().manual_seed(rows)
        cuts = sorted(torch.randint(0, rows + 1, (G - 1,), generator=g).tolist())
        offsets = [0, *cuts, rows]
        X, W = operands(form, rows, 264, 392, G, seed=2)
        out = call(form, X, W, offsets, G, rows, 264, 392)
        check(form, X, W, offsets, G, rows, 264, 392, out, C.BF16)


@pytest.mark.parametrize("form", ["fwd", "dgrad"])
@pytest.mark.parametrize("out_type", [C.BF16, C.F32])
@pytest.mark.parametrize("rows", [40, 900])
def test_perm_and_pitches(form, out_type, rows):
    N, K, G = 392, 2048, 3
    offsets = [0, rows // 3, rows // 2, rows - 2]
    X, W = operands(form, rows, N, K, G, seed=3, pad=24)
    perm = torch.randperm(rows, generator=torch.Generator().manual_seed(5)).int().cuda()
    cols = N if form == "fwd" else K
    out = call(form, X, W, offsets, G, rows, N, K, out_type, perm=perm, ldo=cols + 8)
    check(form, X, W, offsets, G, rows, N, K, out, out_type, perm=perm)


@pytest.mark.parametrize("rows,G,N,K", [(700, 4, 264, 520), (3000, 1, 136, 512)])
def test_accumulate(rows, G, N, K):
    offsets = [0, 5, 5, 300, rows] if G == 4 else [0, rows]
    X, W = operands("wgrad", rows, N, K, G, seed=4, pad=8)
    before = torch.randn(G, N, K, device="cuda")
    out = before.clone()
    call("wgrad", X, W, offsets, G, rows, N, K, C.F32, accumulate=1, into=out)
    once = call("wgrad", X, W, offsets, G, rows, N, K, C.F32)
    assert C.ec2moe_last_device_error() == C.OK
    # one fp32 addition more than the call without it
    assert torch.equal(out, before + once)
    check("wgrad", X, W, offsets, G, rows, N, K, once, C.F32)
    if G == 4:
        assert torch.equal(out[1], before[1])


def test_no_rows():
    X, W = torch.zeros(0, 64, device="cuda", dtype=BF), torch.zeros(0, 32, device="cuda", dtype=BF)
    out = torch.full((3, 64, 32), SENTINEL, device="cuda")
    C.ec2moe_grouped_gemm_wgrad(3, 0, 64, 32, 0, 64, 0, 32, torch.zeros(4, dtype=torch.int32, device="cuda"), C.F32, 1, out)
    assert bool((out == SENTINEL).all())
    C.ec2moe_grouped_gemm_wgrad(3, 0, 64, 32, 0, 64, 0, 32, torch.zeros(4, dtype=torch.int32, device="cuda"), C.F32, 0, out)
    assert bool((out == 0).all())


@pytest.mark.parametrize("out_type", [C.BF16, C.F32])
@pytest.mark.parametrize("lengths", [[379, 379, 379], [443, 443, 443], [379, 384, 320, 443, 448, 379], [5, 64, 3, 128, 9, 0, 70, 2048, 1921]])
def test_ragged_sums_of_many_tiles(lengths, out_type):
    """Several tiles per CTA pair, each sum ending inside a block, with as many blocks as the pipeline has
    stages (6, 7) or with whole sums in between: blocks that end a sum come to the same stage one after the other."""
    offsets = [0]
    for n in lengths:
        offsets.append(offsets[-1] + n)
    G, rows, N, K = len(lengths), offsets[-1], 3000, 2560
    X, W = operands("wgrad", rows, N, K, G, seed=14)
    for _ in range(2):
        out = call("wgrad", X, W, offsets, G, rows, N, K, out_type)
        check("wgrad", X, W, offsets, G, rows, N, K, out, out_type)


@pytest.mark.parametrize("out_type,accumulate", [(C.BF16, 0), (C.F32, 0), (C.F32, 1)])
@pytest.mark.parametrize("form", FORMS)
@pytest.mark.parametrize("lengths,N,K", [([0, 3000, 1], 264, 520), ([900, 0, 40, 1500], 520, 1024), ([130], 264, 2048), ([7], 2048, 264),
                                         ([2, 1, 300, 0, 5], 1032, 1544)])
def test_few_tiles(form, lengths, N, K, out_type, accumulate):
    """Sums that are cut into ranges, for groups with many, few and no rows."""
    offsets = [0]
    for n in lengths:
        offsets.append(offsets[-1] + n)
    G, rows = len(lengths), offsets[-1]
    X, W = operands(form, rows, N, K, G, seed=15)
    out = call(form, X, W, offsets, G, rows, N, K, out_type)
    check(form, X, W, offsets, G, rows, N, K, out, out_type)
    if accumulate and form == "wgrad":
        twice = call(form, X, W, offsets, G, rows, N, K, out_type, accumulate=1, into=out.clone())
        assert torch.equal(twice, out + out)
    elif form != "wgrad":
        perm = torch.arange(rows, dtype=torch.int32, device="cuda").flip(0).contiguous()
        other = call(form, X, W, offsets, G, rows, N, K, out_type, perm=perm)
        assert torch.equal(other, out.flip(0))


@pytest.mark.parametrize("form", FORMS)
def test_other_groups_values_stay_out(form):
    """Infinities and NaN in one group's rows, and in rows of no group, reach no other group's results."""
    offsets, N, K = [0, 37, 101, 170, 300], 200, 328
    G, rows = 4, 310
    X, W = operands(form, rows, N, K, G, seed=6)
    for t in ((X,) if form != "wgrad" else (X, W)):
        t[37:101:2] = float("inf")
        t[38:101:2] = float("nan")
        t[300:] = float("nan")
    if form != "wgrad":
        W[1] = float("inf")
    out = call(form, X, W, offsets, G, rows, N, K, C.F32)
    assert C.ec2moe_last_device_error() == C.OK
    value, mag = ref.grouped(form, X, W, ref.groups(offsets, rows))
    for g, (a, b) in enumerate(zip(offsets[:-1], offsets[1:])):
        if g == 1:
            continue
        got, v, m = (out[g], value[g], mag[g]) if form == "wgrad" else (out[a:b], value[a:b], mag[a:b])
        depth = {"fwd": K, "dgrad": N, "wgrad": b - a}[form]
        assert bool(((got.double() - v).abs() <= tolerance(v, m, C.F32, depth)).all()), g
    if form != "wgrad":
        assert bool((out[300:] == SENTINEL).all())


@pytest.mark.parametrize("form", FORMS)
@pytest.mark.parametrize("offsets", [[0, 50, 20, 90, 120], [0, 60, 400, 100, 120], [-4, 60, 90, 100, 120], [0, 80, 60, 120, 120]])
def test_bad_ranges_are_skipped_and_reported(form, offsets):
    G, rows, N, K = 4, 120, 136, 200
    X, W = operands(form, rows, N, K, G, seed=7)
    out = call(form, X, W, offsets, G, rows, N, K)
    check(form, X, W, offsets, G, rows, N, K, out, C.BF16, error=C.ERR_INVALID_ARG)
    assert C.ec2moe_last_device_error() == C.OK


@pytest.mark.parametrize("form", ["fwd", "dgrad"])
@pytest.mark.parametrize("N,K", [(136, 200), (256, 8192), (8192, 256)])
def test_bad_destinations_are_skipped_and_reported(form, N, K):
    rows = 20
    X, W = operands(form, rows, N, K, 1, seed=8)
    perm = torch.arange(rows, dtype=torch.int32, device="cuda")
    perm[3], perm[7] = -1, rows
    out = call(form, X, W, None, 1, rows, N, K, perm=perm)
    assert C.ec2moe_last_device_error() == C.ERR_INVALID_ARG
    value, mag = ref.grouped(form, X, W, [(0, rows)])
    keep = torch.tensor([i for i in range(rows) if i not in (3, 7)], device="cuda")
    err = (out[keep].double() - value[keep]).abs()
    assert bool((err <= tolerance(value[keep], mag[keep], C.BF16, K if form == "fwd" else N)).all())
    assert bool((out[[3, 7]] == SENTINEL).all())


@pytest.mark.parametrize("form", FORMS)
@pytest.mark.parametrize("rows,N,K", [(500, 264, 4096), (9000, 512, 512)])
def test_same_bits_again(form, rows, N, K):
    offsets = [0, rows // 7, rows // 2, rows]
    X, W = operands(form, rows, N, K, 3, seed=9)
    a = call(form, X, W, offsets, 3, rows, N, K, C.F32)
    b = call(form, X, W, offsets, 3, rows, N, K, C.F32)
    assert torch.equal(a, b)


def test_gradients_by_differences():
    """<dC, C(A + e dA)> and <dC, C(B + e dB)> change as dgrad and wgrad say: the products are linear in each
    operand, so the difference with e = 1 is exact up to the sums' roundings (fp32 results)."""
    offsets, N, K, G, rows = [0, 70, 70, 200], 136, 264, 3, 200
    A, W = operands("fwd", rows, N, K, G, seed=10)
    dC, _ = operands("dgrad", rows, N, K, G, seed=11)
    eA, eW = operands("fwd", rows, N, K, G, seed=12)
    C0 = call("fwd", A, W, offsets, G, rows, N, K, C.F32).double()
    dA = call("dgrad", dC, W, offsets, G, rows, N, K, C.F32).double()
    dW = call("wgrad", dC, A, offsets, G, rows, N, K, C.F32).double()
    dc = dC.double()
    for step, change in ((eA, (dA * eA.double()).sum()), (eW, (dW * eW.double()).sum())):
        moved = call("fwd", A if step is eW else step, step if step is eW else W, offsets, G, rows, N, K, C.F32).double()
        # C(e) alone is the change of C, by linearity
        assert abs(float((dc * moved).sum() - change)) <= 1e-5 * float((dc * moved).abs().sum())
    assert torch.isfinite(C0).all()


def test_graph_replay_and_streams():
    offsets, N, K, G, rows = [0, 70, 70, 1200], 512, 1024, 3, 1200
    cases = {f: operands(f, rows, N, K, G, seed=13) for f in FORMS}
    want = {f: call(f, *cases[f], offsets, G, rows, N, K) for f in FORMS}
    offs = torch.tensor(offsets, dtype=torch.int32, device="cuda")
    n_ws = max(16, C.ec2moe_grouped_gemm_workspace_size(G, rows, N, K))
    side = torch.cuda.Stream()
    outs = {f: torch.empty_like(want[f]) for f in FORMS}
    ws = {f: torch.empty(n_ws, dtype=torch.uint8, device="cuda") for f in FORMS}
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        for f in FORMS:
            X, W = cases[f]
            if f == "wgrad":
                C.ec2moe_grouped_gemm_wgrad(G, rows, N, K, X, N, W, K, offs, C.BF16, 0, outs[f], ws[f], n_ws)
            elif f == "fwd":
                C.ec2moe_grouped_gemm(G, rows, N, K, X, K, offs, W, None, C.BF16, outs[f], N, ws[f], n_ws)
            else:
                C.ec2moe_grouped_gemm_dgrad(G, rows, N, K, X, N, offs, W, None, C.BF16, outs[f], K, ws[f], n_ws)
    for _ in range(3):
        for f in FORMS:
            outs[f].zero_()
        graph.replay()
        torch.cuda.synchronize()
        for f in FORMS:
            assert torch.equal(outs[f], want[f]), f
    # two calls at once, on streams and workspaces of their own
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    got = {}
    for s, f in zip(streams, ("fwd", "wgrad")):
        got[f] = torch.full_like(want[f], SENTINEL)
        s.wait_stream(torch.cuda.current_stream())
    for s, f in zip(streams, ("fwd", "wgrad")):
        call(f, *cases[f], offsets, G, rows, N, K, into=got[f], stream=s, ws=ws[f])
    torch.cuda.synchronize()
    for f in got:
        assert torch.equal(got[f], want[f]), f
