"""GPU parity of the matrix product over rows (mnn_linear_*) against its definition in fp64.

Tolerance, per element, with S = the sum of the absolute terms (products, bias, residual):
* products of 16-bit values are exact in fp32; the tensor core adds 16 of them per step and cuts the sum off, at most 2^-23 of
  the running sum, which never exceeds S: (K / 16 + 8) 2^-23 S, the 8 for the joins of a cluster, bias and residual;
* up to four rows are summed by 32 lanes or more, each at most K / 32 + 8 rounded additions, far inside the bounds below;
* fp32 operands lose at most 2^-20 each to the cut of their low halves and 2^-20 to the product of the low halves (both halves
  are cut off, not rounded: |lo| < 2^-10 |v|): 3 * 2^-20 S; at most 24 steps of 8 elements between additions
  to registers, cut off: 24 * 2^-23 S, one rounded addition per 64 elements: (K / 64 + 8) 2^-24 S;
* the activations have slopes of at most 1.13; their own evaluation errs by at most 2^-19 of the value with the fast
  exponential and division (16-bit types), 2^-21 of the value with the exact ones;
* one rounding at the store: half an eps of the type.
"""
import numpy as np
import pytest

from oracle import rows as oracle
from paper_2002_12418_b200 import binding as B

pytestmark = pytest.mark.gpu
HALF_EPS = {"fp32": 2.0 ** -24, "bf16": 2.0 ** -8, "fp16": 2.0 ** -11}


def bound(y, s, size, K, dtype):
    if dtype == "fp32":
        err = (3 * 2.0 ** -20 + 24 * 2.0 ** -23 + (K / 64 + 8) * 2.0 ** -24) * size
        own = 2.0 ** -21
    else:
        err = (K / 16 + 8) * 2.0 ** -23 * size
        own = 2.0 ** -19
    err = 1.13 * err + own * np.abs(s) + 1e-30
    tiny = 2.0 ** -25 if dtype == "fp16" else 0.0          # half the spacing of the smallest halves
    return err + HALF_EPS[dtype] * (np.abs(y) + err) + tiny


def make(torch, seed, shape, ld, dtype, scale=1.0, offset=0):
    """Rows `ld` elements apart, `offset` elements behind an aligned address; what lies between rows is NaN."""
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    t = {"fp32": torch.float32, "bf16": torch.bfloat16, "fp16": torch.float16}[dtype]
    flat = torch.full((offset + shape[0] * ld + 16,), float("nan"), dtype=t, device="cuda")
    view = flat[offset:offset + shape[0] * ld].view(shape[0], ld)[:, :shape[1]]
    view.copy_(torch.randn(shape, generator=g, device="cuda") * scale)
    return view


def host(t):
    return None if t is None else t.double().cpu().numpy()


def run_case(M, K, N, dtype, act="none", mode="none", bias=True, pads=(0, 0, 0, 0), offset=0, seed=0, in_place=False):
    import torch
    ldx, ldw, ldy, ldr = K + pads[0], K + pads[1], N + pads[2], N + pads[3]
    x = make(torch, seed, (M, K), ldx, dtype, offset=offset)
    w = make(torch, seed + 1, (N, K), ldw, dtype, K ** -0.5, offset=offset)
    b = make(torch, seed + 2, (1, N), N, dtype, 0.5)[0].contiguous() if bias else None
    r = make(torch, seed + 3, (M, N), ldr, dtype) if mode != "none" else None
    runner = B.LinearRunner(M, N, K, dtype, act, mode, ldx, ldw, ldy, ldr)
    want, s, size = oracle.linear(host(x), host(w), host(b), host(r), act, mode)
    if in_place:
        y = r
    else:
        whole = torch.full((M, ldy), 7.0, dtype=x.dtype, device="cuda")
        y = whole[:, :N]
    runner.run(x, w, b, r, y)
    torch.cuda.synchronize()
    assert runner.device_status() == 0
    got = host(y)
    over = np.abs(got - want) - bound(want, s, size, K, dtype)
    assert np.isfinite(got).all() and (over <= 0).all(), "worst excess %.3e at %s" % (over.max(), np.unravel_index(over.argmax(), over.shape))
    if not in_place and ldy > N:
        assert (whole[:, N:] == 7.0).all(), "columns behind the rows' end were written"
    info = runner.info
    runner.close()
    return got, info


# every type; a single row, a few, and sizes around the tiles of 16..256 rows, 128 features and 32 or 64 elements of K
@pytest.mark.parametrize("dtype", ["fp32", "bf16", "fp16"])
@pytest.mark.parametrize("M,K,N", [(1, 1, 1), (1, 64, 128), (1, 1024, 1000), (3, 72, 130), (16, 512, 640), (17, 96, 256), (33, 200, 129),
                                   (64, 2048, 512), (100, 328, 385), (129, 640, 127), (257, 256, 300), (700, 136, 1000)])
def test_sizes(M, K, N, dtype):
    run_case(M, K, N, dtype, seed=M + K + N)


@pytest.mark.parametrize("dtype", ["fp32", "bf16", "fp16"])
@pytest.mark.parametrize("act", ["none", "relu", "gelu", "gelu_tanh", "silu"])
@pytest.mark.parametrize("mode", ["none", "after", "before"])
def test_epilogues(act, mode, dtype):
    run_case(37, 264, 200, dtype, act, mode, seed=5)
    run_case(300, 264, 1040, dtype, act, mode, bias=False, seed=6)


# rows that TMA cannot copy: odd lengths and strides, odd base addresses
@pytest.mark.parametrize("dtype", ["fp32", "bf16", "fp16"])
@pytest.mark.parametrize("M,K,N,pads,offset", [(1, 7, 5, (0, 0, 0, 0), 0), (5, 1001, 131, (0, 0, 0, 0), 1), (77, 1001, 513, (3, 0, 3, 3), 0),
                                               (40, 64, 96, (1, 8, 0, 0), 0), (130, 333, 260, (2, 5, 1, 7), 3), (16, 4096, 300, (0, 0, 0, 0), 1),
                                               (600, 129, 700, (0, 0, 0, 0), 0)])
def test_unaligned_rows(M, K, N, pads, offset, dtype):
    run_case(M, K, N, dtype, "silu", "after", pads=pads, offset=offset, seed=M + K)


# tensors that start at odd addresses, with rows that TMA could copy otherwise
@pytest.mark.parametrize("dtype", ["fp32", "bf16", "fp16"])
@pytest.mark.parametrize("M,K,N", [(2, 256, 300), (4, 1000, 77), (20, 256, 300), (70, 1032, 260), (300, 96, 1000)])
def test_unaligned_starts(M, K, N, dtype):
    run_case(M, K, N, dtype, "relu", "before", pads=(16 - K % 16, 32 - K % 16, 0, 0), offset=1, seed=M)


# fp32 on pairs: rows of very different sizes (each has its own scale), and values of very different sizes within a row
def test_scales_of_rows():
    import torch
    M, K, N = 1500, 640, 1300
    x, w = make(torch, 1, (M, K), K, "fp32"), make(torch, 2, (N, K), K, "fp32")
    x *= 10.0 ** torch.linspace(-18, 18, M, device="cuda")[:, None]
    w *= 10.0 ** torch.linspace(18, -18, N, device="cuda")[:, None]
    x[7], x[8], w[9] = 0.0, 1e-42, 1e-44                  # nothing, and denormals
    x[:, ::5] *= 1e-4
    w[:, 1::3] *= 1e-3
    r = B.LinearRunner(M, N, K, "fp32")
    assert r.info.form == B.LINEAR_PAIRS
    got = host(r.run(x, w))
    want, s, size = oracle.linear(host(x), host(w))
    # beside the bounds of above: 2^-38 of the largest values' products per term, and fp32's own smallest step
    most = np.abs(host(x)).max(1)[:, None] * np.abs(host(w)).max(1)[None, :]
    assert (np.abs(got - want) <= bound(want, s, size, K, "fp32") + K * 2.0 ** -38 * most + 2.0 ** -149).all()


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
def test_padded_rows_by_tma(dtype):
    _, info = run_case(70, 128, 200, dtype, "relu", "before", pads=(8, 16, 1, 24), seed=9)
    assert info.form == B.LINEAR_TILES


def test_residual_in_place():
    run_case(50, 256, 300, "bf16", "none", "after", seed=11, in_place=True)
    run_case(520, 256, 2048, "fp32", "relu", "before", seed=12, in_place=True)


# the kernel on pairs of SMs, at sizes off its 256 x 256 blocks
@pytest.mark.parametrize("dtype,M,K,N", [("bf16", 2048, 512, 4096), ("fp16", 1900, 520, 4200), ("bf16", 4001, 392, 3003), ("fp32", 1500, 640, 1030),
                                         ("fp32", 2100, 260, 1700), ("fp32", 1300, 771, 1100), ("bf16", 2000, 1537, 4000), ("fp16", 1201, 2051, 3333)])
def test_pairs(dtype, M, K, N):
    _, info = run_case(M, K, N, dtype, "silu", "after", seed=21)
    assert info.form == B.LINEAR_PAIRS


# integers small enough that every sum is exact: any correct evaluation is bit-identical
@pytest.mark.parametrize("dtype,M,K,N", [("fp32", 200, 300, 260), ("bf16", 200, 296, 260), ("fp16", 200, 299, 260), ("bf16", 2048, 256, 4096),
                                         ("fp32", 4, 4096, 256), ("bf16", 4, 4096, 256), ("fp32", 1, 4096, 5000), ("bf16", 1, 4097, 256),
                                         ("bf16", 3, 1000, 9000), ("fp16", 2, 72, 20), ("fp32", 1700, 256, 1800), ("fp32", 1700, 257, 1800), ("fp32", 12, 4096, 256)])
def test_integers_are_exact(dtype, M, K, N):
    import torch
    g = torch.Generator(device="cuda")
    g.manual_seed(3)
    t = {"fp32": torch.float32, "bf16": torch.bfloat16, "fp16": torch.float16}[dtype]
    x = torch.randint(-4, 5, (M, K), generator=g, device="cuda").to(t)
    w = torch.randint(-4, 5, (N, K), generator=g, device="cuda").to(t)
    b = torch.randint(-4, 5, (N,), generator=g, device="cuda").to(t)
    r = B.LinearRunner(M, N, K, dtype)
    y = r.run(x, w, b)
    want = (x.double() @ w.double().t() + b.double()).to(t)
    assert torch.equal(y, want) and r.device_status() == 0
    y2 = r.run(x, w, b)
    assert torch.equal(y, y2)


@pytest.mark.parametrize("dtype", ["fp32", "bf16", "fp16"])
@pytest.mark.parametrize("K", [96, 101, 1024])
def test_infinities_and_nan(dtype, K):
    import torch
    for rows in (1, 20, 1400):       # the kernels for few rows, for tiles and on pairs
        check_infinities(torch, rows, K, 140 if rows < 1000 else 1540, dtype)


def check_infinities(torch, M, K, N, dtype):
    x = make(torch, 1, (M, K), K, dtype)
    w = make(torch, 2, (N, K), K, dtype)
    x[3 % M, 5], x[4 % M, K - 1], x[6 % M, 2], w[7, 9] = (float("inf"), float("-inf"), float("nan"), float("inf")) if M > 1 else (float("inf"), 1.0, 1.0, float("inf"))
    w[9, 5] = 0.0                                    # infinity times zero
    r = B.LinearRunner(M, N, K, dtype)
    got = host(r.run(x, w))
    want, s, size = oracle.linear(host(x), host(w))
    assert np.array_equal(np.isnan(got), np.isnan(want)) and np.array_equal(np.isinf(got), np.isinf(want))
    assert np.array_equal(got[np.isinf(want)], want[np.isinf(want)])
    fine = np.isfinite(want)
    assert (np.abs(got[fine] - want[fine]) <= bound(want, s, size, K, dtype)[fine]).all()
    assert r.device_status() == 0


@pytest.mark.parametrize("dtype", ["fp32", "bf16", "fp16"])
@pytest.mark.parametrize("M,K,N,pads,offset", [(5, 256, 48, (0, 0, 0, 0), 0), (13, 101, 7, (0, 3, 1, 2), 0), (7, 1000, 77, (0, 0, 0, 0), 1),
                                               (100, 256, 48, (0, 0, 0, 0), 0), (1001, 40, 1, (0, 0, 0, 0), 0), (5903, 19, 2, (0, 0, 1, 0), 0)])
def test_groups_of_four_rows(M, K, N, pads, offset, dtype):
    _, info = run_case(M, K, N, dtype, "silu", "before", pads=pads, offset=offset, seed=M)
    assert info.form == B.LINEAR_FEW


@pytest.mark.parametrize("M,K,N", [(5, 12009, 700), (19, 4099, 530), (200, 4100, 260), (192, 1027, 16), (260, 4099, 300)])
@pytest.mark.parametrize("dtype", ["fp32", "fp16"])
def test_operands_laid_out_by_several_warps_a_row(M, K, N, dtype):
    _, info = run_case(M, K, N, dtype, "none", "after", pads=(1, 0, 0, 0), seed=K)
    assert info.launches_per_run == 2 or info.form == B.LINEAR_FEW


@pytest.mark.parametrize("M,K,N,pads", [(80, 1001, 8000, (0, 0, 0, 0)), (114, 707, 6225, (0, 2, 1, 0))])
def test_pairs_of_fewer_unaligned_rows(M, K, N, pads):
    _, info = run_case(M, K, N, "fp32", "relu", "before", pads=pads, seed=M)
    assert info.form == B.LINEAR_PAIRS


@pytest.mark.parametrize("dtype,M,K,N,few", [("bf16", 1, 1000, 40000, False), ("fp16", 2, 1024, 14000, False), ("bf16", 2, 1024, 9001, True),
                                            ("fp32", 4, 1000, 9001, True), ("fp32", 3, 4096, 3100, False), ("fp16", 4, 1022, 5001, True)])
def test_few_rows_of_large_products(dtype, M, K, N, few):
    _, info = run_case(M, K, N, dtype, "gelu", "after", seed=N)
    assert (info.form == B.LINEAR_FEW) == few


@pytest.mark.parametrize("M,N,form", [(2048, 4096, B.LINEAR_PAIRS), (64, 4096, B.LINEAR_TILES)])
def test_nothing_but_nan(M, N, form):
    """Every sum is taken a second time, without a wait that runs out; the workspace is good for the next run."""
    import torch
    K = 16384
    r = B.LinearRunner(M, N, K)
    assert r.info.form == form
    x, w = torch.full((M, K), float("nan"), device="cuda"), torch.ones(N, K, device="cuda")
    y = r.run(x, w)
    torch.cuda.synchronize()
    assert r.device_status() == 0 and torch.isnan(y).all()
    x.fill_(0.5)
    y = r.run(x, w)
    torch.cuda.synchronize()
    assert r.device_status() == 0 and (y == 0.5 * K).all()
    r.close()


def test_relu_keeps_nan_and_half_overflows_to_infinity():
    import torch
    x = torch.full((2, 64), 200.0, dtype=torch.float16, device="cuda")
    w = torch.full((3, 64), 200.0, dtype=torch.float16, device="cuda")
    x[1, 0] = float("nan")
    y = B.LinearRunner(2, 3, 64, "fp16", act="relu").run(x, w)
    assert torch.isinf(y[0]).all() and torch.isnan(y[1]).all()


def test_graph_replay_other_stream_and_two_plans_at_once():
    import torch
    M, K, N = 24, 512, 1024
    x, w = make(torch, 1, (M, K), K, "bf16"), make(torch, 2, (N, K), K, "bf16")
    r, r2 = B.LinearRunner(M, N, K, "bf16", act="gelu"), B.LinearRunner(M, N, K, "bf16", act="gelu")
    want = r.run(x, w)
    y = torch.empty_like(want)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        r.run(x, w, y=y)
    y.zero_()
    x2 = x.clone()
    for _ in range(3):
        graph.replay()
    torch.cuda.synchronize()
    assert torch.equal(y, want)
    x.mul_(2)                                        # a replay reads what lies there now
    graph.replay()
    torch.cuda.synchronize()
    assert torch.equal(y, r2.run(x, w)) and not torch.equal(y, want)
    with torch.cuda.stream(side):
        a = r.run(x2, w)
    b = r2.run(x2, w)
    torch.cuda.synchronize()
    assert torch.equal(a, want) and torch.equal(b, want)


# forms that lay operands out in the workspace first, captured and replayed on new inputs
@pytest.mark.parametrize("dtype,M,K,N", [("fp32", 1500, 640, 1300), ("bf16", 77, 1001, 513)])
def test_graph_replay_with_operands_laid_out(dtype, M, K, N):
    import torch
    x, w = make(torch, 1, (M, K), K, dtype), make(torch, 2, (N, K), K, dtype)
    r, other = B.LinearRunner(M, N, K, dtype), B.LinearRunner(M, N, K, dtype)
    assert r.info.launches_per_run == 2
    r.run(x, w)
    torch.cuda.synchronize()
    y = torch.empty(M, N, dtype=x.dtype, device="cuda")
    graph, side = torch.cuda.CUDAGraph(), torch.cuda.Stream()
    with torch.cuda.graph(graph, stream=side):
        r.run(x, w, y=y)
        r.run(x, w, y=y)
    x.mul_(0.5)
    w.add_(0.25)
    graph.replay()
    torch.cuda.synchronize()
    assert torch.equal(y, other.run(x, w)) and r.device_status() == 0


def test_refusals_of_tensors():
    import torch
    r = B.LinearRunner(4, 8, 16, "bf16", residual="after")
    x, w, y = (torch.zeros(s, dtype=torch.bfloat16, device="cuda") for s in ((4, 16), (8, 16), (4, 8)))
    res = torch.zeros_like(y)
    r.run(x, w, None, res, y)
    for bad in (dict(x=x.float()), dict(x=x[:3]), dict(x=x.cpu()), dict(w=w.t()), dict(residual=None), dict(bias=torch.zeros(7, device="cuda", dtype=torch.bfloat16)),
                dict(y=torch.zeros(4, 9, dtype=torch.bfloat16, device="cuda")[:, :8])):
        a = dict(x=x, w=w, bias=None, residual=res, y=y)
        a.update(bad)
        with pytest.raises(B.MnnError) as e:
            r.run(a["x"], a["w"], a["bias"], a["residual"], a["y"])
        assert e.value.code == B.MNN_EINVAL
    # overlapping memory: y inside x; y one row behind its residual
    flat = torch.zeros(16 * 16, dtype=torch.bfloat16, device="cuda")
    with pytest.raises(B.MnnError):
        r.run(flat[:64].view(4, 16), w, None, res, flat[8:40].view(4, 8))
    with pytest.raises(B.MnnError):
        r.run(x, w, None, flat[:32].view(4, 8), flat[8:40].view(4, 8))
    # columns side by side in one buffer do not overlap
    both = torch.zeros(4, 24, dtype=torch.bfloat16, device="cuda")
    B.LinearRunner(4, 8, 16, "bf16", ldx=24, ldy=24).run(both[:, :16], w, y=both[:, 16:])
    torch.cuda.synchronize()


# every sum infinite and K so long that taking the sums of one work item again lasts longer than a wait may (1.8 and 1.5 s, a wait one
# second): a second item's waits must not run out meanwhile.  A record of two SMs gives one SM, or the pair of them, two items at small
# sizes.
@pytest.mark.parametrize("M,N,K,form", [(96, 384, 1 << 18, B.LINEAR_TILES), (256, 512, 1 << 16, B.LINEAR_PAIRS)])
def test_infinite_sums_of_a_very_long_k(M, N, K, form):
    import torch
    before = B.mnn_get_calibration()
    try:
        record = list(before)
        record[7] = 2
        B.mnn_set_calibration(record)
        r = B.LinearRunner(M, N, K)
    finally:
        B.mnn_set_calibration(before)
    assert r.info.form == form and r.info.split == 1 and r.info.items > (2 if form == B.LINEAR_TILES else 1)
    g = torch.Generator(device="cuda")
    g.manual_seed(7)
    x, w = torch.full((M, K), 0.5, device="cuda"), torch.ones(N, K, device="cuda")
    at = torch.randint(0, K, (M,), generator=g, device="cuda")
    rows = torch.arange(M, device="cuda")
    x[rows, at] = torch.where(rows % 2 == 0, float("inf"), float("-inf"))
    y = r.run(x, w)
    torch.cuda.synchronize()
    assert r.device_status() == 0
    assert (y[0::2] == float("inf")).all() and (y[1::2] == float("-inf")).all()
    x[rows, at] = 0.5                                # and the workspace is good for the next run
    y = r.run(x, w)
    torch.cuda.synchronize()
    assert r.device_status() == 0 and (y == 0.5 * K).all()


# GELU's tail: with sums that are exact (one term, of 8 bits), what is left is the evaluation of v h(|v|) or v (1 - h), h = erfc(|v| / sqrt 2) / 2 =
# e^(-v^2/2) q(t), t = 1 / (1 + c |v|).  Relative errors in units of 2^-24: the exponent v^2 / 2 is rounded twice and its factor once, 1.5 v^2;
# the exponential 4; t 3 (fp32: 2.2) that q's slope of 2.7 makes 8 (6); q's own roundings 6.5; its fit 32 (0.5); three products and a difference 3.
@pytest.mark.parametrize("dtype", ["fp32", "bf16", "fp16"])
@pytest.mark.parametrize("M,N,form", [(1, 4096, B.LINEAR_FEW), (64, 4096, B.LINEAR_TILES), (2048, 4096, B.LINEAR_PAIRS)])
def test_gelu_far_from_zero(M, N, form, dtype):
    import math

    import torch
    K = 256
    t = {"fp32": torch.float32, "bf16": torch.bfloat16, "fp16": torch.float16}[dtype]
    v = (torch.arange(N, device="cuda") / (N / 24.0) - 12.0).bfloat16()          # -12 to 12 in 8 bits
    x, w = torch.zeros(M, K, dtype=t, device="cuda"), torch.zeros(N, K, dtype=t, device="cuda")
    x[:, 3], w[:, 3] = 1.0, v.to(t)
    r = B.LinearRunner(M, N, K, dtype, act="gelu")
    assert r.info.form == form
    got = host(r.run(x, w))
    s = host(v)
    want = np.array([0.5 * a * math.erfc(-a / math.sqrt(2.0)) for a in s])
    err = (1.5 * s * s + (20.0 if dtype == "fp32" else 54.0)) * 2.0 ** -24 * np.abs(want)
    err += HALF_EPS[dtype] * (np.abs(want) + err) + (2.0 ** -25 if dtype == "fp16" else 0.0)
    over = np.abs(got - want[None, :]) - err[None, :]
    assert (over <= 0).all(), (over.max(), s[over.max(0).argmax()])


def test_gelu_of_infinities_and_far_values():
    import torch
    inf = float("inf")
    for dtype, N in (("fp32", 8), ("bf16", 8), ("fp32", 300000), ("bf16", 300000)):
        t = torch.float32 if dtype == "fp32" else torch.bfloat16
        w = torch.zeros(N, 8, dtype=t, device="cuda")
        w[:8, 0] = torch.tensor([inf, -inf, float("nan"), 1e38, -1e38, -40.0, 1e19, -1e19], device="cuda").to(t)
        x = torch.zeros(1, 8, dtype=t, device="cuda")
        x[0, 0] = 1.0
        r = B.LinearRunner(1 if N == 8 else 40, N, 8, dtype, act="gelu")
        y = r.run(x if N == 8 else x.repeat(40, 1), w).float()
        v = w[:8, 0].float()
        for row in (y[0], y[-1]):
            assert row[0] == inf and torch.isnan(row[1:3]).all()                 # minus infinity times nothing
            # fp32 operands on tiles are two halves of 11 bits, each off by less than 2^-10 of it: 2^-20 of a value (the sum is 1 * v)
            assert ((row[[3, 6]] - v[[3, 6]]).abs() <= 2.0 ** -20 * v[[3, 6]]).all() and (row[[4, 5, 7]] == 0).all() and (row[8:] == 0).all()


# fp32 on tiles, one term: hi hi + lo hi + hi lo with hi the upper 11 bits of a value and lo what is left of it, rounded to 11 bits.  lo is smaller
# than 2^-10 of the value (of its power of two), so that its rounding is off by at most half of 2^-10 2^-11: 2^-22.  Beside the missing lo lo, which is
# known, the product is off by 2^-22 for each operand, by 2^-24 for the rounding of the sum, and by what is cut off lo hi + hi lo, 2^-23 of it, 2^-32.
@pytest.mark.parametrize("offset", [0, 1])
def test_low_halves_are_rounded(offset):
    import torch
    M, N, K = 64, 4096, 256
    x, w = make(torch, 1, (M, K), K, "fp32", offset=offset), make(torch, 2, (N, K), K, "fp32", offset=offset)
    x[:, :7], x[:, 8:] = 0.0, 0.0
    w[:, 7].copy_(w[:, 3])
    r = B.LinearRunner(M, N, K)
    assert r.info.form == B.LINEAR_TILES and r.info.form_unaligned == B.LINEAR_COPIED
    got = host(r.run(x, w))
    assert r.device_status() == 0
    a, b = x[:, 7].contiguous(), w[:, 7].contiguous()
    lo = lambda t: host(t) - host((t.view(torch.int32) & -8192).view(torch.float32))  # noqa: E731
    product = host(a)[:, None] * host(b)[None, :]
    want = product - lo(a)[:, None] * lo(b)[None, :]
    over = np.abs(got - want) - (2 * 2.0 ** -22 + 2.0 ** -24 + 2.0 ** -32) * np.abs(product)
    assert (over <= 0).all(), over.max()


# tensors that start off 16 bytes, fetched by copier warps: several work items to a CTA (a record of three SMs), so that the ring of stages goes on
# from one to the next at every phase, and K loops shared by a cluster.
@pytest.mark.parametrize("dtype", ["fp32", "bf16", "fp16"])
@pytest.mark.parametrize("sms,M,K,N", [(3, 70, 264, 1300), (3, 130, 1032, 900), (3, 33, 72, 2000), (148, 40, 4104, 500), (148, 12, 4104, 400)])
def test_copiers_over_many_items_and_shared_loops(sms, M, K, N, dtype):
    before = B.mnn_get_calibration()
    try:
        record = list(before)
        record[7] = sms
        B.mnn_set_calibration(record)
        _, info = run_case(M, K, N, dtype, "relu", "after", pads=(8, 16, 1, 0), offset=1, seed=K)
    finally:
        B.mnn_set_calibration(before)
    assert info.form_unaligned == B.LINEAR_COPIED and (info.items > sms if sms == 3 else info.split > 1)


def test_the_status_word_is_read_and_cleared():
    import torch
    r = B.LinearRunner(40, 300, 256)
    x, w = torch.ones(40, 256, device="cuda"), torch.ones(300, 256, device="cuda")
    r.run(x, w)
    assert r.device_status() == 0
    at = r._ws_ptr - r.workspace.data_ptr()
    r.workspace[at:at + 4].view(torch.int32).fill_(53)       # as a wait that ran out leaves it
    r.run(x, w)
    assert r.device_status() == 53 and r.device_status() == 0
    assert (r.run(x, w) == 256).all() and r.device_status() == 0
