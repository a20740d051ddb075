"""GPU parity of sampling (mnn_sample_*) against its definition in fp64, row by row.  Tokens have to be equal; a probability is
a quotient of two fp64 figures rounded once to fp32, where the mass in the denominator is a sum of weights rounded to 2^-43 or
finer each: 2^-23 relative covers both, and 1e-37 what fp32 cannot hold."""
import numpy as np
import pytest

from oracle import rows as oracle
from paper_2002_12418_b200 import binding as B

pytestmark = pytest.mark.gpu


def types(torch):
    return {"fp32": torch.float32, "bf16": torch.bfloat16, "fp16": torch.float16}


def check(logits, u, probs=True, runner=None, **given):
    import torch
    rows, vocab = logits.shape
    name = {v: k for k, v in types(torch).items()}[logits.dtype]
    r = runner or B.SampleRunner(rows, vocab, name, ld=logits.stride(0) if rows > 1 else 0)
    token, prob, dist = r.run(logits, u, probs=probs, **given)
    token2, prob2, _ = r.run(logits, u, probs=probs, **given)
    torch.cuda.synchronize()
    assert torch.equal(token, token2) and torch.equal(prob, prob2)
    token, prob = token.cpu().numpy(), prob.double().cpu().numpy()
    dist = dist.double().cpu().numpy() if dist is not None else None
    l = logits.double().cpu().numpy()
    par = {k: v.double().cpu().numpy() for k, v in given.items() if v is not None}
    uu = u.double().cpu().numpy()
    for i in range(rows):
        a = {k: (int(v[i]) if k == "top_k" else v[i]) for k, v in par.items()}
        t, pr, ps = oracle.sample_row(l[i], uu[i], **a)
        assert token[i] == t, "row %d: token %d, wanted %d (%s, u = %r)" % (i, token[i], t, a, uu[i])
        assert abs(prob[i] - pr) <= 2.0 ** -23 * pr + 1e-37
        if dist is not None:
            assert (np.abs(dist[i] - ps) <= 2.0 ** -23 * ps + 1e-37).all()
    return token


def make(torch, seed, rows, vocab, dtype, pad=0, scale=2.0):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    l = torch.randn(rows, vocab + pad, generator=g, device="cuda") * scale
    return l.to(types(torch)[dtype])[:, :vocab], torch.rand(rows, generator=g, device="cuda"), g


@pytest.mark.parametrize("dtype", ["fp32", "bf16", "fp16"])
@pytest.mark.parametrize("rows,vocab,pad", [(1, 1, 0), (3, 2, 1), (5, 33, 0), (1, 1000, 0), (40, 1001, 3), (9, 4099, 0), (4, 32000, 0), (2, 100003, 1), (1, 131072, 0)])
def test_sizes(rows, vocab, pad, dtype):
    import torch
    l, u, g = make(torch, rows + vocab, rows, vocab, dtype, pad)
    t = torch.rand(rows, generator=g, device="cuda") + 0.3
    k = torch.randint(1, max(2, min(vocab, 300)), (rows,), generator=g, device="cuda", dtype=torch.int32)
    p = torch.rand(rows, generator=g, device="cuda") * 0.5 + 0.5
    q = torch.rand(rows, generator=g, device="cuda") * 0.1
    check(l, u)
    check(l, u, temperature=t)
    check(l, u, temperature=t, top_k=k)
    check(l, u, temperature=t, top_p=p)
    check(l, u, temperature=t, min_p=q)
    check(l, u, temperature=t, top_k=k, top_p=p, min_p=q)
    check(l, u, probs=False, temperature=t, top_p=p, min_p=q)


def test_largest_vocabulary():
    import torch
    for dtype in ("fp32", "bf16"):
        l, u, g = make(torch, 5, 2, B.SAMPLE_MAX_VOCAB, dtype, 1)
        check(l, u, top_p=torch.tensor([0.9, 0.5], device="cuda"), top_k=torch.tensor([100000, 0], device="cuda", dtype=torch.int32))


def test_many_rows():
    import torch
    l, u, g = make(torch, 6, 700, 257, "fp32")
    check(l, u, top_p=torch.rand(700, generator=g, device="cuda"))


# more clusters than run at one time
@pytest.mark.parametrize("dtype", ["fp32", "bf16", "fp16"])
def test_many_rows_of_several_ctas(dtype):
    import torch
    rows, vocab = 420, 50001
    l, u, g = make(torch, 13, rows, vocab, dtype, 1)
    r = B.SampleRunner(rows, vocab, dtype, ld=vocab + 1)
    assert r.info.ctas_per_row > 1
    p = torch.rand(rows, generator=g, device="cuda")
    k = torch.randint(0, 300, (rows,), generator=g, device="cuda", dtype=torch.int32)
    check(l, u, probs=False, runner=r, top_p=p)
    check(l, u, probs=False, runner=r, top_k=k, top_p=p, min_p=p * 0.01)


# masks: rows half hidden, rows with one candidate, rows with none; the lowest value of the type instead of -infinity
@pytest.mark.parametrize("dtype", ["fp32", "bf16", "fp16"])
@pytest.mark.parametrize("vocab", [50, 9000])
def test_masks(vocab, dtype):
    import torch
    l, u, g = make(torch, 8, 12, vocab, dtype)
    low = torch.finfo(l.dtype).min
    l[0] = float("-inf")
    l[1] = float("nan")
    l[2] = low
    l[3, 1:] = float("-inf")
    l[4, :-1] = low
    l[5, torch.rand(vocab, generator=g, device="cuda") < 0.7] = float("-inf")
    l[6, torch.rand(vocab, generator=g, device="cuda") < 0.7] = float("nan")
    l[7, torch.rand(vocab, generator=g, device="cuda") < 0.7] = low
    l[8, 3], l[8, 40] = float("inf"), float("inf")
    l[9] = 0.0
    l[10] = torch.where(torch.rand(vocab, generator=g, device="cuda") < 0.5, 0.0, -0.0).to(l.dtype)
    l[11, 7] = torch.finfo(l.dtype).max
    k = torch.full((12,), 20, dtype=torch.int32, device="cuda")
    p = torch.full((12,), 0.8, device="cuda")
    for given in ({}, dict(top_k=k), dict(top_p=p), dict(top_k=k, top_p=p), dict(min_p=p), dict(temperature=p * 0), dict(temperature=p / 0),
                  dict(temperature=p / 0, top_k=k, top_p=p)):
        token = check(l, u, **given)
        assert token[0] == -1 and token[1] == -1 and token[3] == 0


# long rows of which nothing is left, in clusters, whatever they were given: nothing in the kernel needs these values before its last barrier
@pytest.mark.parametrize("dtype", ["fp32", "bf16", "fp16"])
@pytest.mark.parametrize("vocab", [20000, 200001])
def test_rows_of_nothing(vocab, dtype):
    import torch
    rows = 64
    l = torch.full((rows, vocab), float("-inf"), device="cuda").to(types(torch)[dtype])
    l[1::3] = float("nan")
    g = torch.Generator(device="cuda")
    g.manual_seed(4)
    given = {k: torch.rand(rows, generator=g, device="cuda") for k in ("temperature", "top_p", "min_p")}
    u = torch.rand(rows, generator=g, device="cuda")
    k = torch.randint(0, 300, (rows,), generator=g, device="cuda", dtype=torch.int32)
    given["temperature"][0:2], k[0:4] = float("nan"), -1
    for t in (given["top_p"], u):
        t.view(torch.int32)[2:4] = -1                # a NaN of nothing but ones
    r = B.SampleRunner(rows, vocab, dtype)
    assert vocab < 100000 or r.info.ctas_per_row > 1
    for _ in range(20):
        token, prob, dist = r.run(l, u, top_k=k, probs=True, **given)
        assert (token == -1).all() and (prob == 0).all() and (dist == 0).all()
    # and a draw from the last value alone
    l[:, -1] = 1.0
    token, prob, dist = r.run(l, u, top_k=k, probs=True, **given)
    assert (token == vocab - 1).all() and (prob == 1).all() and (dist[:, -1] == 1).all() and (dist[:, :-1] == 0).all()


# values that tie by the thousand: the first ones by index stay
@pytest.mark.parametrize("vocab", [100, 20011])
@pytest.mark.parametrize("levels", [1, 2, 5])
def test_ties(vocab, levels):
    import torch
    g = torch.Generator(device="cuda")
    g.manual_seed(levels)
    rows = 16
    l = torch.randint(0, levels, (rows, vocab), generator=g, device="cuda").to(torch.bfloat16)
    u = torch.rand(rows, generator=g, device="cuda")
    k = torch.randint(1, vocab + 2, (rows,), generator=g, device="cuda", dtype=torch.int32)
    p = torch.rand(rows, generator=g, device="cuda")
    check(l, u, top_k=k)
    check(l, u, top_p=p)
    check(l, u, top_k=k, top_p=p)
    check(l, u, temperature=torch.zeros(rows, device="cuda"))


# parameters at and beyond their ends
def test_edges_of_the_parameters():
    import torch
    nan, inf = float("nan"), float("inf")
    l, _, _ = make(torch, 9, 12, 700, "fp32")
    u = torch.tensor([0.0, 1.0 - 2.0 ** -24, 1.0, 2.0, -1.0, nan, 0.5, 0.5, 0.5, 0.5, 0.5, 0.5], device="cuda")
    t = torch.tensor([1.0, 1.0, 1.0, 1.0, 1.0, 1.0, 0.0, -1.0, nan, 1e-30, 1e30, inf], device="cuda")
    check(l, u, temperature=t)
    k = torch.tensor([0, -5, 1, 2, 699, 700, 701, 2 ** 31 - 1, 3, 3, 3, 3], device="cuda", dtype=torch.int32)
    check(l, u, top_k=k)
    p = torch.tensor([0.0, -1.0, 1.0, 2.0, 1e-30, 1.0 - 2.0 ** -24, 0.5, nan, 0.3, 0.3, 0.3, 0.3], device="cuda")
    check(l, u, top_p=p)
    q = torch.tensor([0.0, -1.0, 1.0, 2.0, 1e-30, 1.0 - 2.0 ** -24, 0.5, 0.1, 0.3, 0.3, 0.3, 0.3], device="cuda")
    check(l, u, min_p=q)
    check(l, u, temperature=t, top_k=k, top_p=p, min_p=q)


@pytest.mark.parametrize("dtype", ["fp32", "bf16", "fp16"])
@pytest.mark.parametrize("vocab", [5000, 40001])
def test_wide_and_narrow_rows(vocab, dtype):
    import torch
    for scale in (1e-6, 1e-3, 30.0, 1e4, 1e30):
        l, u, g = make(torch, 10, 8, vocab, dtype, scale=scale)
        l = torch.where(torch.isinf(l), torch.finfo(l.dtype).max * torch.sign(l), l)
        p = torch.rand(8, generator=g, device="cuda")
        k = torch.randint(1, 3000, (8,), generator=g, device="cuda", dtype=torch.int32)
        t = torch.full((8,), scale, device="cuda")
        check(l, u, top_p=p)
        check(l, u, top_k=k, top_p=p)
        check(l, u, temperature=t, top_k=k, top_p=p, min_p=p * 0.01)
        check(l, u, temperature=t, min_p=p * 0.1)


# rows that lie around zero, wholly below it, and borders among the smallest values
@pytest.mark.parametrize("dtype", ["fp32", "bf16", "fp16"])
def test_rows_around_zero(dtype):
    import torch
    l, u, g = make(torch, 12, 10, 6000, dtype, scale=1.0)
    l[0:2] -= 20.0
    l[2:4] = -l[2:4].abs()
    l[4:6] *= 1e-3
    l[6:8] = torch.where(l[6:8].abs() < 1.0, l[6:8] * 1e-4, -l[6:8].abs())
    l[8:10] = torch.where(l[8:10] > 2.0, l[8:10], l[8:10] * 1e-3)
    p = torch.rand(10, generator=g, device="cuda")
    k = torch.randint(1, 5000, (10,), generator=g, device="cuda", dtype=torch.int32)
    for given in ({}, dict(top_k=k), dict(top_p=p), dict(top_k=k, top_p=p), dict(min_p=p), dict(top_p=p, min_p=p), dict(temperature=p * 1e-3, top_p=p)):
        check(l, u, **given)


# BF16 rows on both sides of the length from which they are cut by values
@pytest.mark.parametrize("vocab", [300, 4095, 4096, 4097])
def test_short_bf16_rows(vocab):
    import torch
    l, u, g = make(torch, vocab, 12, vocab, "bf16", 1, scale=1.0)
    l[0:2] -= 20.0
    l[2:4] *= 1e-3
    l[4:6] = torch.where(l[4:6].abs() < 1.0, l[4:6] * 1e-4, -l[4:6].abs())
    l[6:8] = l[6:8].round()
    l[8, ::3], l[9, 5], l[10] = float("-inf"), float("nan"), float("-inf")
    p = torch.rand(12, generator=g, device="cuda")
    k = torch.randint(0, vocab + 2, (12,), generator=g, device="cuda", dtype=torch.int32)
    for given in ({}, dict(top_k=k), dict(top_p=p), dict(top_k=k, top_p=p), dict(min_p=p), dict(top_p=p, min_p=p * 0.1), dict(temperature=p * 1e-3, top_p=p)):
        check(l, u, **given)


# the draws follow the distribution: 20000 equal rows, the frequency of each token within 6 standard deviations
def test_draws_follow_the_distribution():
    import torch
    g = torch.Generator(device="cuda")
    g.manual_seed(1)
    n = 20000
    l = torch.tensor([0.0, 1.0, 2.0, float("-inf"), 0.5, -1.0, 2.0, -3.0], device="cuda").repeat(n, 1)
    token, _, dist = B.SampleRunner(n, 8).run(l, torch.rand(n, generator=g, device="cuda"), probs=True)
    p = dist[0].double().cpu().numpy()
    seen = np.bincount(token.cpu().numpy(), minlength=8) / n
    assert (np.abs(seen - p) <= 6 * np.sqrt(p * (1 - p) / n) + 1e-12).all()


def test_what_lies_around_is_left_alone_and_graphs_replay():
    import torch
    l, u, g = make(torch, 11, 6, 999, "bf16", 1)
    r = B.SampleRunner(6, 999, "bf16", ld=1000)
    before = l.clone()
    token = torch.full((8,), 77, dtype=torch.int32, device="cuda")
    prob = torch.full((8,), 7.0, device="cuda")
    whole = torch.full((7 * 999,), 7.0, device="cuda")
    r.run(l, u, token=token[1:7], prob=prob[1:7], probs=whole[:6 * 999].view(6, 999))
    torch.cuda.synchronize()
    assert token[0] == 77 and token[7] == 77 and prob[0] == 7.0 and prob[7] == 7.0 and (whole[6 * 999:] == 7.0).all()
    assert torch.equal(l, before)
    want = token[1:7].clone()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    out, pr = torch.empty_like(want), torch.empty(6, device="cuda")
    with torch.cuda.graph(graph, stream=side):
        r.run(l, u, token=out, prob=pr)
    out.zero_()
    graph.replay()
    torch.cuda.synchronize()
    assert torch.equal(out, want)
    u.fill_(0.999)
    graph.replay()
    torch.cuda.synchronize()
    assert torch.equal(out, r.run(l, u)[0])


def test_refusals_of_tensors():
    import torch
    r = B.SampleRunner(4, 100, "bf16")
    l, u = torch.zeros(4, 100, dtype=torch.bfloat16, device="cuda"), torch.zeros(4, device="cuda")
    r.run(l, u)
    for a in ((l.float(), u), (l[:3], u), (l, u.double()), (l, u[:3]), (l, None), (l.cpu(), u)):
        with pytest.raises(B.MnnError) as e:
            r.run(*a)
        assert e.value.code == B.MNN_EINVAL
    with pytest.raises(B.MnnError):
        r.run(l, u, top_k=torch.zeros(4, device="cuda"))
    with pytest.raises(B.MnnError):
        r.run(l, u, probs=torch.zeros(4, 100, device="cuda", dtype=torch.float64))
    torch.cuda.synchronize()


# the run of both: logits from the product, a token from the logits
def test_logits_and_draw_together():
    import torch
    g = torch.Generator(device="cuda")
    g.manual_seed(2)
    for dtype, M, K, V in (("bf16", 5, 256, 5003), ("fp32", 3, 128, 1000), ("fp16", 33, 264, 2048)):
        t = types(torch)[dtype]
        h = torch.randn(M, K, generator=g, device="cuda").to(t)
        table = torch.randn(V, K, generator=g, device="cuda").mul_(0.3).to(t)
        logits = B.LinearRunner(M, V, K, dtype).run(h, table)
        check(logits, torch.rand(M, generator=g, device="cuda"), top_p=torch.full((M,), 0.9, device="cuda"))


# rows of the distribution further apart than their length; what lies between them is left as it was
@pytest.mark.parametrize("dtype,vocab", [("fp32", 1001), ("bf16", 40001), ("fp16", 70000)])
def test_distribution_rows_apart(dtype, vocab):
    import torch
    rows, pad = 5, 7
    l, u, g = make(torch, 21, rows, vocab, dtype)
    l = l.contiguous()
    p = torch.rand(rows, generator=g, device="cuda")
    want = B.SampleRunner(rows, vocab, dtype).run(l, u, top_p=p, probs=True)
    plan = B.mnn_sample_plan(rows, vocab, B.make_sample_opts(dtype, 0, vocab + pad))
    token, prob = torch.empty(rows, dtype=torch.int32, device="cuda"), torch.empty(rows, device="cuda")
    probs = torch.full((rows, vocab + pad), 7.0, device="cuda")
    B.mnn_sample_run(plan, l.data_ptr(), u.data_ptr(), None, None, p.data_ptr(), None, token.data_ptr(), prob.data_ptr(), probs.data_ptr(),
                     torch.cuda.current_stream().cuda_stream)
    torch.cuda.synchronize()
    B.mnn_sample_destroy(plan)
    assert torch.equal(token, want[0]) and torch.equal(prob, want[1]) and torch.equal(probs[:, :vocab], want[2]) and (probs[:, vocab:] == 7.0).all()
