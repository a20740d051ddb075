"""From an image to an answer: a stack of convolutions, its pooled features through the matrix product over rows, a class drawn from
the logits, all on one stream and in one graph; and tokens through a feed-forward block and a vocabulary.  Every step is held to
the oracle on the inputs that it was given."""
import numpy as np
import pytest

from oracle import direct_conv as oc
from oracle import rows as oracle
from paper_2002_12418_b200 import binding as B
from paper_2002_12418_b200 import workloads as W
from tests.util import rel_l2, to_dev

pytestmark = pytest.mark.gpu


def test_network_classifier_and_draw():
    import torch
    N, classes = 5, 37
    layers = [W.ConvLayer("a", N, 3, 32, 40, 40, 3, 2, 1, seed=1), W.ConvLayer("b", N, 32, 64, 20, 20, 3, 1, 1, seed=2),
              W.ConvLayer("c", N, 64, 96, 20, 20, 1, 1, 0, seed=3)]
    x = W.make_inputs(layers[0])[0]
    ws, bs = zip(*[W.make_inputs(l.with_batch(1))[1:] for l in layers])
    net = B.NetRunner(N, 40, 40, layers)
    wd, bd = [to_dev(torch, w) for w in ws], [to_dev(torch, b) for b in bs]
    net.prepare(wd)
    net.bind(wd, bd)
    g = torch.Generator(device="cuda")
    g.manual_seed(1)
    table, bias = torch.randn(classes, 96, generator=g, device="cuda"), torch.randn(classes, generator=g, device="cuda")
    u, k = torch.rand(N, generator=g, device="cuda"), torch.full((N,), 5, dtype=torch.int32, device="cuda")
    head, draw = B.LinearRunner(N, classes, 96, "fp32"), B.SampleRunner(N, classes, "fp32")
    xd = to_dev(torch, x)
    y = torch.empty((N, 96, 20, 20), device="cuda")
    pooled, logits = torch.empty(N, 96, device="cuda"), torch.empty(N, classes, device="cuda")
    token, prob = torch.empty(N, dtype=torch.int32, device="cuda"), torch.empty(N, device="cuda")

    def step():
        net.run(xd, y)
        torch.mean(y, dim=(2, 3), out=pooled)
        head.run(pooled, table, bias, y=logits)
        draw.run(logits, u, top_k=k, token=token, prob=prob)

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step()
    torch.cuda.synchronize()
    eager = [t.clone() for t in (y, logits, token, prob)]
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        step()
    for t in (y, logits, token, prob):
        t.zero_()
    graph.replay()
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(eager, (y, logits, token, prob)))
    assert net.device_status() == (0, -1) and head.device_status() == 0
    a = x
    for l, w, b in zip(layers, ws, bs):
        a = oc.direct_conv(a.astype(np.float32), w, b, l.stride, l.pad, l.dilation, l.groups, l.relu)
    assert rel_l2(y.cpu().numpy(), a) <= 3e-3
    want, _, size = oracle.linear(pooled.double().cpu().numpy(), table.double().cpu().numpy(), bias.double().cpu().numpy())
    assert (np.abs(logits.double().cpu().numpy() - want) <= 2.0 ** -18 * size).all()      # (24 bits of which 96 terms lose at most 6)
    for i in range(N):
        t, p, _ = oracle.sample_row(logits[i].double().cpu().numpy(), float(u[i]), top_k=5)
        assert int(token[i]) == t and abs(float(prob[i]) - p) <= 2.0 ** -23 * p


def test_block_of_tokens_and_vocabulary():
    import torch
    g = torch.Generator(device="cuda")
    g.manual_seed(2)
    for M in (1, 6, 300):
        D, F, V = 256, 1024, 4099
        rnd = lambda *s, scale=1.0: torch.randn(*s, generator=g, device="cuda").mul_(scale).bfloat16()  # noqa: E731
        h, up, down, table = rnd(M, D), rnd(F, D, scale=D ** -0.5), rnd(D, F, scale=F ** -0.5), rnd(V, D, scale=0.1)
        b1 = rnd(F, scale=0.1)
        wide = B.LinearRunner(M, F, D, "bf16", act="gelu_tanh").run(h, up, b1)
        out = B.LinearRunner(M, D, F, "bf16", residual="after").run(wide, down, None, h)
        logits = B.LinearRunner(M, V, D, "bf16").run(out, table)
        u, p = torch.rand(M, generator=g, device="cuda"), torch.full((M,), 0.9, device="cuda")
        token, prob, _ = B.SampleRunner(M, V, "bf16").run(logits, u, top_p=p)
        f = lambda t: t.double().cpu().numpy()  # noqa: E731
        for got, (want, s, size) in ((wide, oracle.linear(f(h), f(up), f(b1), None, "gelu_tanh")), (out, oracle.linear(f(wide), f(down), None, f(h), "none", "after")),
                                     (logits, oracle.linear(f(out), f(table)))):
            err = 1.13 * (1024 / 16 + 8) * 2.0 ** -23 * size + 2.0 ** -19 * np.abs(s)
            assert (np.abs(f(got) - want) <= err + 2.0 ** -8 * (np.abs(want) + err)).all()
        for i in range(M):
            t, q, _ = oracle.sample_row(f(logits[i]), float(u[i]), top_p=float(p[i].double()))
            assert int(token[i]) == t and abs(float(prob[i]) - q) <= 2.0 ** -23 * q


# product, product and draw again and again on one stream over the same buffers, with inputs whose size changes by 2^3 from one to the next: each
# kernel may start while the one before it still runs, and has to see what that one writes
@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("M,D,F,V", [(1, 256, 512, 1000), (4, 512, 512, 3000), (33, 129, 257, 1001), (300, 512, 1024, 4100), (1500, 640, 1300, 1040)])
def test_chains_over_the_same_buffers(M, D, F, V, dtype):
    import torch
    t = torch.float32 if dtype == "fp32" else torch.bfloat16
    g = torch.Generator(device="cuda")
    g.manual_seed(M)
    xs = [(torch.randn(M, D, generator=g, device="cuda") * 2.0 ** (i % 7 * 3 - 9)).to(t) for i in range(60)]
    w1, w2 = [(torch.randn(n, k, generator=g, device="cuda") * k ** -0.5).to(t) for n, k in ((F, D), (V, F))]
    a, b, draw = B.LinearRunner(M, F, D, dtype, act="relu"), B.LinearRunner(M, V, F, dtype), B.SampleRunner(M, V, dtype)
    h, logits = torch.empty(M, F, device="cuda", dtype=t), torch.empty(M, V, device="cuda", dtype=t)
    u, p = torch.rand(M, generator=g, device="cuda"), torch.full((M,), 0.9, device="cuda")

    def buffers():
        return [(torch.empty(M, dtype=torch.int32, device="cuda"), torch.empty(M, device="cuda")) for _ in xs]

    def go(out, between=lambda: None):
        for x, (token, prob) in zip(xs, out):
            a.run(x, w1, y=h)
            between()
            b.run(h, w2, y=logits)
            between()
            draw.run(logits, u, top_p=p, token=token, prob=prob)
            between()

    want, eager, replayed = buffers(), buffers(), buffers()
    go(want, torch.cuda.synchronize)
    go(eager)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        go(replayed)
    for _ in range(3):
        graph.replay()
    torch.cuda.synchronize()
    for out in (eager, replayed):
        assert all(torch.equal(c[0], d[0]) and torch.equal(c[1], d[1]) for c, d in zip(want, out))
    assert a.device_status() == 0 and b.device_status() == 0
