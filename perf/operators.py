"""The work behind the last feature map or token state that the performance of this repository is judged by.

``listed()`` holds twelve cases, ``draw(rng)`` more of the same ranges.  A case is one of

* ``linear``  y = act(x w^T + b) with a residual, through ``LinearRunner`` (``mnn_linear_plan`` / ``mnn_linear_run``);
* ``sample``  a token per row of logits, through ``SampleRunner`` (``mnn_sample_plan`` / ``mnn_sample_run``).

``own`` chooses between the library's kernels and the plain forms, which compute in 32 bits (sampling in 64: which token is
drawn hangs on sums next to a border) and round once at the end.
"""
from __future__ import annotations

import math

import numpy as np
import torch

own = False

DTYPES = {"fp32": torch.float32, "bf16": torch.bfloat16, "fp16": torch.float16}
ACTS = ("none", "relu", "gelu", "gelu_tanh", "silu")
# the largest listed product, and the largest listed rows x vocabulary: no drawn case is larger
MAX_MACS = 8192 * 4096 * 16384
MAX_LOGITS = 512 * 131072


def _linear(name, M, K, N, dtype, act="none", bias=True, residual="none", pad=0):
    """pad: elements between the end of a row of x, r and y and the start of the next one."""
    return dict(name=name, kind="linear", M=M, K=K, N=N, dtype=dtype, act=act, bias=bias, residual=residual, pad=pad)


def _sample(name, rows, vocab, dtype, temperature=True, top_k=0, top_p=0.0, min_p=0.0, probs=False, masked=False, pad=0):
    """top_k, top_p, min_p: 0 = not given; else every row has a value of its own around it.  masked: some logits are -inf."""
    return dict(name=name, kind="sample", rows=rows, vocab=vocab, dtype=dtype, temperature=temperature, top_k=top_k, top_p=top_p,
                min_p=min_p, probs=probs, masked=masked, pad=pad)


def listed():
    return [
        # the classifier behind one image's pooled features: the smallest product, latency is all of it
        _linear("classifier_1x1024x1000_fp32", 1, 1024, 1000, "fp32"),
        # one token of one sequence through a square projection onto the residual stream: the weights' bytes
        _linear("token_1x4096x4096_bf16", 1, 4096, 4096, "bf16", residual="after"),
        # sixteen sequences' tokens through the wide half of a feed-forward block
        _linear("tokens_16x4096x16384_fp16", 16, 4096, 16384, "fp16", act="gelu_tanh"),
        # sizes off every tile, rows that start at odd addresses
        _linear("odd_77x1001x513_bf16", 77, 1001, 513, "bf16", act="silu", residual="before", pad=3),
        # a batch of 64 feature maps of 7 x 7 positions as rows, in the library's own type: a residual block's last product
        _linear("positions_3136x1024x1024_fp32", 3136, 1024, 1024, "fp32", act="relu", residual="before"),
        # the logits of 32 sequences: a vocabulary's weights against few rows
        _linear("logits_32x2048x131072_bf16", 32, 2048, 131072, "bf16", bias=False),
        # prompts of 8192 tokens in all through the wide half of a feed-forward block: the tensor cores' rate
        _linear("prompt_8192x4096x16384_bf16", 8192, 4096, 16384, "bf16", act="gelu"),
        # one class answer among the five best: the smallest draw
        _sample("class_1x1000_fp32", 1, 1000, "fp32", top_k=5),
        # one sequence's next token
        _sample("token_1x131072_bf16", 1, 131072, "bf16", top_p=0.95),
        # a batch of requests, each with its own settings, over rows of odd length and stride, some under a grammar's mask
        _sample("requests_64x100003_fp32", 64, 100003, "fp32", top_k=50, top_p=0.9, min_p=0.02, masked=True, pad=1),
        # the filtered distribution itself, as a verifier of drafted tokens wants it
        _sample("probs_64x32000_fp16", 64, 32000, "fp16", top_p=0.9, probs=True),
        # a large serving batch
        _sample("batch_512x131072_bf16", 512, 131072, "bf16", top_p=0.95, min_p=0.001),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    if rng.random() < 0.55:
        while True:
            M, K, N = _log_int(rng, 1, 8192), _log_int(rng, 16, 16384), _log_int(rng, 16, 131072)
            if rng.random() < 0.6:      # most layers have such sizes; the rest stay odd
                K, N = max(16, K // 16 * 16), max(16, N // 16 * 16)
            if M * K * N <= MAX_MACS // 2 and N * K <= 1 << 28 and M * N <= 1 << 27 and M * K <= 1 << 27:
                break
        return dict(kind="linear", M=M, K=K, N=N, dtype=rng.choice(["bf16", "bf16", "fp16", "fp32"]), act=rng.choice(ACTS),
                    bias=rng.random() < 0.7, residual=rng.choice(["none", "after", "before"]), pad=rng.choice([0, 0, 0, 8, 5]))
    while True:
        rows, vocab = _log_int(rng, 1, 512), _log_int(rng, 32, 262144)
        if rows * vocab <= MAX_LOGITS:
            break
    return dict(kind="sample", rows=rows, vocab=vocab, dtype=rng.choice(["bf16", "bf16", "fp16", "fp32"]), temperature=rng.random() < 0.9,
                top_k=rng.choice([0, 0, 1, 20, 200]), top_p=rng.choice([0.0, 0.5, 0.9, 0.99]), min_p=rng.choice([0.0, 0.0, 0.05]),
                probs=rng.random() < 0.3 and rows * vocab <= 1 << 23, masked=rng.random() < 0.4, pad=rng.choice([0, 0, 1, 8]))


def _rows(gen, rows, cols, pad, dtype, scale=1.0):
    """rows x cols values of N(0, scale^2), each row `pad` elements behind the last one's end."""
    t = torch.randn(rows, cols + pad, generator=gen, device="cuda", dtype=torch.float32).mul_(scale).to(dtype)
    return t[:, :cols]


def prepare(case, seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(int(seed))
    dtype = DTYPES[case["dtype"]]
    s = {"case": case}
    if case["kind"] == "linear":
        M, K, N, pad = case["M"], case["K"], case["N"], case["pad"]
        s["x"] = _rows(gen, M, K, pad, dtype)
        s["w"] = _rows(gen, N, K, 0, dtype, K ** -0.5)
        s["bias"] = torch.randn(N, generator=gen, device="cuda").mul_(0.1).to(dtype) if case["bias"] else None
        s["residual"] = _rows(gen, M, N, pad, dtype) if case["residual"] != "none" else None
        if own:
            from paper_2002_12418_b200 import binding as B
            ldr = N + pad if s["residual"] is not None else 0
            s["runner"] = B.LinearRunner(M, N, K, case["dtype"], act=case["act"], residual=case["residual"], ldx=K + pad, ldr=ldr)
        return s
    rows, vocab, pad = case["rows"], case["vocab"], case["pad"]
    # logits as a language model's: masses by a power law of the rank, with noise
    l = torch.rand(rows, vocab + pad, generator=gen, device="cuda").mul_(vocab).add_(1.0).log_().mul_(-1.3)
    l.add_(torch.randn(rows, vocab + pad, generator=gen, device="cuda").mul_(1.5))
    if case["masked"]:                  # every second row under a mask, the fourth of eight under one that leaves nothing
        hidden = torch.rand(rows, vocab + pad, generator=gen, device="cuda") < 0.5
        at = torch.arange(rows, device="cuda")[:, None]
        l.masked_fill_((hidden & (at % 2 == 1)) | (at % 8 == 3), -math.inf)
    s["logits"] = l.to(dtype)[:, :vocab]
    uniform = lambda: torch.rand(rows, generator=gen, device="cuda")  # noqa: E731
    s["u"] = uniform()
    s["temperature"] = uniform() + 0.5 if case["temperature"] else None
    s["top_k"] = (uniform() * case["top_k"]).int() + (case["top_k"] + 1) // 2 if case["top_k"] else None
    s["top_p"] = 1.0 - (1.0 - case["top_p"]) * (uniform() + 0.5) if case["top_p"] else None
    s["min_p"] = case["min_p"] * (uniform() + 0.5) if case["min_p"] else None
    if own:
        from paper_2002_12418_b200 import binding as B
        s["runner"] = B.SampleRunner(rows, vocab, case["dtype"], ld=vocab + pad)
    return s


def _act(v, act):
    if act == "relu":
        return v.clamp_min(0.0)
    if act == "gelu":
        return 0.5 * v * (1.0 + torch.erf(v * math.sqrt(0.5)))
    if act == "gelu_tanh":
        return 0.5 * v * (1.0 + torch.tanh(math.sqrt(2.0 / math.pi) * (v + 0.044715 * v * v * v)))
    if act == "silu":
        return v / (1.0 + torch.exp(-v))
    return v


def _plain_linear(s):
    case = s["case"]
    v = s["x"].float() @ s["w"].float().t()
    if s["bias"] is not None:
        v = v + s["bias"].float()
    if case["residual"] == "before":
        v = v + s["residual"].float()
    v = _act(v, case["act"])
    if case["residual"] == "after":
        v = v + s["residual"].float()
    return v.to(DTYPES[case["dtype"]])


def _plain_sample(s):
    case = s["case"]
    l = s["logits"].float()
    rows, vocab = l.shape
    l = torch.where(torch.isnan(l), -math.inf, l)
    v, idx = torch.sort(l, dim=1, descending=True, stable=True)
    m = v[:, :1].double()
    some = m > -math.inf
    d = torch.where(v.double() == m, 0.0, v.double() - m)        # infinite where the largest logit is
    t = s["temperature"].double()[:, None] if s["temperature"] is not None else torch.ones_like(m)
    w = torch.where(d == 0.0, 1.0, torch.exp(d / t))
    at = torch.arange(vocab, device=l.device)[None, :]
    keep = (v > -math.inf) & ((t > 0.0) | (at == 0)) & ((m < math.inf) | (d == 0.0))
    if s["top_k"] is not None:
        k = s["top_k"][:, None]
        keep = keep & ((at < k) | (k <= 0))
    if s["top_p"] is not None:
        p = s["top_p"].double()[:, None]
        mass = torch.where(keep, w, 0.0).cumsum(1)
        before = torch.cat([torch.zeros_like(m), mass[:, :-1]], 1)
        keep = keep & ((before < p * mass[:, -1:]) | (p >= 1.0) | (at == 0))
    if s["min_p"] is not None:
        keep = keep & (w >= s["min_p"].double()[:, None].clamp_max(1.0))
    kept = torch.zeros_like(w).scatter_(1, idx, torch.where(keep, w, 0.0))
    mass = kept.cumsum(1)
    total = mass[:, -1:]
    token = (mass <= s["u"].double()[:, None] * total).sum(1, keepdim=True).clamp_max(vocab - 1)
    share = kept / torch.where(some, total, 1.0)
    out = {"token": torch.where(some, token, -1)[:, 0].int(), "prob": torch.where(some, share.gather(1, token), 0.0)[:, 0].float()}
    if case["probs"]:
        out["probs"] = share.float()
    return out


def run(s):
    if own:
        r = s["runner"]
        if s["case"]["kind"] == "linear":
            return r.run(s["x"], s["w"], s["bias"], s["residual"])
        out = dict(zip(("token", "prob", "probs"), r.run(s["logits"], s["u"], s["temperature"], s["top_k"], s["top_p"], s["min_p"],
                                                          probs=s["case"]["probs"])))
        return {k: v for k, v in out.items() if v is not None}
    return _plain_linear(s) if s["case"]["kind"] == "linear" else _plain_sample(s)


def work(case):
    size = 4 if case["dtype"] == "fp32" else 2
    if case["kind"] == "linear":
        M, K, N = case["M"], case["K"], case["N"]
        elems = M * K + N * K + M * N * (2 if case["residual"] != "none" else 1) + (N if case["bias"] else 0)
        return {"bytes": elems * size, "flops": 2 * M * N * K}
    rows, vocab = case["rows"], case["vocab"]
    given = 1 + sum(bool(case[k]) for k in ("temperature", "top_k", "top_p", "min_p"))
    nbytes = rows * vocab * (size + (4 if case["probs"] else 0)) + rows * 4 * (given + 2)
    return {"bytes": nbytes, "flops": 20 * rows * vocab}


def _exact_linear(case, s):
    def gate(v):
        if case["act"] == "relu":
            return torch.maximum(v, torch.zeros_like(v))
        if case["act"] == "gelu":
            return v * torch.special.ndtr(v)
        if case["act"] == "gelu_tanh":          # (1 + tanh z) / 2 is the logistic function of 2 z
            return v * torch.sigmoid(2.0 * math.sqrt(2.0 / math.pi) * (v + 0.044715 * v ** 3))
        if case["act"] == "silu":
            return v * torch.sigmoid(v)
        return v

    y = torch.empty(case["M"], case["N"], dtype=torch.float64, device="cuda")
    w = s["w"].double()
    step = 2048
    for i in range(0, case["M"], step):
        v = torch.einsum("mk,nk->mn", s["x"][i:i + step].double(), w)
        v += 0.0 if s["bias"] is None else s["bias"].double()
        r = 0.0 if s["residual"] is None else s["residual"][i:i + step].double()
        y[i:i + step] = gate(v + r) if case["residual"] == "before" else gate(v) + r
    return y


def _exact_row(l, u, temperature, top_k, top_p, min_p):
    """The definition of one row, candidate by candidate of the sorted order: (token, prob, probs)."""
    vocab = len(l)
    probs = np.zeros(vocab)
    cand = np.flatnonzero(l > -np.inf)           # a NaN compares false
    if not len(cand):
        return -1, 0.0, probs
    order = cand[np.lexsort((cand, -l[cand]))]
    top = l[order[0]]
    if not temperature > 0.0:
        order = order[:1]
    elif np.isinf(top):
        order = order[l[order] == top]
    if top_k > 0:
        order = order[:top_k]
    w = np.ones(len(order)) if np.isinf(top) else np.exp((l[order] - top) / temperature) if temperature > 0.0 else np.ones(1)
    if top_p < 1.0:
        n = max(1, int(np.searchsorted(np.cumsum(w), top_p * np.sum(w), side="left")) + 1)
        order, w = order[:n], w[:n]
    n = int(np.sum(w >= min(min_p, 1.0)))
    order, w = order[:n], w[:n]
    by_index = np.argsort(order)
    order, w = order[by_index], w[by_index]
    run_mass = np.cumsum(w)
    at = min(int(np.searchsorted(run_mass, u * run_mass[-1], side="right")), len(order) - 1)
    probs[order] = w / run_mass[-1]
    return int(order[at]), float(probs[order[at]]), probs


def exact(case, seed):
    s = prepare(case, seed)
    if case["kind"] == "linear":
        return _exact_linear(case, s)
    logits = s["logits"].double().cpu().numpy()
    given = {k: s[k].double().cpu().numpy() if s[k] is not None else None for k in ("u", "temperature", "top_k", "top_p", "min_p")}
    value = lambda k, i, off: off if given[k] is None else given[k][i]  # noqa: E731
    rows = [_exact_row(logits[i], given["u"][i], value("temperature", i, 1.0), int(value("top_k", i, 0)), value("top_p", i, 1.0),
                       value("min_p", i, 0.0)) for i in range(case["rows"])]
    out = {"token": np.array([r[0] for r in rows], dtype=np.int32), "prob": np.array([r[1] for r in rows])}
    if case["probs"]:
        out["probs"] = np.stack([r[2] for r in rows])
    return out
