"""Operators on 4-bit codes with group scales, and the distillation loss, as cases that can be timed and compared.

Three uses of paper_2312_07759_b200.binding:

"groups"   assign_groups: the export of a trained layer, W [rows][cols] -> 4-bit codes and one scale per `group` weights of a
           row (cols for a single one), and on demand the dequantised weights;
"matmul"   matmul_codes: Y = X W^T on such codes, for one token, a few, or a prompt;
"distill"  the Kullback-Leibler divergence of a student's logits from a teacher's top logits: its value ("loss"), its gradient
           ("grad", from the statistics that the value's call keeps) or both in one call ("step").

With `own` false the same results come from elementary torch operations in 32 bits (64 where a comparison is near its
border).
"""
from __future__ import annotations

import math

import torch

own = False

_TYPES = {"fp32": torch.float32, "bf16": torch.bfloat16, "fp16": torch.float16}
_BYTES = {"fp32": 4.0, "bf16": 2.0, "fp16": 2.0}


def _groups(name, rows, cols, *, group=128, k=16, weights="fp32", type="bf16", wq=False):
    return {"name": name, "use": "groups", "rows": rows, "cols": cols, "group": group, "k": k, "weights": weights, "type": type,
            "wq": wq}


def _matmul(name, tokens, rows, cols, *, group=128, k=16, type="bf16"):
    return {"name": name, "use": "matmul", "tokens": tokens, "rows": rows, "cols": cols, "group": group, "k": k, "type": type}


def _distill(name, part, rows, vocab, top, *, tau=2.0, type="bf16", teacher="fp32", padded=False):
    return {"name": name, "use": "distill", "part": part, "rows": rows, "vocab": vocab, "top": top, "tau": tau, "type": type,
            "teacher": teacher, "padded": padded}


def listed():
    return [
        # the smallest export: the 1000-way classifier on 512 features, with the dequantised weights to check it by
        _groups("export_classifier", 1000, 512, group=64, type="fp16", wq=True),
        # a large square layer of full-precision weights; traffic is all
        _groups("export_8192", 8192, 8192),
        # one sample through that classifier: launches and latency are everything
        _matmul("token_classifier", 1, 1000, 512, group=64, type="fp16"),
        # one token through an ordinary layer of a language model
        _matmul("token_4096", 1, 4096, 4096),
        # ... and through a large one, which no longer fits in L2
        _matmul("token_28672", 1, 28672, 8192),
        # eight sequences decoded together, an odd layer, small groups
        _matmul("batch8_ragged", 8, 11007, 4099, group=32, type="fp16"),
        # a few samples in full precision on codes without scales, as the export of one codebook per layer leaves them
        _matmul("batch5_fp32_plain", 5, 4096, 4608, group=0, type="fp32"),
        # a prompt
        _matmul("prompt_2048", 2048, 8192, 8192),
        # the loss of a few long rows, for an evaluation: the rows have to be shared by many multiprocessors
        _distill("loss_few_rows", "loss", 6, 151937, 50, type="fp32"),
        # a small training step of the 1000-way network: full-precision logits, few teacher entries, some rows padded away
        _distill("step_classes", "step", 64, 1000, 5, tau=4.0, type="fp32", padded=True),
        # a training step on a batch of tokens
        _distill("step_tokens", "step", 4096, 32000, 64),
        # the gradient alone, odd vocabulary
        _distill("grad_ragged", "grad", 1021, 100003, 100, type="fp16", teacher="fp16", padded=True),
    ]


def _log_uniform(rng, low, high):
    return int(math.exp(rng.uniform(math.log(low), math.log(high + 0.99))))


def draw(rng):
    """One more case of the same ranges."""
    use = rng.choice(["groups", "matmul", "matmul", "distill", "distill"])
    k = rng.choice([16, 16, 16, rng.randint(5, 15)])
    if use == "groups":
        while True:
            rows, cols = _log_uniform(rng, 64, 16384), _log_uniform(rng, 128, 16384)
            if rng.random() < 0.6:
                cols &= ~63
            if 64 * 256 <= rows * cols <= 8192 * 8192:
                break
        c = _groups("", rows, cols, group=rng.choice([32, 64, 128, 128, 256, cols]), k=k,
                    weights=rng.choice(["fp32", "fp32", "bf16", "fp16"]), type=rng.choice(["bf16", "fp16", "fp32"]),
                    wq=rng.random() < 0.3)
    elif use == "matmul":
        t = rng.choice(["bf16", "bf16", "fp16", "fp16", "fp32"])
        while True:
            tokens = rng.choice([1, 1, rng.randint(2, 16), _log_uniform(rng, 17, 2048)])
            if t == "fp32":
                tokens = min(tokens, 16)
            rows, cols = _log_uniform(rng, 256, 28672), _log_uniform(rng, 256, 16384)
            if rng.random() < 0.7:
                cols &= ~63
            if 256 * 1024 <= rows * cols <= 28672 * 8192 and tokens * rows * cols <= 2048 * 8192 * 8192:
                break
        c = _matmul("", tokens, rows, cols, group=rng.choice([0, 32, 64, 128, 128, 128, 256, cols]), k=k, type=t)
    else:
        t = rng.choice(["bf16", "bf16", "fp16", "fp32"])
        while True:
            rows, vocab = _log_uniform(rng, 1, 8192), _log_uniform(rng, 1000, 200000)
            if rng.random() < 0.5:
                vocab &= ~127
            if rows * vocab <= 4096 * 32000:
                break
        c = _distill("", rng.choice(["loss", "grad", "step", "step"]), rows, vocab, rng.randint(1, 128),
                     tau=rng.choice([1.0, 2.0, 4.0]), type=t, teacher=rng.choice([t, "fp32"]), padded=rng.random() < 0.5)
    del c["name"]
    return c


def _codebook(k, g, type):
    """What k-means finds on normal weights over their largest: about the quantiles, closer together in the middle."""
    u = (torch.arange(k, device="cuda", dtype=torch.float64) + 0.5) / k
    c = torch.erfinv(2.0 * u - 1.0)
    c = (c / c.abs().max()) * (1.0 + 0.02 * torch.randn(k, device="cuda", generator=g, dtype=torch.float64))
    return c.sort()[0].to(_TYPES[type]).contiguous()


def _span(case):
    """Weights that share a scale."""
    return case["group"] if case["group"] else case["cols"]


def prepare(case, seed):
    g = torch.Generator(device="cuda").manual_seed(int(seed))
    s = {"case": case}
    if case["use"] == "distill":
        R, V, J = case["rows"], case["vocab"], case["top"]
        z = torch.randn(R, V, device="cuda", generator=g) * 2.0
        # a teacher that the student is near to: its largest logits are a noisy form of the student's largest
        z[torch.arange(R, device="cuda"), torch.randint(0, V, (R,), device="cuda", generator=g)] += 9.0
        top, idx = torch.topk(z, J, dim=1)
        t = top + torch.randn(R, J, device="cuda", generator=g)
        if case["padded"]:   # rows of which no entry counts, and rows with fewer
            keep = torch.randint(0, J + 1, (R, 1), device="cuda", generator=g)
            keep = torch.where(torch.rand(R, 1, device="cuda", generator=g) < 0.5, torch.full_like(keep, J), keep)
            idx = torch.where(torch.arange(J, device="cuda")[None] < keep, idx, torch.full_like(idx, -1))
        s["z"] = z.to(_TYPES[case["type"]])
        s["t"], s["idx"] = t.to(_TYPES[case["teacher"]]), idx
        s["weight"] = torch.rand(R, device="cuda", generator=g) + 0.5
        if case["part"] == "grad":   # what the loss of the same logits leaves
            s["stats"] = _statistics(s["z"].float(), s["idx"], s["t"].float(), case["tau"])
        return s
    T = _TYPES[case["type"]]
    rows, cols, span = case["rows"], case["cols"], _span(case)
    s["C"] = _codebook(case["k"], g, case["type"])
    if case["use"] == "groups":
        W = torch.randn(rows, cols, device="cuda", generator=g) * math.sqrt(2.0 / cols)
        W *= torch.exp(0.3 * torch.randn(rows, 1, device="cuda", generator=g))
        if cols > span:   # a group of weights that were pruned
            W[rows // 2, :span] = 0.0
        s["W"] = W.to(_TYPES[case["weights"]])
        return s
    # codes as often as normal weights take them
    c = s["C"].float()
    cut = (c[1:] + c[:-1]) * 0.5
    codes = torch.zeros(rows, (cols + 31) // 32 * 32, device="cuda", dtype=torch.uint8)
    for a in range(0, rows, 2048):
        w = torch.randn(min(2048, rows - a), cols, device="cuda", generator=g) * 0.4
        codes[a:a + w.shape[0], :cols] = torch.bucketize(w, cut).to(torch.uint8)
    s["codes"] = codes[:, 0::2] | (codes[:, 1::2] << 4)
    if case["group"]:
        n = (cols + span - 1) // span
        s["scales"] = (torch.exp(0.3 * torch.randn(rows, n, device="cuda", generator=g)) * math.sqrt(2.0 / cols) * 2.5).to(T)
    else:
        s["scales"] = None
    s["X"] = torch.randn(case["tokens"], cols, device="cuda", generator=g).to(T)
    return s


# ---- plain forms ---------------------------------------------------------------------------------------------------


def _export(W, C, span, T, want_Wq):
    rows, cols = W.shape
    n = (cols + span - 1) // span
    w = torch.nn.functional.pad(W.float(), (0, n * span - cols)).view(rows, n, span)
    c = C.float()
    scales = (w.abs().amax(2) / c.abs().max()).to(T)
    reach = scales.double()[:, :, None] * c.double()
    codes = (w.double()[:, :, :, None] - reach[:, :, None, :]).abs_().argmin(3)   # ties: the lowest index
    codes = codes.to(torch.uint8).view(rows, n * span)[:, :cols]
    out = {"scales": scales}
    if want_Wq:
        out["Wq"] = (scales.float().repeat_interleave(span, 1)[:, :cols] * c[codes.int()]).to(W.dtype)
    codes = torch.nn.functional.pad(codes, (0, (cols + 31) // 32 * 32 - cols))
    out["codes"] = codes[:, 0::2] | (codes[:, 1::2] << 4)
    return out


def _dequantised(codes, C, scales, span, cols):
    both = torch.stack((codes & 15, codes >> 4), dim=2).view(codes.shape[0], -1)[:, :cols]
    w = C.float()[both.int()]
    return w if scales is None else w * scales.float().repeat_interleave(span, 1)[:, :cols]


def _statistics(z, idx, t, tau):
    """Logarithms of the normalisers: of the student's softmax over the vocabulary, of the teacher's over its entries."""
    fine = (idx >= 0) & (idx < z.shape[1])
    t = torch.where(fine, t / tau, torch.full_like(t, -math.inf))
    return torch.stack((torch.logsumexp(z / tau, 1), torch.logsumexp(t, 1)), 1)


def _teacher(idx, t, tau, lse_t, vocab):
    """The teacher's probabilities (0 where an entry is padding) and whether a row has any."""
    fine = (idx >= 0) & (idx < vocab)
    some = torch.isfinite(lse_t)[:, None]
    lp = torch.where(fine & some, t / tau - lse_t[:, None], torch.full_like(t, -math.inf))
    return torch.exp(lp), lp, some


def _loss(z, idx, t, tau, stats):
    lse_z, lse_t = stats.unbind(1)
    p, lp, _ = _teacher(idx, t, tau, lse_t, z.shape[1])
    lq = torch.gather(z, 1, idx.clamp(0, z.shape[1] - 1)) / tau - lse_z[:, None]
    return tau * tau * torch.where(p > 0, p.double() * (lp.double() - lq.double()), torch.zeros_like(p, dtype=torch.float64)).sum(1).float()


def _gradient(z, idx, t, tau, stats, weight):
    lse_z, lse_t = stats.unbind(1)
    p, _, some = _teacher(idx, t, tau, lse_t, z.shape[1])
    d = torch.where(some, torch.exp(z / tau - lse_z[:, None]), torch.zeros_like(z))
    d.scatter_add_(1, idx.clamp(0, z.shape[1] - 1), -p)
    return d * (tau * weight)[:, None]


def _run_plain(state):
    case = state["case"]
    if case["use"] == "groups":
        return _export(state["W"], state["C"], _span(case), _TYPES[case["type"]], case["wq"])
    if case["use"] == "matmul":
        w = _dequantised(state["codes"], state["C"], state["scales"], _span(case), case["cols"])
        return {"Y": (state["X"].float() @ w.T).to(state["X"].dtype)}
    z, idx, t, tau = state["z"].float(), state["idx"], state["t"].float(), case["tau"]
    if case["part"] == "grad":
        return {"dz": _gradient(z, idx, t, tau, state["stats"], state["weight"]).to(state["z"].dtype)}
    stats = _statistics(z, idx, t, tau)
    out = {"loss": _loss(z, idx, t, tau, stats)}
    if case["part"] == "step":
        out["dz"] = _gradient(z, idx, t, tau, stats, state["weight"]).to(state["z"].dtype)
    return out


# ---- the framework's calls -----------------------------------------------------------------------------------------


def _run_own(state):
    from paper_2312_07759_b200 import binding as B
    case = state["case"]
    if case["use"] == "groups":
        codes, scales, Wq = B.assign_groups(state["W"], state["C"], case["group"], want_Wq=case["wq"])
        return {"scales": scales, "Wq": Wq, "codes": codes} if case["wq"] else {"scales": scales, "codes": codes}
    if case["use"] == "matmul":
        return {"Y": B.matmul_codes(state["X"], state["codes"], state["C"], state["scales"], case["group"])}
    if case["part"] == "grad":
        return {"dz": B.distill_backward(state["z"], state["idx"], state["t"], case["tau"], state["stats"], state["weight"])}
    if case["part"] == "step":
        loss, dz = B.distill_step(state["z"], state["idx"], state["t"], case["tau"], state["weight"])
        return {"loss": loss, "dz": dz}
    loss, _ = B.distill_forward(state["z"], state["idx"], state["t"], case["tau"])
    return {"loss": loss}


def run(state):
    if own:
        return _run_own(state)
    return _run_plain(state)


# ---- 64 bits, from the definitions ---------------------------------------------------------------------------------


def _exact_groups(s):
    case, W, C = s["case"], s["W"].double(), s["C"].double()
    rows, cols, span = case["rows"], case["cols"], _span(case)
    largest = torch.stack([W[:, a:a + span].abs().max(1)[0] for a in range(0, cols, span)], 1)
    scales = largest / C.abs().max()
    out = {"scales": scales, "codes": None}
    if case["wq"]:
        # the stored scale is a value of its type; the codebook entry nearest to w over that scale
        held = scales.float().to(_TYPES[case["type"]]).double()
        out["Wq"] = torch.empty_like(W)
        for i, a in enumerate(range(0, cols, span)):
            reach = held[:, i, None, None] * C[None, None, :]
            j = (W[:, a:a + span, None] - reach).abs().argmin(2)
            out["Wq"][:, a:a + span] = held[:, i, None] * C[j]
    return out


def _exact_matmul(s):
    case, X, C = s["case"], s["X"].double(), s["C"].double()
    cols, span = case["cols"], _span(case)
    Y = torch.empty(case["tokens"], case["rows"], device="cuda", dtype=torch.float64)
    at = torch.arange(cols, device="cuda")
    for a in range(0, case["rows"], 1024):
        b = s["codes"][a:a + 1024].long()
        w = C[(b[:, at // 2] >> (4 * (at % 2))) & 15]
        if s["scales"] is not None:
            w = w * s["scales"][a:a + 1024].double()[:, at // span]
        Y[:, a:a + 1024] = torch.einsum("mk,nk->mn", X, w)
    return {"Y": Y}


def _exact_distill(s):
    case, tau = s["case"], s["case"]["tau"]
    R, V = s["z"].shape
    loss, dz = torch.empty(R, device="cuda", dtype=torch.float64), None
    if case["part"] != "loss":
        dz = torch.empty(R, V, device="cuda", dtype=torch.float64)
    for a in range(0, R, 256):
        z, idx, t = (s[x][a:a + 256] for x in ("z", "idx", "t"))
        lq = torch.log_softmax(z.double() / tau, 1)
        fine = (idx >= 0) & (idx < V)
        any_ = fine.any(1)
        lp = torch.log_softmax(torch.where(fine, t.double() / tau, torch.full_like(t, -1e30, dtype=torch.float64)), 1)
        p = lp.exp() * fine
        at = torch.where(fine, idx, torch.zeros_like(idx))
        loss[a:a + 256] = torch.where(any_, tau * tau * (p * (lp - lq.gather(1, at))).sum(1), torch.zeros((), device="cuda", dtype=torch.float64))
        if dz is not None:
            target = torch.zeros_like(lq).scatter_add_(1, at, p)
            dz[a:a + 256] = tau * s["weight"][a:a + 256].double()[:, None] * (lq.exp() - target) * any_[:, None]
    out = {} if case["part"] == "grad" else {"loss": loss}
    if dz is not None:
        out["dz"] = dz
    return out


def exact(case, seed):
    s = prepare(case, seed)
    return {"groups": _exact_groups, "matmul": _exact_matmul, "distill": _exact_distill}[case["use"]](s)


def work(case):
    """Every input read once, every output written once; two operations per multiply-add, four per exponential and its sum, one
    per comparison of a weight with a border between codebook entries (log2 k of them)."""
    b = _BYTES[case["type"]]
    if case["use"] == "distill":
        n, j = float(case["rows"]) * case["vocab"], float(case["rows"]) * case["top"]
        by = n * b + j * (8.0 + _BYTES[case["teacher"]]) + 4.0 * case["rows"]
        if case["part"] != "loss":
            by += n * b + 4.0 * case["rows"]
        return {"bytes": by, "flops": n * (6.0 if case["part"] == "loss" else 8.0) + 8.0 * j}
    n, groups = float(case["rows"]) * case["cols"], float(case["rows"]) * math.ceil(case["cols"] / _span(case))
    if case["use"] == "groups":
        w = _BYTES[case["weights"]]
        return {"bytes": n * w * (2.0 if case["wq"] else 1.0) + n / 2.0 + groups * b + case["k"] * b,
                "flops": n * (2.0 + math.log2(case["k"]))}
    return {"bytes": n / 2.0 + (groups * b if case["group"] else 0.0) + case["tokens"] * b * (case["rows"] + case["cols"]),
            "flops": 2.0 * n * case["tokens"]}
