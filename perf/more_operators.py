"""What the embedding lookup, the softmax cross entropy and the distillation over a large vocabulary are timed on.

A model over learned embeddings takes its features from a table of nodes, entities or tokens (``embedding``) and
answers with one of them: its loss is a softmax over the whole table, against the right answer
(``linear_cross_entropy``) or against a teacher's best answers (``linear_distill``).  A case is a dict of plain
values.  ``kind`` names the calls:

    lookup    rows of the table (embedding)
    scatter   the table's gradient (embedding_backward), into a fresh gradient or added to one that is there (``add``)
    score     the loss alone (linear_cross_entropy), as in an evaluation
    train     the loss and its gradients (linear_cross_entropy, linear_cross_entropy_backward)
    distill   the loss against a teacher's top ``K`` logits and its gradients (linear_distill, linear_distill_backward)

``n`` rows or tokens, ``V`` rows of the table (the vocabulary), ``k`` features.  ``skew``: tokens are drawn as
V u^skew for uniform u, so 1 is even and more is a few frequent ones.  ``pad``: the share of rows without a token
or target, as padded batches have them.
"""
from __future__ import annotations

import math

import numpy as np
import torch

own = False

DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}


def listed():
    return [
        # the seeds of one query looked up in a citation-sized table: latency
        {"name": "lookup_few", "kind": "lookup", "n": 8, "V": 2708, "k": 256, "dtype": "bf16", "out": "same",
         "skew": 1.0, "pad": 0.0},
        # the neighbours of a sampled batch in a table of the benchmark's 2.4M nodes, some places padded
        {"name": "lookup_nodes", "kind": "lookup", "n": 1500000, "V": 2400000, "k": 128, "dtype": "bf16", "out": "same",
         "skew": 2.0, "pad": 0.05},
        # the gradient of a small table of types, fp32, every token frequent
        {"name": "scatter_types", "kind": "scatter", "n": 4096, "V": 90, "k": 64, "dtype": "f32", "out": "same",
         "skew": 1.5, "pad": 0.0, "add": False},
        # the gradient of a token table, a few tokens most of the batch
        {"name": "scatter_tokens", "kind": "scatter", "n": 1000000, "V": 131072, "k": 256, "dtype": "bf16",
         "out": "same", "skew": 3.0, "pad": 0.02, "add": False},
        # a batch's gradient added to that of an ogbn-arxiv-sized table, 300 wide (word vectors), fp32 sums
        {"name": "scatter_add", "kind": "scatter", "n": 262144, "V": 169343, "k": 300, "dtype": "f16", "out": "f32",
         "skew": 1.3, "pad": 0.0, "add": True},
        # one query scored against 50000 entities: the table's read is all there is
        {"name": "score_one", "kind": "score", "n": 1, "V": 50000, "k": 512, "dtype": "bf16", "bias": False, "pad": 0.0},
        # an evaluation over 14951 entities (odd), 200 features
        {"name": "score_entities", "kind": "score", "n": 2048, "V": 14951, "k": 200, "dtype": "f16", "bias": True,
         "pad": 0.0},
        # a small batch over a small set of answers: latency of a training step's end
        {"name": "train_small", "kind": "train", "n": 256, "V": 1433, "k": 128, "dtype": "bf16", "bias": True,
         "pad": 0.1},
        # a padded batch over 40943 entities (odd)
        {"name": "train_padded", "kind": "train", "n": 4096, "V": 40943, "k": 512, "dtype": "f16", "bias": False,
         "pad": 0.3},
        # the largest: 8192 tokens over a vocabulary of 131072
        {"name": "train_large", "kind": "train", "n": 8192, "V": 131072, "k": 1024, "dtype": "bf16", "bias": False,
         "pad": 0.0},
        # a small student of 602 features over 10007 answers (odd), a teacher's top 10
        {"name": "distill_small", "kind": "distill", "n": 1000, "V": 10007, "k": 602, "dtype": "f16", "bias": True,
         "pad": 0.1, "K": 10, "T": 2.0},
        # a student over a vocabulary of 65536, a teacher's top 64
        {"name": "distill_tokens", "kind": "distill", "n": 4096, "V": 65536, "k": 768, "dtype": "bf16", "bias": False,
         "pad": 0.05, "K": 64, "T": 1.0},
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _width(rng, lo, hi):
    """A width: half of them multiples of 8, the others any number."""
    w = _log(rng, lo, hi)
    return max(8, w // 8 * 8) if rng.random() < 0.5 else w


def draw(rng):
    kind = rng.choice(["lookup", "scatter", "scatter", "score", "score", "train", "train", "distill"])
    pad = rng.choice([0.0, 0.0, 0.05, 0.3])
    if kind in ("lookup", "scatter"):
        k = _width(rng, 8, 1024)
        c = {"kind": kind, "n": min(_log(rng, 1, 1_500_000), 250_000_000 // k),
             "V": min(_log(rng, 2, 2_400_000), 300_000_000 // k), "k": k, "dtype": rng.choice(["f32", "bf16", "f16"]),
             "out": rng.choice(["same", "same", "f32"]), "skew": rng.choice([1.0, 1.5, 2.0, 3.0]), "pad": pad}
        if kind == "scatter":
            c["add"] = rng.random() < 0.3
        return c
    k, V = _width(rng, 16, 1536), _log(rng, 500, 131072)
    n = min(_log(rng, 1, 8192), 1_000_000_000_000 // (V * k))
    c = {"kind": kind, "n": n, "V": V, "k": k, "dtype": rng.choice(["bf16", "f16"]), "bias": rng.random() < 0.5, "pad": pad}
    if kind == "distill":
        c["K"], c["T"] = _log(rng, 1, 128), rng.choice([1.0, 2.0, 4.0])
    return c


# ----------------------------------------------------------------- inputs

def _tokens(n, V, skew, pad, g):
    """Tokens by frequency; which are the frequent ones changes with the seed."""
    rank = (torch.rand(n, generator=g, device="cuda", dtype=torch.float64) ** skew * V).long().clamp_(max=V - 1)
    t = torch.randperm(V, generator=g, device="cuda")[rank]
    return torch.where(torch.rand(n, generator=g, device="cuda") < pad, -1, t).to(torch.int32)


def prepare(case, seed):
    g = torch.Generator(device="cuda").manual_seed(int(seed) * 7919 + 23)
    dt = DTYPES[case["dtype"]]
    n, V, k = case["n"], case["V"], case["k"]
    s = {"kind": case["kind"], "V": V}
    if case["kind"] in ("lookup", "scatter"):
        s["out"] = dt if case["out"] == "same" else DTYPES[case["out"]]
        s["index"] = _tokens(n, V, case["skew"], case["pad"], g)
        if case["kind"] == "lookup":
            s["scale"] = k ** 0.5
            s["table"] = (torch.randn((V, k), generator=g, device="cuda") * k ** -0.5).to(dt)
        else:
            s["scale"] = k ** 0.5
            s["dY"] = (torch.randn((n, k), generator=g, device="cuda") * k ** -0.5).to(dt)
            s["grad"] = torch.randn((V, k), generator=g, device="cuda").to(s["out"]) if case["add"] else None
        return s
    # answers by frequency; the features of most rows lean towards their answer, as those of a model in training
    # do: its logit rises by up to log V, where the sum over the others lies a little higher
    W = torch.randn((V, k), generator=g, device="cuda") * (3.0 * k ** -0.5)
    target = _tokens(n, V, 1.5, case["pad"], g)
    lean = torch.rand((n, 1), generator=g, device="cuda") * (math.log(V) / 9.0)
    X = torch.randn((n, k), generator=g, device="cuda") + lean * W[target.clamp(min=0).long()]
    s["X"], s["W"] = X.to(dt), W.to(dt)
    s["bias"] = torch.randn(V, generator=g, device="cuda") if case["bias"] else None
    if case["kind"] == "distill":
        # the best K of the teacher, the best first: the answer and K - 1 others
        K = min(case["K"], V)
        others = torch.arange(K, device="cuda") * max(1, V // K)
        index = (target.clamp(min=0).long()[:, None] + others) % V
        s["teacher"] = (torch.randn((n, K), generator=g, device="cuda") * 3.0 + 10.0).sort(1, descending=True)[0]
        # a teacher sends fewer where fewer matter, none for a padded place
        fewer = torch.randint(1, K + 1, (n, 1), generator=g, device="cuda")
        index = torch.where(torch.rand((n, 1), generator=g, device="cuda") < 0.5,
                            torch.where(torch.arange(K, device="cuda") < fewer, index, -1), index)
        s["index"] = torch.where(target[:, None] < 0, -1, index).to(torch.int32)
        s["T"] = case["T"]
    else:
        s["target"] = target
    if case["kind"] != "score":
        # the mean over the rows that count, under the scale of a loss
        s["dloss"] = torch.full((n,), 1.0 / max(1, int((target >= 0).sum())), device="cuda")
    return s


# ------------------------------------------------------------- plain forms

def _logits(s, rows):
    z = s["X"][rows].float() @ s["W"].float().t()
    return z if s["bias"] is None else z + s["bias"]


def _pieces(s):
    """Rows in pieces whose logits stay under 2 GB."""
    n, V = s["X"].shape[0], s["V"]
    per = max(1, (1 << 29) // V)
    return [slice(at, min(at + per, n)) for at in range(0, n, per)]


def _lse(z):
    top = z.max(1, keepdim=True)[0]
    return top[:, 0] + (z - top).exp().sum(1).log()


def _plain_head(s):
    """The losses of both kinds: the answer is a teacher's only entry, of weight 1."""
    distill = s["kind"] == "distill"
    T = s["T"] if distill else 1.0
    index = s["index"] if distill else s["target"][:, None]
    held = index >= 0
    if distill:
        t = torch.where(held, s["teacher"] / T, -math.inf)
        top = t.max(1, keepdim=True)[0]
        e = torch.where(held, (t - torch.where(held.any(1, keepdim=True), top, 0.0)).exp(), 0.0)
        q = e / e.sum(1, keepdim=True).clamp(min=1e-37)
    else:
        q = held.float()
    live = held.any(1)
    train = s["kind"] != "score"
    n, k = s["X"].shape
    loss, lse = torch.empty(n, device="cuda"), torch.empty(n, device="cuda")
    logp = torch.zeros_like(q)
    if train:
        dX = torch.empty((n, k), device="cuda")
        dW = torch.zeros((s["V"], k), device="cuda")
        db = torch.zeros(s["V"], device="cuda")
    for rows in _pieces(s):
        z = _logits(s, rows) / T
        at = index[rows].clamp(min=0).long()
        lse[rows] = torch.where(live[rows], _lse(z), 0.0)
        logp[rows] = torch.where(held[rows], z.gather(1, at) - lse[rows][:, None], 0.0)
        logq = torch.where(q[rows] > 0, q[rows], 1.0).log()
        loss[rows] = T * T * (q[rows] * (logq - logp[rows])).sum(1)
        if train:
            p = (z - lse[rows][:, None]).exp()
            p.scatter_add_(1, at, -q[rows])
            p *= torch.where(live[rows], T * s["dloss"][rows], 0.0)[:, None]
            dX[rows] = p @ s["W"].float()
            dW += p.t() @ s["X"][rows].float()
            db += p.sum(0)
    out = [loss, lse] + ([logp] if distill else [])
    if train:
        out += [dX.to(s["X"].dtype), dW.to(s["W"].dtype)] + ([] if s["bias"] is None else [db])
    return out


def _plain(s):
    if s["kind"] == "lookup":
        rows = s["table"][s["index"].clamp(min=0).long()].float() * s["scale"]
        return torch.where(s["index"][:, None] >= 0, rows, 0.0).to(s["out"])
    if s["kind"] == "scatter":
        # the rows in the tokens' order, and differences of their running sums (long ones: 64 bits)
        token, order = s["index"].sort()
        ends = torch.searchsorted(token, torch.arange(-1, s["V"], device="cuda", dtype=torch.int32), right=True)
        run = (s["dY"][order].t().double() * s["scale"]).contiguous().cumsum(1)
        run = torch.cat([torch.zeros_like(run[:, :1]), run], 1)[:, ends]
        sums = (run[:, 1:] - run[:, :-1]).t().contiguous()
        if s["grad"] is not None:
            sums += s["grad"]
        return sums.to(s["out"])
    return _plain_head(s)


# ------------------------------------------------------------ the operators

def run(s):
    if not own:
        return _plain(s)
    import paper_2103_00959_amd as cg
    kind = s["kind"]
    if kind == "lookup":
        return cg.embedding(s["table"], s["index"], scale=s["scale"], out_dtype=s["out"])
    if kind == "scatter":
        if s["grad"] is not None:       # onto a copy: the pass can be made again
            return cg.embedding_backward(s["dY"], s["index"], s["V"], scale=s["scale"], out=s["grad"].clone(), accumulate=True)
        return cg.embedding_backward(s["dY"], s["index"], s["V"], scale=s["scale"], out_dtype=s["out"])
    if kind == "distill":
        loss, lse, logp = cg.linear_distill(s["X"], s["W"], s["index"], s["teacher"], s["bias"], temperature=s["T"])
        g = cg.linear_distill_backward(s["dloss"], s["X"], s["W"], s["index"], s["teacher"], lse, logp, s["bias"],
                                       temperature=s["T"])
        return [loss, lse, logp, g["dX"], g["dW"]] + ([] if s["bias"] is None else [g["db"]])
    loss, lse = cg.linear_cross_entropy(s["X"], s["W"], s["target"], s["bias"])
    if kind == "score":
        return [loss, lse]
    g = cg.linear_cross_entropy_backward(s["dloss"], s["X"], s["W"], s["target"], loss, lse, s["bias"])
    return [loss, lse, g["dX"], g["dW"]] + ([] if s["bias"] is None else [g["db"]])


def work(case):
    n, V, k = case["n"], case["V"], case["k"]
    b = 4 if case["dtype"] == "f32" else 2
    if case["kind"] in ("lookup", "scatter"):
        o = b if case["out"] == "same" else 4
        if case["kind"] == "lookup":
            # the distinct rows that n such tokens can be expected to name
            share = np.diff((np.arange(V + 1) / V) ** (1.0 / case["skew"])) * (1.0 - case["pad"])
            rows = float((1.0 - np.exp(n * np.log1p(-share))).sum())
            return {"bytes": 4 * n + rows * k * b + n * k * o, "flops": n * k}
        # (padded places have no gradient to read)
        return {"bytes": 4 * n + n * (1.0 - case["pad"]) * k * b + V * k * o * (2 if case["add"] else 1), "flops": 2 * n * k}
    # padded rows have no loss and no gradient; logits that are not kept are computed again for the gradients
    live = n * (1.0 - case["pad"])
    bias = 4 * V if case["bias"] else 0
    per_row = 8 * case["K"] if case["kind"] == "distill" else 4
    if case["kind"] == "score":
        return {"bytes": live * k * b + V * k * b + bias + n * (per_row + 8), "flops": 2 * live * V * k}
    return {"bytes": 2 * (live * k * b + V * k * b + bias) + n * (per_row + 12), "flops": 8 * live * V * k}


# --------------------------------------------------- the definition in 64 bits

def exact(case, seed):
    s = prepare(case, seed)
    if case["kind"] == "lookup":
        T = torch.cat([s["table"].double() * s["scale"], torch.zeros((1, case["k"]), dtype=torch.float64, device="cuda")])
        return T[torch.where(s["index"] < 0, case["V"], s["index"].long())]
    if case["kind"] == "scatter":
        sums = torch.zeros((case["V"] + 1, case["k"]), dtype=torch.float64, device="cuda")
        sums.index_add_(0, torch.where(s["index"] < 0, case["V"], s["index"].long()), s["dY"].double())
        sums = sums[:-1] * s["scale"]
        return sums if s["grad"] is None else sums + s["grad"].double()
    n, V, k = case["n"], case["V"], case["k"]
    kind = case["kind"]
    X, Wt = s["X"].double(), s["W"].double().t().contiguous()
    T = float(case.get("T", 1.0))
    dX, dW = torch.zeros((n, k), dtype=torch.float64, device="cuda"), torch.zeros((V, k), dtype=torch.float64, device="cuda")
    db = torch.zeros(V, dtype=torch.float64, device="cuda")
    losses, lses, logps = [], [], []
    step = max(1, (1 << 28) // V)
    for a in range(0, n, step):
        z = X[a:a + step] @ Wt
        if s["bias"] is not None:
            z += s["bias"].double()
        logp = torch.log_softmax(z / T, 1)
        lse = torch.logsumexp(z / T, 1)
        want = torch.zeros_like(z)           # the distribution asked for
        if kind == "distill":
            ix = s["index"][a:a + step].long()
            t = (s["teacher"][a:a + step].double() / T).masked_fill(ix < 0, -math.inf)
            some = (ix >= 0).any(1)
            q = torch.zeros_like(t)
            q[some] = torch.softmax(t[some], 1)
            want.scatter_add_(1, ix.clamp(min=0), q)
            entropy = torch.special.entr(q).sum(1)
            mine = logp.gather(1, ix.clamp(min=0)) * (ix >= 0)
            logps.append(mine)
            losses.append(T * T * (-(q * mine).sum(1) - entropy))
        else:
            tg = s["target"][a:a + step].long()
            some = tg >= 0
            want[some, tg[some]] = 1.0
            losses.append(-(want * torch.where(want > 0, logp, 0.0)).sum(1))
        lses.append(lse * some)
        if kind != "score":
            d = (logp.exp() - want) * (T * s["dloss"][a:a + step].double() * some)[:, None]
            dX[a:a + step] = d @ Wt.t()
            dW += d.t() @ X[a:a + step]
            db += d.sum(0)
    out = [torch.cat(losses), torch.cat(lses)] + ([torch.cat(logps)] if kind == "distill" else [])
    if kind != "score":
        out += [dX, dW] + ([] if s["bias"] is None else [db])
    return out
