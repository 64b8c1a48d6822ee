"""What the products of typed rows and the 8-bit activation checkpoints are timed on.

Rows of several types (node types, relations, experts) lie sorted by type; each type has a weight matrix of
its own.  A case is a dict of plain values.  ``kind`` names the calls:

    trip      activations into an 8-bit checkpoint (act_checkpoint) and back (act_restore)
    linear    the forward product (grouped_linear)
    backward  its gradients (grouped_linear_backward), the input given as it was or as its checkpoint (``keep``)
    step      a training pass of one layer: the forward that also writes the checkpoint of its input, then the
              backward that reads it (the activation follows the aggregation, as in a relational GCN layer)

``n`` rows, ``pad`` more behind the last group; ``E`` groups whose sizes fall as rank^-skew (0: even), the
last ``empty`` ones having no rows; ``k`` features to ``m`` outputs.  Sizes are those of this repository's
workloads (citation, ogbn and Reddit graphs, the 2.4M-node benchmark), of its tests, and generic ones.
"""
from __future__ import annotations

import math

import torch

own = False

DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
BLOCK = 32          # features that share a scale


def listed():
    return [
        # raw citation-graph features (1433 wide, an odd width), the smallest round trip: latency
        {"name": "trip_small", "kind": "trip", "n": 2708, "F": 1433, "dtype": "bf16"},
        # 300-wide input features (word vectors) of an ogbn-arxiv-sized graph in fp32, a ragged last block
        {"name": "trip_words", "kind": "trip", "n": 169343, "F": 300, "dtype": "f32"},
        # 256-wide hidden activations of the benchmark's 2.4M nodes
        {"name": "trip_large", "kind": "trip", "n": 2400000, "F": 256, "dtype": "bf16"},
        # serving: one token, its 8 experts of 64; the weights' reads are all there is
        {"name": "linear_token", "kind": "linear", "n": 8, "pad": 0, "E": 64, "empty": 56, "skew": 0.0,
         "k": 2048, "m": 1024, "dtype": "bf16", "out": "same", "act": "none", "bias": False},
        # the input layer of a Reddit-sized graph with 7 node types: 602 features (rows off the 16-byte grid)
        {"name": "linear_typed", "kind": "linear", "n": 232965, "pad": 0, "E": 7, "empty": 0, "skew": 1.0,
         "k": 602, "m": 128, "dtype": "bf16", "out": "same", "act": "relu", "bias": True},
        # messages of 90 relations, 64 wide, in fp16 to fp32 sums; most relations are rare
        {"name": "linear_relations", "kind": "linear", "n": 2501829, "pad": 0, "E": 90, "empty": 5, "skew": 1.2,
         "k": 64, "m": 64, "dtype": "f16", "out": "f32", "act": "none", "bias": False},
        # 64 experts over 32k rows, wide layers: the matrix cores' rate
        {"name": "linear_experts", "kind": "linear", "n": 32768, "pad": 0, "E": 64, "empty": 0, "skew": 0.5,
         "k": 2048, "m": 2048, "dtype": "bf16", "out": "same", "act": "none", "bias": False},
        # gradients on a citation-sized graph, 24 relations, some without rows; input kept as it was
        {"name": "backward_small", "kind": "backward", "n": 2708, "pad": 100, "E": 24, "empty": 6, "skew": 1.0,
         "k": 64, "m": 48, "dtype": "bf16", "dw": "f32", "act": "relu", "keep": "input"},
        # gradients of a hidden layer of the 2.4M-node benchmark with 8 node types, input kept in 8 bits
        {"name": "backward_large", "kind": "backward", "n": 2400000, "pad": 0, "E": 8, "empty": 0, "skew": 1.0,
         "k": 256, "m": 128, "dtype": "bf16", "dw": "same", "act": "none", "keep": "8bit"},
        # gradients of the wide experts, input kept in 8 bits
        {"name": "backward_experts", "kind": "backward", "n": 32768, "pad": 0, "E": 64, "empty": 0, "skew": 0.5,
         "k": 2048, "m": 2048, "dtype": "bf16", "dw": "same", "act": "none", "keep": "8bit"},
        # a training pass over 300-wide features of an ogbn-arxiv-sized graph, 4 node types, 47 outputs (odd)
        {"name": "step_words", "kind": "step", "n": 169343, "pad": 0, "E": 4, "empty": 0, "skew": 1.0,
         "k": 300, "m": 47, "dtype": "f16", "dw": "f32", "act": "none", "bias": True},
        # a training pass of a hidden layer, 600k nodes of 12 types
        {"name": "step_hidden", "kind": "step", "n": 600000, "pad": 0, "E": 12, "empty": 1, "skew": 0.7,
         "k": 256, "m": 256, "dtype": "bf16", "dw": "f32", "act": "none", "bias": True},
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _width(rng, lo, hi):
    """A layer width: half of them multiples of 8, the others any number (classes, raw features)."""
    w = _log(rng, lo, hi)
    return max(8, w // 8 * 8) if rng.random() < 0.5 else w


def draw(rng):
    kind = rng.choice(["trip", "linear", "linear", "backward", "backward", "step"])
    if kind == "trip":
        F = _width(rng, 8, 2048)
        return {"kind": kind, "n": min(_log(rng, 1000, 2_400_000), 600_000_000 // F), "F": F,
                "dtype": rng.choice(["f32", "bf16", "f16"])}
    E, k, m = _log(rng, 1, 256), _width(rng, 16, 2048), _width(rng, 16, 2048)
    E = max(1, min(E, 200_000_000 // (k * m)))
    n = min(_log(rng, 1, 2_400_000), 80_000_000_000 // (k * m), 500_000_000 // (k + m))
    c = {"kind": kind, "n": n, "pad": rng.choice([0, 0, 0, rng.randint(1, 300)]), "E": E,
         "empty": rng.randint(0, E // 2), "skew": rng.choice([0.0, 0.5, 1.0, 1.5]), "k": k, "m": m,
         "dtype": rng.choice(["bf16", "f16"]),
         "act": "none" if kind == "step" else rng.choice(["none", "none", "relu", "elu"])}
    if kind != "backward":
        c["bias"] = rng.random() < 0.5
    if kind == "linear":
        c["out"] = rng.choice(["same", "same", "f32"])
    else:
        # gradients of the weights in fp32 for optimizers that keep fp32 weights
        c["dw"] = "same" if c["act"] == "elu" else rng.choice(["same", "f32"])
    if kind == "backward":
        c["keep"] = rng.choice(["input", "8bit"])
    return c


def sizes(case):
    """Rows of each group by rank: shares rank^-skew of n over the groups that have any, largest remainders first."""
    live = case["E"] - case["empty"]
    share = [(r + 1.0) ** -case["skew"] for r in range(live)]
    exact_rows = [case["n"] * s / sum(share) for s in share]
    rows = [int(x) for x in exact_rows]
    by_rest = sorted(range(live), key=lambda r: rows[r] - exact_rows[r])
    for r in by_rest[:case["n"] - sum(rows)]:
        rows[r] += 1
    return rows + [0] * case["empty"]


# ----------------------------------------------------------------- inputs

def _activations(shape, g, dtype, act="none"):
    """Hidden activations: features of different scales, and the values an activation leaves."""
    x = torch.randn(shape, generator=g, device="cuda")
    x *= torch.randn(shape[-1], generator=g, device="cuda").mul_(0.5).exp_()
    if act == "relu":
        x.relu_()
    elif act == "elu":
        x = torch.where(x > 0, x, torch.expm1(x))
    return x.to(dtype)


def prepare(case, seed):
    g = torch.Generator(device="cuda").manual_seed(int(seed) * 7919 + 17)
    dt = DTYPES[case["dtype"]]
    s = {"kind": case["kind"], "case": case}
    if case["kind"] == "trip":
        s["A"] = _activations((case["n"], case["F"]), g, dt, "relu" if int(seed) % 2 else "none")
        return s
    E, k, m, rows = case["E"], case["k"], case["m"], case["n"] + case["pad"]
    # which group has how many rows changes with the seed; a program's plain form knows the sizes on the host
    order = torch.randperm(E, generator=torch.Generator().manual_seed(int(seed) + 5)).tolist()
    by_rank = sizes(case)
    s["rows"] = [by_rank[r] for r in order]
    s["offsets"] = torch.tensor([0] + s["rows"]).cumsum(0).to(torch.int32).cuda()
    s["W"] = (torch.randn((E, m, k), generator=g, device="cuda") * k ** -0.5).to(dt)
    if case.get("bias"):
        s["bias"] = torch.randn((E, m), generator=g, device="cuda") * 0.1
    if case["kind"] in ("linear", "step") or case["keep"] == "input":
        s["X"] = _activations((rows, k), g, dt)
    else:
        s["codes"], s["exps"] = _checkpoint(_activations((rows, k), g, dt))
    if case["kind"] in ("backward", "step"):
        s["dY"] = (torch.randn((rows, m), generator=g, device="cuda") * 0.02).to(dt)
    if case["kind"] == "backward" and case["act"] != "none":
        s["Y"] = _activations((rows, m), g, dt, case["act"])
    # rows behind the last group are the caller's: its buffers hold zeros there
    if case["pad"]:
        if case["kind"] != "backward":
            s["Yout"] = torch.zeros((rows, m), dtype=_out_dtype(case), device="cuda")
        if case["kind"] != "linear":
            s["dXout"] = torch.zeros((rows, k), dtype=dt, device="cuda")
    return s


def _out_dtype(case):
    return torch.float32 if case.get("out") == "f32" else DTYPES[case["dtype"]]


def _dw_dtype(case):
    return torch.float32 if case["dw"] == "f32" else DTYPES[case["dtype"]]


# ------------------------------------------------------------- plain forms

def _checkpoint(A):
    """Codes and exponent bytes of A: a power-of-two scale for each 32 features of a row, codes to nearest even."""
    n, F = A.shape
    nb = (F + BLOCK - 1) // BLOCK
    x = torch.nn.functional.pad(A.float(), (0, nb * BLOCK - F)).view(n, nb, BLOCK)
    top = x.abs().amax(-1)
    lo, hi = (103, 136) if A.dtype == torch.float16 else (1, 248)
    b = (((top.view(torch.int32) + 0x10000) >> 23) - 6).clamp_(lo, hi)
    q = torch.round(x * _pow2(254 - b).unsqueeze(-1)).clamp_(-127, 127)
    bad = ~torch.isfinite(top)
    b[bad] = 255
    q[bad] = 0
    return q.to(torch.int8).view(n, nb * BLOCK)[:, :F].contiguous(), b.to(torch.uint8)


def _pow2(b):
    """2^(b - 127) of whole numbers from 1 to 254, by its fp32 bits."""
    return (b.to(torch.int32) << 23).view(torch.float32)


def _restore(codes, exps, F):
    s = torch.where(exps == 255, math.nan, _pow2(exps.to(torch.int32).clamp(max=254)))
    return codes.float() * s.repeat_interleave(BLOCK, 1)[:, :F]


def _act(v, act):
    return v.relu() if act == "relu" else torch.where(v > 0, v, torch.expm1(v)) if act == "elu" else v


def _spans(s):
    """(group, first row, end row) of the groups that have rows: one product each, as their sizes differ."""
    end, spans = 0, []
    for g, r in enumerate(s["rows"]):
        if r:
            spans.append((g, end, end + r))
        end += r
    return spans


def _plain_linear(s):
    case = s["case"]
    X, W, bias = s["X"], s["W"], s.get("bias")
    Y = torch.zeros((X.shape[0], case["m"]), dtype=_out_dtype(case), device=X.device)
    for g, a, b in _spans(s):
        v = X[a:b].float() @ W[g].float().t()
        Y[a:b] = _act(v if bias is None else v + bias[g], case["act"])
    return Y


def _plain_backward(s, Xf, Y):
    case, dY, W = s["case"], s["dY"], s["W"]
    E, m, k = W.shape
    dX = torch.zeros((dY.shape[0], k), dtype=dY.dtype, device=dY.device)
    dW = torch.zeros((E, m, k), dtype=_dw_dtype(case), device=dY.device)
    db = torch.zeros((E, m), dtype=torch.float32, device=dY.device)
    for g, a, b in _spans(s):
        dZ = dY[a:b].float()
        if case["act"] == "relu":
            dZ = dZ * (Y[a:b] > 0)
        elif case["act"] == "elu":
            y = Y[a:b].float()
            dZ = dZ * torch.where(y > 0, 1.0, y + 1.0)
        dX[a:b] = dZ @ W[g].float()
        dW[g] = dZ.t() @ Xf[a:b]
        db[g] = dZ.sum(0)
    return {"dX": dX, "dW": dW, "db": db}


def _plain(s):
    case = s["case"]
    if s["kind"] == "trip":
        codes, exps = _checkpoint(s["A"])
        return {"A": _restore(codes, exps, case["F"]).to(s["A"].dtype), "exps": exps}
    if s["kind"] == "linear":
        return {"Y": _plain_linear(s)}
    if s["kind"] == "backward":
        Xf = s["X"].float() if "X" in s else _restore(s["codes"], s["exps"], case["k"])
        return _plain_backward(s, Xf, s.get("Y"))
    Y = _plain_linear(s)
    Xf = _restore(*_checkpoint(s["X"]), case["k"])
    return dict(_plain_backward(s, Xf, None), Y=Y)


# --------------------------------------------------------------- one pass

def run(s):
    return _run_own(s) if own else _plain(s)


def _run_own(s):
    import paper_2103_00959_amd as cg
    case = s["case"]
    if s["kind"] == "trip":
        codes, exps = cg.act_checkpoint(s["A"])
        return {"A": cg.act_restore(codes, exps, out_dtype=s["A"].dtype), "exps": exps}
    if s["kind"] == "linear":
        return {"Y": cg.grouped_linear(s["X"], s["W"], s["offsets"], s.get("bias"), case["act"],
                                       out_dtype=_out_dtype(case), out=s.get("Yout"))}
    if s["kind"] == "step":
        Y, codes, exps = cg.grouped_linear(s["X"], s["W"], s["offsets"], s.get("bias"), case["act"],
                                           out=s.get("Yout"), save=True)
        kept = {"codes": codes, "exps": exps}
    else:
        kept = {"X": s["X"]} if "X" in s else {"codes": s["codes"], "exps": s["exps"]}
    o = cg.grouped_linear_backward(s["dY"], s["W"], s["offsets"], **kept, act=case["act"],
                                   Y=s.get("Y"), dw_dtype=_dw_dtype(case),
                                   out={"dX": s["dXout"]} if "dXout" in s else None)
    got = {"dX": o["dX"], "dW": o["dW"], "db": o["db"]}
    return dict(got, Y=Y) if s["kind"] == "step" else got


# ------------------------------------------------------------------- work

def work(case):
    """Each input read once, each output written once; products of the rows that belong to a group."""
    b = 4 if case["dtype"] == "f32" else 2
    if case["kind"] == "trip":
        nF, blocks = case["n"] * case["F"], case["n"] * ((case["F"] + BLOCK - 1) // BLOCK)
        return {"bytes": 2 * nF * b + 2 * (nF + blocks), "flops": 0}
    n, E, k, m = case["n"], case["E"], case["k"], case["m"]
    live = sum(r > 0 for r in sizes(case))
    kept = n * k + n * ((k + BLOCK - 1) // BLOCK)
    weights = live * k * m * b + (4 * live * m if case.get("bias") else 0)
    dw = E * k * m * (4 if case.get("dw") == "f32" else b) + 4 * E * m
    if case["kind"] == "linear":
        return {"bytes": n * k * b + weights + n * m * (4 if case["out"] == "f32" else b), "flops": 2 * n * k * m}
    if case["kind"] == "backward":
        read = n * m * b * (2 if case["act"] != "none" else 1) + (kept if case["keep"] == "8bit" else n * k * b)
        return {"bytes": read + weights + n * k * b + dw, "flops": 4 * n * k * m}
    back = n * m * b + kept + n * k * b          # dY and the checkpoint read back, dX written
    return {"bytes": n * k * b + weights + n * m * b + kept + back + dw, "flops": 6 * n * k * m}


# ------------------------------------------------------------ in 64 bits

def _two_to(e):
    """2^e in 64 bits, by its bits (the device's power function is not exact there)."""
    return ((e.long() + 1023) << 52).view(torch.float64)


def _exact_values(A):
    """The values a checkpoint of A stands for: frexp gives each block's exponent."""
    n, F = A.shape
    nb = -(-F // BLOCK)
    lo, hi = (-24, 9) if A.dtype == torch.float16 else (-126, 121)
    v = torch.zeros((n, nb * BLOCK), dtype=torch.float64, device=A.device)
    v[:, :F] = A
    v = v.reshape(-1, BLOCK)
    mant, e = torch.frexp(v.abs().max(dim=1).values)
    e = torch.where(mant * 128 >= 127.5, e - 6, e - 7).clamp(lo, hi)
    e[mant == 0] = lo
    step = _two_to(e)[:, None]
    q = (v / step).round().clamp(-127, 127) * step
    return q.reshape(n, nb * BLOCK)[:, :F], (e + 127).reshape(n, nb)


def exact(case, seed):
    s = prepare(case, seed)
    if s["kind"] == "trip":
        v, e = _exact_values(s["A"])
        return {"A": v, "exps": e.to(torch.uint8)}
    rows = case["n"] + case["pad"]
    group = torch.full((rows,), -1, device="cuda")
    group[:case["n"]] = torch.repeat_interleave(torch.arange(case["E"], device="cuda"),
                                                torch.tensor(s["rows"], device="cuda"))
    got = {}
    if s["kind"] != "backward":
        got["Y"] = torch.zeros((rows, case["m"]), dtype=torch.float64, device="cuda")
    if s["kind"] != "linear":
        got["dX"] = torch.zeros((rows, case["k"]), dtype=torch.float64, device="cuda")
        got["dW"] = torch.zeros(s["W"].shape, dtype=torch.float64, device="cuda")
        got["db"] = torch.zeros(s["W"].shape[:2], dtype=torch.float64, device="cuda")
    for g in torch.unique(group[group >= 0]).tolist():
        at = torch.nonzero(group == g)[:, 0]
        W = s["W"][g].double()
        if "Y" in got:
            z = torch.mm(s["X"][at].double(), W.t().contiguous())
            if "bias" in s:
                z += s["bias"][g].double()
            if case["act"] == "relu":
                z.clamp_(min=0)
            elif case["act"] == "elu":
                z = z.clamp(min=0) + torch.expm1(z.clamp(max=0))
            got["Y"][at] = z
        if s["kind"] == "linear":
            continue
        if s["kind"] == "step":
            X = _exact_values(s["X"][at])[0]
        elif "X" in s:
            X = s["X"][at].double()
        else:
            step = _two_to(s["exps"][at].long() - 127)
            X = s["codes"][at].double() * step[:, torch.arange(case["k"], device="cuda") // BLOCK]
        d, y = s["dY"][at].double(), s["Y"][at].double() if "Y" in s else None
        if case["act"] == "relu":
            d = torch.where(y > 0, d, 0.0)
        elif case["act"] == "elu":
            d = d * (1 + y.clamp(max=0))
        got["dX"][at] = torch.mm(d, W)
        got["dW"][g] = torch.mm(d.t().contiguous(), X)
        got["db"][g] = d.sum(0)
    return got
