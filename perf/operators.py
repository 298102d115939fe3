"""The operators of a quantised, sampling actor: rows of floats to 8-bit levels with a scale each, the product of such
levels with scales for each row and each output channel, and the draw of an index from a row of scores under temperature,
top-k, top-p and min-p with given random numbers.  Cases, inputs, plain forms and 64-bit values of each."""
from __future__ import annotations

import numpy as np
import torch

own = False   # False: the operators in elementary torch operations; True: the framework's kernels

TYPES = {"fp32": torch.float32, "bf16": torch.bfloat16, "fp16": torch.float16}
BYTES = {"fp32": 4, "bf16": 2, "fp16": 2}
CODES = {"fp32": 0, "bf16": 1, "fp16": 2}   # the framework's DQN_TYPE_FP32, DQN_TYPE_BF16, DQN_TYPE_FP16


def pitch(n):
    """Bytes of a row of n levels when rows start on 16-byte borders."""
    return (n + 15) // 16 * 16


def listed():
    return [
        # the inputs of the Q-network's fully connected layer for 32 acting states: a small call, latency counts
        {"name": "quantize act 32x3136", "op": "quantize", "rows": 32, "cols": 3136, "dtype": "bf16", "pad": 0},
        # a large activation matrix with what its levels stand for, as training with quantisation in mind has it
        {"name": "quantize 8192x8192", "op": "quantize", "rows": 8192, "cols": 8192, "dtype": "bf16", "pad": 0},
        # odd lengths inside a wider matrix, full precision
        {"name": "quantize odd 1001x5003", "op": "quantize", "rows": 1001, "cols": 5003, "dtype": "fp32", "pad": 5},
        # fc1 of the Q-network for the benchmark's eight environments
        {"name": "linear act 8x512x3136", "op": "linear", "M": 8, "N": 512, "K": 3136, "dtype": "fp32", "relu": True, "bias": True, "dense": False},
        # one token against a wide layer: the weights' bytes are everything
        {"name": "linear token 1x16384x4096", "op": "linear", "M": 1, "N": 16384, "K": 4096, "dtype": "bf16", "relu": False, "bias": False, "dense": False},
        # fc1 of the Q-network for the largest minibatch of the benchmark's sweep
        {"name": "linear 512x512x3136", "op": "linear", "M": 512, "N": 512, "K": 3136, "dtype": "fp32", "relu": True, "bias": True, "dense": False},
        # ragged sizes, rows packed without a gap (so at every alignment)
        {"name": "linear odd 1111x2051x2003", "op": "linear", "M": 1111, "N": 2051, "K": 2003, "dtype": "fp16", "relu": False, "bias": True, "dense": True},
        # a large product: arithmetic is everything
        {"name": "linear 8192x8192x8192", "op": "linear", "M": 8192, "N": 8192, "K": 8192, "dtype": "bf16", "relu": False, "bias": False, "dense": False},
        # a Boltzmann policy over Q rows of 18 actions
        {"name": "sample 512x18", "op": "sample", "rows": 512, "n": 18, "dtype": "fp32", "spread": 2.0, "filters": "temperature", "masked": 0.0},
        # one long row, top-k and top-p together: a single sequence being continued
        {"name": "sample 1x131072", "op": "sample", "rows": 1, "n": 131072, "dtype": "bf16", "spread": 3.0, "filters": "k+p", "masked": 0.0},
        # many long rows, top-p alone
        {"name": "sample 256x131072", "op": "sample", "rows": 256, "n": 131072, "dtype": "bf16", "spread": 3.0, "filters": "p", "masked": 0.0},
        # odd length, full precision, part of each row masked away, every row with settings of its own
        {"name": "sample odd 33x50021", "op": "sample", "rows": 33, "n": 50021, "dtype": "fp32", "spread": 3.0, "filters": "mixed", "masked": 0.1},
    ]


def spread_size(rng, lo, hi):
    """A whole number from lo to hi, evenly over its logarithm."""
    return min(hi, max(lo, int(round(lo * (hi / lo) ** rng.random()))))


def draw(rng):
    op = rng.choice(["quantize", "linear", "sample"])
    dtype = rng.choice(["fp32", "bf16", "fp16"])
    if op == "quantize":
        cols = spread_size(rng, 1, 16384)
        rows = spread_size(rng, 1, min(16384, (1 << 25) // cols))
        return {"op": op, "rows": rows, "cols": cols, "dtype": dtype, "pad": rng.choice([0, 0, 1, 8])}
    if op == "linear":
        M, N, K = spread_size(rng, 1, 8192), spread_size(rng, 1, 16384), spread_size(rng, 16, 16384)
        while M * N * K > 1 << 38:
            M, N, K = (M + 1) // 2, N, (K + 1) // 2
        return {"op": op, "M": M, "N": N, "K": K, "dtype": dtype, "relu": rng.random() < 0.3, "bias": rng.random() < 0.5, "dense": rng.random() < 0.3}
    n = spread_size(rng, 2, 262144)
    rows = spread_size(rng, 1, min(4096, (1 << 24) // n))
    return {"op": op, "rows": rows, "n": n, "dtype": dtype, "spread": rng.choice([1.0, 2.0, 4.0]),
            "filters": rng.choice(["temperature", "k", "p", "k+p", "min_p", "mixed"]), "masked": rng.choice([0.0, 0.0, 0.2])}


def floats(g, *shape):
    return torch.randn(*shape, generator=g, device="cuda", dtype=torch.float32)


def levels_of(x):
    """8-bit levels and scales of x's rows, for the inputs of a product."""
    a = x.abs().amax(1, keepdim=True).clamp_min(1e-30)
    return torch.round(x * (127.0 / a)).to(torch.int8), (a / 127.0).squeeze(1)


def settings(case, g):
    """Temperature, top-k, top-p and min-p of every row (None: off), as a server or an actor sets them."""
    rows, n, f = case["rows"], case["n"], case["filters"]
    pick = lambda values: torch.tensor(values, device="cuda")[torch.randint(len(values), (rows,), generator=g, device="cuda")]  # noqa: E731
    if f == "temperature":
        return pick([0.5, 0.7, 1.0, 1.3]), None, None, None
    if f == "k":
        return pick([0.7, 1.0]), pick([20, 40, 50]).int(), None, None
    if f == "p":
        return pick([0.7, 0.8, 1.0]), None, pick([0.9, 0.95]), None
    if f == "k+p":
        return pick([0.7, 0.8, 1.0]), pick([40, 50, 100]).int(), pick([0.9, 0.95]), None
    if f == "min_p":
        return pick([1.0, 1.5]), None, None, pick([0.02, 0.05, 0.1])
    return pick([0.0, 0.5, 1.0, 1.0, 2.0]), pick([0, 0, 1, 40, 1000, max(1, n // 2)]).int(), pick([0.3, 0.9, 0.95, 1.0]), pick([0.0, 0.0, 0.02, 0.1])


def prepare(case, seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    s = dict(case)
    s["stream"] = torch.cuda.current_stream()
    if case["op"] == "quantize":
        rows, cols = case["rows"], case["cols"]
        # rows of very different size, as activations of different tokens are
        x = floats(g, rows, cols + case["pad"]) * torch.exp(floats(g, rows, 1))
        s["x"] = x.to(TYPES[case["dtype"]])
        s["q"] = torch.zeros(rows, pitch(cols), dtype=torch.int8, device="cuda")
        s["scale"] = torch.zeros(rows, device="cuda")
        s["out"] = torch.zeros(rows, cols, dtype=TYPES[case["dtype"]], device="cuda")
    elif case["op"] == "linear":
        M, N, K = case["M"], case["N"], case["K"]
        ld = K if case["dense"] else pitch(K)
        s["ld"] = ld
        x, w = torch.zeros(M, ld, dtype=torch.int8, device="cuda"), torch.zeros(N, ld, dtype=torch.int8, device="cuda")
        x[:, :K], s["sx"] = levels_of(floats(g, M, K) * torch.exp(0.5 * floats(g, M, 1)))
        w[:, :K], s["sw"] = levels_of(floats(g, N, K) * (K ** -0.5))
        s["x"], s["w"] = x, w
        s["b"] = 0.1 * floats(g, N) if case["bias"] else None
        s["y"] = torch.zeros(M, N, dtype=TYPES[case["dtype"]], device="cuda")
    else:
        rows, n = case["rows"], case["n"]
        x = case["spread"] * floats(g, rows, n)
        if case["masked"]:
            x = x.masked_fill(torch.rand(rows, n, generator=g, device="cuda") < case["masked"], float("-inf"))
        s["x"] = x.to(TYPES[case["dtype"]])
        s["t"], s["k"], s["p"], s["m"] = settings(case, g)
        s["u"] = torch.rand(rows, generator=g, device="cuda")
        s["index"] = torch.zeros(rows, dtype=torch.int32, device="cuda")
        s["logp"] = torch.zeros(rows, device="cuda")
        s["work"] = None   # the framework's workspace for this size, made on the first call as a server makes it
    return s


def run(s):
    if own:
        return run_own(s)
    return {"quantize": plain_quantize, "linear": plain_linear, "sample": plain_sample}[s["op"]](s)


def run_own(s):
    import paper_2111_01264_amd as P
    if s["op"] == "quantize":
        P.q8_quantize_rows(s["x"], CODES[s["dtype"]], s["cols"] + s["pad"], s["rows"], s["cols"], s["q"], pitch(s["cols"]), s["scale"], s["out"], s["cols"], s["stream"])
        return {"values": s["out"], "scale": s["scale"]}   # (the levels themselves, held in 8 bits, are in s["q"])
    if s["op"] == "linear":
        P.q8_linear(s["x"], s["ld"], s["sx"], s["w"], s["ld"], s["sw"], s["b"], int(s["relu"]), s["M"], s["N"], s["K"], s["y"], CODES[s["dtype"]], s["N"], s["stream"])
        return {"y": s["y"]}
    if s["work"] is None:
        s["work"] = torch.empty(max(1, P.policy_sample_workspace(s["rows"], s["n"])), dtype=torch.uint8, device="cuda")
    P.policy_sample(s["x"], CODES[s["dtype"]], s["n"], s["rows"], s["n"], s["t"], s["k"], s["p"], s["m"], s["u"], s["index"], s["logp"], s["work"], s["work"].numel(), s["stream"])
    return {"index": s["index"], "logp": s["logp"]}


def plain_quantize(s):
    # 64 bits: a quotient next to the border between two levels has to fall on its own side
    x = s["x"][:, :s["cols"]].double()
    a = x.abs().amax(1, keepdim=True)
    q = torch.where(a > 0, torch.round(127.0 * x / a), 0.0)
    scale = (a / 127.0).float()
    return {"values": (q.float() * scale).to(TYPES[s["dtype"]]), "scale": scale.squeeze(1)}


def plain_linear(s):
    K = s["K"]
    y = s["x"][:, :K].float() @ s["w"][:, :K].float().t()
    y = y * s["sx"][:, None] * s["sw"][None, :]
    if s["b"] is not None:
        y = y + s["b"]
    if s["relu"]:
        y = torch.clamp_min(y, 0.0)
    return {"y": y.to(TYPES[s["dtype"]])}


def plain_sample(s):
    # 64 bits: sums over a long row, and random numbers next to a border between two entries
    x, rows, n = s["x"].double(), s["rows"], s["n"]
    t = torch.ones(rows, 1, device=x.device, dtype=torch.float64) if s["t"] is None else s["t"].double()[:, None]
    x, order = torch.sort(x, dim=1, descending=True, stable=True)   # ties: lowest index first
    at = torch.arange(n, device=x.device)[None, :]
    top = x[:, :1]
    w = torch.where(x == top, 1.0, torch.exp((x - top) / t))
    w = torch.where(t == 0, (at == 0).double(), w)
    c = torch.cumsum(w, 1)
    keep = torch.ones_like(w, dtype=torch.bool)
    mass = c[:, -1:]
    if s["k"] is not None:
        k = s["k"].long()[:, None]
        k = torch.where((k <= 0) | (k > n), n, k)
        keep &= at < k
        mass = c.gather(1, k - 1)
    if s["p"] is not None:
        p = s["p"].double()[:, None]
        keep &= (c - w < p * mass) | (p >= 1) | (at == 0)
    if s["m"] is not None:
        keep &= w >= s["m"].double()[:, None].clamp_max(1.0)
    w = torch.zeros_like(w).scatter_(1, order, torch.where(keep, w, 0.0))   # back to the order of the indices
    c = torch.cumsum(w, 1)
    total = c[:, -1:]
    index = (c <= s["u"].double()[:, None] * total).sum(1, keepdim=True)
    empty = top == float("-inf")   # a mask that leaves nothing
    logp = torch.where(empty, float("nan"), torch.log(w.gather(1, index) / total))
    index = torch.where(empty, -1, index)
    return {"index": index.squeeze(1).int(), "logp": logp.squeeze(1).float()}


def work(case):
    if case["op"] == "quantize":
        cells, e = case["rows"] * case["cols"], BYTES[case["dtype"]]
        return {"bytes": 2 * cells * e + cells + 4 * case["rows"], "flops": 2 * cells}
    if case["op"] == "linear":
        M, N, K = case["M"], case["N"], case["K"]
        return {"bytes": M * K + N * K + 4 * (M + N + (N if case["bias"] else 0)) + M * N * BYTES[case["dtype"]], "flops": 2 * M * N * K}
    cells = case["rows"] * case["n"]
    return {"bytes": cells * BYTES[case["dtype"]] + 28 * case["rows"], "flops": 2 * cells}


def exact(case, seed):
    s = prepare(case, seed)
    if case["op"] == "quantize":
        x = s["x"][:, :case["cols"]].float().cpu().numpy().astype(np.float64)
        a = np.max(np.abs(x), axis=1, keepdims=True)
        levels = np.rint(np.divide(x * 127.0, a, out=np.zeros_like(x), where=a > 0))
        return {"values": levels * (a / 127.0), "scale": a[:, 0] / 127.0}
    if case["op"] == "linear":
        K = case["K"]
        # whole numbers below 2^53: the sums are exact
        y = torch.matmul(s["x"][:, :K].to(torch.float64), s["w"][:, :K].to(torch.float64).t().contiguous())
        y *= torch.outer(s["sx"].to(torch.float64), s["sw"].to(torch.float64))
        if s["b"] is not None:
            y += s["b"].to(torch.float64)
        return {"y": torch.relu(y) if case["relu"] else y}
    x, u = s["x"].float().cpu().numpy().astype(np.float64), s["u"].cpu().numpy().astype(np.float64)
    t, k, p, m = (None if s[v] is None else s[v].cpu().numpy().astype(np.float64) for v in "tkpm")
    index, logp = np.zeros(case["rows"], np.int32), np.zeros(case["rows"])
    for r in range(case["rows"]):
        if not np.any(x[r] > -np.inf):
            index[r], logp[r] = -1, np.nan
            continue
        if t is not None and t[r] == 0:
            index[r] = np.argmax(x[r])
            continue
        w = np.exp((x[r] - x[r].max()) / (1.0 if t is None else t[r]))
        order = np.argsort(-x[r], kind="stable")
        if k is not None and 0 < k[r] < case["n"]:
            order = order[:int(k[r])]
        before = np.cumsum(w[order]) - w[order]
        if p is not None and p[r] < 1:
            inside = before < p[r] * w[order].sum()
            inside[0] = True
            order = order[inside]
        if m is not None:
            order = order[w[order] >= min(m[r], 1.0)]
        order = np.sort(order)
        c = np.cumsum(w[order])
        index[r] = order[np.searchsorted(c, u[r] * c[-1], side="right")]
        logp[r] = np.log(w[index[r]] / c[-1])
    return {"index": index, "logp": logp}
