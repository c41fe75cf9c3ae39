"""Attention over a stored pattern as it is trained and served: a position bias, dropout, several heads, gradients.

Operations
  forward   out = dropout(softmax_rows(scale * X Y^T + bias at the pattern)) @ H and the rows' log-sum-exp
  backward  the gradients of X, Y, H and of the bias table
  bias      scaled scores plus bias, on a value array (the chain of separate calls)
  bias_grad the gradient of the bias table from the gradient of a value array
  dropout   dropout on a value array, the probabilities' or their gradient's

Patterns
  band       a sequence: a token sees the ``window`` last tokens up to itself and the first ``sinks``
  rows       the last M tokens of a sequence of K alone: one step of serving
  rmat       power-law graph (a/b/c/d = .57/.19/.19/.05)
  lognormal  row degrees exp(N(2.5, 1)), columns uniform
  uniform    about ``deg`` entries a row at random columns, every 16th row empty, any M x K

The bias of an entry is that of the bucket of its clamped relative position col - row - shift: distances below a quarter
of the buckets have one each, longer ones share logarithmically many.  An entry is dropped where the first word of
Threefry-2x32 with 13 rounds at the counter (row, column) is below p * 2^32; the key comes from seed, step and head.
"""
import math
from functools import reduce

import numpy as np
import torch

own = False

MASK = 0xFFFFFFFF
TURNS = (13, 15, 26, 6, 17, 29, 16, 24)  # Threefry-2x32's rotations
PARITY = 0x1BD11BDA


# ------------------------------------------------------------------------------------------------ the cases
def listed():
    return [
        # one new token of a sequence, all heads: the smallest call, where latency counts
        dict(name="forward_token", op="forward", pattern="rows", M=1, K=2048, window=1024, sinks=4, heads=8, kv_heads=2, d=64, N=64,
             p=0.0, buckets=32, reach=128, dtype="bf16"),
        # a training pass over a sequence with a sliding window, eight heads that share two of keys and values
        dict(name="forward_band_4k", op="forward", pattern="band", M=4096, window=256, sinks=4, heads=8, kv_heads=2, d=64, N=64,
             p=0.1, buckets=32, reach=128, dtype="bf16"),
        # graph attention over 65 k nodes, unequal widths
        dict(name="forward_rmat16", op="forward", pattern="rmat", scale=16, edge_factor=16, heads=1, kv_heads=1, d=32, N=128,
             p=0.3, buckets=32, reach=128, dtype="f16"),
        # the backward passes of a small graph, of the sequence and of a large graph
        dict(name="backward_rmat13", op="backward", pattern="rmat", scale=13, edge_factor=16, heads=1, kv_heads=1, d=32, N=64,
             p=0.3, buckets=32, reach=128, dtype="f16"),
        dict(name="backward_band_4k", op="backward", pattern="band", M=4096, window=256, sinks=4, heads=8, kv_heads=2, d=64, N=64,
             p=0.1, buckets=32, reach=128, dtype="bf16"),
        dict(name="backward_lognormal", op="backward", pattern="lognormal", M=262144, heads=2, kv_heads=2, d=64, N=64,
             p=0.1, buckets=32, reach=128, dtype="f16"),
        # the separate calls of the chain: a bipartite matrix of odd sizes, power-law graphs, a sequence of several heads
        dict(name="bias_odd", op="bias", pattern="uniform", M=30011, K=50021, deg=11, heads=2, p=0.0, buckets=20, reach=300, dtype="bf16"),
        dict(name="bias_rmat18", op="bias", pattern="rmat", scale=18, edge_factor=16, heads=1, p=0.0, buckets=32, reach=128, dtype="f16"),
        dict(name="bias_grad_rmat13", op="bias_grad", pattern="rmat", scale=13, edge_factor=16, heads=1, p=0.0, buckets=32, reach=128, dtype="f16"),
        dict(name="bias_grad_band_4k", op="bias_grad", pattern="band", M=4096, window=256, sinks=4, heads=8, p=0.0, buckets=32, reach=128, dtype="bf16"),
        dict(name="dropout_rmat16", op="dropout", pattern="rmat", scale=16, edge_factor=16, heads=1, p=0.3, buckets=0, reach=0, dtype="f16"),
        dict(name="dropout_lognormal", op="dropout", pattern="lognormal", M=262144, heads=2, p=0.5, buckets=0, reach=0, dtype="bf16"),
    ]


def draw(rng):
    def spread(lo, hi):
        return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))

    op = rng.choice(["forward", "forward", "backward", "backward", "bias", "bias_grad", "dropout"])
    pattern = rng.choice(["band", "band", "rmat", "lognormal", "uniform"] + (["rows"] if op == "forward" else []))
    case = dict(op=op, pattern=pattern)
    if pattern == "band":
        case.update(M=spread(16, 8192), window=spread(4, 384), sinks=rng.randint(0, 8))
        entries = case["M"] * (case["window"] + case["sinks"])
    elif pattern == "rows":
        case.update(M=rng.randint(1, 16), K=spread(17, 30000), sinks=rng.randint(0, 8))
        case["window"] = spread(1, case["K"] - case["M"] + 1)
        entries = case["M"] * (case["window"] + case["sinks"])
    elif pattern == "rmat":
        case.update(scale=rng.randint(9, 18), edge_factor=rng.randint(6, 18))
        entries = case["edge_factor"] << case["scale"]
    elif pattern == "lognormal":
        case.update(M=spread(500, 200000))
        entries = 20 * case["M"]
    else:
        case.update(M=spread(300, 100000), K=spread(300, 100000), deg=rng.randint(2, 40))
        entries = case["deg"] * case["M"]
    if op in ("forward", "backward"):
        case.update(d=8 * rng.randint(1, 16), N=8 * rng.randint(1, 16))
    width = case.get("d", 128) + case.get("N", 0)
    case["heads"] = rng.choice([h for h in (1, 2, 3, 4, 6, 8) if h == 1 or entries * h * width <= 1.1e9])
    if op in ("forward", "backward"):
        case["kv_heads"] = rng.choice([k for k in (1, 2, 3, 4, 6, 8) if case["heads"] % k == 0])
    case["p"] = rng.choice([0.0, 0.1, 0.35, 0.6]) if op in ("forward", "backward") else rng.choice([0.05, 0.3, 0.6]) if op == "dropout" else 0.0
    if op == "dropout" or (op in ("forward", "backward") and rng.random() < 0.25):
        case.update(buckets=0, reach=0)
    else:
        case.update(buckets=4 * rng.randint(2, 16), reach=spread(17, 1000))
    case["dtype"] = rng.choice(["f16", "bf16"])
    return case


# --------------------------------------------------------------------------------------------------- inputs
def _shape(case):
    if case["pattern"] in ("uniform", "rows"):
        return case["M"], case["K"]
    n = 1 << case["scale"] if case["pattern"] == "rmat" else case["M"]
    return n, n


def _shift(case):
    """Position of row 0 (the rows of ``rows`` are the last of the sequence)."""
    return case["K"] - case["M"] if case["pattern"] == "rows" else 0


def _pattern(case, turn, device):
    """(row, column) of every entry, in CSR order.  The draws belong to the case; columns are numbered from another one
    on for each ``turn`` (a sequence has one numbering)."""
    M, K = _shape(case)
    gen = torch.Generator(device=device).manual_seed(0)
    if case["pattern"] in ("band", "rows"):
        i = torch.arange(M, device=device)[:, None]
        j = i + _shift(case) - torch.arange(case["window"], device=device)[None]
        k = torch.arange(case["sinks"], device=device)[None].expand(M, -1)
        rows = torch.cat([i.expand_as(j)[j >= 0], i.expand_as(k)[k <= i + _shift(case)]])
        cols = torch.cat([j[j >= 0], k[k <= i + _shift(case)]])
        turn = 0
    elif case["pattern"] == "rmat":
        n = case["edge_factor"] << case["scale"]
        u = torch.rand((case["scale"], n), generator=gen, device=device)
        bit = (1 << torch.arange(case["scale"], device=device))[:, None]
        rows = ((u >= 0.76) * bit).sum(0)
        cols = ((((u >= 0.57) & (u < 0.76)) | (u >= 0.95)) * bit).sum(0)
    else:
        if case["pattern"] == "uniform":
            deg = torch.full((M,), case["deg"], device=device)
            deg[5::16] = 0
        else:
            deg = torch.exp(torch.randn(M, generator=gen, device=device) + 2.5).round().clamp(1, min(4096, K)).to(torch.int64)
        rows = torch.arange(M, device=device).repeat_interleave(deg)
        cols = torch.randint(0, K, (rows.numel(),), generator=gen, device=device)
    key = torch.unique(rows * K + (cols + turn) % K)  # sorted: CSR order
    return key // K, key % K


def _bucket_of(case):
    """Bucket of each relative position -reach .. reach: half of the buckets for either sign, each half with distances of its
    own up to its half, then logarithmically many a bucket."""
    half, reach = case["buckets"] // 2, case["reach"]
    near = half // 2
    r = np.arange(-reach, reach + 1)
    n = np.abs(r)
    far = near + np.floor(np.log(np.maximum(n, near) / near) / np.log(max(reach, near + 1) / near) * (half - near) + 1e-9).astype(np.int64)
    return torch.from_numpy((np.where(n < near, n, np.minimum(far, half - 1)) + (r > 0) * half).astype(np.uint8))


def _blocks(row, col, M, K):
    """Where CSR entries lie in a value array of windows of eight rows and blocks of 32 columns' vectors, and its length."""
    cell, vector = torch.unique((row >> 3) * K + col, return_inverse=True)
    first = torch.searchsorted(cell, torch.arange((M + 7) // 8 + 1, device=row.device) * K)
    start, end = first[row >> 3], first[(row >> 3) + 1]
    block = start + (vector - start) // 32 * 32
    return 8 * block + (row & 7) * torch.clamp(end - block, max=32) + vector - block, 8 * cell.numel()


def prepare(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    dt = torch.float16 if case["dtype"] == "f16" else torch.bfloat16
    M, K = _shape(case)
    op, heads = case["op"], case["heads"]
    row, col = _pattern(case, int(torch.randint(0, K, (1,), generator=gen, device="cuda")), "cuda")

    def normal(*shape, std=1.0):
        return (torch.randn(shape, generator=gen, device="cuda") * std).to(dt)

    s = dict(op=op, M=M, K=K, heads=heads, p=case["p"], shift=_shift(case), dt=dt, row=row, col=col)
    s["rng"] = torch.tensor([seed * 0x9E3779B97F4A7C15 % (1 << 63), seed % 1000], device="cuda")  # seed and step
    if case["buckets"]:
        s["bucket"] = _bucket_of(case).cuda()
        s["table"] = normal(heads, case["buckets"], std=0.5)
    if op in ("forward", "backward"):
        s["kv"] = case["kv_heads"]
        s["X"], s["Y"] = normal(M, heads, case["d"]), normal(K, s["kv"], case["d"])
        s["H"] = normal(K, s["kv"], case["N"])
        s["scale"] = case["d"] ** -0.5
    else:
        s["slot"], s["length"] = _blocks(row, col, M, K)
        s["scale"] = 0.125
        s["vals"] = torch.zeros((heads, s["length"]), dtype=dt, device="cuda")
        # scores, gradients that arrive at them, probabilities
        v = normal(heads, row.numel(), std={"bias": 8.0, "bias_grad": 0.1, "dropout": 1.0}[op])
        s["vals"][:, s["slot"]] = v.abs() / 16 if op == "dropout" else v
    if own:
        import paper_2412_11007_amd as fs
        rowptr = torch.searchsorted(row, torch.arange(M + 1, device="cuda")).to(torch.int32)
        colidx = col.to(torch.int32)
        s["fmt"] = fs.fs_convert(rowptr, colidx, None, M, K, torch_dtype=dt, V=0 if op in ("forward", "backward") else 8)
        s["bias"] = fs.FsBucketBias(s["table"], s["bucket"], shift=s["shift"]) if case["buckets"] else None
        s["drop"] = fs.FsDropout(case["p"], s["rng"]) if case["p"] else None
    if op == "backward":
        s["dOut"] = normal(M, heads, case["N"])
        if own:
            s["out"], s["lse"] = fs.fs_attention_forward(s["fmt"], s["X"], s["Y"], s["H"], scale=s["scale"], bias=s["bias"], dropout=s["drop"])
            rowptr_t, colidx_t, _ = fs.fs_csr_transpose(rowptr, colidx, M, K)
            s["fmt_t"] = fs.fs_convert(rowptr_t, colidx_t, None, K, M, torch_dtype=dt)
        else:
            s["out"], s["lse"] = _forward(s)
    return s


# ------------------------------------------------------------------------------------------------- one pass
def run(s):
    if own:
        return _calls(s)
    if s["op"] == "forward":
        return dict(zip(("out", "lse"), _forward(s)))
    if s["op"] == "backward":
        return _backward(s)
    v = s["vals"][:, s["slot"]].float()
    if s["op"] == "bias_grad":
        return _by_bucket(s, v).to(s["dt"])
    v = v * s["scale"] + _bias(s).T if s["op"] == "bias" else v * _keep(s).T
    out = torch.zeros_like(s["vals"])
    out[:, s["slot"]] = v.to(s["dt"])
    return out


def _calls(s):
    import paper_2412_11007_amd as fs
    if s["op"] == "forward":
        out, lse = fs.fs_attention_forward(s["fmt"], s["X"], s["Y"], s["H"], scale=s["scale"], bias=s["bias"], dropout=s["drop"])
        return {"out": out, "lse": lse}
    if s["op"] == "backward":
        got = fs.fs_attention_backward(s["fmt"], s["fmt_t"], s["X"], s["Y"], s["H"], s["out"], s["lse"], s["dOut"], scale=s["scale"],
                                       bias=s["bias"], dropout=s["drop"])
        return {k: g for k, g in zip(("dX", "dY", "dH", "dTable"), got) if g is not None}
    if s["op"] == "bias":
        return fs.fs_edge_bias(s["fmt"], s["vals"], s["bias"], scale=s["scale"])
    if s["op"] == "bias_grad":
        return fs.fs_edge_bias_backward(s["fmt"], s["vals"], s["bias"])
    return fs.fs_edge_dropout(s["fmt"], s["vals"], s["drop"])


# ----------------------------------------------------------------------------------------- the plain form
def _threefry(key, ctr, rounds):
    """Both words of Threefry-2x32 on 64-bit tensors that hold 32-bit values."""
    ks = (key[0], key[1], key[0] ^ key[1] ^ PARITY)

    def step(x, i):
        a = (x[0] + x[1]) & MASK
        b = ((x[1] << TURNS[i % 8] & MASK) | x[1] >> (32 - TURNS[i % 8])) ^ a
        if i % 4 == 3:
            n = i // 4 + 1
            a, b = (a + ks[n % 3]) & MASK, (b + ks[(n + 1) % 3] + n) & MASK
        return a, b

    return reduce(step, range(rounds), ((ctr[0] + ks[0]) & MASK, (ctr[1] + ks[1]) & MASK))


def _keep(s):
    """What each entry's probability is multiplied with, (entries, heads)."""
    seed, step = s["rng"][0], s["rng"][1]
    k = _threefry((seed & MASK, seed >> 32 & MASK), (step & MASK, step >> 32 & MASK), 20)
    head = torch.arange(s["heads"], device="cuda")
    word = _threefry(_threefry(k, (head, 0 * head), 20), (s["row"][:, None], s["col"][:, None]), 13)[0]
    return (word >= math.floor(s["p"] * 2.0 ** 32)).float() / (1 - s["p"])


def _buckets(s):
    reach = s["bucket"].numel() // 2
    return s["bucket"].long()[torch.clamp(s["col"] - s["row"] - s["shift"], -reach, reach) + reach]


def _bias(s):
    return s["table"].float().T[_buckets(s)]  # (entries, heads)


def _by_bucket(s, v):
    """Sums of (heads, entries) over the entries of each bucket: long sums, in 64 bits."""
    mine = _buckets(s)[:, None] == torch.arange(s["table"].shape[1], device="cuda")
    return torch.where(mine, v[..., None], 0.0).sum(1, dtype=torch.float64)


def _over_heads(s, t):
    """(K, kv_heads, .) as every query head sees it, in 32 bits."""
    return t.float().repeat_interleave(s["heads"] // s["kv"], 1)


def _scores(s):
    v = s["scale"] * (s["X"].float()[s["row"]] * _over_heads(s, s["Y"])[s["col"]]).sum(-1)
    return v + _bias(s) if "bucket" in s else v


def _forward(s):
    M, row, v = s["M"], s["row"], _scores(s)
    index = row[:, None].expand_as(v)
    top = torch.full((M, s["heads"]), -math.inf, device="cuda").scatter_reduce(0, index, v, "amax")
    e = torch.exp(v - top[row])
    total = torch.zeros_like(top).index_add(0, row, e)
    w = e / total[row] * _keep(s) if s["p"] else e / total[row]
    out = torch.zeros((M, s["heads"], s["H"].shape[2]), device="cuda").index_add(0, row, w[..., None] * _over_heads(s, s["H"])[s["col"]])
    return out.to(s["dt"]), (top + torch.log(total)).T.contiguous()


def _backward(s):
    row, col = s["row"], s["col"]
    H, dOut = _over_heads(s, s["H"]), s["dOut"].float()
    w = torch.exp(_scores(s) - s["lse"].T[row])
    keep = _keep(s) if s["p"] else torch.ones_like(w)
    D = (dOut * s["out"].float()).sum(-1)
    ds = w * (keep * (dOut[row] * H[col]).sum(-1) - D[row])

    def onto(shape, index, weight, values):  # sum of weighted rows
        return torch.zeros(shape, device="cuda").index_add(0, index, weight[..., None] * values)

    def group(t):  # the query heads that share keys and values
        return t.reshape(t.shape[0], s["kv"], -1, t.shape[2]).sum(2).to(s["dt"])

    g = {"dX": s["scale"] * onto(s["X"].shape, row, ds, _over_heads(s, s["Y"])[col]),
         "dY": s["scale"] * onto((s["K"], s["heads"], s["X"].shape[2]), col, ds, s["X"].float()[row]),
         "dH": onto((s["K"], s["heads"], H.shape[2]), col, w * keep, dOut[row])}
    g = {"dX": g["dX"].to(s["dt"]), "dY": group(g["dY"]), "dH": group(g["dH"])}
    if "bucket" in s:
        g["dTable"] = _by_bucket(s, ds.T).to(s["dt"])
    return g


# ----------------------------------------------------------------------------------- the definition in 64 bits
def _words(key, row, col, rounds):
    """Both words, on numpy's 32-bit integers."""
    k = [np.uint32(key[0]), np.uint32(key[1])]
    k.append(k[0] ^ k[1] ^ np.uint32(PARITY))
    a, b = np.uint32(row) + k[0], np.uint32(col) + k[1]
    for i in range(rounds):
        t = np.uint32(TURNS[i % 8])
        a = a + b
        b = (b << t | b >> (np.uint32(32) - t)) ^ a
        if i % 4 == 3:
            a = a + k[(i // 4 + 1) % 3]
            b = b + k[(i // 4 + 2) % 3] + np.uint32(i // 4 + 1)
    return a, b


def _sums(index, n, values):
    """Sums of rows of ``values`` by ``index``, segment by segment of the sorted order."""
    order = torch.argsort(index, stable=True)
    return torch.segment_reduce(values[order], "sum", lengths=torch.bincount(index, minlength=n), initial=0.0)


def exact(case, seed):
    global own
    was, own = own, False
    try:
        s = prepare(case, seed)
    finally:
        own = was
    M, K, row, col = s["M"], s["K"], s["row"].cpu().numpy(), s["col"].cpu().numpy()
    with np.errstate(over="ignore"):
        seed_, step = int(s["rng"][0]), int(s["rng"][1])
        a = _words((seed_ & MASK, seed_ >> 32 & MASK), np.array([step & MASK]), np.array([step >> 32 & MASK]), 20)
        keep = []
        for h in range(s["heads"]):
            k = _words((a[0][0], a[1][0]), np.array([h]), np.array([0]), 20)
            word = _words((k[0][0], k[1][0]), row, col, 13)[0]
            keep.append(torch.from_numpy(np.where(word.astype(np.int64) >= int(s["p"] * 4294967296), 1 / (1 - s["p"]), 0.0)).cuda())
    bias = [0.0] * s["heads"]
    if "bucket" in s:
        lut = s["bucket"].cpu().numpy().astype(np.int64)
        bucket = torch.from_numpy(lut[np.clip(col - row - s["shift"], -(lut.size // 2), lut.size // 2) + lut.size // 2]).cuda()
        bias = [t[bucket] for t in s["table"].double()]
    if case["op"] not in ("forward", "backward"):
        if case["op"] == "bias_grad":
            return _sums(bucket, s["table"].shape[1], s["vals"][:, s["slot"]].double().T).T
        out = s["vals"].double()
        for h in range(s["heads"]):
            v = out[h, s["slot"]]
            out[h, s["slot"]] = s["scale"] * v + bias[h] if case["op"] == "bias" else v * keep[h]
        return out
    r, c, share = s["row"], s["col"], s["heads"] // s["kv"]
    empty = torch.bincount(r, minlength=M) == 0
    got = {k: [] for k in ("out", "lse", "dX", "dTable")}
    dY = [0.0] * s["kv"]
    dH = [0.0] * s["kv"]
    for h in range(s["heads"]):
        x, y, v = s["X"][:, h].double(), s["Y"][:, h // share].double(), s["H"][:, h // share].double()
        t = s["scale"] * (x[r] * y[c]).sum(1) + bias[h]
        top = t.max()  # one for all rows: exponentials in 64 bits reach far
        lse = torch.where(empty, -math.inf, top + torch.log(_sums(r, M, torch.exp(t - top)[:, None])[:, 0]))
        p = torch.exp(t - lse[r])
        w = p * keep[h] if s["p"] else p
        out = _sums(r, M, w[:, None] * v[c])
        got["out"].append(out)
        got["lse"].append(lse)
        if case["op"] == "backward":
            g = s["dOut"][:, h].double()
            ds = (w * (g[r] * v[c]).sum(1) - p * (g * out).sum(1)[r])[:, None]
            got["dX"].append(s["scale"] * _sums(r, M, ds * y[c]))
            dY[h // share] = dY[h // share] + s["scale"] * _sums(c, K, ds * x[r])
            dH[h // share] = dH[h // share] + _sums(c, K, w[:, None] * g[r])
            if "bucket" in s:
                got["dTable"].append(_sums(bucket, s["table"].shape[1], ds)[:, 0])
    if case["op"] == "forward":
        return {"out": torch.stack(got["out"], 1), "lse": torch.stack(got["lse"])}
    both = {"dX": torch.stack(got["dX"], 1), "dY": torch.stack(dY, 1), "dH": torch.stack(dH, 1)}
    if "bucket" in s:
        both["dTable"] = torch.stack(got["dTable"])
    return both


# ------------------------------------------------------------------------- what a pass cannot do without
def work(case):
    M, K = _shape(case)
    row, col = _pattern(case, 0, "cuda" if torch.cuda.is_available() else "cpu")
    nnz, heads, op = row.numel(), case["heads"], case["op"]
    if op in ("forward", "backward"):
        kv, d, N = case["kv_heads"], case["d"], case["N"]
        seen = torch.unique(col).numel()  # rows of Y and H that are read
        pattern, queries, keys = 4 * (nnz + M + 1), 2 * M * heads, 2 * seen * kv
        if op == "forward":  # X read, out and lse written
            return {"bytes": pattern + queries * (d + N) + 4 * M * heads + keys * (d + N), "flops": 2 * nnz * heads * (d + N)}
        # X, out, dOut and lse read, dX written; Y and H read, their gradients written
        return {"bytes": 2 * pattern + queries * (2 * d + 2 * N) + 4 * M * heads + keys * (d + N) + 2 * K * kv * (d + N),
                "flops": 2 * nnz * heads * (3 * d + 2 * N)}
    nvec = torch.unique((row >> 3) * K + col).numel()
    values = 16 * nvec * heads
    return {"bytes": 5 * nvec + values * (1 if op == "bias_grad" else 2), "flops": 2 * nnz * heads}
