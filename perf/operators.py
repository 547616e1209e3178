"""The operators on 8-bit rows by which their speed is judged: what a GNN program does with a table of
features, layer inputs or past embeddings that it keeps as int8 codes with one fp32 scale per row.

Definitions.  A row x of F numbers is held as
    scale = fp32(max|x| / 127),   code_c = x_c / scale rounded to nearest, ties to even,
and stands for the values scale * code_c.  The codes of N rows are an int8 matrix whose row stride is F
rounded up to 16.  sample_W keeps k = min(n, W) of the n entries of each row of a CSR matrix: the first k
("bucket"), entry (off + i * P) mod n for i < k ("fastrand", n > W: P is the first of 577, 587, 593, 599 that
does not divide n, off the high half of SplitMix64(seed)'s output number r + 1 mod n, or 0 for seed 0), or all
("full").  A row's factor f is 1, 1 / k ("mean") or 1 / n ("inv_degree").

A case's "op":
  store        es_q8_write of rows of X, then es_q8_read: of all rows (a checkpoint of a layer's input, taken in
               the forward pass and read back in the backward pass), or written at `n` ids and read at `m` (a table
               of past embeddings: a batch's nodes are pushed, their neighbours pulled)
  spmm         es_spmm_q8: Y[i] = f * sum over the kept entries of row rows[i] of value * scale_c * code_c
  edge_grad    es_spmm_q8_backward_vals: the gradient of that product with respect to the entries' values
  weight_grad  es_q8_weight_grad: dW = (scale * codes)^T G, the gradient of a dense layer's weight
Graphs are those of perf/cases.py, smaller in code; everything is made on the GPU from the seed.
"""
import math

import numpy as np
import torch

own = False

_TYPES = {"fp32": torch.float32, "fp16": torch.float16, "bf16": torch.bfloat16}
_EXPONENT = 2.1


# ---- the cases --------------------------------------------------------------------------------
def _store(name, N, F, type, n=0, m=0):
    return dict(name=name, op="store", N=N, F=F, type=type, n=n, m=m)


def _graph_case(name, op, N, mean, dmax, F, mode, W, seed, values, norm, targets=0, clustered=False):
    return dict(name=name, op=op, N=N, mean=float(mean), dmax=dmax, F=F, mode=mode, W=W, rotation=seed, values=values,
                norm=norm, targets=targets, clustered=clustered)


def _weight_grad(name, N, F, out):
    return dict(name=name, op="weight_grad", N=N, F=F, out=out)


def listed():
    return [
        # one small batch in serving: 64 nodes' embeddings pushed, some thousand neighbours' pulled; launches count
        _store("push_64_pull_1024_f128", 170_000, 128, "fp32", 64, 1024),
        # a training batch on a table of raw features of 602 columns, in bf16
        _store("push_16k_pull_64k_f602_bf16", 233_000, 602, "bf16", 16_384, 65_536),
        # the last layer's input on the dense graph, 41 classes: rows that tile no line
        _store("checkpoint_233k_f41", 233_000, 41, "fp32"),
        # a hidden layer's input on the largest graph: the checkpoint that 8 bits are wanted for
        _store("checkpoint_2450k_f128", 2_450_000, 128, "fp32"),
        # serving: the exact aggregation of 32 asked nodes of the dense graph, latency
        _graph_case("serve_32_exact_f64", "spmm", 233_000, 490, 21_000, 64, "full", 0, 0, "mean", "none", targets=32),
        # exact inference on a citation graph, hubs of thousands of entries among rows of ten, 100 columns
        _graph_case("citation_exact_f100", "spmm", 170_000, 14, 13_000, 100, "full", 0, 0, "sym", "none"),
        # the sampled products the method is made for: short kept rows on the dense graph, unweighted mean
        _graph_case("social_bucket_w64_f64", "spmm", 233_000, 490, 21_000, 64, "bucket", 64, 0, "unit", "mean"),
        # and on the largest graph, a table of 314 MB, with a rotation per row
        _graph_case("copurchase_fastrand_w64_f128", "spmm", 2_450_000, 50, 20_000, 128, "fastrand", 64, 11, "sym", "none",
                    clustered=True),
        # learned edge values on the citation graph
        _graph_case("citation_edge_grad_bucket_w16_f128", "edge_grad", 170_000, 14, 13_000, 128, "bucket", 16, 0, "sym",
                    "none"),
        # the same on the dense graph, 41 columns, a seed of its own per step: most entries' gradients are zeros
        _graph_case("social_edge_grad_fastrand_w64_f41", "edge_grad", 233_000, 490, 21_000, 41, "fastrand", 64, 7, "mean",
                    "mean"),
        # first layer's weight on the dense graph: 602 features to 256
        _weight_grad("weight_grad_233k_602x256", 233_000, 602, 256),
        # a hidden layer's on the largest graph
        _weight_grad("weight_grad_2450k_128x128", 2_450_000, 128, 128),
    ]


def draw(rng):
    """One more case of the same ranges."""
    def log_uniform(lo, hi):
        return math.exp(rng.uniform(math.log(lo), math.log(hi)))

    while True:
        op = rng.choice(["store", "store", "spmm", "spmm", "spmm", "edge_grad", "weight_grad"])
        N = int(log_uniform(2_700, 2_450_000))
        F = int(log_uniform(8, 640))
        if rng.random() < 0.4:
            F = (F + 15) // 16 * 16
        if op == "store":
            kind = rng.choice(["fp32", "fp32", "fp16", "bf16"])
            c = _store("", N, F, kind)
            if rng.random() < 0.5:
                c["n"] = int(log_uniform(1, min(N, 100_000)))
                c["m"] = min(16 * c["n"], int(log_uniform(1, 400_000)))
            if max(N, c["m"]) * F > 2_450_000 * 128:
                continue
        elif op == "weight_grad":
            c = _weight_grad("", N, F, int(log_uniform(8, 256)))
            if N * (F + 4 * c["out"]) > 2_450_000 * 640 or N * F * c["out"] > 2_450_000 * 128 * 128:
                continue
        else:
            mean = round(log_uniform(4.5, 490), 1)
            dmax = max(16, int(min(N // 8, mean * log_uniform(40, 900), 21_000)))
            if dmax < 3 * mean or N * mean > 120.0e6:
                continue
            mode = rng.choice(["full", "bucket", "fastrand", "fastrand"])
            values, norm = rng.choice([("sym", "none"), ("mean", "none"), ("unit", "mean"), ("unit", "inv_degree")])
            c = _graph_case("", op, N, mean, dmax, F, mode, 0 if mode == "full" else int(log_uniform(4, 256)),
                            rng.choice([0, rng.randrange(1, 1 << 40)]), values, norm,
                            clustered=rng.random() < 0.4)
            if op == "spmm" and rng.random() < 0.3:
                c["targets"] = int(log_uniform(1, 4096))
            elif _entries(c)[1] * F > 2_450_000 * 20 * 128:
                continue
        del c["name"]
        return c


# ---- sizes, without building the graph --------------------------------------------------------
def _capped_mean(dmin, cap):
    """Mean of min(d, cap) for density ~ d**-2.1 from dmin on."""
    a = _EXPONENT - 1.0
    if cap <= dmin:
        return cap
    return dmin * a / (a - 1.0) - dmin ** a * cap ** (1.0 - a) / (a - 1.0)


def _dmin(mean, dmax):
    """Lower end of the degree law that gives `mean` (floor allowed for)."""
    lo, hi = 0.05, float(dmax)
    for _ in range(80):
        mid = 0.5 * (lo + hi)
        lo, hi = (mid, hi) if _capped_mean(mid, dmax) < mean + 0.5 else (lo, mid)
    return hi


def _entries(case):
    """(stored, kept) entries of the asked rows, to within a few percent."""
    rows = case["targets"] or case["N"]
    stored = rows * case["mean"]
    if case["mode"] == "full":
        return stored, stored
    return stored, min(stored, rows * _capped_mean(_dmin(case["mean"], case["dmax"]), case["W"]))


def work(case):
    N, F = case["N"], case["F"]
    row = (F + 15) // 16 * 16 + 4                              # a row's codes and its scale
    if case["op"] == "store":
        b = _TYPES[case["type"]].itemsize
        n, m = case["n"] or N, case["m"] or N
        return {"bytes": float(n * (F * b + row) + m * (F * b + row)), "flops": 2.0 * n * F + m * F}
    if case["op"] == "weight_grad":
        return {"bytes": float(N * (row + 4 * case["out"]) + 4 * F * case["out"]), "flops": 2.0 * N * F * case["out"]}
    stored, kept = _entries(case)
    rows = case["targets"] or N
    entry = 4 if case["values"] == "unit" or case["op"] == "edge_grad" else 8
    out = 4.0 * stored if case["op"] == "edge_grad" else 0.0   # its dense operand is read, the product's written
    return {"bytes": 4.0 * rows + entry * kept + min(float(N), kept) * row + 4.0 * rows * F + out, "flops": 2.0 * kept * F}


# ---- inputs -----------------------------------------------------------------------------------
def _graph(case, gen, dev):
    N, dmax = case["N"], case["dmax"]
    dmin = _dmin(case["mean"], dmax)
    # the law's N quantiles in random order: every seed has another graph of the same size
    u = (torch.randperm(N, device=dev, generator=gen).double() + 0.5) / N
    deg = (dmin * (1.0 - u).pow(-1.0 / (_EXPONENT - 1.0))).floor().clamp(1, dmax).long()
    rowptr = torch.zeros(N + 1, dtype=torch.int64, device=dev)
    rowptr[1:] = deg.cumsum(0)
    nnz = int(rowptr[-1])
    rows = torch.repeat_interleave(torch.arange(N, device=dev), deg)
    cols = torch.randint(N, (nnz,), device=dev, generator=gen)
    if case["clustered"]:                                      # 64 blocks of ids, 80 % of the entries inside their own
        size = -(-N // 64)
        start = rows // size * size
        near = start + (torch.rand(nnz, device=dev, generator=gen) * (N - start).clamp(max=size)).long()
        cols = torch.where(torch.rand(nnz, device=dev, generator=gen) < 0.8, near.clamp(max=N - 1), cols)
    cols = (rows * N + cols).sort().values - rows * N          # in increasing order inside each row
    vals = None
    if case["values"] == "sym":
        vals = (deg.double().rsqrt()[rows] * deg.double().rsqrt()[cols]).float()
    elif case["values"] == "mean":
        vals = deg.double().reciprocal()[rows].float()
    return rowptr.int(), cols.int(), vals


def _activations(n, F, gen, dev):
    """Layer inputs: rows of different size, every second number cut off by a relu, some rows all zero."""
    x = torch.randn((n, F), device=dev, generator=gen).clamp_(min=0)
    size = torch.randn((n, 1), device=dev, generator=gen).exp_()
    return x.mul_(size * (torch.rand((n, 1), device=dev, generator=gen) > 0.01))


def _quantise(x):
    """(codes, scale) of the rows of x; quotients in 64 bits, so that what lies next to a border is decided exactly."""
    scale = (x.abs().amax(1).double() / 127.0).float()
    q = (x.double() / scale.double().clamp(min=1e-38)[:, None]).round_().to(torch.int8)
    return q, scale


def _empty_table(N, F, dev):
    return (torch.zeros((N, (F + 15) // 16 * 16), dtype=torch.int8, device=dev), torch.zeros(N, device=dev))


def prepare(case, seed):
    dev = torch.device("cuda")
    gen = torch.Generator(device=dev)
    gen.manual_seed(int(seed) * 1_000_003 + 17)
    N, F = case["N"], case["F"]
    s = {"case": case}
    if case["op"] == "store":
        kind = _TYPES[case["type"]]
        n, m = case["n"] or N, case["m"] or N
        s["X"] = _activations(n, F, gen, dev).to(kind)
        s["codes"], s["scale"] = _empty_table(N, F, dev)
        s["Y"] = torch.zeros((m, F), dtype=kind, device=dev)
        s["push"] = s["pull"] = None
        if case["n"]:
            s["push"] = torch.randperm(N, device=dev, generator=gen)[:n].int()
            pull = torch.randint(N, (m,), device=dev, generator=gen).int()
            near = torch.randint(n, (m,), device=dev, generator=gen)
            s["pull"] = torch.where(torch.rand(m, device=dev, generator=gen) < 0.5, s["push"][near], pull)
            # what earlier batches left in the table
            q, s["scale"][:] = _quantise(_activations(N, F, gen, dev))
            s["codes"][:, :F] = q
        return s
    x = _activations(N, F, gen, dev)
    if case["op"] == "spmm" and not case["targets"]:
        x -= 0.3                                               # features that have both signs
    s["codes"], s["scale"] = _empty_table(N, F, dev)
    q, s["scale"] = _quantise(x)
    s["codes"][:, :F] = q
    del x, q
    if case["op"] == "weight_grad":
        s["G"] = torch.randn((N, case["out"]), device=dev, generator=gen) / math.sqrt(N)
        s["dW"] = torch.zeros((F, case["out"]), device=dev)
        return s
    s["rowptr"], s["colidx"], s["vals"] = _graph(case, gen, dev)
    s["rows"] = None
    if case["op"] == "edge_grad":
        s["dY"] = torch.randn((N, F), device=dev, generator=gen)
        s["dvals"] = torch.zeros(s["colidx"].numel(), device=dev)
        return s
    if case["targets"]:
        s["rows"] = torch.randint(N, (case["targets"],), device=dev, generator=gen).int()
    s["Y"] = torch.zeros((case["targets"] or N, F), device=dev)
    return s


# ---- the plain forms --------------------------------------------------------------------------
def _srl(z, bits):
    """Logical shift of a 64-bit pattern held in int64."""
    return (z >> bits) & ((1 << (64 - bits)) - 1)


def _signed(v):
    return v - (1 << 64) if v >= 1 << 63 else v


def _kept(s):
    """(place of each kept entry's row among the asked ones, its position in colidx, the rows' n and k)."""
    c = s["case"]
    start = s["rowptr"].long()
    rows = torch.arange(c["N"], device=start.device) if s["rows"] is None else s["rows"].long()
    first = start[rows]
    n = start[rows + 1] - first
    k = n if c["mode"] == "full" else n.clamp(max=c["W"])
    at = torch.repeat_interleave(torch.arange(rows.numel(), device=start.device), k)
    slot = torch.arange(at.numel(), device=start.device) - (k.cumsum(0) - k)[at]
    if c["mode"] == "fastrand":
        P = torch.where(n % 577 != 0, 577, torch.where(n % 587 != 0, 587, torch.where(n % 593 != 0, 593, 599)))
        off = torch.zeros_like(n)
        if c["rotation"]:
            z = (rows + 1) * _signed(0x9E3779B97F4A7C15) + _signed(c["rotation"])
            z = (z ^ _srl(z, 30)) * _signed(0xBF58476D1CE4E5B9)
            z = (z ^ _srl(z, 27)) * _signed(0x94D049BB133111EB)
            off = _srl(z ^ _srl(z, 31), 32) % n.clamp(min=1)
        entry = (off[at] + slot * P[at]) % n[at]
        slot = torch.where((n > c["W"])[at], entry, slot)
    return at, first[at] + slot, n, k


def _factor(norm, n, k):
    if norm == "mean":
        return torch.where(k > 0, 1.0 / k.clamp(min=1).float(), 0.0)
    if norm == "inv_degree":
        return torch.where(k > 0, 1.0 / n.clamp(min=1).float(), 0.0)
    return torch.ones(n.numel(), device=n.device)


def _plain(s):
    c = s["case"]
    F = c["F"]
    if c["op"] == "store":
        q, scale = _quantise(s["X"].float())
        if s["push"] is None:
            s["codes"][:, :F], s["scale"][:] = q, scale
            s["Y"][:] = s["codes"][:, :F].float() * s["scale"][:, None]
        else:
            s["codes"][:, :F].index_copy_(0, s["push"].long(), q)
            s["scale"].index_copy_(0, s["push"].long(), scale)
            pull = s["pull"].long()
            s["Y"][:] = s["codes"][pull, :F].float() * s["scale"][pull][:, None]
        return s["Y"]
    if c["op"] == "weight_grad":
        s["dW"][:] = (s["codes"][:, :F].float() * s["scale"][:, None]).t() @ s["G"]
        return s["dW"]
    at, p, n, k = _kept(s)
    col = s["colidx"][p].long()
    f = _factor(c["norm"], n, k)
    if c["op"] == "edge_grad":
        dot = (s["codes"][col, :F].float() * s["dY"][at]).sum(1)
        s["dvals"].zero_()
        s["dvals"][p] = dot * s["scale"][col] * f[at]
        return s["dvals"]
    w = s["scale"][col] if s["vals"] is None else s["scale"][col] * s["vals"][p]
    s["Y"].zero_().index_add_(0, at, s["codes"][col, :F].float().mul_(w[:, None]))
    s["Y"].mul_(f[:, None])
    return s["Y"]


def run(state):
    if not own:
        return _plain(state)
    import paper_2104_10716_amd as es
    s, c = state, state["case"]
    if c["op"] == "store":
        es.es_q8_write(s["X"], s["codes"], s["scale"], rows=s["push"])
        return es.es_q8_read(s["codes"], s["scale"], s["Y"], rows=s["pull"])
    if c["op"] == "weight_grad":
        return es.es_q8_weight_grad(s["codes"], s["scale"], s["G"], s["dW"])
    if c["op"] == "edge_grad":
        return es.es_spmm_q8_backward_vals(s["rowptr"], s["colidx"], s["dY"], s["codes"], s["scale"], s["dvals"], c["W"],
                                           c["mode"], c["rotation"], c["norm"])
    return es.es_spmm_q8(s["rowptr"], s["colidx"], s["vals"], s["codes"], s["scale"], s["Y"], c["W"], c["mode"],
                         c["rotation"], c["norm"], rows=s["rows"])


# ---- the definitions in 64 bits ---------------------------------------------------------------
def _splitmix_high(seed, count):
    """High halves of SplitMix64's outputs number `count` (unsigned, so that products wrap by themselves)."""
    with np.errstate(over="ignore"):
        z = np.uint64(seed) + count.astype(np.uint64) * np.uint64(0x9E3779B97F4A7C15)
        z = (z ^ (z >> np.uint64(30))) * np.uint64(0xBF58476D1CE4E5B9)
        z = (z ^ (z >> np.uint64(27))) * np.uint64(0x94D049BB133111EB)
        return ((z ^ (z >> np.uint64(31))) >> np.uint64(32)).astype(np.float64)


def _exact_entries(s, lo, hi):
    """Asked rows lo .. hi - 1: (row counted from lo, position, n, k) per kept entry, from a rectangle of slots."""
    c = s["case"]
    ptr = s["rowptr"].double()
    ids = torch.arange(lo, hi, device=ptr.device) if s["rows"] is None else s["rows"][lo:hi].long()
    begin = ptr[ids]
    n = ptr[ids + 1] - begin                                   # whole numbers, exact in 64 bits
    k = n if c["mode"] == "full" else n.clamp(max=float(c["W"]))
    width = int(k.max()) if k.numel() else 0
    slot = torch.arange(width, device=ptr.device, dtype=torch.float64)[None, :].expand(hi - lo, width)
    present = slot < k[:, None]
    if c["mode"] == "fastrand":
        P = torch.full_like(n, 599.0)
        for p in (593.0, 587.0, 577.0):
            P[torch.remainder(n, p) != 0] = p
        off = torch.zeros_like(n)
        if c["rotation"]:
            high = torch.from_numpy(_splitmix_high(c["rotation"], ids.cpu().numpy() + 1)).to(ptr.device)
            off = torch.remainder(high, n.clamp(min=1.0))
        entry = torch.remainder(off[:, None] + slot * P[:, None], n.clamp(min=1.0)[:, None])
        slot = torch.where((n > c["W"])[:, None], entry, slot)
    at = present.nonzero()[:, 0]
    pos = (begin[:, None] + slot)[present].long()
    return at, pos, n, k


def exact(case, seed):
    s = prepare(case, seed)
    F, op = case["F"], case["op"]
    table = lambda i: s["codes"][i, :F].double() * s["scale"][i].double()[:, None]  # noqa: E731
    if op == "store":
        x = s["X"].double()
        scale = (x.abs().max(1).values / 127.0).float().double()
        value = torch.where(scale[:, None] > 0, (x / scale[:, None]), torch.zeros_like(x)).round() * scale[:, None]
        if s["push"] is None:
            return value
        full = table(slice(None))
        full[s["push"].long()] = value
        return full[s["pull"].long()]
    if op == "weight_grad":
        out = torch.zeros((F, case["out"]), dtype=torch.float64, device=s["G"].device)
        for lo in range(0, case["N"], 262_144):
            i = slice(lo, lo + 262_144)
            out += table(i).t().contiguous() @ s["G"][i].double()
        return out
    rows = case["targets"] or case["N"]
    if op == "edge_grad":
        result = torch.zeros(s["colidx"].numel(), dtype=torch.float64, device=s["dY"].device)
    else:
        result = torch.zeros((rows, F), dtype=torch.float64, device=s["Y"].device)
    # rows per step: a rectangle of at most 2^27 slots, some 2^31 products
    longest = int((s["rowptr"][1:] - s["rowptr"][:-1]).max())
    width = longest if case["mode"] == "full" else min(longest, case["W"])
    step = max(1, min((1 << 27) // max(width, 1), (1 << 31) // max(1, int(F * max(4.0, min(width, case["mean"]))))))
    for lo in range(0, rows, step):
        hi = min(rows, lo + step)
        at, pos, n, k = _exact_entries(s, lo, hi)
        f = torch.ones_like(n)
        if case["norm"] == "mean":
            f = torch.where(k > 0, 1.0 / k, 0.0)
        elif case["norm"] == "inv_degree":
            f = torch.where(k > 0, 1.0 / n, 0.0)
        col = s["colidx"][pos].long()
        if op == "edge_grad":
            result[pos] = (table(col) * s["dY"][lo:hi][at].double()).sum(1) * f[at]
        else:
            value = f[at] if s["vals"] is None else f[at] * s["vals"][pos].double()
            result[lo:hi].index_add_(0, at, table(col) * value[:, None])
    return result
