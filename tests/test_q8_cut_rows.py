"""es_spmm_q8 where rows are longer than a wave should take alone: cut into pieces whose sums meet in the workspace, on
graphs whose rows have every length around the borders, with every kind of workspace.  Definitions and
tolerances are those of test_q8: a sum of k products is off by at most (k + 5) 2^-24 times the sum of their magnitudes."""
import numpy as np
import pytest

import paper_2104_10716_amd as es
from test_q8 import U, dev, filled, near

GUARD = 256


def spread_graph(N, mean, seed, most=2600):
    """Rows of lengths around the borders (0, 1, 1023 .. 1025, ..., 2049), the others at random with the given mean."""
    rng = np.random.default_rng(seed)
    deg = np.minimum(rng.gamma(0.7, mean / 0.7, N).astype(np.int64), min(most, N))
    edge = np.array([0, 1, 255, 256, 257, 1023, 1024, 1025, 1026, 1199, 1200, 1201, 1499, 1500, 1501, 1959, 1960, 1961, 2047, 2048,
                     2049, 2500])
    edge = edge[edge <= N]
    deg[rng.permutation(N)[:edge.size]] = edge
    rowptr = np.zeros(N + 1, dtype=np.int32)
    rowptr[1:] = np.cumsum(deg)
    return rowptr, rng.integers(0, N, rowptr[-1]).astype(np.int32)


def kept_mask(rowptr, nnz, W, mode, seed):
    import oracle
    if mode == "full":
        return np.ones(nnz, bool)
    keep = np.zeros(nnz, bool)
    pos, cnt = oracle.kept(rowptr, W, mode, seed)
    keep[pos[np.arange(pos.shape[1])[None, :] < cnt[:, None]]] = True
    return keep


def definition(rowptr, colidx, vals, v, W, mode, seed):
    """(Y, tolerance) in 64 bits of all rows, and what each keeps."""
    from scipy.sparse import csr_matrix
    N = rowptr.size - 1
    keep = kept_mask(rowptr, colidx.size, W, mode, seed)
    k = np.add.reduceat(np.concatenate([keep, [False]]).astype(np.int64), rowptr[:-1]) * (np.diff(rowptr) > 0)
    A = csr_matrix((np.where(keep, vals, 0).astype(np.float64), colidx, rowptr), shape=(N, N))
    B = csr_matrix((np.abs(A.data), colidx, rowptr), shape=(N, N))
    return A @ v, (B @ np.abs(v)) * ((k + 5) * U)[:, None], k


def workspaces(N, nnz, F, W, mode, n_rows):
    """(name, workspace) of every kind: the library's own, one of the asked size full of NaN with a guard
    behind it, one full of zeros, one byte too few, none at all."""
    import torch
    need = es.es_spmm_q8_workspace_bytes(N, nnz, F, W, mode, n_rows)
    yield "lent", None
    for name, byte in (("NaN", 255), ("zeros", 0)):            # 0xFFFFFFFF is a NaN
        w = torch.full((need + GUARD,), byte, dtype=torch.uint8, device="cuda:0")
        w[need:] = 201
        yield name, w
    if need:
        yield "too small", torch.full((need - 1,), 255, dtype=torch.uint8, device="cuda:0")
    yield "empty", torch.empty(0, dtype=torch.uint8, device="cuda:0")


def check_every_workspace(graph, codes, scale, F, W, mode, seed, rows, want, tol, what):
    import torch
    N, nnz = graph[0].numel() - 1, graph[1].numel()
    n = N if rows is None else rows.numel()
    need = es.es_spmm_q8_workspace_bytes(N, nnz, F, W, mode, n)
    seen = {}
    for name, w in workspaces(N, nnz, F, W, mode, n):
        Y = torch.full((n, F), float("nan"), device="cuda:0")
        es.es_spmm_q8(*graph, codes, scale, Y, W, mode, seed, rows=rows, workspace=w)
        near(Y.cpu().numpy(), want, tol, f"{what} {mode} {W} {name}")
        if name in ("NaN", "zeros"):
            assert bool((w[need:] == 201).all()), (what, name)     # nothing behind what it asked for
        seen[name] = Y
    assert torch.equal(seen["lent"], seen["NaN"]) and torch.equal(seen["lent"], seen["zeros"])


@pytest.mark.gpu
@pytest.mark.parametrize("N,mean,F", [(10_000, 490, 64), (20_000, 300, 64), (12_000, 300, 100), (4000, 350, 16), (2000, 600, 300),
                                      (1500, 500, 602), (1500, 500, 1040), (700, 300, 2304)])
def test_rows_between_a_wave_and_a_piece(N, mean, F):
    """Small dense graphs, on which a wave takes rows of up to four times the mean alone."""
    rowptr, colidx = spread_graph(N, mean, N + F, 5 * mean)
    rng = np.random.default_rng(F)
    vals = rng.standard_normal(colidx.size).astype(np.float32)
    codes, scale, q, s, v = filled(rng.standard_normal((N, F)).astype(np.float32))
    graph = dev(rowptr), dev(colidx), dev(vals)
    ids = rng.integers(-2, N + 2, 2000).astype(np.int32)
    ids[:1000] = np.argsort(-np.diff(rowptr), kind="stable")[rng.integers(0, min(N, 400), 1000)]      # long ones, many times
    inside = (ids >= 0) & (ids < N)
    at = np.where(inside, ids, 0)
    for mode, W, seed in (("full", 0, 0), ("fastrand", 1500, 3), ("bucket", 1500, 0), ("bucket", 1100, 0), ("fastrand", 1024, 0)):
        want, tol, k = definition(rowptr, colidx, vals, v, W, mode, seed)
        assert k.max() > 1024 or W == 1024 or F == 2304
        check_every_workspace(graph, codes, scale, F, W, mode, seed, None, want, tol, "all rows")
        check_every_workspace(graph, codes, scale, F, W, mode, seed, dev(ids), np.where(inside[:, None], want[at], 0),
                              np.where(inside[:, None], tol[at], 0), "2000 rows")


@pytest.mark.gpu
@pytest.mark.parametrize("F", [64, 300, 602, 1040])
def test_cut_rows_of_several_blocks_of_columns(F):
    """Hubs above the shortest piece in a sparse graph, rows of one to five blocks of columns."""
    N = 6000
    rowptr, colidx = spread_graph(N, 8, F)
    rng = np.random.default_rng(F)
    vals = rng.standard_normal(colidx.size).astype(np.float32)
    codes, scale, q, s, v = filled(rng.standard_normal((N, F)).astype(np.float32))
    graph = dev(rowptr), dev(colidx), dev(vals)
    for mode, W, seed in (("full", 0, 0), ("fastrand", 2040, 8), ("bucket", 1025, 0)):
        want, tol, k = definition(rowptr, colidx, vals, v, W, mode, seed)
        check_every_workspace(graph, codes, scale, F, W, mode, seed, None, want, tol, f"F={F}")


@pytest.mark.gpu
@pytest.mark.parametrize("F", [1, 8, 64, 100, 300])
@pytest.mark.parametrize("n", [1, 7, 512])
def test_few_asked_rows_with_every_workspace(n, F):
    N = 5000
    rowptr, colidx = spread_graph(N, 60, n)
    rng = np.random.default_rng(n + F)
    vals = rng.standard_normal(colidx.size).astype(np.float32)
    codes, scale, q, s, v = filled(rng.standard_normal((N, F)).astype(np.float32))
    graph = dev(rowptr), dev(colidx), dev(vals)
    longest = np.argsort(-np.diff(rowptr), kind="stable")
    ids = np.where(rng.random(n) < 0.5, longest[rng.integers(0, 30, n)], rng.integers(-2, N + 2, n)).astype(np.int32)
    ids[0] = longest[0]
    inside = (ids >= 0) & (ids < N)
    at = np.where(inside, ids, 0)
    for mode, W, seed in (("full", 0, 0), ("fastrand", 1500, 3), ("bucket", 129, 0), ("bucket", 128, 0)):
        want, tol, k = definition(rowptr, colidx, vals, v, W, mode, seed)
        check_every_workspace(graph, codes, scale, F, W, mode, seed, dev(ids), np.where(inside[:, None], want[at], 0),
                              np.where(inside[:, None], tol[at], 0), f"n={n} F={F}")


@pytest.mark.gpu
def test_wide_rows_whose_time_moves_the_border():
    """2304 columns on 200 k rows: by the time that the launch takes, a wave may have rows of more than a thousand
    entries.  The rows around that border, and others, against their definition in 64 bits on the device."""
    import torch
    N, F = 200_000, 2304
    rng = np.random.default_rng(1)
    deg = rng.integers(30, 50, N)
    hubs = rng.permutation(N)[:300]
    deg[hubs] = rng.integers(1000, 1300, 300)
    deg[hubs[:8]] = (1023, 1024, 1025, 1026, 1111, 1112, 1113, 2600)
    rowptr = np.zeros(N + 1, dtype=np.int32)
    rowptr[1:] = np.cumsum(deg)
    colidx = rng.integers(0, N, rowptr[-1]).astype(np.int32)
    vals = rng.standard_normal(colidx.size).astype(np.float32)
    gen = torch.Generator(device="cuda:0").manual_seed(5)
    codes = torch.randint(-127, 128, (N, F), device="cuda:0", generator=gen, dtype=torch.int8)
    scale = torch.rand(N, device="cuda:0", generator=gen) + 0.25
    graph = dev(rowptr), dev(colidx), dev(vals)
    need = es.es_spmm_q8_workspace_bytes(N, colidx.size, F, 0, "full", N)
    w = torch.full((need + GUARD,), 255, dtype=torch.uint8, device="cuda:0")
    Y = torch.full((N, F), float("nan"), device="cuda:0")
    es.es_spmm_q8(*graph, codes, scale, Y, 0, "full", workspace=w)
    assert not bool(Y.isnan().any())
    for r in np.concatenate([hubs[:60], rng.integers(0, N, 40)]):
        e = slice(int(rowptr[r]), int(rowptr[r + 1]))
        c = graph[1][e].long()
        x = codes[c].double() * scale[c].double()[:, None] * graph[2][e].double()[:, None]
        near(Y[r].cpu().numpy(), x.sum(0).cpu().numpy(), x.abs().sum(0).cpu().numpy() * (deg[r] + 5) * U, f"row {r} of {deg[r]}")


@pytest.mark.gpu
def test_a_row_of_all_entries_that_there_can_be():
    """2^31 - 1 entries, all of one row: counts past the last one do not fit 31 bits.  Every entry but a handful names a row
    of zeros, so the sums are exact."""
    import torch
    n, F = 2 ** 31 - 1, 16
    colidx = torch.zeros(n, dtype=torch.int32, device="cuda:0")            # 8.6 GB
    named = [0, 1023, 2 ** 30, n - 1025, n - 1024, n - 2, n - 1]
    colidx[torch.tensor(named, device="cuda:0")] = 1
    rowptr = torch.tensor([0, 0, n], dtype=torch.int32, device="cuda:0")
    codes = torch.tensor([[0] * F, list(range(-8, 8))], dtype=torch.int8, device="cuda:0")
    scale = torch.tensor([1.0, 0.5], device="cuda:0")
    want = codes[1].float() * (0.5 * len(named))
    none = torch.empty(0, dtype=torch.uint8, device="cuda:0")
    # one workgroup takes the row; 64 share it; every entry but one, in another order
    for mode, W, workspace in (("full", 0, none), ("full", 0, None), ("fastrand", n - 1, None)):
        Y = torch.full((2, F), float("nan"), device="cuda:0")
        es.es_spmm_q8(rowptr, colidx, None, codes, scale, Y, W, mode, workspace=workspace)
        torch.cuda.synchronize()
        assert bool((Y[0] == 0).all()) and torch.equal(Y[1], want), (mode, Y)
    dY = torch.ones((2, F), device="cuda:0")
    dvals = torch.full((n,), 7.0, device="cuda:0")
    each = float(codes[1].float().sum() * 0.5)
    for mode, W in (("full", 0), ("bucket", n - 1), ("fastrand", n - 1)):
        es.es_spmm_q8_backward_vals(rowptr, colidx, dY, codes, scale, dvals, W, mode)
        left = {"full": -1, "bucket": n - 1, "fastrand": (n - 1) * 577 % n}[mode]
        for p in named:
            assert float(dvals[p]) == (0.0 if p == left else each), (mode, p)
        assert int(torch.count_nonzero(dvals)) == len(named) - (left in named), mode
        dvals.fill_(7.0)
