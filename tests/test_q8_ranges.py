"""The operators on 8-bit rows at the ends of what they take."""
import pytest

import paper_2104_10716_amd as es


@pytest.mark.gpu
@pytest.mark.parametrize("kind", ["float32", "float16"])
def test_more_rows_than_one_launch_takes(kind):
    """2^24 rows and more: whole tables and lists of ids go in several launches.  Rows of whole numbers with a largest one of
    127 2^e, so that what is read back is what was written, bit for bit."""
    import torch
    N, F = 2 ** 24 + 1000, 5
    r = torch.arange(N, device="cuda:0")
    X = torch.stack([torch.full_like(r, 127), r % 127, -(r % 91), r % 3, r % 128 - 64], 1).float()
    X = (X * torch.exp2((r % 7 - 4).float())[:, None]).to(getattr(torch, kind))
    codes = torch.full((N, 32), 77, dtype=torch.int8, device="cuda:0")
    scale = torch.full((N,), 0.25, device="cuda:0")
    es.es_q8_write(X, codes, scale)
    assert torch.equal(scale, torch.exp2((r % 7 - 4).float()))
    assert bool((codes[:, 5:16] == 0).all()) and bool((codes[:, 16:] == 77).all())
    Y = torch.full((N, F + 1), 3.0, device="cuda:0", dtype=X.dtype)
    assert torch.equal(es.es_q8_read(codes, scale, Y[:, :F]), X) and bool((Y[:, F] == 3.0).all())
    # the same rows backwards: read at ids, then written at ids
    ids = torch.arange(N - 1, -1, -1, dtype=torch.int32, device="cuda:0")
    assert torch.equal(es.es_q8_read(codes, scale, Y[:, :F], rows=ids), X.flip(0))
    es.es_q8_write(X, codes, scale, rows=ids)
    assert torch.equal(es.es_q8_read(codes, scale, Y[:, :F]), X.flip(0))


def test_sizes_beyond_the_abi_are_not_cut_to_their_low_bits():
    assert [es.es_q8_row_bytes(F) for F in (2 ** 32 + 16, 2 ** 64 + 16, -2 ** 32 + 16)] == [0, 0, 0]
    ask = es.es_spmm_q8_workspace_bytes
    assert ask(170_000, 2_400_000, 100, 0, "full", 170_000) > 0
    for bad in ((2 ** 64 + 170_000, 2_400_000, 100, 0, "full", 170_000), (170_000, 2 ** 64 + 2_400_000, 100, 0, "full", 170_000),
                (170_000, 2_400_000, 2 ** 32 + 100, 0, "full", 170_000), (170_000, 2_400_000, 100, 5000, 2 ** 32, 170_000),
                (170_000, 2_400_000, 100, 0, "full", 2 ** 64 + 170_000), (170_000, 2_400_000, 100, -2 ** 32 + 5000, "bucket", 170_000)):
        assert ask(*bad) == 0, bad
    # a sample that is wider than any row can be is every row
    assert ask(170_000, 2_400_000, 100, 2 ** 32 + 4, "bucket", 170_000) == ask(170_000, 2_400_000, 100, 2 ** 31 - 1, "bucket", 170_000) > 0
    ask = es.es_q8_weight_grad_workspace_bytes
    assert ask(1_000_000, 128, 128) > 0
    assert ask(2 ** 64 + 1_000_000, 128, 128) == ask(1_000_000, 2 ** 32 + 128, 128) == ask(1_000_000, 128, 2 ** 32 + 128) == 0


@pytest.mark.gpu
def test_arguments_beyond_the_abi_are_not_cut_to_their_low_bits():
    import torch
    d = "cuda:0"
    rowptr = torch.tensor([0, 3, 9, 9], dtype=torch.int32, device=d)
    colidx = torch.tensor([0, 1, 2, 0, 1, 2, 2, 1, 0], dtype=torch.int32, device=d)
    codes = torch.arange(-24, 24, dtype=torch.int8, device=d).reshape(3, 16)
    scale = torch.tensor([1.0, 0.5, 2.0], device=d)
    dY = torch.arange(48, dtype=torch.float32, device=d).reshape(3, 16)
    new = lambda: torch.full((3, 16), 5.0, device=d)  # noqa: E731
    want = es.es_spmm_q8(rowptr, colidx, None, codes, scale, new(), 0, "full")
    da = es.es_spmm_q8_backward_vals(rowptr, colidx, dY, codes, scale, torch.empty(9, device=d), 0, "full")
    for mode in ("bucket", "fastrand"):
        for W in (2 ** 31, 2 ** 32 + 1, 2 ** 64 + 2):
            assert torch.equal(es.es_spmm_q8(rowptr, colidx, None, codes, scale, new(), W, mode), want)
            assert torch.equal(es.es_spmm_q8_backward_vals(rowptr, colidx, dY, codes, scale, torch.full((9,), 5.0, device=d), W, mode), da)
    for W, mode, norm in ((4, 2 ** 32 + 1, "none"), (4, "bucket", 2 ** 32), (-2 ** 32 + 4, "bucket", "none")):
        Y = new()
        with pytest.raises(es.EsSpmmError):
            es.es_spmm_q8(rowptr, colidx, None, codes, scale, Y, W, mode, 0, norm)
        with pytest.raises(es.EsSpmmError):
            es.es_spmm_q8_backward_vals(rowptr, colidx, dY, codes, scale, torch.empty(9, device=d), W, mode, 0, norm)
        assert bool((Y == 5.0).all())


@pytest.mark.gpu
@pytest.mark.parametrize("exponent", [-95, -105, -110, -111, -118, -126, -130, -140])
def test_weight_gradient_of_very_small_numbers(exponent):
    """scale * G goes to the matrix cores as three bf16 numbers, whose last place is 2^-133: what is below it is lost, at
    most |code| 2^-133 per product, beside the roundings of any other sum (three per row).  From 2^-110 on nothing is below it."""
    import numpy as np
    import torch
    N, F, H = 200, 40, 70
    rng = np.random.default_rng(-exponent)
    q = rng.integers(-127, 128, (N, F)).astype(np.int8)
    s = np.exp2(rng.integers(-3, 4, N)).astype(np.float32)
    g = (rng.uniform(1, 2, (N, H)) * np.exp2(exponent) / s[:, None]).astype(np.float32) * rng.choice([-1, 1], (N, H)).astype(np.float32)
    codes = torch.zeros((N, 48), dtype=torch.int8, device="cuda:0")
    codes[:, :F] = torch.from_numpy(q).cuda()
    dW = es.es_q8_weight_grad(codes, torch.from_numpy(s).cuda(), torch.from_numpy(g).cuda(), torch.empty((F, H), device="cuda:0"))
    x, y = q.astype(np.float64), g.astype(np.float64) * s.astype(np.float64)[:, None]
    tol = np.abs(x).T @ np.abs(y) * (3 * N + 8) * 2.0 ** -24 + (N + 1) * 2.0 ** -150
    if exponent < -110:
        tol += np.abs(x).sum(0)[:, None] * 2.0 ** -133
    err = np.abs(dW.cpu().numpy().astype(np.float64) - x.T @ y)
    assert (err <= 1.01 * tol).all(), (err / tol).max()
