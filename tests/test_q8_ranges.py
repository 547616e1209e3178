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
