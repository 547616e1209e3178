"""The operators on 8-bit rows (es_q8_write, es_q8_read, es_spmm_q8, es_spmm_q8_backward_vals,
es_q8_weight_grad) against their definitions in 64 bits, computed here with NumPy from the
oracle's sampled entries.

Tolerances, derived before the first run: u = 2^-24 is fp32's unit of rounding.  A sum of k
products in fp32, in any order, is off by at most (k + c) u times the sum of their magnitudes, where c counts
the other roundings: the weight a * scale (1), the row factor (at most 2: 1 / sqrt) and its product (1).
The codes and scales themselves, and the zeros of what is not kept, have to be equal."""
import ctypes

import numpy as np
import pytest

import paper_2104_10716_amd as es

U = 2.0 ** -24
FAKE = ctypes.c_void_p(0x1000)


# ---- the definitions --------------------------------------------------------------------------
def quantise(X):
    """(codes, scale, values in 64 bits) of fp32 rows; the quotient of two fp32 numbers of at most 127 is either a
    half-integer or 2^-25 and more away from one (relative), which 64 bits resolve."""
    X = np.asarray(X, dtype=np.float32)
    mag = np.abs(X).max(axis=1) if X.shape[1] else np.zeros(X.shape[0], np.float32)
    bad = ~np.isfinite(X).all(axis=1)
    scale = (np.where(bad, 0.0, mag).astype(np.float64) / 127.0).astype(np.float32)
    scale = np.minimum(scale, np.nextafter(np.float32(np.finfo(np.float32).max / 127.0), np.float32(0)))
    scale[mag < np.float32(127.0) * np.float32(2.0 ** -126)] = 0.0
    safe = np.where(scale > 0, scale, 1.0).astype(np.float64)
    X64 = np.where(bad[:, None] | (scale == 0)[:, None], 0.0, X).astype(np.float64)
    codes = np.rint(X64 / safe[:, None]).astype(np.int8)
    scale[bad] = np.nan
    return codes, scale, codes.astype(np.float64) * scale.astype(np.float64)[:, None]


def kept_lists(rowptr, W, mode, seed):
    """Kept CSR positions per row, in slot order."""
    import oracle
    if mode == "full":
        return [np.arange(rowptr[r], rowptr[r + 1]) for r in range(len(rowptr) - 1)]
    pos, cnt = oracle.kept(rowptr, W, mode, seed)
    return [pos[r, :cnt[r]].astype(np.int64) for r in range(len(cnt))]


def factors(rowptr, kept, norm):
    import oracle
    return np.array([oracle.row_factor(norm, int(rowptr[r + 1] - rowptr[r]), len(p)) for r, p in enumerate(kept)])


def product(rowptr, colidx, vals, value, W, mode, seed, norm):
    """(Y, tolerance) in 64 bits."""
    kept = kept_lists(rowptr, W, mode, seed)
    f = factors(rowptr, kept, norm)
    Y = np.zeros((len(kept), value.shape[1]))
    tol = np.zeros_like(Y)
    for r, p in enumerate(kept):
        a = np.ones(len(p)) if vals is None else vals[p].astype(np.float64)
        x = value[colidx[p]]
        Y[r] = f[r] * (a[:, None] * x).sum(0)
        tol[r] = abs(f[r]) * (np.abs(a)[:, None] * np.abs(x)).sum(0) * (len(p) + 5) * U
    return Y, tol


def edge_gradient(rowptr, colidx, dY, codes, scale, W, mode, seed, norm):
    kept = kept_lists(rowptr, W, mode, seed)
    f = factors(rowptr, kept, norm)
    out, tol = np.zeros(colidx.size), np.zeros(colidx.size)
    F = dY.shape[1]
    for r, p in enumerate(kept):
        c = colidx[p]
        s = np.abs(f[r]) * np.abs(scale[c].astype(np.float64))
        d, q = dY[r].astype(np.float64), codes[c].astype(np.float64)
        out[p] = s * (q * d).sum(1)
        tol[p] = s * (np.abs(q) * np.abs(d)).sum(1) * (F + 6) * U
    return out, tol


def near(got, want, tol, what):
    got = np.asarray(got, dtype=np.float64)
    assert got.shape == want.shape, (what, got.shape, want.shape)
    bad = ~(np.abs(got - want) <= 1.01 * tol)
    if bad.any():
        i = np.unravel_index(np.argmax(np.where(bad, np.abs(got - want) - tol, -1)), bad.shape)
        raise AssertionError(f"{what}: {int(bad.sum())} of {bad.size} off, worst at {i}: {got[i]!r} for {want[i]!r} +- {tol[i]!r}")


# ---- without a GPU ----------------------------------------------------------------------------
def test_row_bytes():
    assert [es.es_q8_row_bytes(F) for F in (1, 15, 16, 17, 41, 602, 2 ** 31 - 16)] == [16, 16, 16, 32, 48, 608, 2 ** 31 - 16]
    assert [es.es_q8_row_bytes(F) for F in (0, -1, 2 ** 31 - 15, 2 ** 31 - 1)] == [0, 0, 0, 0]


def test_refusals_answer_on_the_host():
    """Every refused call returns before any HIP call; the fake pointers are never dereferenced."""
    lib = es.load_library()
    odd = ctypes.c_void_p(0x1001)

    def write(X=FAKE, type=0, n=4, F=20, ldx=20, rows=None, N=4, codes=FAKE, ldq=32, scale=FAKE):
        return lib.es_q8_write(X, type, n, F, ldx, rows, N, codes, ldq, scale, None)

    def read(codes=FAKE, ldq=32, scale=FAKE, N=4, F=20, rows=None, n=4, Y=FAKE, type=0, ldy=20):
        return lib.es_q8_read(codes, ldq, scale, N, F, rows, n, Y, type, ldy, None)

    for call, dense in ((write, "X"), (read, "Y")):
        ld = "ld" + dense.lower()
        for bad in (dict(type=3), dict(type=-1), dict(n=-1), dict(n=5), dict(F=0), dict(F=33), {ld: 19}, dict(N=-1), dict(N=2 ** 31),
                    dict(ldq=24), dict(ldq=16), dict(codes=None), dict(scale=None), {dense: None}, {dense: odd},
                    {dense: odd, "type": 1}, dict(codes=ctypes.c_void_p(0x1008)), dict(scale=odd), dict(rows=odd),
                    dict(rows=FAKE, n=2 ** 31)):
            assert call(**bad) == -1, bad
        assert call(n=0, **{dense: None}) == 0
    assert write(rows=FAKE, N=0, n=3, codes=None, scale=None) == 0         # every id is outside an empty table

    def spmm(rowptr=FAKE, colidx=FAKE, codes=FAKE, ldq=32, scale=FAKE, Y=FAKE, N=4, nnz=9, F=20, ldy=20, W=2, mode=1, norm=0,
             rows=None, n=4, ws=None):
        return lib.es_spmm_q8(rowptr, colidx, None, codes, ldq, scale, Y, N, nnz, F, ldy, W, mode, 0, norm, rows, n, ws,
                              0, None)

    def grad(rowptr=FAKE, colidx=FAKE, dY=FAKE, codes=FAKE, ldq=32, scale=FAKE, dvals=FAKE, N=4, nnz=9, F=20, ldy=20, W=2,
             mode=1, norm=0):
        return lib.es_spmm_q8_backward_vals(rowptr, colidx, dY, ldy, codes, ldq, scale, dvals, N, nnz, F, W, mode, 0, norm, None)

    both = (dict(N=-1), dict(N=2 ** 31), dict(nnz=-1), dict(nnz=2 ** 31), dict(F=0), dict(F=33), dict(ldq=24), dict(ldq=16),
            dict(ldy=19), dict(W=0), dict(W=0, mode=2), dict(mode=3), dict(mode=-1), dict(norm=5), dict(norm=-1),
            dict(rowptr=None), dict(colidx=None), dict(codes=None), dict(scale=None), dict(codes=ctypes.c_void_p(0x1008)),
            dict(scale=odd))
    for bad in both + (dict(Y=None), dict(Y=odd), dict(n=3), dict(n=-1), dict(rows=FAKE, n=2 ** 31), dict(rows=odd), dict(ws=odd)):
        assert spmm(**bad) == -1, bad
    for bad in both + (dict(dvals=None), dict(dvals=odd), dict(dY=None), dict(dY=odd)):
        assert grad(**bad) == -1, bad
    assert spmm(N=0, n=0) == 0 and spmm(rows=FAKE, n=0, Y=None) == 0 and grad(N=0) == 0 and grad(nnz=0) == 0

    def weight(codes=FAKE, ldq=32, scale=FAKE, G=FAKE, ldg=8, dW=FAKE, ldw=8, N=4, F=20, H=8, ws=None):
        return lib.es_q8_weight_grad(codes, ldq, scale, G, ldg, dW, ldw, N, F, H, ws, 0, None)

    for bad in (dict(ldq=24), dict(ldq=16), dict(codes=None), dict(scale=None), dict(G=None), dict(G=odd), dict(ldg=7),
                dict(dW=None), dict(dW=odd), dict(ldw=7), dict(N=-1), dict(N=2 ** 31), dict(F=0), dict(H=0), dict(ws=odd)):
        assert weight(**bad) == -1, bad
    ask = es.es_q8_weight_grad_workspace_bytes
    assert ask(0, 16, 16) == ask(-1, 16, 16) == ask(5, 0, 16) == ask(5, 16, 0) == ask(2 ** 31, 16, 16) == 0
    assert ask(100, 16, 16) == 0 and ask(1_000_000, 128, 128) > 0


def test_widths_beyond_the_kernels_offsets_are_refused():
    lib = es.load_library()
    F = 2 ** 30 + 1
    assert lib.es_spmm_q8_backward_vals(FAKE, FAKE, FAKE, F, FAKE, F + 15, FAKE, FAKE, 4, 9, F, 2, 1, 0, 0, None) == -2
    for ldq, ldg, H in ((32, 2 ** 26, 8), (32, 2 ** 27 - 1, 2 ** 27 - 1), (2 ** 27, 8, 8)):
        assert lib.es_q8_weight_grad(FAKE, ldq, FAKE, FAKE, ldg, FAKE, H, 100, 20, H, None, 0, None) == -2


def test_python_refuses_what_it_cannot_read():
    import torch
    from torch._subclasses.fake_tensor import FakeTensorMode
    host = torch.zeros(4, 16)
    codes, scale = torch.zeros(4, 16, dtype=torch.int8), torch.zeros(4)
    for call in (lambda: es.es_q8_write(host, codes, scale), lambda: es.es_q8_read(codes, scale, host),
                 lambda: es.es_q8_write(None, codes, scale), lambda: es.es_q8_weight_grad(codes, scale, host, host)):
        with pytest.raises(ValueError, match="device tensor"):
            call()
    with FakeTensorMode():
        x = torch.empty(4, 16, device="cuda")
        q, s = torch.empty(4, 16, dtype=torch.int8, device="cuda"), torch.empty(4, device="cuda")
        with pytest.raises((ValueError, RuntimeError)):
            es.es_q8_write(x, q, s)


def test_no_kernel_of_8_bit_rows_spills(tmp_path):
    """From the library's own metadata: every code object that is linked into it, one per source file."""
    import os
    import re
    import subprocess
    from paper_2104_10716_amd import build
    llvm = "/opt/rocm/llvm/bin"
    if not os.path.exists(f"{llvm}/clang-offload-bundler"):
        pytest.skip("no LLVM tools")
    es.load_library()
    fat = str(tmp_path / "fat")
    subprocess.run([f"{llvm}/llvm-objcopy", "--dump-section", f".hip_fatbin={fat}", build.LIB, os.devnull], check=True)
    data, magic, kernels = open(fat, "rb").read(), b"__CLANG_OFFLOAD_BUNDLE__", {}
    starts = [m.start() for m in re.finditer(re.escape(magic), data)]
    for a, b in zip(starts, starts[1:] + [len(data)]):
        bundle, code = str(tmp_path / "bundle"), str(tmp_path / "code")
        open(bundle, "wb").write(data[a:b])
        subprocess.run([f"{llvm}/clang-offload-bundler", "--type=o", "--unbundle", "--targets=hipv4-amdgcn-amd-amdhsa--gfx950",
                        f"--input={bundle}", f"--output={code}"], check=True)
        notes = subprocess.run([f"{llvm}/llvm-readelf", "--notes", code], check=True, capture_output=True, text=True).stdout
        found = re.findall(r"\.name: +(_Z\w+kernel\w+)\n.*?\.private_segment_fixed_size: +(\d+)\n.*?\.vgpr_spill_count: +(\d+)\n",
                           notes, re.S)
        kernels.update({name: (int(scratch), int(spilled)) for name, scratch, spilled in found if "es_q8" in name})
    assert len(kernels) > 100 and any("es_q8_grad_kernel" in k for k in kernels)
    assert {k: v for k, v in kernels.items() if v != (0, 0)} == {}


# ---- on the GPU -------------------------------------------------------------------------------
def dev(a):
    import torch
    return None if a is None else torch.from_numpy(np.ascontiguousarray(a)).to("cuda:0")


def table(N, F, pad=0):
    """A table on the device, filled with what no write leaves."""
    import torch
    ld = es.es_q8_row_bytes(F) + 16 * pad
    codes = torch.full((N, ld), 77, dtype=torch.int8, device="cuda:0")
    return codes, torch.full((N,), 0.5, dtype=torch.float32, device="cuda:0")


def filled(X):
    """(codes, scale) on the device and (codes, scale, value) on the host, from the definition."""
    q, s, v = quantise(X)
    codes, scale = table(*X.shape)
    codes.zero_()
    codes[:, :X.shape[1]] = dev(q)
    scale.copy_(dev(s))
    return codes, scale, q, s, v


def awkward_rows(rng, F):
    """Rows at which rounding, scales and the held formats have their borders."""
    X = rng.standard_normal((48, F)).astype(np.float32) * np.exp(rng.uniform(-20, 20, (48, 1))).astype(np.float32)
    X[0] = 0.0
    X[1] = -0.0
    X[2, 0] = np.nan
    X[3, F - 1] = -np.inf
    X[4] = 0.0
    X[4, F // 2] = np.float32(3.4028235e38)                    # the largest number
    X[5] = rng.uniform(-1, 1, F).astype(np.float32) * np.float32(3.4e38)
    X[6] = np.float32(1e-40)                                   # subnormal: held as zeros
    small = np.float32(127.0) * np.float32(2.0 ** -126)
    X[7] = np.nextafter(small, np.float32(0))                  # just below the smallest scale: zeros
    X[8] = rng.uniform(-1, 1, F).astype(np.float32) * small    # the smallest scale, subnormal quotients' operands
    X[8, 0] = small
    for i, e in ((9, 0), (10, -126), (11, 100), (12, 3)):      # ties: scale is exactly 2^e
        k = rng.integers(-127, 127, F).astype(np.float32) + np.float32(0.5)
        X[i] = k * np.float32(2.0 ** e)
        X[i, 0] = np.float32(127.0 * 2.0 ** e)
    X[13] = np.nextafter(X[9], np.float32(np.inf))             # one step off a tie
    X[14] = np.nextafter(X[9], np.float32(-np.inf))
    X[13, 0] = X[14, 0] = 127.0
    for i in range(15, 30):                                    # next to a border of a scale that is no power of two
        top = np.float32(rng.uniform(0.5, 2.0))
        s = np.float64(np.float32(np.float64(top) / 127.0))
        near_tie = ((rng.integers(-126, 126, F) + 0.5) * s).astype(np.float32)
        step = rng.integers(-1, 2, F)
        X[i] = np.where(step < 0, np.nextafter(near_tie, np.float32(-9)), np.where(step > 0, np.nextafter(near_tie, np.float32(9)), near_tie))
        X[i, 0] = -top
    return X


def torch_type(name):
    import torch
    return {"fp32": torch.float32, "fp16": torch.float16, "bf16": torch.bfloat16}[name]


@pytest.mark.gpu
@pytest.mark.parametrize("kind", ["fp32", "fp16", "bf16"])
@pytest.mark.parametrize("F", [1, 3, 4, 15, 16, 17, 31, 41, 64, 100, 128, 130, 256, 257, 602, 1024, 1025, 2048, 2049, 5000])
def test_write_and_read_every_row(kind, F):
    import torch
    rng = np.random.default_rng(F)
    X = dev(awkward_rows(rng, F)).to(torch_type(kind))
    q, s, v = quantise(X.float().cpu().numpy())
    N = X.shape[0]
    for pad, shift in ((0, 0), (2, 1)):                        # rows back to back; strided ones, off every alignment
        src = X
        if shift:
            wide = torch.full((N + 1, F + 5), 9.0, device=X.device, dtype=X.dtype)
            src = wide[1:, shift:shift + F]
            src.copy_(X)
        codes, scale = table(N, F, pad)
        es.es_q8_write(src, codes, scale)
        torch.cuda.synchronize()
        got = codes.cpu().numpy()
        np.testing.assert_array_equal(scale.cpu().numpy(), s)
        np.testing.assert_array_equal(got[:, :F], q)
        row = es.es_q8_row_bytes(F)
        assert (got[:, F:row] == 0).all() and (got[:, row:] == 77).all()
        Y = torch.full((N, F + 3 * shift), 5.0, device=X.device, dtype=X.dtype)
        out = es.es_q8_read(codes, scale, Y[:, shift:shift + F])
        torch.cuda.synchronize()
        want = torch.from_numpy(q.astype(np.float32) * s[:, None]).to(X.dtype)      # one product in fp32, one rounding
        assert torch.equal(torch.nan_to_num(out.cpu().float(), nan=1.25), torch.nan_to_num(want.float(), nan=1.25))
        assert bool((Y[:, :shift] == 5.0).all()) and bool((Y[:, shift + F:] == 5.0).all())
        fine = np.isfinite(s)
        np.testing.assert_allclose(want.double().numpy()[fine & (np.abs(v).max(1) < 6e4)], v[fine & (np.abs(v).max(1) < 6e4)],
                                   rtol=1.01 * (torch.finfo(X.dtype).eps / 2 + U), atol=6.1e-8 if kind == "fp16" else 0)


@pytest.mark.gpu
@pytest.mark.parametrize("n", [1, 5, 64, 2047, 2048, 2049, 9000])
@pytest.mark.parametrize("F", [3, 128, 700, 3000])
def test_write_at_ids(n, F):
    """Ids in any order, some outside the table, many more than once: the last row of equal ids is the one that is
    held, and rows that no id names keep what they had."""
    import torch
    rng = np.random.default_rng(n + F)
    N = 700
    X = rng.standard_normal((n, F)).astype(np.float32)
    X[::7] = 0.0                                               # scale 0 beside the marks
    X[3::11, 0] = np.nan
    for ids in (rng.integers(-3, N + 3, n), rng.integers(5, 9, n), np.full(n, 699), np.full(n, -1),
                np.concatenate([rng.permutation(N)[:min(n, N)], np.full(max(0, n - N), -2 ** 31)])):
        ids = ids.astype(np.int32)
        codes, scale = table(N, F)
        scale[5:8] = 0.0
        before_q, before_s = codes.cpu().numpy(), scale.cpu().numpy()
        es.es_q8_write(dev(X), codes, scale, rows=dev(ids))
        torch.cuda.synchronize()
        q, s, _ = quantise(X)
        for i, r in enumerate(ids):
            if 0 <= r < N:
                before_q[r, :F], before_q[r, F:], before_s[r] = q[i], 0, s[i]
        np.testing.assert_array_equal(scale.cpu().numpy(), before_s)
        np.testing.assert_array_equal(codes.cpu().numpy(), before_q)
        Y = torch.full((n, F), 3.0, device="cuda:0")
        es.es_q8_read(codes, scale, Y, rows=dev(ids))
        torch.cuda.synchronize()
        inside = (ids >= 0) & (ids < N)
        want = np.where(inside[:, None], before_q[np.where(inside, ids, 0), :F] * before_s[np.where(inside, ids, 0)][:, None], 0)
        np.testing.assert_array_equal(Y.cpu().numpy(), want.astype(np.float32))


@pytest.mark.gpu
@pytest.mark.parametrize("kind,F", [("fp32", 3), ("fp32", 32), ("fp32", 64), ("fp32", 128), ("fp32", 256), ("bf16", 20), ("fp16", 130), ("bf16", 602)])
def test_write_at_ids_where_the_way_to_tell_equal_ones_changes(kind, F):
    import torch
    rng = np.random.default_rng(F)
    N = 900
    whole = dev(rng.standard_normal((3201, F)).astype(np.float32)).to(torch_type(kind))
    q, s, _ = quantise(whole.float().cpu().numpy())
    for n in (199, 200, 201, 400, 401, 800, 801, 1600, 1601, 3200, 3201):
        for ids in (rng.integers(-3, N + 3, n), rng.integers(0, 10, n)):
            ids = ids.astype(np.int32)
            codes, scale = table(N, F)
            want_q, want_s = codes.cpu().numpy(), scale.cpu().numpy()
            es.es_q8_write(whole[:n], codes, scale, rows=dev(ids))
            for i, r in enumerate(ids):
                if 0 <= r < N:
                    want_q[r, :F], want_q[r, F:], want_s[r] = q[i], 0, s[i]
            np.testing.assert_array_equal(scale.cpu().numpy(), want_s)
            np.testing.assert_array_equal(codes.cpu().numpy(), want_q)


@pytest.mark.gpu
def test_more_ids_than_marks():
    """More rows than one pass can tell apart: later pieces replace earlier ones."""
    import torch
    n, N = 2 ** 23 + 1000, 50
    ids = torch.arange(n, device="cuda:0", dtype=torch.int32) % N
    X = torch.arange(n, device="cuda:0", dtype=torch.float32)[:, None].contiguous()
    codes, scale = table(N, 1)
    es.es_q8_write(X, codes, scale, rows=ids)
    torch.cuda.synchronize()
    last = np.array([n - 1 - ((n - 1 - r) % N) for r in range(N)], dtype=np.float32)
    np.testing.assert_array_equal(scale.cpu().numpy(), (last.astype(np.float64) / 127).astype(np.float32))
    assert bool((codes[:, 0] == 127).all())


@pytest.mark.gpu
def test_tables_beyond_32_bit_offsets():
    import torch
    N, F = 4_400_000, 1000                                     # 4.4 GB of codes
    codes = torch.empty((N, es.es_q8_row_bytes(F)), dtype=torch.int8, device="cuda:0")
    scale = torch.empty(N, device="cuda:0")
    rng = np.random.default_rng(3)
    ids = np.array([0, N - 1, 2 ** 21 - 1, 2 ** 21, 2 ** 22 - 1, 2 ** 22 + 7, N - 2], dtype=np.int32)
    X = rng.standard_normal((len(ids), F)).astype(np.float32)
    q, s, v = quantise(X)
    es.es_q8_write(dev(X), codes, scale, rows=dev(ids))
    Y = torch.empty((len(ids), F), device="cuda:0")
    es.es_q8_read(codes, scale, Y, rows=dev(ids))
    np.testing.assert_array_equal(Y.cpu().numpy(), q.astype(np.float32) * s[:, None])
    # a graph whose last row gathers them
    rowptr = np.zeros(N + 1, dtype=np.int32)
    rowptr[N] = len(ids)
    col = np.sort(ids)
    order = np.argsort(ids)
    a = rng.standard_normal(len(ids)).astype(np.float32)
    Z = torch.empty((2, F), device="cuda:0")
    es.es_spmm_q8(dev(rowptr), dev(col), dev(a), codes, scale, Z, 0, "full", rows=dev(np.array([N - 1, 0], np.int32)))
    want = (a[:, None].astype(np.float64) * v[order]).sum(0)
    tol = (np.abs(a)[:, None] * np.abs(v[order])).sum(0) * (len(ids) + 5) * U
    near(Z[0].cpu().numpy(), want, tol, "far rows")
    assert bool((Z[1] == 0).all())


@pytest.mark.gpu
def test_tables_beyond_64_gib():
    """Rows 16 KiB apart: the largest offset no longer fits 32 bits of 16-byte units."""
    import torch
    N, F = 4_200_000, 40
    whole = torch.empty((N, 16_384), dtype=torch.int8, device="cuda:0")        # 69 GB, hardly any of it touched
    codes, scale = whole[:, 16:16 + es.es_q8_row_bytes(F)], torch.zeros(N, device="cuda:0")
    rng = np.random.default_rng(3)
    ids = np.array([1, 7, 2 ** 22, N - 2, N - 1], dtype=np.int32)
    X = rng.standard_normal((len(ids), F)).astype(np.float32)
    q, s, v = quantise(X)
    es.es_q8_write(dev(X), codes, scale, rows=dev(ids))
    Y = torch.empty((len(ids), F), device="cuda:0")
    es.es_q8_read(codes, scale, Y, rows=dev(ids))
    np.testing.assert_array_equal(Y.cpu().numpy(), q.astype(np.float32) * s[:, None])
    rowptr = np.zeros(N + 1, dtype=np.int32)
    rowptr[N - 2:] = len(ids)                                  # row N - 3 gathers them
    a = rng.standard_normal(len(ids)).astype(np.float32)
    g = dev(rowptr), dev(ids)
    for rows in (dev(np.array([N - 3, 0], np.int32)), dev(np.concatenate([np.full(600, N - 3), np.zeros(600)]).astype(np.int32))):
        Z = torch.empty((rows.numel(), F), device="cuda:0")
        for mode, W in (("full", 0), ("fastrand", 7)):
            es.es_spmm_q8(*g, dev(a), codes, scale, Z, W, mode, rows=rows)
            tol = (np.abs(a)[:, None] * np.abs(v)).sum(0) * (len(ids) + 5) * U
            near(Z[0].cpu().numpy(), (a[:, None].astype(np.float64) * v).sum(0), tol, "far rows")
            assert bool((Z[-1] == 0).all())
    dY = torch.zeros((N, F), device="cuda:0")
    row = rng.standard_normal(F).astype(np.float32)
    dY[N - 3] = dev(row)
    for mode, W in (("full", 0), ("bucket", 9), ("fastrand", 9)):
        da = es.es_spmm_q8_backward_vals(*g, dY, codes, scale, torch.empty(len(ids), device="cuda:0"), W, mode)
        near(da.cpu().numpy(), (v * row).sum(1), (np.abs(v) * np.abs(row)).sum(1) * (F + 6) * U, "far da")


def graph(N, avg, seed, long_row=0, dense_row=None):
    from workloads import random_csr
    rowptr, colidx = random_csr(N, avg, seed, empty_frac=0.1)
    if long_row:                                               # one row that holds the first `long_row` columns
        r = N // 2 if dense_row is None else dense_row
        head, tail = colidx[:rowptr[r]], colidx[rowptr[r + 1]:]
        grown = long_row - (rowptr[r + 1] - rowptr[r])
        colidx = np.concatenate([head, np.arange(long_row, dtype=np.int32), tail]).astype(np.int32)
        rowptr = rowptr.copy()
        rowptr[r + 1:] += grown
    return rowptr.astype(np.int32), colidx


MODES = [("full", 0, 0), ("bucket", 1, 0), ("bucket", 7, 0), ("fastrand", 5, 0), ("fastrand", 16, 99), ("fastrand", 300, 2 ** 40 + 1)]


@pytest.mark.gpu
@pytest.mark.parametrize("F", [1, 3, 16, 17, 33, 41, 64, 100, 128, 130, 256, 300, 602, 1040, 2500])
def test_product_all_rows(F):
    import torch
    N = 333
    rowptr, colidx = graph(N, 12.0, F, long_row=329)
    rng = np.random.default_rng(F)
    vals = rng.standard_normal(colidx.size).astype(np.float32)
    X = rng.standard_normal((N, F)).astype(np.float32) * np.exp(rng.uniform(-6, 6, (N, 1))).astype(np.float32)
    codes, scale, q, s, v = filled(X)
    for mode, W, seed in MODES:
        for norm, a in (("none", vals), ("mean", None), ("rsqrt", vals), ("rescale", None), ("inv_degree", vals)):
            ld = F + (3 if norm == "mean" else 0)
            Y = torch.full((N, ld), float("nan"), device="cuda:0")
            es.es_spmm_q8(dev(rowptr), dev(colidx), dev(a), codes, scale, Y[:, :F], W, mode, seed, norm)
            torch.cuda.synchronize()
            want, tol = product(rowptr, colidx, a, v, W, mode, seed, norm)
            near(Y[:, :F].cpu().numpy(), want, tol, f"{mode} {W} {norm} F={F}")
            assert bool(Y[:, F:].isnan().all())


@pytest.mark.gpu
@pytest.mark.parametrize("N,avg,long_row", [(1, 1, 0), (2, 1.5, 2), (64, 60, 64), (5000, 2, 0), (3000, 4, 2999), (20_000, 6, 20_000),
                                            (40_000, 30, 17_777)])
@pytest.mark.parametrize("F", [16, 41, 128])
def test_product_on_row_lengths(N, avg, long_row, F):
    """From empty rows to one that holds every column, the same bits each time."""
    import torch
    rowptr, colidx = graph(N, avg, N, long_row)
    rng = np.random.default_rng(N)
    vals = rng.standard_normal(colidx.size).astype(np.float32)
    codes, scale, q, s, v = filled(rng.standard_normal((N, F)).astype(np.float32))
    for mode, W, seed in (("full", 0, 0), ("bucket", 600, 0), ("fastrand", 9000, 3), ("fastrand", 12, 0)):
        d = dev(rowptr), dev(colidx), dev(vals), codes, scale
        Y = [es.es_spmm_q8(*d, torch.full((N, F), float("nan"), device="cuda:0"), W, mode, seed) for _ in range(2)]
        want, tol = product(rowptr, colidx, vals, v, W, mode, seed, "none")
        near(Y[0].cpu().numpy(), want, tol, f"{mode} {W}")
        assert torch.equal(Y[0], Y[1])


@pytest.mark.gpu
@pytest.mark.parametrize("n", [0, 1, 2, 33, 500, 3000])
@pytest.mark.parametrize("F", [8, 64, 100])
def test_product_of_asked_rows(n, F):
    """Rows in any order, more than once, outside the graph; a hub among them."""
    import torch
    N = 9000
    rowptr, colidx = graph(N, 20.0, 5, long_row=8500)
    rng = np.random.default_rng(n)
    vals = rng.standard_normal(colidx.size).astype(np.float32)
    codes, scale, q, s, v = filled(rng.standard_normal((N, F)).astype(np.float32))
    ids = rng.integers(-2, N + 2, n).astype(np.int32)
    ids[n // 2:n // 2 + 1] = N // 2                            # the hub
    ids[n - 1:] = ids[:1]
    for mode, W, seed in (("full", 0, 0), ("bucket", 40, 0), ("fastrand", 16, 7), ("fastrand", 4000, 7)):
        Y = torch.full((n, F), float("nan"), device="cuda:0")
        es.es_spmm_q8(dev(rowptr), dev(colidx), dev(vals), codes, scale, Y, W, mode, seed, "mean", rows=dev(ids))
        torch.cuda.synchronize()
        want, tol = product(rowptr, colidx, vals, v, W, mode, seed, "mean")
        inside = (ids >= 0) & (ids < N)
        at = np.where(inside, ids, 0)
        near(Y.cpu().numpy(), np.where(inside[:, None], want[at], 0), np.where(inside[:, None], tol[at], 0), f"{mode} {W} n={n}")


@pytest.mark.gpu
def test_rows_that_no_kept_entry_names_have_no_influence():
    import torch
    N, F = 400, 48
    rowptr, colidx = graph(N, 9.0, 8)
    codes, scale, q, s, v = filled(np.random.default_rng(0).standard_normal((N, F)).astype(np.float32))
    used = np.zeros(N, bool)
    for p in kept_lists(rowptr, 3, "fastrand", 5):
        used[colidx[p]] = True
    assert 0 < used.sum() < N
    bad = scale.clone()
    bad[dev(~used)] = float("nan")
    g = dev(rowptr), dev(colidx), None
    Y, Z = torch.empty((N, F), device="cuda:0"), torch.empty((N, F), device="cuda:0")
    es.es_spmm_q8(*g, codes, scale, Y, 3, "fastrand", 5)
    es.es_spmm_q8(*g, codes, bad, Z, 3, "fastrand", 5)
    assert torch.equal(Y, Z)
    # a row that a kept entry does name: NaN in every column, there alone
    one = int(np.flatnonzero(used)[0])
    bad = scale.clone()
    bad[one] = float("nan")
    es.es_spmm_q8(*g, codes, bad, Z, 3, "fastrand", 5)
    hit = dev(np.array([one in colidx[p] for p in kept_lists(rowptr, 3, "fastrand", 5)]))
    assert bool(Z[hit].isnan().all()) and torch.equal(Z[~hit], Y[~hit])


@pytest.mark.gpu
@pytest.mark.parametrize("F", [1, 3, 16, 17, 41, 64, 100, 128, 256, 300, 602, 1024, 1040, 3000])
def test_edge_gradient(F):
    import torch
    N = 300
    rowptr, colidx = graph(N, 12.0, F + 1, long_row=297)
    rng = np.random.default_rng(F)
    dY = rng.standard_normal((N, F)).astype(np.float32)
    X = rng.standard_normal((N, F)).astype(np.float32) * np.exp(rng.uniform(-6, 6, (N, 1))).astype(np.float32)
    codes, scale, q, s, v = filled(X)
    for shift in (0, 1):
        wide = torch.zeros((N, F + 4 * shift), device="cuda:0")
        grad = wide[:, shift:shift + F]
        grad.copy_(dev(dY))
        for mode, W, seed in MODES:
            for norm in ("none", "mean", "rsqrt", "rescale", "inv_degree"):
                out = torch.full((colidx.size,), float("nan"), device="cuda:0")
                es.es_spmm_q8_backward_vals(dev(rowptr), dev(colidx), grad, codes, scale, out, W, mode, seed, norm)
                torch.cuda.synchronize()
                want, tol = edge_gradient(rowptr, colidx, dY, q, s, W, mode, seed, norm)
                near(out.cpu().numpy(), want, tol, f"{mode} {W} {norm} F={F}")


@pytest.mark.gpu
@pytest.mark.parametrize("N,avg,long_row", [(1, 1, 0), (2, 1.5, 2), (5000, 2, 0), (3000, 4, 2999), (20_000, 6, 20_000), (2000, 300, 1999)])
def test_edge_gradient_on_row_lengths(N, avg, long_row):
    import torch
    F = 41
    rowptr, colidx = graph(N, avg, N, long_row)
    rng = np.random.default_rng(N)
    dY = rng.standard_normal((N, F)).astype(np.float32)
    codes, scale, q, s, v = filled(rng.standard_normal((N, F)).astype(np.float32))
    for mode, W, seed in (("full", 0, 0), ("bucket", 600, 0), ("fastrand", 9000, 3), ("fastrand", 12, 0), ("fastrand", 290, 1),
                          ("fastrand", 64, 5), ("fastrand", 65, 5), ("fastrand", 1024, 5), ("fastrand", 1025, 0), ("fastrand", 1100, 9)):
        outs = [es.es_spmm_q8_backward_vals(dev(rowptr), dev(colidx), dev(dY), codes, scale,
                                            torch.full((colidx.size,), float("nan"), device="cuda:0"), W, mode, seed)
                for _ in range(2)]
        want, tol = edge_gradient(rowptr, colidx, dY, q, s, W, mode, seed, "none")
        near(outs[0].cpu().numpy(), want, tol, f"{mode} {W}")
        assert torch.equal(outs[0], outs[1])


@pytest.mark.gpu
@pytest.mark.parametrize("N,avg,long_row", [(3000, 6, 2900), (9000, 6, 7000), (26_000, 4, 25_000), (26_000, 60, 3000), (120_000, 3, 9000)])
@pytest.mark.parametrize("F", [8, 20, 41, 100, 250])
def test_every_share_of_a_wave(N, avg, long_row, F):
    """Both products where a row is a whole wave's, half a wave's, and that of as few lanes as cover its columns."""
    import oracle
    import torch
    from scipy.sparse import csr_matrix
    rowptr, colidx = graph(N, avg, F, long_row)
    rng = np.random.default_rng(N + F)
    vals = rng.standard_normal(colidx.size).astype(np.float32)
    dY = rng.standard_normal((N, F)).astype(np.float32)
    X = rng.standard_normal((N, F)).astype(np.float32) * np.exp(rng.uniform(-3, 3, (N, 1))).astype(np.float32)
    codes, scale, q, s, v = filled(X)
    rows = np.repeat(np.arange(N), np.diff(rowptr))
    d = dev(rowptr), dev(colidx)
    for mode, W, seed in (("full", 0, 0), ("bucket", 24, 0), ("fastrand", 50, 9)):
        keep = np.ones(colidx.size, bool)
        if mode != "full":
            pos, cnt = oracle.kept(rowptr, W, mode, seed)
            keep[:] = False
            keep[pos[np.arange(pos.shape[1])[None, :] < cnt[:, None]]] = True
        k = np.add.reduceat(np.concatenate([keep, [False]]).astype(np.int64), rowptr[:-1]) * (np.diff(rowptr) > 0)
        A = csr_matrix((np.where(keep, vals, 0).astype(np.float64), colidx, rowptr), shape=(N, N))
        B = csr_matrix((np.abs(A.data), colidx, rowptr), shape=(N, N))
        Y = es.es_spmm_q8(*d, dev(vals), codes, scale, torch.full((N, F), float("nan"), device="cuda:0"), W, mode, seed)
        near(Y.cpu().numpy(), A @ v, (B @ np.abs(v)) * ((k + 5) * U)[:, None], f"{mode} {W}")
        da = es.es_spmm_q8_backward_vals(*d, dev(dY), codes, scale, torch.full((colidx.size,), float("nan"), device="cuda:0"),
                                         W, mode, seed)
        want, tol = np.zeros(colidx.size), np.zeros(colidx.size)
        for lo in range(0, colidx.size, 100_000):
            e = slice(lo, lo + 100_000)
            x, g = v[colidx[e]], dY[rows[e]].astype(np.float64)
            want[e], tol[e] = (x * g).sum(1) * keep[e], (np.abs(x) * np.abs(g)).sum(1) * keep[e] * (F + 6) * U
        near(da.cpu().numpy(), want, tol, f"da {mode} {W}")


@pytest.mark.gpu
@pytest.mark.parametrize("N,avg,long_row", [(3000, 6, 2900), (9000, 20, 7000), (26_000, 12, 25_000), (120_000, 6, 9000)])
@pytest.mark.parametrize("F", [16, 41, 250, 300, 520])
def test_edge_gradient_of_a_random_sample(N, avg, long_row, F):
    """Every number of lanes that a row of FastRand's takes, at the widths where that changes."""
    import oracle
    import torch
    rowptr, colidx = graph(N, avg, F, long_row)
    rng = np.random.default_rng(N + F)
    dY = rng.standard_normal((N, F)).astype(np.float32)
    codes, scale, q, s, v = filled(rng.standard_normal((N, F)).astype(np.float32))
    rows = np.repeat(np.arange(N), np.diff(rowptr))
    want, tol = np.zeros(colidx.size), np.zeros(colidx.size)
    for lo in range(0, colidx.size, 100_000):
        e = slice(lo, lo + 100_000)
        x, g = v[colidx[e]], dY[rows[e]].astype(np.float64)
        want[e], tol[e] = (x * g).sum(1), (np.abs(x) * np.abs(g)).sum(1) * (F + 6) * U
    d = dev(rowptr), dev(colidx), dev(dY)
    for W, seed in ((1, 0), (5, 2), (64, 9), (65, 9), (127, 0), (128, 3), (224, 9), (225, 9), (256, 0), (257, 1), (384, 9), (385, 9), (1024, 9)):
        pos, cnt = oracle.kept(rowptr, W, "fastrand", seed)
        keep = np.zeros(colidx.size, bool)
        keep[pos[np.arange(pos.shape[1])[None, :] < cnt[:, None]]] = True
        da = es.es_spmm_q8_backward_vals(*d, codes, scale, torch.full((colidx.size,), float("nan"), device="cuda:0"), W, "fastrand", seed)
        near(da.cpu().numpy(), want * keep, tol * keep, f"W={W}")


@pytest.mark.gpu
def test_edge_gradient_against_differences():
    """The product is linear in the values, so a central difference of L = <dY, Y> has no truncation error, only the
    product's own rounding: two evaluations, each off by at most its tolerance, over a step of 2 h."""
    import torch
    N, F, h = 60, 24, 1.0
    rowptr, colidx = graph(N, 5.0, 11)
    rng = np.random.default_rng(1)
    vals = rng.standard_normal(colidx.size).astype(np.float32)
    dY = rng.standard_normal((N, F)).astype(np.float32)
    codes, scale, q, s, v = filled(rng.standard_normal((N, F)).astype(np.float32))
    for mode, W, seed, norm in (("full", 0, 0, "none"), ("fastrand", 3, 5, "mean"), ("bucket", 2, 0, "rescale")):
        g = torch.empty(colidx.size, device="cuda:0")
        es.es_spmm_q8_backward_vals(dev(rowptr), dev(colidx), dev(dY), codes, scale, g, W, mode, seed, norm)
        g = g.cpu().numpy()
        for p in range(0, colidx.size, 7):
            L, tol = [], edge_gradient(rowptr, colidx, dY, q, s, W, mode, seed, norm)[1][p]
            for sign in (1, -1):
                a = vals.copy()
                a[p] += np.float32(sign * h)
                Y = torch.empty((N, F), device="cuda:0")
                es.es_spmm_q8(dev(rowptr), dev(colidx), dev(a), codes, scale, Y, W, mode, seed, norm)
                L.append((Y.cpu().numpy().astype(np.float64) * dY).sum())
                tol += (product(rowptr, colidx, a, v, W, mode, seed, norm)[1] * np.abs(dY)).sum() / (2 * h)
                step = np.float64(a[p]) - np.float64(vals[p])
                tol += abs(abs(step) - h) / h * abs(g[p])       # the perturbed value is rounded too
            assert abs((L[0] - L[1]) / (2 * h) - g[p]) <= tol, (mode, p)


@pytest.mark.gpu
@pytest.mark.parametrize("N,F,H", [(0, 20, 8), (1, 1, 1), (7, 16, 5), (15, 130, 41), (16, 64, 64), (17, 33, 129), (255, 128, 128),
                                   (1000, 41, 7), (1025, 602, 256), (5000, 100, 3), (20_011, 128, 128), (40_000, 16, 250), (3000, 1100, 300)])
def test_weight_gradient(N, F, H):
    """Each product is exact but for the scale's and the sum's roundings, of which there are at most three per row."""
    import torch
    rng = np.random.default_rng(N + F)
    X = rng.standard_normal((N, F)).astype(np.float32) * np.exp(rng.uniform(-4, 4, (N, 1))).astype(np.float32)
    G = rng.standard_normal((N, H)).astype(np.float32)
    if N:
        G[rng.integers(0, N)] *= 1e4
        codes, scale, q, s, v = filled(X)
    else:
        codes, scale = table(0, F)
        v = X.astype(np.float64)
    want = v.T @ G.astype(np.float64)
    tol = np.abs(v).T @ np.abs(G).astype(np.float64) * (3 * N + 8) * U
    need = es.es_q8_weight_grad_workspace_bytes(N, F, H)
    outs = []
    for workspace in (None, torch.full((need + 256,), 201, dtype=torch.uint8, device="cuda:0"),
                      torch.empty(0, dtype=torch.uint8, device="cuda:0")):
        for shift in (0, 1):                                   # rows back to back; strided, off every alignment
            g = torch.zeros((N, H + 2 * shift), device="cuda:0")[:, shift:shift + H]
            g.copy_(dev(G))
            dW = torch.full((F, H + 3 * shift), float("nan"), device="cuda:0")
            es.es_q8_weight_grad(codes, scale, g, dW[:, shift:shift + H], workspace)
            torch.cuda.synchronize()
            near(dW[:, shift:shift + H].cpu().numpy(), want, tol, f"N={N} F={F} H={H}")
            assert bool(dW[:, :shift].isnan().all()) and bool(dW[:, shift + H:].isnan().all())
            outs.append(dW[:, shift:shift + H].clone())
        if workspace is not None and workspace.numel():
            assert bool((workspace[need:] == 201).all())       # nothing behind what it asked for
    assert torch.equal(outs[0], outs[2])                       # a workspace of the asked size: the same bits


@pytest.mark.gpu
def test_a_training_step_from_8_bit_checkpoints():
    """Z = X W1, H = relu(A(a) Z), P = H W2, Y = A(a) P with learned edge values a: the inputs X and H and the products' operands Z and
    P are kept as 8-bit rows, and the gradients of W1, W2 and a are those of the formulas on the kept values."""
    import torch
    N, F0, F1, C = 500, 70, 48, 9
    rowptr, colidx = graph(N, 8.0, 21)
    rng = np.random.default_rng(2)
    rp, ci = dev(rowptr), dev(colidx)
    a = dev(rng.uniform(0.1, 1.0, colidx.size).astype(np.float32))
    X, W1, W2 = (dev(rng.standard_normal(s).astype(np.float32)) for s in ((N, F0), (F0, F1), (F1, C)))
    W, mode, seed, norm = 5, "fastrand", 77, "mean"
    new = lambda n, f: torch.empty((n, f), device="cuda:0")  # noqa: E731

    def keep(T):
        codes = torch.empty((T.shape[0], es.es_q8_row_bytes(T.shape[1])), dtype=torch.int8, device="cuda:0")
        return es.es_q8_write(T, codes, torch.empty(T.shape[0], device="cuda:0"))

    # forward
    kX = keep(X)
    Z = X @ W1
    kZ = keep(Z)
    H = es.es_spmm_norm(rp, ci, a, Z, new(N, F1), W, mode, seed, norm).relu_()
    mask = H > 0
    kH = keep(H)
    P = H @ W2
    kP = keep(P)
    es.es_spmm_norm(rp, ci, a, P, new(N, C), W, mode, seed, norm)
    dY = dev(rng.standard_normal((N, C)).astype(np.float32))
    # backward
    dP = es.es_spmm_backward(rp, ci, a, dY, new(N, C), W, mode, seed, norm)
    da2 = es.es_spmm_q8_backward_vals(rp, ci, dY, *kP, torch.empty_like(a), W, mode, seed, norm)
    dW2 = es.es_q8_weight_grad(*kH, dP, new(F1, C))
    dH = (dP @ W2.t()) * mask
    dZ = es.es_spmm_backward(rp, ci, a, dH, new(N, F1), W, mode, seed, norm)
    da1 = es.es_spmm_q8_backward_vals(rp, ci, dH, *kZ, torch.empty_like(a), W, mode, seed, norm)
    dW1 = es.es_q8_weight_grad(*kX, dZ, new(F0, F1))
    torch.cuda.synchronize()
    for (codes, scale), T, G, dW in ((kH, H, dP, dW2), (kX, X, dZ, dW1)):
        q, s, v = quantise(T.cpu().numpy())
        np.testing.assert_array_equal(codes[:, :T.shape[1]].cpu().numpy(), q)
        g = G.cpu().numpy().astype(np.float64)
        near(dW.cpu().numpy(), v.T @ g, np.abs(v).T @ np.abs(g) * (3 * N + 8) * U, "dW")
        assert np.abs(v - T.cpu().numpy()).max() <= np.nanmax(s) * 0.5 * (1 + 1e-6)    # half a step of the codes
    for T, G, da in ((P, dY, da2), (Z, dH, da1)):
        q, s, v = quantise(T.cpu().numpy())
        want, tol = edge_gradient(rowptr, colidx, G.cpu().numpy(), q, s, W, mode, seed, norm)
        near(da.cpu().numpy(), want, tol, "da")


@pytest.mark.gpu
def test_serving_from_a_table_of_past_embeddings():
    """Batches of nodes push their new embeddings and ask for their neighbourhoods' sums, as a serving program does, on a
    side stream, then from a captured graph whose inputs change between replays."""
    import torch
    N, F, B = 3000, 64, 32
    rowptr, colidx = graph(N, 15.0, 4, long_row=2900)
    rng = np.random.default_rng(9)
    vals = rng.standard_normal(colidx.size).astype(np.float32)
    g = dev(rowptr), dev(colidx), dev(vals)
    X = rng.standard_normal((N, F)).astype(np.float32)
    codes, scale = table(N, F)
    es.es_q8_write(dev(X), codes, scale)
    new_x, ids = torch.zeros((B, F), device="cuda:0"), torch.zeros(B, dtype=torch.int32, device="cuda:0")
    Y, Z = torch.zeros((B, F), device="cuda:0"), torch.zeros((B, F), device="cuda:0")
    side = torch.cuda.Stream()

    def step():
        es.es_q8_write(new_x, codes, scale, rows=ids)
        es.es_spmm_q8(*g, codes, scale, Y, 0, "full", 0, "mean", rows=ids)
        es.es_q8_read(codes, scale, Z, rows=ids)

    def batch(t):
        x = rng.standard_normal((B, F)).astype(np.float32)
        i = rng.permutation(N)[:B].astype(np.int32)
        i[0], i[-1] = N // 2, -1                               # the hub, and a padded place
        new_x.copy_(dev(x))
        ids.copy_(dev(i))
        X[i[:-1]] = x[:-1]
        return i

    def check(i, what):
        q, s, v = quantise(X)
        want, tol = product(rowptr, colidx, vals, v, 0, "full", 0, "mean")
        near(Y[:-1].cpu().numpy(), want[i[:-1]], tol[i[:-1]], what)
        np.testing.assert_array_equal(Z[:-1].cpu().numpy(), q[i[:-1]].astype(np.float32) * s[i[:-1]][:, None])
        assert bool((Y[-1] == 0).all()) and bool((Z[-1] == 0).all())

    for t in range(3):
        i = batch(t)
        torch.cuda.synchronize()
        with torch.cuda.stream(side):
            step()
        side.synchronize()
        check(i, f"side stream {t}")
    captured = torch.cuda.CUDAGraph()
    with torch.cuda.graph(captured):
        step()
    for t in range(4):
        i = batch(3 + t)
        captured.replay()
        torch.cuda.synchronize()
        check(i, f"replay {t}")
        torch.empty(1 << 20, device="cuda:0").normal_()        # the program's own work between replays


@pytest.mark.gpu
def test_a_captured_backward_pass():
    """Both gradients captured with a workspace of their own, replayed on changing inputs, beside eager calls."""
    import torch
    N, F, H = 3000, 96, 40
    rowptr, colidx = graph(N, 10.0, 6)
    rng = np.random.default_rng(1)
    rp, ci = dev(rowptr), dev(colidx)
    codes, scale, q, s, v = filled(rng.standard_normal((N, F)).astype(np.float32))
    dY, G = torch.zeros((N, F), device="cuda:0"), torch.zeros((N, H), device="cuda:0")
    da, dW = torch.zeros(colidx.size, device="cuda:0"), torch.zeros((F, H), device="cuda:0")
    ws = torch.empty(max(16, es.es_q8_weight_grad_workspace_bytes(N, F, H)), dtype=torch.uint8, device="cuda:0")

    def step(da, dW, ws):
        es.es_spmm_q8_backward_vals(rp, ci, dY, codes, scale, da, 4, "fastrand", 3)
        es.es_q8_weight_grad(codes, scale, G, dW, ws)

    step(da, dW, ws)
    torch.cuda.synchronize()
    captured = torch.cuda.CUDAGraph()
    with torch.cuda.graph(captured):
        step(da, dW, ws)
    for t in range(3):
        dY.normal_()
        G.normal_()
        da.fill_(9.0)
        dW.fill_(9.0)
        captured.replay()
        da2, dW2 = torch.empty_like(da), torch.empty_like(dW)
        step(da2, dW2, ws)
        torch.cuda.synchronize()
        assert torch.equal(da, da2) and torch.equal(dW, dW2)
        want, tol = edge_gradient(rowptr, colidx, dY.cpu().numpy(), q, s, 4, "fastrand", 3, "none")
        near(da.cpu().numpy(), want, tol, "captured da")


@pytest.mark.gpu
def test_python_refusals_on_device_tensors():
    import torch
    d = "cuda:0"
    N, F = 8, 20
    codes, scale = table(N, F)
    X, Y = torch.zeros((N, F), device=d), torch.zeros((N, F), device=d)
    rp, ci = torch.zeros(N + 1, dtype=torch.int32, device=d), torch.zeros(3, dtype=torch.int32, device=d)
    ids = torch.zeros(N, dtype=torch.int32, device=d)
    bad_tables = [(codes[:, :16], scale), (codes.float(), scale), (codes, scale.double()), (codes, scale[:5]),
                  (torch.zeros((N, 24), dtype=torch.int8, device=d), scale), (codes[:, 1:], scale),
                  (codes, torch.zeros(2 * N, device=d)[::2]), (torch.zeros(N * 32, dtype=torch.int8, device=d), scale)]
    for q, s in bad_tables:
        for call in (lambda: es.es_q8_write(X, q, s), lambda: es.es_q8_read(q, s, Y), lambda: es.es_spmm_q8(rp, ci, None, q, s, Y, 4, "full"),
                     lambda: es.es_spmm_q8_backward_vals(rp, ci, X, q, s, torch.zeros(3, device=d), 4, "full"),
                     lambda: es.es_q8_weight_grad(q, s, X, torch.zeros((F, F), device=d))):
            with pytest.raises(ValueError):
                call()
    for call in (lambda: es.es_q8_write(X.double(), codes, scale), lambda: es.es_q8_write(X.t(), codes, scale),
                 lambda: es.es_q8_write(X[:1].expand(N, F), codes, scale), lambda: es.es_q8_write(X, codes, scale, rows=ids.long()),
                 lambda: es.es_q8_write(X, codes, scale, rows=ids[:4]), lambda: es.es_q8_write(X.cpu(), codes, scale),
                 lambda: es.es_q8_write(torch.zeros((N + 1, F), device=d), codes, scale),
                 lambda: es.es_q8_read(codes, scale, torch.zeros((N + 1, F), device=d)), lambda: es.es_q8_read(codes, scale, Y[:, ::2]),
                 lambda: es.es_spmm_q8(rp, ci, None, codes, scale, Y[:4], 4, "full"), lambda: es.es_spmm_q8(rp, ci, scale[:2], codes, scale, Y, 4, "full"),
                 lambda: es.es_spmm_q8(rp.long(), ci, None, codes, scale, Y, 4, "full"), lambda: es.es_spmm_q8(rp[:5], ci, None, codes, scale, Y, 4, "full"),
                 lambda: es.es_spmm_q8(rp, ci, None, codes, scale, Y.half(), 4, "full"), lambda: es.es_spmm_q8(rp, ci.cpu(), None, codes, scale, Y, 4, "full"),
                 lambda: es.es_spmm_q8_backward_vals(rp, ci, X[:4], codes, scale, torch.zeros(3, device=d), 4, "full"),
                 lambda: es.es_spmm_q8_backward_vals(rp, ci, X, codes, scale, torch.zeros(2, device=d), 4, "full"),
                 lambda: es.es_q8_weight_grad(codes, scale, X[:4], torch.zeros((F, F), device=d)),
                 lambda: es.es_q8_weight_grad(codes, scale, X, torch.zeros((F, F + 1), device=d)),
                 lambda: es.es_q8_weight_grad(codes, scale, X, torch.zeros((F, F), device=d), torch.zeros((4, 8), device=d)[:, ::2])):
        with pytest.raises(ValueError):
            call()
    for call in (lambda: es.es_spmm_q8(rp, ci, None, codes, scale, Y, 0, "bucket"), lambda: es.es_spmm_q8(rp, ci, None, codes, scale, Y, 4, 7),
                 lambda: es.es_spmm_q8(rp, ci, None, codes, scale, Y, 4, "full", norm=9)):
        with pytest.raises(es.EsSpmmError):
            call()
    torch.cuda.synchronize()
    assert bool((codes == 77).all()) and bool((scale == 0.5).all()) and bool((Y == 0).all())


def test_workspaces_of_the_asked_size_are_taken():
    """A size that the plan asks for is one that the plan is content with: per part F * H sums, and one part more or
    less would show in a size between two multiples."""
    ask = es.es_q8_weight_grad_workspace_bytes
    for N in (1, 255, 256, 511, 513, 1025, 9_999, 40_000, 233_000, 1_000_003, 2_450_000, 2 ** 31 - 1):
        for F, H in ((1, 1), (16, 16), (41, 7), (128, 128), (130, 65), (602, 256), (1100, 300), (5000, 4000)):
            need = ask(N, F, H)
            assert need % (4 * F * H) == 0
            parts = need // (4 * F * H)
            if parts:                                          # every part has rows: whole steps of 64, the last one some
                rows = -(-(-(-N // parts)) // 64) * 64
                assert 1 < parts <= 512 and rows * (parts - 1) < N <= rows * parts
    ask = es.es_spmm_q8_workspace_bytes
    assert ask(233_000, 10 ** 8, 64, 64, "bucket", 233_000) == 0           # no row is cut
    assert ask(170_000, 2_400_000, 100, 0, "full", 170_000) == 4 * 100 * 2 * (2_400_000 // 1024 + 1)
    assert ask(233_000, 114_000_000, 64, 0, "full", 32) == 4 * 64 * 32 * 64   # a few rows: 64 pieces each
    assert ask(233_000, 300, 64, 0, "full", 32) == 4 * 64 * 32 * 3            # no row has more than 300 entries
    for bad in ((-1, 5, 64, 4, 0, 1), (5, -1, 64, 4, 0, 1), (5, 5, 0, 4, 0, 1), (5, 5, 64, 0, 1, 1), (5, 5, 64, 4, 0, 0), (5, 5, 64, 4, 9, 1)):
        assert ask(*bad) == 0


@pytest.mark.gpu
def test_native_marshalling_agrees_with_the_checks_in_python(monkeypatch):
    """The plain calls go through the native marshalling; what it hands back goes through the checks in Python to
    the same kernels.  Streams and integers of every kind."""
    import torch
    m = es.load_marshal()
    N, F, H = 600, 40, 24
    rowptr, colidx = graph(N, 10.0, 3, long_row=590)
    rng = np.random.default_rng(3)
    rp, ci, a = dev(rowptr), dev(colidx), dev(rng.standard_normal(colidx.size).astype(np.float32))
    X = dev(rng.standard_normal((N, F)).astype(np.float32))
    G = dev(rng.standard_normal((N, H)).astype(np.float32))
    ids = dev(rng.integers(-1, N, 50).astype(np.int32))
    side = torch.cuda.Stream()

    def everything(stream, W, seed):
        new = lambda *s: torch.zeros(s, device="cuda:0")  # noqa: E731
        codes, scale = table(N, F)
        torch.cuda.synchronize()
        es.es_q8_write(X, codes, scale, stream=stream)
        es.es_q8_write(X[:50], codes, scale, rows=ids, stream=stream)
        out = [codes, scale, es.es_q8_read(codes, scale, new(50, F), rows=ids, stream=stream),
               es.es_q8_read(codes, scale, new(N, F).bfloat16(), stream=stream),
               es.es_spmm_q8(rp, ci, a, codes, scale, new(N, F), W, "full", seed, "mean", stream=stream),
               es.es_spmm_q8(rp, ci, None, codes, scale, new(50, F), W, "fastrand", seed, "none", rows=ids, stream=stream),
               es.es_spmm_q8_backward_vals(rp, ci, X, codes, scale, new(colidx.size), W, "fastrand", seed, stream=stream),
               es.es_q8_weight_grad(codes, scale, G, new(F, H), stream=stream)]
        torch.cuda.synchronize()
        return out

    want = everything(None, 7, 5)
    taken = m.q8_write(X, want[0].clone(), want[1].clone(), None, None)
    assert taken == 0                                          # the native path, not a fallback
    for stream, W, seed in ((side, np.int64(7), np.uint64(5)), (side.cuda_stream, 7, 2 ** 64 + 5), (0, True * 7, 5)):
        for got, w in zip(everything(stream, W, seed), want):
            assert torch.equal(got, w)

    class Refusing:
        readable = staticmethod(m.readable)

        def __getattr__(self, name):
            return lambda *a: None

    monkeypatch.setattr(es.binding, "_marshal", Refusing())
    for stream in (None, side, side.cuda_stream):
        for got, w in zip(everything(stream, 7, 5), want):
            assert torch.equal(got, w)
