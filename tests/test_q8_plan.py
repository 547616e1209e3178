"""What the host decides for the operators on 8-bit rows, without a GPU: tests/q8_plan.cpp is the host source itself
with every launch printed instead of made, built with UBSan in trap mode (undefined behaviour in the
planning arithmetic ends the process, and the test with it)."""
import os
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
FULL, BUCKET, FASTRAND = 0, 1, 2


@pytest.fixture(scope="module")
def ask(tmp_path_factory):
    """ask(queries) -> one line of answer per query, each a tuple (what, number, ...)."""
    from paper_2104_10716_amd import build
    out = str(tmp_path_factory.mktemp("q8_plan") / "q8_plan")
    flags = [f for f in build.HIPCC_FLAGS if f not in ("-O3", "-shared", "-fPIC", "-Wall", "-Wextra")]
    subprocess.run([os.environ.get("HIPCC", "/opt/rocm/bin/hipcc"), "-O1", "-w"] + flags +
                   ["-Xarch_host", "-fsanitize=undefined,integer-divide-by-zero,float-cast-overflow",
                    "-Xarch_host", "-fsanitize-trap=all", "-x", "hip", os.path.join(ROOT, "tests", "q8_plan.cpp"), "-o", out],
                   check=True, capture_output=True, text=True)

    def run(queries):
        text = "".join(" ".join(str(x) for x in q) + "\n" for q in queries)
        res = subprocess.run([out], input=text, capture_output=True, text=True, timeout=300)
        lines = res.stdout.splitlines()
        assert res.returncode == 0 and len(lines) == len(queries), \
            f"ended with {res.returncode} at {queries[len(lines)] if len(lines) < len(queries) else None}"
        return lines
    return run


def plans(ask, queries):
    out = []
    for line in ask([("plan",) + q for q in queries]):
        words = line.split()
        out.append(dict(zip(words[::2], map(int, words[1::2]))))
    return out


def sweep():
    """(N, nnz, F, W, mode, n_rows) over the whole range, dense small graphs and wide rows among them."""
    for N in (1, 3, 513, 2700, 10_000, 15_000, 20_000, 60_000, 200_000, 700_000, 2_450_000, 40_000_000, 2 ** 31 - 1):
        for mean in (0.0, 1.0, 4.6, 14.0, 42.0, 50.0, 256.0, 300.0, 490.0, 1400.0, 9000.0, 200_000.0):
            nnz = int(N * mean)
            if nnz >= 2 ** 31 or mean > 64 * N:
                continue
            for F in (1, 16, 41, 64, 100, 128, 256, 300, 602, 1040, 2304, 2500, 9000, 1_000_000, 16_000_000):
                for W, mode in ((0, FULL), (4, BUCKET), (64, FASTRAND), (129, BUCKET), (1024, BUCKET), (1025, FASTRAND), (1500, FASTRAND),
                                (1500, BUCKET), (5000, BUCKET), (20_000, FASTRAND), (2 ** 31 - 1, FASTRAND)):
                    for n_rows in {1, 32, 512, 513, 2000, 100_000, N}:
                        yield N, nnz, F, W, mode, n_rows


def test_rows_that_the_join_sums_are_rows_that_were_cut(ask):
    """The join takes every row that keeps more than `piece` entries.  All of those have to be long rows (more than
    `long_k`), which workgroups cut and whose sums they leave in the workspace; a wave stores any other row by itself."""
    queries = list(sweep())
    cut = 0
    for q, p in zip(queries, plans(ask, queries)):
        N, nnz, F, W, mode, n_rows = q
        if p["few"] or not p["pieces"]:
            continue
        cut += 1
        assert p["piece"] >= p["long_k"], (q, p)               # more than `piece` is more than `long_k`
        assert p["long_blocks"] > 0, (q, p)                    # and there is somebody to cut them
        most = nnz if mode == FULL else min(W, nnz)
        assert p["piece"] < most, (q, p)
        assert p["pieces"] == 2 * (nnz // p["piece"] + 1), (q, p)      # a place for either end of every span
    assert cut > 10_000


def test_rows_that_wait_in_lds_fit(ask):
    """A wave holds up to 64 rows, as many at least as run side by side."""
    queries = list(sweep())[::7]
    for q, p in zip(queries, plans(ask, queries)):
        if not p["few"]:
            assert p["team"] in (4, 8, 16, 32, 64) and p["team"] >= p["G"], (q, p)
            assert 64 // p["team"] <= p["wave_rows"] <= 64, (q, p)
            assert p["nblocks"] * 4 * p["wave_rows"] >= q[5], (q, p)
        else:
            assert 1 <= p["splits"] <= 64 and p["grid_x"] == q[5] * p["splits"], (q, p)


def test_the_asked_workspace_is_the_planned_one(ask):
    queries = list(sweep())[::11]
    for q, p, size in zip(queries, plans(ask, queries), ask([("bytes",) + q for q in queries])):
        assert int(size) == 4 * q[2] * p["pieces"], (q, p)


def launches(line, fields):
    """(status, [(blocks, threads, ...)]) of an answer."""
    words = list(map(int, line.split()))
    rest = words[1:]
    assert len(rest) % fields == 0, line
    return words[0], [tuple(rest[i:i + fields]) for i in range(0, len(rest), fields)]


def test_every_launch_has_fewer_than_2_to_32_threads(ask):
    """That is what a launch can hold along x.  Beyond it a call is refused before its first launch."""
    many = (1, 5000, 2_450_000, 2 ** 24, 20_000_000, 70_000_000, 300_000_000, 700_000_000, 900_000_000, 2 ** 31 - 1)
    queries = []
    for N in many:
        for F in (1, 16, 100, 256, 1000, 4000):
            for nnz in (N // 2 + 1, N, min(3 * N, 2 ** 31 - 1), 2 ** 31 - 1):
                for W, mode in ((0, FULL), (4, BUCKET), (900, FASTRAND), (5000, FASTRAND)):
                    queries.append(("vals", N, nnz, F, W, mode))
                    queries += [("spmm", N, nnz, F, W, mode, n, ws) for n in (1, 512, N) for ws in (0, 1)]
            queries += [("grad", N, F, H, ws) for H in (1, 100, 5000, 2_000_000) for ws in (0, 1)]
    queries += [("grad", 100, F, H, 1) for F in (1, 100, 2 ** 26, 2 ** 27 - 16) for H in (1, 2 ** 20, 2 ** 26 - 1)]
    served = refused = 0
    for q, line in zip(queries, ask(queries)):
        status, made = launches(line, 2)
        assert status in (0, -2), (q, line)
        assert (status == 0) == (len(made) > 0), (q, line)
        assert all(0 < blocks * threads < 2 ** 32 for blocks, threads in made), (q, line)
        if q[1] <= 700_000_000 and q[0] != "grad":
            assert status == 0, (q, line)
        served += status == 0
        refused += status == -2
    assert served > 1000 and refused > 20


def test_long_lists_of_rows_are_written_and_read_in_order(ask):
    """Whole tables and lists of ids in one launch after the other, none too large, none left out."""
    queries = [(what, kind, n, F, ids, n) for what in ("write", "read") for kind in (0, 1, 2) for ids in (0, 1)
               for n in (1, 4000, 2 ** 23 - 2, 2 ** 24 - 1, 2 ** 24, 2 ** 25 + 3, 700_000_000, 2 ** 31 - 1)
               for F in (1, 16, 64, 100, 128, 300, 600, 700, 1024, 1500, 2048, 2049, 4096, 100_000)]
    for q, line in zip(queries, ask(queries)):
        status, made = launches(line, 4)
        assert status == 0 and made, (q, line)
        assert all(0 < blocks * threads < 2 ** 32 for blocks, threads, _, _ in made), (q, line)
        marks = q[0] == "write" and q[4] and len(made) % 3 == 0 and q[2] > 3200
        pieces = made[2::3] if marks else made
        done = 0
        for blocks, threads, rows, first in pieces:
            assert first == (0 if q[4] else done), (q, line)
            done += rows
        assert done == q[2], (q, line)


def test_staged_entries_are_aligned_for_16_byte_reads(tmp_path):
    """Staged entries are read from LDS 16 bytes at a time: the arrays that hold them say so, wherever the compiler lays them."""
    import re
    from paper_2104_10716_amd import build
    src = tmp_path / "aligned.hip"
    src.write_text('#include "es_q8_spmm.h"\nnamespace {\n'
                   'template __global__ void es_q8_few_kernel<4, false>(const Q8Args);\n'
                   'template __global__ void es_q8_spmm_kernel<4, 32, true, false>(const Q8Args);\n'
                   'template __global__ void es_q8_spmm_kernel<1, 4, false, false>(const Q8Args);\n}\n')
    out = str(tmp_path / "aligned.ll")
    flags = [f for f in build.HIPCC_FLAGS if f not in ("-O3", "-shared", "-fPIC", "-Wall", "-Wextra")]
    subprocess.run([os.environ.get("HIPCC", "/opt/rocm/bin/hipcc"), "-w", "-O1", "-Xclang", "-disable-llvm-passes"] + flags +
                   ["--cuda-device-only", "-S", "-emit-llvm", str(src), "-o", out], check=True, capture_output=True)
    arrays = re.findall(r"^@(\S*E3lds) = .*addrspace\(3\) global .*, align (\d+)", open(out).read(), re.M)
    assert len(arrays) == 3, arrays
    assert all(int(align) >= 16 for _, align in arrays), arrays
