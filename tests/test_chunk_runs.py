"""How the attention kernels for chunks share out their work, worked out on the host by the kernels' own sums and steps (chunk_runs.cu): whatever the lengths, a call's
runs have to begin with its first item, end with its last and lie in order within the items that there are, and no sum may leave its 32 bits."""
import ctypes as C
import os
import re
import subprocess

import numpy as np
import pytest

HERE = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(HERE)
CSRC = os.path.join(ROOT, "paper_2402_13720_b200", "csrc")
KEYS = 64


def constants(prefix, source):
    """Cost of an item, border and shortest run of a kernel, from its source."""
    text = open(os.path.join(CSRC, source)).read()
    assert re.search(r"KEYS = 64\b", text)
    cost = re.search(r"constexpr int ITEM_COST = (\d+), SNAP = (\d+), MIN_RUN = (\d+);", text)
    return [f"-D{prefix}_{n}={x}" for n, x in zip(("ITEM_COST", "SNAP", "MIN_RUN"), cost.groups())]


@pytest.fixture(scope="module")
def lib(tmp_path_factory):
    out = str(tmp_path_factory.mktemp("runs") / "chunk_runs.so")
    nvcc = os.environ.get("NVCC", "/usr/local/cuda/bin/nvcc")
    subprocess.run([nvcc, "-std=c++17", "-O1", "-Xcompiler", "-fPIC", "-shared", "-gencode", "arch=compute_100a,code=sm_100a", "-I", os.path.join(ROOT, "include"), "-I", CSRC,
                    *constants("TC", "paged_chunk_tc.cu"), *constants("ROW", "paged_chunk.cu"), "-o", out, os.path.join(HERE, "chunk_runs.cu")], check=True)
    f = C.CDLL(out).chunk_runs
    f.restype = C.c_int64
    f.argtypes = [C.c_int, C.c_void_p, C.c_void_p, C.c_int, C.c_int, C.c_int, C.c_int, C.c_int, C.c_int64, C.c_int, C.c_void_p]
    return f


def play(lib, tc, chunks, Hkv, group, cap, grid=None):
    R = 256 if tc else 64
    grid = grid or (148 if tc else 296)
    lens = np.array([n for n, _ in chunks], dtype=np.int32)
    starts = np.concatenate([[0], np.cumsum([m for _, m in chunks])]).astype(np.int32)
    rows, n = int(starts[-1]), len(chunks)
    tiles = -(-rows * group // 64) + min(n, rows)
    begins = np.zeros((grid + 1, 4), dtype=np.int32)
    total = lib(int(tc), lens.ctypes.data, starts.ctypes.data, n, rows, Hkv, group, cap, tiles, grid, begins.ctypes.data)
    assert 0 < total <= 2 ** 31 - 1
    at = [tuple(int(x) for x in b) for b in begins]
    first = next(i for i, (_, m) in enumerate(chunks) if m > 0)
    assert at[0] == (first, 0, 0, 0) and at[-1] == (n, 0, 0, 0)
    for i, (s, head, rt, unit) in enumerate(at):
        assert i == 0 or at[i] >= at[i - 1], i
        if s == n:
            assert (head, rt, unit) == (0, 0, 0)
            continue
        m, length = chunks[s][1], min(max(chunks[s][0], 0), cap)
        assert 0 <= head < Hkv and 0 <= rt < -(-m * group // R)
        seen = length - m + 1 + min(m * group - 1, rt * R + R - 1) // group
        assert unit == 0 or 0 < unit < -(-seen // KEYS)
        # what is cut: the run in front has the piece before, and is not empty
        assert unit == 0 or at[i - 1] < at[i]


CALLS = [
    # (len, new) of the sequences, kv heads, group, tokens of a row of the table
    ([(1, 1)], 1, 1, 16),
    ([(2048, 2048)], 32, 1, 2048),
    ([(24061, 61)], 8, 7, 24064),
    ([(5596, 4096), (1501, 1), (900, 800), (3000, 2000), (4100, 4000)], 8, 8, 5632),
    ([(0, 0), (300, 257), (1, 1), (0, 0), (256, 256)], 1, 8, 320),
    ([(60 + i, i % 4) for i in range(1024)], 1, 2, 1088),
    ([(20, 30), (0, 4), (1, 2), (64, 65)], 2, 2, 80),
]
# Far more new rows than a row of the table holds.
CROWDED = [
    ([(16, 46500)], 8, 8, 16),
    ([(1024, 46500)], 8, 8, 1024),
    ([(128, 24000)], 8, 8, 128),
    ([(1024, 70000)], 4, 8, 1024),
    ([(64, 17000)], 1, 64, 64),
    ([(64, 166000)], 8, 8, 64),
    ([(256, 90000)], 8, 8, 256),
    ([(0, 1 << 20), (16, 16), (16, 1 << 20)], 2, 1, 16),
    ([(100, 1 << 27), (7, 7)], 1, 8, 128),
]


@pytest.mark.parametrize("tc", [True, False])
@pytest.mark.parametrize("chunks,Hkv,group,cap", CALLS)
def test_runs(lib, tc, chunks, Hkv, group, cap):
    for grid in (1, 2, 7, None):
        play(lib, tc, chunks, Hkv, group, cap, grid)


@pytest.mark.parametrize("tc", [True, False])
@pytest.mark.parametrize("chunks,Hkv,group,cap", CROWDED)
def test_runs_of_more_new_rows_than_there_is_room_for(lib, tc, chunks, Hkv, group, cap):
    play(lib, tc, chunks, Hkv, group, cap)


# A table whose rows have room for a very long text, short sequences, and many rows.
WIDE = [
    ([(1, 1), (3, 2), (5000, 4000)], 8, 1, 1 << 30),
    ([(1, 1)] * 1024, 32, 1, 1 << 30),
    ([(2, 2), (0, 0), (7, 7), (1 << 20, 1 << 16), (1, 1)], 4, 2, 1 << 29),
    ([(1, 1), (100, 60000), (5, 5)], 128, 1, 1 << 28),
]


@pytest.mark.parametrize("tc", [True, False])
@pytest.mark.parametrize("chunks,Hkv,group,cap", WIDE)
def test_runs_of_short_sequences_in_a_wide_table(lib, tc, chunks, Hkv, group, cap):
    for grid in (1, 3, None):
        play(lib, tc, chunks, Hkv, group, cap, grid)
