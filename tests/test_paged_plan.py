"""How the paged attention's work is cut, and division by a page's length, checked on the host: csrc/paged_plan.cuh is
compiled with a host compiler and run for many problems."""
import ctypes
import os
import random
import subprocess

import numpy as np
import pytest

HERE = os.path.dirname(os.path.abspath(__file__))
COST = 1                            # what an item costs beside its steps


@pytest.fixture(scope="module")
def lib(tmp_path_factory):
    so = str(tmp_path_factory.mktemp("plan") / "paged_plan.so")
    subprocess.run(["g++", "-std=c++17", "-O1", "-shared", "-fPIC", "-o", so, os.path.join(HERE, "paged_plan_host.cpp")], check=True)
    return ctypes.CDLL(so)


def ptr(a):
    return a.ctypes.data_as(ctypes.c_void_p)


def test_division_by_a_page(lib):
    rng = random.Random(1)
    top = 2 ** 31 - 1
    for d in list(range(1, 300)) + [1560, 4680, 65535, 65536, 65537, 2 ** 30 - 1, 2 ** 30, 2 ** 30 + 1, top] + [rng.randint(1, top) for _ in range(300)]:
        n = [0, 1, d - 1, d, d + 1, top, top - 1, top // d * d, top // d * d - 1] + [rng.randint(0, top) for _ in range(200)]
        n += [k * d + e for k in (1, 2, 3, 1000) for e in (-1, 0, 1)]
        n = np.array([v for v in n if 0 <= v <= top], dtype=np.uint32)
        assert lib.divides(ctypes.c_uint32(d), ptr(n), len(n)), d


def check(lib, steps, grid):
    """Every step is some CTA's, the pieces that an item's CTAs count on are those that there are, each CTA ends at most one
    item that others began and begins at most one that others end, and no CTA has much more than an even share."""
    steps = np.array(steps, dtype=np.int32)
    out, pieces, snap = np.zeros(2 * grid, dtype=np.int64), np.zeros((len(steps), 2), dtype=np.int32), ctypes.c_int32(0)
    n = lib.plan(len(steps), ptr(steps), grid, ptr(out), ptr(pieces), ctypes.byref(snap))
    assert 1 <= n <= grid and snap.value >= 1
    starts, ends = out[0:2 * n:2], out[1:2 * n:2]
    end_of = np.cumsum(steps.astype(np.int64) + COST)
    all_ = int(end_of[-1])
    assert starts[0] == 0 and ends[-1] == all_ and np.array_equal(starts[1:], ends[:-1]) and np.all(ends >= starts)
    share = all_ / n
    assert (ends - starts).max() <= share + 1 + 2 * snap.value
    at = 0
    for i, s in enumerate(steps):
        s = int(s)
        lo = int(np.searchsorted(ends, at, side="right"))                 # the CTA that holds the item's first position
        mine, k = [], lo
        while k < n and starts[k] < at + s:
            a, b = max(int(starts[k]) - at, 0), min(int(ends[k]) - at, s)
            if a < b:
                mine.append((k, a, b))
            k += 1
        assert mine[0][1] == 0 and mine[-1][2] == s and all(x[2] == y[1] for x, y in zip(mine, mine[1:]))
        if len(mine) == 1:
            assert pieces[i, 1] <= 1, (i, mine, pieces[i])
        else:
            assert pieces[i].tolist() == [mine[0][0], len(mine)], (i, mine, pieces[i])
            assert [k for k, _, _ in mine] == list(range(mine[0][0], mine[0][0] + len(mine)))
            assert min(b - a for _, a, b in mine) >= min(snap.value - COST + 1, 1)
        at += s + COST


@pytest.mark.parametrize("grid", [1, 2, 148, 296, 444, 1024])
def test_every_step_is_taken_once(lib, grid):
    rng = random.Random(grid)
    for steps in ([1], [2], [3126] * 4, [1] * 600, [3] * 600, [17] * 1024, [100000], [1, 100000, 1], [40000000, 1, 30000000]):
        check(lib, steps, grid)
    for _ in range(150):
        top = rng.choice([1, 2, 5, 20, 200, 5000])
        check(lib, [rng.randint(1, top) for _ in range(rng.choice([1, 2, 7, 50, 700]))], grid)
