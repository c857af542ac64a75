"""The cut of an attention call into pieces, replayed on the CPU: whatever the
launch was planned for, the pieces cover the tiles' steps once, and the joining
launch reads the sums that a workgroup wrote and no others."""
import ctypes
import os
import shutil
import subprocess

import numpy as np
import pytest

HERE = os.path.dirname(os.path.abspath(__file__))


@pytest.fixture(scope="module")
def cut(tmp_path_factory):
    compiler = shutil.which("g++") or shutil.which("clang++") or "/opt/rocm/bin/amdclang++"
    so = str(tmp_path_factory.mktemp("cut") / "libcut_model.so")
    subprocess.run([compiler, "-O1", "-std=c++17", "-shared", "-fPIC", os.path.join(HERE, "cut_model.cpp"), "-o", so],
                   check=True)
    return ctypes.CDLL(so)


def replay(cut, steps, workgroups):
    """`steps` of each tile that has some: the sums written (workgroup, begins a
    tile), those read for each tile, and how often each step is done."""
    total = sum(steps)
    first = np.concatenate([[0], np.cumsum(steps)])
    n = cut.cut_n(total, workgroups)
    assert 0 < n <= workgroups and n <= total
    done = np.zeros(total, int)
    written, pieces, whole = set(), {}, set()
    for w in range(n):
        at, end = cut.cut_start(total, workgroups, w), cut.cut_start(total, workgroups, w + 1)
        assert at < end
        done[at:end] += 1
        tile = int(np.searchsorted(first, at, "right")) - 1
        parts = 0
        while at < end:
            u0, u1 = at - first[tile], min(steps[tile], end - first[tile])
            part = u0 != 0 or u1 != steps[tile]
            if part:
                slot = 2 * w + (u0 == 0)
                assert slot not in written
                written.add(slot)
                parts += 1
            else:
                whole.add(tile)
            if u0 == 0:
                pieces[tile] = (w, cut.cut_owner(total, workgroups, int(first[tile + 1]) - 1) if part else w)
            at = first[tile] + u1
            tile += 1
        assert parts <= 2
    assert cut.cut_start(total, workgroups, n) == total and np.all(done == 1)
    read = []
    for tile in range(len(steps)):
        w0, w1 = pieces[tile]
        assert (w1 == w0) == (tile in whole)
        if w1 > w0:
            read += [2 * (w0 + i) + (i == 0) for i in range(w1 - w0 + 1)]
    assert len(read) == len(set(read)) and set(read) == written


PLANNED = [  # steps of the tiles, workgroups launched
    ([19] * 4, 300), ([19] * 16, 768), ([16] * 8, 768), ([5] * 32, 512), ([1], 768), ([1], 1),
    ([19, 19, 21, 20] * 2, 210), ([259] * 8 + [1] * 100, 512), ([7] * 300, 512), ([1] * 511, 512),
    ([1 << 20] * 40, 768), ([(1 << 31) - 2], 768),
]


@pytest.mark.parametrize("case", PLANNED[:-2])
def test_pieces_of_planned_calls(cut, case):
    replay(cut, *case)


def test_pieces_of_any_call(cut):
    rng = np.random.default_rng(0)
    for _ in range(300):
        steps = np.maximum(1, rng.geometric(1.0 / rng.integers(1, 40), rng.integers(1, 200))).tolist()
        replay(cut, steps, int(rng.integers(1, 900)))


def test_steps_up_to_31_bits(cut):
    for steps, workgroups in PLANNED[-2:]:
        total = sum(steps)
        n = cut.cut_n(total, workgroups)
        assert n == workgroups
        starts = [cut.cut_start(total, workgroups, w) for w in range(n + 1)]
        assert starts == [w * total // n for w in range(n + 1)]
        for step in (0, 1, total // 3, total - 1):
            w = cut.cut_owner(total, workgroups, step)
            assert starts[w] <= step < starts[w + 1]


def test_no_steps(cut):
    assert cut.cut_n(0, 768) == 0
