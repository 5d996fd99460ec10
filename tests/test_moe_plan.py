"""How w2_moe_experts cuts its rows and columns and its workspace (csrc/moe_plan.h, compiled by itself), walked on the CPU from one row
to the entry's largest sizes: bounds on what the kernels write, offsets that 32 bits reach, workspaces that no larger batch shrinks."""
import os
import shutil
import subprocess

import numpy as np
import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
PROGRAM = r"""
#include <cstdio>
#include "%s/paper_2508_06753_amd/csrc/moe_plan.h"
using namespace w2::moe;
int main()
{
    long long hidden, inter, E, G, M, k;
    while (scanf("%%lld %%lld %%lld %%lld %%lld %%lld", &hidden, &inter, &E, &G, &M, &k) == 6) {
        const long long rows = most_rows(hidden, inter, (int)k), m = M < rows ? M : rows, A = m * k;
        const Plan p = plan(hidden, inter, (int)E, (int)G, A);
        const Tiny t = tiny(hidden, inter, (int)E, (int)G, A);
        const Workspace w = workspace(hidden, inter, (int)E, (int)G, M, (int)k);
        printf("%%lld %%d %%d %%lld %%d %%d %%d %%d %%d %%d %%zu %%zu %%zu %%zu %%zu %%zu %%zu %%zu %%zu %%zu %%zu\n", rows, p.few, p.rows, (long long)p.tiles, p.ks_up, p.ks_down,
               t.fits, t.tiles, t.rows, t.units, t.lds, w.tiles, w.tile_rows, w.place, w.xs, w.xe, w.hs, w.he, w.z, w.ze, w.total);
    }
}
"""
SIZES = [(256, 256, 1, 64, 1), (256, 256, 1, 128, 64), (4096, 1024, 128, 128, 8), (4096, 14336, 8, 128, 2), (5120, 1280, 40, 64, 5), (2048, 768, 64, 128, 6),
         (131072, 131072, 1024, 128, 64), (131072, 256, 1024, 64, 1), (256, 131072, 7, 64, 64), (1280, 512, 24, 128, 10)]


@pytest.fixture(scope="module")
def walk(tmp_path_factory):
    if shutil.which("g++") is None:
        pytest.skip("no g++")
    d = tmp_path_factory.mktemp("moe_plan")
    (d / "p.cpp").write_text(PROGRAM % ROOT)
    subprocess.run(["g++", "-O1", "-std=c++17", "-Wall", "-Werror", "-o", str(d / "p"), str(d / "p.cpp")], check=True)

    def run(queries):
        text = "\n".join(" ".join(map(str, q)) for q in queries)
        out = subprocess.run([str(d / "p")], input=text, capture_output=True, text=True, check=True).stdout
        return [list(map(int, line.split())) for line in out.splitlines()]

    return run


def batches(k):
    top = (1 << 24) // k
    return sorted({m for m in list(range(1, 140)) + [2 ** b + d for b in range(7, 25) for d in (-1, 0, 1)] + [top] if 1 <= m <= top})


@pytest.mark.parametrize("hidden,inter,E,G,k", SIZES)
def test_workspace_and_bounds(walk, hidden, inter, E, G, k):
    ms = batches(k)
    last = 0
    for m, r in zip(ms, walk([(hidden, inter, E, G, m, k) for m in ms])):
        rows, few, tile, tiles, ks_up, ks_down, fits, t_tiles, t_rows, units, lds = r[:11]
        at, total = r[11:20], r[20]
        m = min(m, rows)                                      # rows that go together
        A = m * k
        assert total >= last, "a larger batch wants less"
        last = total
        # what the kernels write lies in its own part
        need = [256 + 16 * tiles, 4 * tiles * tile, 4 * A, 2 * m * hidden, m * hidden // 32, 2 * A * inter, A * inter // 32,
                A * hidden * (4 if few else 2), A * hidden // 32]
        for begin, size, end in zip(at, need, at[1:] + [total]):
            assert begin % 256 == 0 and begin + size <= end, (m, begin, size, end)
        # offsets of 32 bits, a grid's limits
        assert 2 * m * hidden <= 1 << 31 and 2 * A * inter <= 1 << 31 or m == 1
        assert tile in (8, 32) and ks_up in (1, 2) and ks_down in (1, 2)
        if fits:
            assert A <= 64 and lds <= 128 << 10 and t_rows == min(A, 8) and t_tiles <= 64 and m * 512 <= 1 << 15
            assert inter // 32 % units == 0 and t_rows >= min(m, 2)


def test_tiles_are_enough(walk):
    """However the choices fall on the experts, there are no more tiles than the plan says."""
    rng = np.random.default_rng(1)
    for hidden, inter, E, G, k in SIZES[:6] + SIZES[9:]:
        for m in (1, 2, 3, 7, 30, 100, 333, 2000):
            _, _, tile, tiles, *rest = walk([(hidden, inter, E, G, m, k)])[0]
            t_tiles = rest[3]
            for skew in (0.0, 1.0, 4.0):
                p = 1.0 / (1 + np.arange(E)) ** skew
                for A in {m * k, max(1, m * k // 3)}:         # some may be no one's
                    counts = np.bincount(rng.choice(E, A, p=p / p.sum()), minlength=E)
                    assert np.ceil(counts / tile).sum() <= tiles
                    if m * k <= 64:
                        assert np.ceil(counts / 8).sum() <= t_tiles
