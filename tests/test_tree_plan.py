"""How the attention of drafted tokens is cut up (csrc/tree_plan.h, compiled by itself), up to the largest sizes that its entry takes."""
import os
import shutil
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def compiled(tmp_path_factory, name, program):
    if shutil.which("g++") is None:
        pytest.skip("no g++")
    d = tmp_path_factory.mktemp(name)
    (d / "p.cpp").write_text(f'#include "{ROOT}/paper_2508_06753_amd/csrc/tree_plan.h"\n' + program)
    subprocess.run(["g++", "-O2", "-fwrapv", "-std=c++17", "-o", str(d / "p"), str(d / "p.cpp")], check=True)
    return subprocess.run([str(d / "p")], capture_output=True, text=True, check=True).stdout.splitlines()


SHARES = r"""
#include <stdio.h>
#include <algorithm>
using namespace w2;
int main()
{
    // packed rows of a request: small ones all, then single cases up to what a grid of 2^24 - 1 workgroups of 128 rows counts
    const auto walk = [](long long rows, int W) {
        const int all = (int)((rows + 31) / 32), tiles = (all + W - 1) / W;
        long long next = 0, bad = 0;
        for (int t = 0; t < tiles; ++t) {
            const tree::Share s = tree::share(all, tiles, t);
            bad += s.first != next || s.count < 1 || s.count > W;
            next = (long long)s.first + s.count;
        }
        printf("%lld %d %lld %lld\n", rows, W, bad, all - next);
    };
    for (int W : {2, 4}) {
        for (long long rows = 1; rows <= 2000; rows += 13) walk(rows, W);
        for (long long rows : {71ll * 42000, 128ll * 23200, 16ll * 186000, 8ll * 371000, 131072ll * 32, (1ll << 24) * 8, ((1ll << 24) - 1) * 32 * W, ((1ll << 24) - 1) * 32 * W - 100})
            walk(rows, W);
    }
}
"""


def test_every_wave_of_rows_is_in_one_tile(tmp_path_factory):
    lines = [tuple(map(int, l.split())) for l in compiled(tmp_path_factory, "share", SHARES)]
    assert len(lines) > 300
    for rows, waves, bad, left in lines:
        assert bad == 0 and left == 0, f"{rows} packed rows, {waves} waves a tile: {bad} tiles are wrong, {left} waves are left over"


PLANS = r"""
#include <stdio.h>
using namespace w2;
int main()
{
    const long long INT_MAX_ = (1ll << 31) - 1;
    for (long long len : {0ll, 1ll, 127ll, 128ll, 129ll, 5000ll, 120000ll, 1ll << 20, 1ll << 30, INT_MAX_ - 128, INT_MAX_ - 127, INT_MAX_ - 126, INT_MAX_ - 1, INT_MAX_})
        for (long long rows : {1ll, 2ll, 4ll, 9ll, 64ll, 1000ll, 1ll << 20})
            for (int G : {1, 4, 16})
                for (int D : {8, 64, 128, 256})
                    for (long long requests : {1ll, 40ll, 65535ll})
                        for (long long room : {0ll, 1ll, 2ll, 3ll, 7ll, 127ll, 128ll}) {
                            tree::Plan p = tree::make_plan(requests, rows, G, 8, D, len, 0);
                            const tree::Plan wish = p;
                            tree::fit(p, len, room);
                            const bool ok = p.chunks >= 1 && p.chunks <= std::max(1ll, room) && p.chunk >= 128 && p.chunk % 128 == 0 &&
                                            p.chunk <= (1u << 31) && (long long)p.chunk * p.chunks >= len &&
                                            (p.chunks == 1 || (long long)p.chunk * (p.chunks - 1) < len) &&
                                            wish.chunks <= tree::MAX_CHUNKS && (room < wish.chunks || (p.chunk == wish.chunk && p.chunks == wish.chunks));
                            if (!ok) printf("%lld keys, %lld rows of %d heads of %d, %lld requests, room for %lld: %d chunks of %u\n", len, rows, G, D, requests, room, p.chunks, p.chunk);
                        }
    printf("done\n");
}
"""


def test_chunks_are_no_more_than_there_is_room_for(tmp_path_factory):
    """Every key is in one chunk, whatever the longest request: parts of more chunks than the workspace holds would be written
    behind it."""
    lines = compiled(tmp_path_factory, "plans", PLANS)
    assert lines == ["done"], lines[:5]


WIDE = r"""
#include <stdio.h>
using namespace w2;
int main()
{
    // limits as wide as they go: more units than run at once by far
    for (long long rows : {1ll << 17, 1ll << 20, (1ll << 20) + 77, (1ll << 21) - 16, (1ll << 24) - 128, 1ll << 24})
        for (int G : {1, 16, 128})
            for (int n_kv : {1, 8, 1024 / G}) {
                const tree::Plan p = tree::make_plan(65535, rows, G, n_kv, 8, (1ll << 31) - 1, 0);
                printf("%lld %d %d %d\n", rows, G, n_kv, p.chunks);
            }
}
"""


def test_plans_of_the_widest_limits(tmp_path_factory):
    """Keys times heads times tiles pass 64 bits there.  Workgroups that are to hold them are at most two a unit and one round, so a
    chunk has half of the longest request or more; a product that wrapped would cut the keys to pieces."""
    for line in compiled(tmp_path_factory, "wide", WIDE):
        assert int(line.split()[3]) <= 2, line
