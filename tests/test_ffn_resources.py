"""What the built kernels of a layer's feed-forward half ask of a CU, as the library's own code objects say (their metadata): local memory
that a launch has to declare, scratch memory.  Read from the built library on the CPU."""
import os
import shutil
import struct
import subprocess

import pytest

msgpack = pytest.importorskip("msgpack")

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
LIB = os.path.join(ROOT, "paper_2508_06753_amd", "libw2mm.so")


def code_objects(data):
    """The device code objects of the bundles in a library: magic, number of entries, then offset, size and name of each."""
    magic, at = b"__CLANG_OFFLOAD_BUNDLE__", 0
    while (at := data.find(magic, at)) >= 0:
        here, n = at + len(magic) + 8, struct.unpack_from("<Q", data, at + len(magic))[0]
        for _ in range(n):
            offset, size, length = struct.unpack_from("<QQQ", data, here)
            if b"gfx950" in data[here + 24:here + 24 + length]:
                yield data[at + offset:at + offset + size]
            here += 24 + length
        at = here


def notes(elf):
    """The AMDGPU metadata of a 64-bit code object: note type 32 of a section of notes (type 7)."""
    begin, (size, count) = struct.unpack_from("<Q", elf, 40)[0], struct.unpack_from("<HH", elf, 58)
    for i in range(count):
        kind, at, length = struct.unpack_from("<I", elf, begin + i * size + 4)[0], *struct.unpack_from("<QQ", elf, begin + i * size + 24)
        if kind != 7:
            continue
        end = at + length
        while at + 12 <= end:
            name, desc, what = struct.unpack_from("<III", elf, at)
            body = at + 12 + (name + 3) // 4 * 4
            if what == 32:
                yield msgpack.unpackb(elf[body:body + desc], strict_map_key=False)
            at = body + (desc + 3) // 4 * 4


@pytest.fixture(scope="module")
def kernels():
    if not os.path.exists(LIB):
        pytest.skip("nothing built")
    with open(LIB, "rb") as f:
        data = f.read()
    found = {k[".name"]: k for elf in code_objects(data) for note in notes(elf) for k in note["amdhsa.kernels"]}
    assert len(found) > 100
    return found


def named(kernels, name):
    some = {n: k for n, k in kernels.items() if name in n}
    assert some, name
    return some


@pytest.mark.parametrize("name", ["moe_tiny_up_kernel", "moe_few_kernel"])
def test_local_memory_is_all_declared_at_the_launch(kernels, name):
    """Kernels that may ask for more than 64 KiB of local memory have none beside what the launch names: the opt-in sees all of it."""
    for n, k in named(kernels, name).items():
        assert k[".group_segment_fixed_size"] == 0, n


TINY = r"""
#include <cstdio>
#include "%s/paper_2508_06753_amd/csrc/moe_plan.h"
int main()
{
    long long hidden, inter, E, G, A;
    while (scanf("%%lld %%lld %%lld %%lld %%lld", &hidden, &inter, &E, &G, &A) == 5) {
        const w2::moe::Tiny t = w2::moe::tiny(hidden, inter, (int)E, (int)G, A);
        printf("%%d %%d %%zu %%zu\n", t.fits, t.rows, t.lds, t.lds_all);
    }
}
"""


def test_two_launches_declare_rows_and_what_leaves(tmp_path):
    """Sums of three ranges of K of two pairs of blocks (2 KiB each), eight choices, and the rows: within a CU's 160 KiB."""
    if shutil.which("g++") is None:
        pytest.skip("no g++")
    (tmp_path / "p.cpp").write_text(TINY % ROOT)
    subprocess.run(["g++", "-O1", "-std=c++17", "-Wall", "-Werror", "-o", str(tmp_path / "p"), str(tmp_path / "p.cpp")], check=True)
    cases = [(hidden, 256, 8, G, A) for hidden in range(256, 1 << 17, 256) for G in (64, 128) for A in (1, 2, 4, 6, 7, 8, 9, 64)]
    out = subprocess.run([str(tmp_path / "p")], input="\n".join(" ".join(map(str, c)) for c in cases), capture_output=True, text=True, check=True).stdout
    window = 0
    for (hidden, _, _, _, A), line in zip(cases, out.splitlines()):
        fits, rows, lds, everything = map(int, line.split())
        assert rows == min(A, 8) and lds == rows * (2 * hidden + 16 + hidden // 32)
        assert everything == lds + 3 * 2 * 2048 + 8 * 4
        assert not fits or everything <= 160 << 10
        window += fits and lds <= 64 << 10 < everything
    assert window                                             # sizes whose rows alone need no opt-in


def test_kernel_for_many_rows_keeps_nothing_in_scratch(kernels):
    for n, k in named(kernels, "moe_tile_kernel").items():
        assert k[".private_segment_fixed_size"] == 0 and k[".vgpr_spill_count"] == 0 and k[".sgpr_spill_count"] == 0, n


def test_norm_keeps_a_row_in_registers(kernels):
    for n, k in named(kernels, "residual_norm_kernel").items():
        assert k[".private_segment_fixed_size"] == 0 and k[".vgpr_spill_count"] == 0, n


# ------------------------------------------------------------------ the counted waits of the kernel for many rows
class Wave:
    """Vector memory operations in the order in which they are asked for, and so complete."""

    def __init__(self):
        self.issued, self.landed = [], 0

    def load(self, what, n=1):
        self.issued += [what] * n

    def wait(self, left):
        self.landed = max(self.landed, len(self.issued) - left)

    def has(self, what):
        return what in self.issued and what not in self.issued[self.landed:]


COUNTS = r"""
#include <cstdio>
#include "%s/paper_2508_06753_amd/csrc/moe_plan.h"
using namespace w2::moe;
int main()
{
    for (int rt = 1; rt <= 2; ++rt) printf("%%d %%d %%d %%d\n", TILE_AHEAD, tile_weights(rt), tile_at_start(rt), tile_at_stage(rt));
}
"""


def tile_stages(rt, n_kt, ahead, weights, at_start, at_stage):
    """-> whether every stage's rows have landed at the barrier in front of their first reads."""
    w = Wave()
    w.load("weights", weights)
    for s in range(ahead):
        w.load(s, rt)
    w.load("weights", weights)
    w.wait(at_start)
    ok = w.has(0)
    for s in range(2 * n_kt):
        w.wait(at_stage)
        ok &= w.has(s + 1)
        w.load(s + ahead, rt)
        if s % 2:
            w.load("weights", weights)
    return ok


def test_counts_of_the_kernel_for_many_rows(tmp_path):
    if shutil.which("g++") is None:
        pytest.skip("no g++")
    (tmp_path / "p.cpp").write_text(COUNTS % ROOT)
    subprocess.run(["g++", "-O1", "-std=c++17", "-o", str(tmp_path / "p"), str(tmp_path / "p.cpp")], check=True)
    lines = subprocess.run([str(tmp_path / "p")], capture_output=True, text=True, check=True).stdout.splitlines()
    for rt, line in enumerate(lines, 1):
        counts = list(map(int, line.split()))
        assert counts[1] == 4 + 4 + rt and max(counts) < 64   # (what a wait can count)
        for n_kt in range(1, 9):
            assert tile_stages(rt, n_kt, *counts)
            for i in (2, 3):                                  # (the walk sees a count that is too high)
                assert not tile_stages(rt, n_kt, *(c + (j == i) for j, c in enumerate(counts)))


OBJDUMP = "/opt/rocm/llvm/bin/llvm-objdump"


def instructions(elf, name, tmp_path):
    """{address: (instruction, address of the next one, target of a branch)} of a kernel of a code object, and where it begins."""
    path = tmp_path / "object"
    path.write_bytes(elf)
    text = subprocess.run([OBJDUMP, "-d", "--disassemble-symbols=" + name, str(path)], capture_output=True, text=True, check=True).stdout
    found, order, start = {}, [], None
    for line in text.splitlines():
        if line.endswith(">:"):
            start = int(line.split()[0], 16)
        elif "//" in line:
            code, _, rest = line.partition("//")
            at = int(rest.split(":")[0], 16)
            target = None
            if "branch" in code.split()[0]:
                target = start + int(rest.rsplit("+0x", 1)[1].rstrip(">"), 16) if "+0x" in rest else start
            order.append(at)
            found[at] = code.strip(), target
    return {at: (*found[at], after) for at, after in zip(order, order[1:] + [None])}, order[0]


def paths(code, at, most=3):
    """Every way through a kernel's branches, each instruction at most `most` times: the vector memory operations, counted waits and
    barriers on it, in order."""
    todo = [(at, (), {})]
    while todo:
        at, events, seen = todo.pop()
        events = list(events)
        while at is not None:
            text, target, after = code[at]
            op = text.split()[0]
            if op.startswith(("buffer_", "global_", "flat_", "scratch_")):
                events.append("rows" if text.endswith("lds") else op)
            elif op == "s_waitcnt" and "vmcnt" in text:
                events.append(int(text.split("vmcnt(")[1].split(")")[0]))
            elif op == "s_barrier":
                events.append("barrier")
            elif op.startswith("s_waitcnt_") or op.startswith("s_setpc"):
                raise AssertionError(text)
            elif op == "s_endpgm":
                yield events
                break
            elif op == "s_branch":
                after = target
            elif target is not None:
                seen = {**seen, at: seen.get(at, 0) + 1}
                if seen[at] > most:
                    break
                todo.append((target, tuple(events), seen))
            at = after


def test_built_kernel_for_many_rows_waits_for_its_rows(kernels, tmp_path):
    """The compiled kernels' own order of loads, walked along every way through them: at the first barrier the first stage's rows have
    landed, at each one behind it another stage's, or all that were ever asked for."""
    if not os.path.exists(OBJDUMP):
        pytest.skip("no llvm-objdump")
    with open(LIB, "rb") as f:
        elves = list(code_objects(f.read()))
    names = set(named(kernels, "moe_tile_kernel"))
    walked = 0
    for elf in elves:
        for name in names & {k[".name"] for note in notes(elf) for k in note["amdhsa.kernels"]}:
            code, start = instructions(elf, name, tmp_path)
            stages = set()
            for events in paths(code, start):
                if "rows" not in events:                      # no tile for this workgroup
                    continue
                rt = events[:events.index("barrier")].count("rows") // 3
                assert rt in (1, 2) and not any(str(e).startswith("scratch") for e in events)
                issued = landed = barriers = 0
                rows = []                                     # which operation each load of rows is
                for e in events:
                    if e == "barrier":
                        ready = sum(r < landed for r in rows)
                        assert landed == issued or ready >= (barriers + 1) * rt, (name, barriers, ready)
                        barriers += 1
                    elif isinstance(e, int):
                        landed = max(landed, issued - e)
                    else:
                        if e == "rows":
                            rows.append(issued)
                        issued += 1
                stages.add((rt, len(rows) // rt - 3))
            walked += 1
            # both heights; 256 of K (two stages) and more, an odd number of them and an even one
            assert {(rt, n) for rt in (1, 2) for n in (2, 4, 6, 8, 10)} <= stages, sorted(stages)
    assert walked == len(names) == 4


# ------------------------------------------------------------------ which kernels the tests' sizes reach
REACH = r"""
#include <cstdio>
#include "%s/paper_2508_06753_amd/csrc/moe_plan.h"
using namespace w2::moe;
int main()
{
    long long hidden, inter, E, G, A;
    while (scanf("%%lld %%lld %%lld %%lld %%lld", &hidden, &inter, &E, &G, &A) == 5) {
        const Tiny t = tiny(hidden, inter, (int)E, (int)G, A);
        const Plan p = plan(hidden, inter, (int)E, (int)G, A);
        printf("%%d %%d %%d %%d %%d\n", t.fits, t.units, p.few, p.ks_up, p.ks_down);
    }
}
"""


def test_sizes_reach_the_kernels_that_they_are_for(tmp_path):
    if shutil.which("g++") is None:
        pytest.skip("no g++")
    from test_ffn_edges import SPLIT, UNITS, WAYS
    (tmp_path / "p.cpp").write_text(REACH % ROOT)
    subprocess.run(["g++", "-O1", "-std=c++17", "-o", str(tmp_path / "p"), str(tmp_path / "p.cpp")], check=True)

    def reach(hidden, inter, E, G, A):
        text = subprocess.run([str(tmp_path / "p")], input=f"{hidden} {inter} {E} {G} {A}", capture_output=True, text=True, check=True).stdout
        return list(map(int, text.split()))

    for G in (64, 128):
        seen = set()
        for hidden, inter, E, k, M in SPLIT:
            fits, _, few, up, down = reach(hidden, inter, E, G, M * k)
            assert not fits and few and (up, down) == (2 if hidden >= 2048 else 1, 2 if inter >= 2048 else 1)
            seen |= {("up", hidden // 256)} if up == 2 else set()
            seen |= {("down", inter // 256)} if down == 2 else set()
        assert seen == {(which, n) for which in ("up", "down") for n in (8, 9, 10, 11, 13)}
        for hidden, inter, E, k, M, units in UNITS:
            fits, got, *_ = reach(hidden, inter, E, G, M * k)
            assert fits and got == units, (hidden, inter, E, k, M, got)
        ways = [reach(256, 256, E, G, M) for M, E in WAYS]
        assert [(w[0], w[2]) for w in ways][0][0] == 1 and ways[1][0] == 0 and ways[1][2] == 1 and ways[2][0] == 0 and ways[2][2] == 0
