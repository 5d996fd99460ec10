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
