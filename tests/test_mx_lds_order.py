"""Lanes of a wavefront that read what its other lanes wrote to LDS, with no barrier of the workgroup between, need a fence of memory there: a wave
barrier orders the scheduling of instructions, and leaves the compiler free to move plain loads and stores across it.  Read from the sources."""
import glob
import os
import re

from paper_1711_00244_amd import binding

MX = os.path.join(os.path.dirname(binding.__file__), "csrc", "mx")


def code(path):
    return re.sub(r"//.*", "", open(path).read())


def test_wave_barriers_stand_between_fences():
    sources = {os.path.basename(p): code(p) for p in glob.glob(os.path.join(MX, "*.h*"))}
    barriers = [(name, m.start()) for name, text in sources.items() for m in re.finditer(r"__builtin_amdgcn_wave_barrier\(\)", text)]
    assert barriers
    fence = r'__builtin_amdgcn_fence\(__ATOMIC_(?:%s|ACQ_REL), "wavefront"\);'
    for name, at in barriers:
        assert re.search(fence % "RELEASE" + r"\s*$", sources[name][:at]), (name, sources[name][:at].count("\n") + 1)
        assert re.match(r"__builtin_amdgcn_wave_barrier\(\);\s*" + fence % "ACQUIRE", sources[name][at:]), (name, sources[name][:at].count("\n") + 1)


def test_where_lanes_exchange():
    # the placing of pairs, the choice of experts (its group scores, its choice), the stores of a tile
    uses = {os.path.basename(p): len(re.findall(r"\blanes_exchange\(\)", code(p))) for p in glob.glob(os.path.join(MX, "*.h*"))}
    assert uses["route.hip"] >= 5 and uses["tile_kernel.hpp"] >= 2, uses
