"""What the tile kernels of the 8-bit linear may touch and hold, from their constants: a host-only compilation of the source, no GPU needed."""
import os
import re
import subprocess

from paper_2506_04985_amd import build
from test_code_objects import code_objects, kernels  # noqa: F401

HEAD = r"""
#include "fptq_grouped.hip"
namespace fptq {
// a list of every tile shape that some kind of group takes
template <class... C> struct List {};
template <template <class> class Check, class... C> constexpr bool all(List<C...>) { return (Check<C>::ok && ...); }
using Tiles = List<Tile0<1>, Tile1<1>, Tile2<1>, Tile3<1>, Tile4<1>, Tile5<1>, Tile6<1>, Tile7<1>, Tile8<1>, Tile9<1>, Tile0<2>, Tile1<2>, Tile2<2>, Tile3<2>, Tile4<2>, Tile5<2>,
                   Tile6<2>, Tile7<2>, Tile8<2>, Tile9<2>, Tile1<4>, Tile3<4>, Tile5<4>, Tile6<4>, Tile7<4>, Tile8<4>, Tile9<4>>;
"""


def compiles(tmp_path, text):
    path = tmp_path / "check.hip"
    path.write_text(HEAD + text + "\n}\n")
    p = subprocess.run([build.HIPCC, *build.FLAGS, "--offload-host-only", "-fsyntax-only", "-Wno-unused-function", str(path)], stdout=subprocess.PIPE, stderr=subprocess.STDOUT, text=True)
    return p.returncode, p.stdout


def holds(tmp_path, text):
    rc, out = compiles(tmp_path, text)
    assert rc == 0, out


def test_the_check_can_fail(tmp_path):
    rc, out = compiles(tmp_path, 'static_assert(Tile0<1>::BM == 1, "not so");')
    assert rc != 0 and "not so" in out


def test_every_load_of_the_tokens_scales_ends_within_the_tiles_lds(tmp_path):
    """A load that writes LDS puts lane l at its base + 4 l: every scale of the tile is brought, and nothing behind the last byte that the launch asks for."""
    holds(tmp_path, r"""
template <class C> struct Within {
    static constexpr bool run()
    {
        bool brought[C::BM] = {};
        for (int piece = 0; piece < C::TOKEN_PIECES; ++piece)
            for (int lane = 0; lane < 64; ++lane) {
                if (!C::loads_token(piece, lane)) continue;
                if (C::SCALES_AT + piece * 256 + lane * 4 + 4 > C::LDS_BYTES) return false;
                brought[piece * 64 + lane] = true;
            }
        for (bool b : brought)
            if (!b) return false;
        return C::TOKEN_PIECES <= C::WAVES * C::KS;      // a wave takes one piece
    }
    static constexpr bool ok = run();
};
static_assert(all<Within>(Tiles()), "a token's scale is missing or lies outside");
""")


def test_the_table_of_times_counts_on_as_many_workgroups_as_a_cu_holds(kernels):  # noqa: F811
    """160 KB of LDS in pieces of 1280 bytes, and 512 registers a lane of a SIMD in pieces of 8, shared by at most eight waves."""
    text = open(os.path.join(build.CSRC, "fptq_grouped.hip")).read()
    shapes = [tuple(int(v) for v in re.findall(r"\d+", m)) for m in re.findall(r"using Tile\d = Tile<([^G]*), GT>;", text)]
    table = re.search(r"COSTS\[3\]\[TILES\] = \{(.*?)\n\};", text, re.S).group(1)
    rows = [(int(a), int(b), int(c), int(d)) for a, b, c, d in re.findall(r"\{(\d+), (\d+), (\d+), (\d+), \d", table)]
    assert len(shapes) == 10 and len(rows) == 30
    registers = {}
    for name, notes in kernels.items():
        m = re.search(r"grouped_tile_kernelINS_4TileI((?:Li\d+E)+)E", name)
        if m:
            registers[tuple(int(v) for v in re.findall(r"\d+", m.group(1)))] = int(re.search(r"\.vgpr_count:\s+(\d+)", notes).group(1))
    assert len(registers) == 27
    for kind, groups in enumerate((1, 2, 4)):
        for shape, (bn, bm, sets, fit) in zip(shapes, rows[10 * kind:]):
            waves_n, waves_m, tn, tm, stages, ks = shape
            assert (bn, bm, sets) == (32 * waves_n * tn, 32 * waves_m * tm, ks)
            if shape + (groups,) not in registers:
                continue
            ring, out = ks * stages * (bm * 128 + bn * 64 + bn * groups * 4), ks * waves_m * 32 * bn * 4
            lds = max(ring, out) + bm * 4
            waves = min(8, 512 // (-(-registers[shape + (groups,)] // 8) * 8)) * 4 // (waves_n * waves_m * ks)
            assert fit == min(160 * 1024 // (-(-lds // 1280) * 1280), waves), (groups, bn, bm, sets)
