"""How the blocks of a chained scan share its tiles, run on the host: the
functions the kernels call (csrc/bc_scan_chain.hpp), built without device code."""
import os
import re
import shutil
import subprocess

import pytest

from paper_1906_11367_amd import build as B
from test_kernel_code import _kernels, device_code  # noqa: F401 (a fixture)

pytestmark = pytest.mark.skipif(shutil.which("hipcc") is None and not os.path.exists("/opt/rocm/bin/hipcc"),
                                reason="no hipcc")


def run_host(tmp_path, body):
    src, exe = tmp_path / "chain.cpp", str(tmp_path / "chain")
    src.write_text('#include "bc_scan_chain.hpp"\n#include <climits>\n#include <cstdio>\n#include <vector>\n'
                   f"using namespace bc::scan;\nint main() {{\n{body}\nreturn 0;\n}}\n")
    for cmd in ([B.hipcc(), "-O1", "-std=c++17", "--offload-host-only", "-x", "hip", "-I", B.CSRC, str(src), "-o", exe],
                [exe]):
        r = subprocess.run(cmd, capture_output=True, text=True)
        assert r.returncode == 0, " ".join(cmd) + "\n" + r.stdout[-2000:] + r.stderr[-2000:]


def test_every_unit_has_its_tiles_blocks(tmp_path):
    run_host(tmp_path, """
      for (int units : {1, 2, 7, 8, 9, 63, 64, 100, 1000})
        for (int tiles : {2, 3, 17}) {
          std::vector<int> blocks(units, 0);
          for (long b = 0; b < (long)units * tiles; ++b) {
            const int u = chain_unit(b, units);
            if (u < 0 || u >= units) return 1;
            ++blocks[u];
          }
          for (int n : blocks) if (n != tiles) return 2;
        }""")


def test_a_number_outside_the_chain_is_no_place(tmp_path):
    """Whatever a counter holds that another call wrote over: a block goes on only
    with a tile of its tensors, in both directions of time."""
    run_host(tmp_path, """
      for (int tiles : {2, 16, 17, 300}) {
        for (long n = -3; n < 2L * tiles + 3; ++n)
          if (chain_has((int)n, tiles) != (n >= 0 && n < tiles)) return 1;
        for (int n : {INT_MIN, INT_MIN + 1, -1, INT_MAX, 0x3f800000}) if (chain_has(n, tiles)) return 2;
        for (int n = 0; n < tiles; ++n) if (tiles - 1 - n < 0) return 3;   // the backward's tile
      }""")


def test_grids_hold_every_word_and_stay_below_2_32_threads(tmp_path):
    """Up to 65536 sequences of 2^20 steps (one word a channel and tile of 128,
    64 channels: 2^36 words and more)."""
    run_host(tmp_path, """
      for (long words = 1; words < 1L << 38; words = words * 3 / 2 + 1) {
        const Grid g = grid_of(clear_blocks(words));
        if ((long)g.x * 256 >= 1L << 32 || g.y > 65535) return 1;
        if ((long)g.x * g.y * 512 < words) return 2;
        if ((long)g.x * (g.y - 1) * 512 >= words) return 3;   // no row of blocks for nothing
      }
      for (long blocks : {1L, 1000L, (1L << 22) - 1, 1L << 22, (1L << 22) + 1, 1L << 31}) {
        const Grid g = grid_of(blocks);
        if ((long)g.x * 512 >= 1L << 32 || (long)g.x * g.y < blocks) return 4;
      }""")


def test_the_kernels_leave_where_there_is_no_place():
    with open(os.path.join(B.CSRC, "bc_scan.hip")) as f:
        text = f.read()
    draw = text[text.index("bool draw_ticket("):]
    assert "return chain_has(place, tiles);" in draw[:draw.index("\n}\n")]
    assert text.count("draw_ticket(p.tickets") == text.count("if (!draw_ticket(p.tickets, p.N * p.slabs, p.tiles, unit, place)) return;") == 2


def test_every_scan_kernel_built_is_one_that_calls_reach(device_code):
    """Cuts of the token kernels (channels a lane, lanes side by side, threads,
    steps a lane): one tile a sequence, or chained."""
    single = {("fwd", 1): {(4, 64, 64, 8), (4, 8, 64, 4), (4, 8, 128, 4), (4, 16, 512, 4), (4, 8, 512, 4)},
              ("fwd", 2): {(4, 64, 64, 8), (4, 16, 64, 8), (4, 16, 128, 8), (4, 16, 256, 8), (4, 16, 512, 8)},
              ("bwd", 1): {(4, 64, 64, 4), (4, 8, 64, 4), (4, 8, 128, 4), (4, 16, 512, 4), (4, 8, 512, 4)},
              ("bwd", 2): {(2, 64, 64, 8), (2, 32, 64, 8), (2, 32, 128, 8), (2, 32, 256, 8), (2, 32, 512, 8)}}
    chained = {("fwd", 1): {(4, 16, 512, 4), (4, 16, 512, 8)}, ("fwd", 2): {(4, 16, 256, 8), (4, 16, 512, 8)},
               ("bwd", 1): {(4, 16, 512, 4)}, ("bwd", 2): {(2, 32, 512, 8)}}
    found = {}
    for _, name in _kernels(device_code, r"k_scan_(fwd|bwd)I"):
        way, *n = re.search(r"k_scan_(fwd|bwd)INS0_3CutILi(\d+)ELi(\d+)ELi(\d+)ELi(\d+)ELi\d+EEELi(\d)ELi(\d)ELi(\d)ELb(\d)E",
                            name).groups()
        *cut, dt, out, form, chain = map(int, n)
        found.setdefault((way, dt, chain), {}).setdefault((out, form), set()).add(tuple(cut))
    for (way, dt), cuts in single.items():
        kinds = [(out, form) for out in ((1, 2) if dt == 1 else (2,)) for form in (0, 1)]
        assert found[way, dt, 0] == {k: cuts for k in kinds}
        assert found[way, dt, 1] == {k: chained[way, dt] for k in kinds}
