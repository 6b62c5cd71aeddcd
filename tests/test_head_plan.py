"""CPU: what the output head plans for its contractions (head_dx_tiles, called through its own header): the scratch of dX's cut tiles has room for every tile of the tokens that are held
in two terms, however wide they are, and is the same as ever for widths that it always had room for."""
import ctypes
import os
import subprocess

import pytest

from paper_2507_09029_amd import build

SOURCE = '''#include "sdp_internal.h"
extern "C" void dx_tiles(int rows, int V, int d, int* to) {
    const sdp::HeadTiles t = sdp::head_dx_tiles(rows, V, d);
    to[0] = t.bm, to[1] = t.bn, to[2] = t.most;
}
extern "C" int two_term_rows() { return sdp::kTwoTermRows; }
'''


@pytest.fixture(scope="module")
def plan(tmp_path_factory):
    d = tmp_path_factory.mktemp("plan")
    (d / "plan.hip").write_text(SOURCE)
    if not os.path.exists(build.LIB):
        build.build_library()
    subprocess.run([build.HIPCC, *build.FLAGS, "--offload-host-only", "-shared", str(d / "plan.hip"), "-o", str(d / "plan.so"), "-L", build.HERE,
                    "-l:" + os.path.basename(build.LIB), f"-Wl,-rpath,{build.HERE}"], check=True)
    return ctypes.CDLL(str(d / "plan.so"))


def test_room_for_two_terms_at_any_width(plan):
    few, to = plan.two_term_rows(), (ctypes.c_int * 3)()
    assert few == 128
    for V in (1, 64, 1000, 2000, 8000, 16000, 32000, 200000, 4194303):
        for d in [8 << i for i in range(18)] + [24, 200, 1200, 40000, 81920, 98304, 114688, 163840, (1 << 20) - 8]:
            if V * d >= 1 << 31:
                continue
            for rows in (1, 5, 31, 64, 65, 100, 127, 128, 129, 200, 600, 5000):
                plan.dx_tiles(rows, V, d, to)
                bm, bn, most = to
                tiles = -(-2 * min(rows, few) // bm) * -(-d // bn)
                assert most == max(tiles, 1024 if bm == bn == 64 else 512), (rows, V, d, list(to), tiles)
