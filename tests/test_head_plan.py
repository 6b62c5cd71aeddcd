"""CPU: what the output head plans (head_dx_tiles, called through its own header) and asks for: the scratch of dX's cut tiles has room for every tile of the tokens that are held
in two terms, however wide they are, and is of one size below; workspaces are as documented."""
import ctypes
import os
import subprocess

import pytest

import paper_2507_09029_amd as sdp
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


def test_workspaces_are_as_large_as_the_header_says():
    """bf16: a piece's logits in 1 GiB; twice that at most, and only from 2 million tokens of vocabulary on, where up to 128 tokens have two rows."""
    size, piece = sdp.lib().sdp_head_loss_workspace_bytes, 1 << 30
    for V in (5, 1000, 32000, 128256, 1000000, 1999999, 2100000, 3000001, 4000000, 4194303):
        ld = (V + 63) // 64 * 64 | 64  # a row of logits in whole lines, an odd number of them
        for d in (8, 504, 2048):
            if V * d >= 1 << 31:
                continue
            for T in (1, 60, 64, 100, 128, 129, 192, 300, 600, 16384, 1 << 20):
                for dx, dw in ((1, 1), (1, 0), (0, 1), (0, 0)):
                    rows = max(64, min(T, piece // (2 * max(ld if dx or dw else V // 8, d)) // 64 * 64, 1 << 15))
                    codes = (min(piece * (2 if V > 2000000 else 1), 2 * (max(rows, 256) * (V + 128))) + 256 * 128 * 2) if dx or dw else 0
                    beside = 5 * T + (2 * rows + 128) * (d + 64) * 2 * (1 + dw) + 8 * rows * (V // 32 + 2) + 1024
                    scratch = 128 << 20 if dx or (dw and T >= 512) else 0
                    sums = (V + 256) * (d + 256) * 4 if dw and T > rows else 0
                    assert size(1, T, V, d, dx, dw) <= codes + beside + scratch + sums + (1 << 16), (T, V, d, dx, dw)
    assert size(1, 128, 4000000, 8, 1, 0) > 1.9 * piece and size(1, 128, 1999999, 8, 1, 0) < 1.05 * piece
    assert size(1, 16384, 32000, 2048, 1, 1) >> 20 == 1320
