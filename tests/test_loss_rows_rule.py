"""CPU: how many waves hold a row of logits, and how many pieces a lane (by_row, sdp_loss_rows.h), for the token loss and for the divergence from a teacher."""
import ctypes
import os
import subprocess

import pytest

from paper_2507_09029_amd import build

SOURCE = '''#include "sdp_loss_rows.h"
template <bool LEAN>
static int tiles(int bf16, int V) {
    int of = -1;
    sdp::by_row<LEAN>(bf16, V, [&](auto, auto waves, auto pieces) { of = waves.value * 100 + pieces.value; });
    return of;
}
extern "C" int token_loss(int bf16, int V) { return tiles<true>(bf16, V); }
extern "C" int divergence(int bf16, int V) { return tiles<false>(bf16, V); }
'''


@pytest.fixture(scope="module")
def rule(tmp_path_factory):
    d = tmp_path_factory.mktemp("rule")
    (d / "rule.hip").write_text(SOURCE)
    subprocess.run([build.HIPCC, *build.FLAGS, "--offload-host-only", "-shared", str(d / "rule.hip"), "-o", str(d / "rule.so")], check=True)
    return ctypes.CDLL(str(d / "rule.so"))


def pairs(f, n, ends):
    """what rows of each number of values and of one more take; n values a piece"""
    return [(f(int(n == 8), e * n), f(int(n == 8), e * n + 1)) for e in ends]


@pytest.mark.parametrize("n", [8, 4])
def test_token_loss_holds_five_to_seven_pieces_in_sixteen_waves(rule, n):
    # 32769 .. 57344 values of bf16, 16385 .. 28672 of fp32
    assert pairs(rule.token_loss, n, (4096, 5120, 6144, 7168)) == [(1604, 1605), (1605, 1606), (1606, 1607), (1607, 816)]
    assert [rule.token_loss(1, V) for V in (40961, 50001, 50257, 50304)] == [1606, 1607, 1607, 1607]


@pytest.mark.parametrize("n", [8, 4])
def test_divergence_holds_them_in_eight_waves(rule, n):
    assert pairs(rule.divergence, n, (4096, 5120, 6144, 7168)) == [(1604, 816), (816, 816), (816, 816), (816, 816)]


@pytest.mark.parametrize("n", [8, 4])
def test_other_rows_alike(rule, n):
    for f in (rule.token_loss, rule.divergence):
        assert pairs(f, n, (64, 128, 256, 512, 1024, 1536, 2048, 2560, 8192, 12288, 16384)) \
            == [(101, 201), (201, 401), (401, 402), (402, 404), (404, 803), (803, 804), (804, 806), (806, 806), (816, 1612), (1612, 1616), (1616, 1600)]
