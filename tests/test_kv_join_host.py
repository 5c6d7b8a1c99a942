"""Which launch joins the pieces of chunks' tiles is host arithmetic: a small C++ program asks the library for it, without a GPU."""

from tests.test_launch_shapes import run_program

PROGRAM = r"""
#include <cstdio>
#include "kv.cuh"
int main() {
    for (int sms = 1; sms <= 1100; sms++)
        for (long long tiles = 0; tiles <= 60; tiles++)
            // 3 CTAs per SM; a tile takes 8 (32 of its 256 rows each) or a multiple of that
            if (kvdro::kv_join_few(tiles, sms) && (tiles * 8 > 3LL * sms || sms > 1024)) {
                std::printf("%lld tiles, %d SMs\n", tiles, sms);
                return 1;
            }
    if (!kvdro::kv_join_few(38, 152) || kvdro::kv_join_few(39, 152) || !kvdro::kv_join_few(7, 20) || kvdro::kv_join_few(8, 20)) return 2;
    return kvdro::kv_join_few(1LL << 40, 152) ? 3 : 0;
}
"""


def test_the_launch_for_few_tiles_holds_every_tile_that_it_is_given(tmp_path):
    """On a full GPU 57 tiles would fit; on 20 SMs 7 do."""
    out = run_program(tmp_path, PROGRAM)
    assert out.returncode == 0, (out.returncode, out.stdout)
