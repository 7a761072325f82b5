"""Where the copies of linear_tile.hip read (the functions of linear.hpp that the kernel calls, compiled for the CPU): of a copy that
the hardware does not drop, no byte lies outside of the rows and weights of the call.  A copy is dropped for sure only where the part of its
address that the lanes hold is past the buffer's length; whether what all lanes share is compared too is left open."""
import os
import subprocess

ROOT = os.path.dirname(os.path.dirname(__file__))
PROBE = r"""
#include <algorithm>
#include <cstdio>
#include <cstdlib>
#include "linear.hpp"
using namespace orthrus;
static long copies = 0, reads = 0;
static void look(const char *what, CopyAt c, int64_t bytes, int64_t room, int rows, int k, int64_t stride) {
    ++copies;
    if ((int64_t)c.lane >= room) return;
    ++reads;
    if ((int64_t)c.lane + c.shared + bytes > room) {
        printf("%s: rows %d, %d of K, stride %ld: byte %ld of %ld\n", what, rows, k, (long)stride, (long)(c.lane + (int64_t)c.shared), (long)room);
        exit(1);
    }
}
int main() {
    const int heights[] = {256, 128, 64}, ks[] = {1, 31, 32, 33, 97, 128, 129, 160, 500, 1003, 14336 / 8};
    for (int bm : heights)
        for (int k : ks)
            for (int dtype : {ORTHRUS_BF16, ORTHRUS_MX8})
                for (int wide = 0; wide < 2; ++wide)
                    for (int rows = 1; rows <= bm; rows += rows < 20 || rows > bm - 20 ? 1 : 13) {
                        const int es = dtype == ORTHRUS_MX8 ? 1 : 2, k_bytes = k * es, blocks = (k + 31) / 32;
                        const int steps = (k_bytes + kStepBytes - 1) / kStepBytes;
                        const int64_t stride = (k_bytes + 15) / 16 * 16 + 4096 * wide, scale_stride = (blocks + 3) / 4 * 4 + 100000 * wide;
                        const int64_t room = x_room(rows, stride, k_bytes);
                        // the whole 16 bytes around the last row's last element
                        if (room > (rows - 1) * stride + (k_bytes + 15) / 16 * 16) return 2;
                        for (int row = 0; row < bm; ++row)
                            for (int chunk = 0; chunk < 8; ++chunk)
                                for (int step = 0; step < steps; ++step) {
                                    const CopyAt c = x_copy(row, chunk, step, (unsigned)stride);
                                    if ((int64_t)c.lane + c.shared != row * stride + step * kStepBytes + chunk * 16) return 3;
                                    look("x", c, 16, room, rows, k, stride);
                                }
                        if (dtype != ORTHRUS_MX8) continue;
                        const int64_t scale_room = x_scale_room(rows, scale_stride, blocks);
                        if (scale_room > (rows - 1) * scale_stride + (blocks + 3) / 4 * 4) return 4;
                        for (int splits = 1; splits <= 8 && (splits == 1 || steps / splits >= 4); ++splits)
                            for (int part = 0; part < splits; ++part)
                                for (int stages : {2, 3}) {
                                    const int from = part * steps / splits, nk = (part + 1) * steps / splits - from;
                                    // the last copy of scales is issued for step nk - 2 + (stages + 3)
                                    for (int q = 0; q <= std::max(stages + 2, nk - 2 + stages + 3) / 4; ++q)
                                        for (int at = 0; at < bm; at += 16)
                                            for (int lane = 0; lane < 64; ++lane)
                                                look("scales of x", x_scale_copy(at, lane / 4, from + 4 * q, lane % 4, (unsigned)scale_stride), 4,
                                                     scale_room, rows, k, scale_stride);
                                }
                    }
    for (int bn : {128, 256})
        for (int k : ks)
            for (int tiles = 1; tiles <= bn / 16; ++tiles) {
                const PackedShape s = packed_shape(ORTHRUS_MX8, tiles * 16, k, 0);
                for (int half = 0; half < bn / 8; ++half)
                    for (int lane = 0; lane < 64; ++lane)
                        for (int step = 0; step < s.steps; ++step) {
                            look("weights", w_copy(half, lane, step, (unsigned)s.tile_bytes), 16, tiles * (int64_t)s.tile_bytes, tiles, k, 0);
                            look("scales of weights", w_scale_copy(half / 8, lane, step, (unsigned)s.steps), 4, (tiles + 3) / 4 * (int64_t)s.steps * 256,
                                 tiles, k, 0);
                        }
            }
    printf("%ld copies, %ld reads\n", copies, reads);
    return reads > 1000 ? 0 : 5;
}
"""


def test_copies_read_inside_the_operands(tmp_path):
    src, exe = tmp_path / "copies.cpp", tmp_path / "copies"
    src.write_text(PROBE)
    subprocess.run(["g++", "-O2", "-std=c++17", "-I", os.path.join(ROOT, "include"), "-I", os.path.join(ROOT, "paper_2609_25405_amd", "csrc"), str(src),
                    "-o", str(exe)], check=True)
    r = subprocess.run([str(exe)], capture_output=True, text=True)
    assert r.returncode == 0, r.stdout
