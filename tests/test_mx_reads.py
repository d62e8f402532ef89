"""Where the tiled microscaled products read scales, on the CPU: the kernel's
own arithmetic (csrc/quick_mx_scales.h) for every lane and step against the
size of the buffer.  What bounds a buffer read is its size against the lane's
offset, word by word; an offset that a wave adds behind that check is not
counted on."""
import os
import subprocess

import paper_2402_10076_amd as Q

SOURCE = r"""
#include <cstdio>
#include <initializer_list>
#include "quick_mx_scales.h"
using namespace quick;

// words of a lane's copy that pass the check and lie outside
static int outside(BufferPlace p, uint32_t size)
{
    int n = 0;
    for (uint32_t w = 0; w < 16; w += 4)
        n += (uint64_t)p.lane + w + 4 <= size && (uint64_t)p.lane + w + p.uniform + 4 > size;
    return n;
}
// words that a step needs, and that the check leaves out or that are another's
static int missing(BufferPlace p, uint32_t size, uint32_t want, int words)
{
    int n = 0;
    for (int w = 0; w < words; w++)
        n += (uint64_t)p.lane + 4 * w + 4 > size || p.lane + p.uniform != want;
    return n;
}

int main()
{
    long bad = 0, lost = 0;
    // rows of activations: whole steps of 128 channels (4 bytes a step)
    for (int T : {1, 2, 3, 33, 64, 130, 512})
        for (int KS = 1; KS <= 90; KS++) {
            const int KB = KS * 4, KQ = (KS + 3) / 4;
            for (int r = 0; r < T; r++)
                for (int q = 0; q < KQ; q++) {
                    const BufferPlace p = scale_copy(row_scales(r, KB), true, q);
                    const int words = KS - 4 * q < 4 ? KS - 4 * q : 4;
                    bad += outside(p, T * KB);
                    lost += missing(p, T * KB, r * KB + q * 16, words);
                }
        }
    // packed scales of the column tiles that there are, of up to 16
    for (int tiles = 1; tiles <= 16; tiles++)
        for (int KQ = 1; KQ <= 30; KQ++)
            for (int t = 0; t < tiles; t++)
                for (int q = 0; q < KQ; q++)
                    for (int lane = 0; lane < 16; lane++) {
                        const BufferPlace p = scale_copy(tile_scales(t, KQ, lane), false, q);
                        bad += outside(p, tiles * KQ * 256);
                        lost += missing(p, tiles * KQ * 256, (t * KQ + q) * 256 + lane * 16, 4);
                    }
    std::printf("%ld words outside, %ld words lost\n", bad, lost);
    return bad || lost;
}
"""


def test_scale_copies_stay_inside(tmp_path):
    src = tmp_path / "t.cpp"
    src.write_text(SOURCE)
    exe = str(tmp_path / "t")
    csrc = os.path.join(os.path.dirname(Q.LIB_PATH), "csrc")
    subprocess.run(["g++", "-std=c++17", "-O1", "-Wall", "-I", csrc, str(src), "-o", exe], check=True)
    r = subprocess.run([exe], capture_output=True, text=True)
    assert r.returncode == 0, r.stdout
