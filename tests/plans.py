"""What csrc/linear_plan.h chooses for a size, asked on the host."""
import ctypes as C
import functools
import os
import subprocess
import tempfile

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2109_04312_amd", "csrc")
SOURCE = """
#include "linear_plan.h"
using namespace mate;
extern "C" {
// few tokens' form [3] (rows 0: none), ranges of a split contraction (0: none), form of the tiles
void forward(int T, int O, int K, int codes, int* out) {
  const ForwardPlan p = plan_forward(T, O, K, codes != 0);
  out[0] = p.few.form.rows; out[1] = p.few.form.blocks; out[2] = p.few.form.tokens; out[3] = p.split.splits; out[4] = p.tiles.form;
}
// one launch, dw's tile, its ranges, are codes copied, dx's form, ranges of its contraction, has a range of dw its own list of blocks
void backward(int T, int E, int F, int* out) {
  const BackwardPlan p = plan_backward(T, E, F, true);
  out[0] = p.one_launch; out[1] = p.tile; out[2] = p.splits; out[3] = p.copy; out[4] = p.product.form; out[5] = p.dx_splits;
  out[6] = !p.one_launch && (T + 63L) / 64 > kMostBlocks;
}
}
"""
TILES = ("256", "128", "128x2", "64", "64x2")


@functools.lru_cache(None)
def lib():
    with tempfile.TemporaryDirectory() as d:
        src, so = os.path.join(d, "plan.hip"), os.path.join(d, "plan.so")
        with open(src, "w") as f:
            f.write(SOURCE)
        subprocess.run(["hipcc", "--offload-arch=gfx950", "--cuda-host-only", "-O1", "-std=c++17", "-fPIC", "-shared", "-w", f"-I{CSRC}", src, "-o", so],
                       check=True, capture_output=True)
        return C.CDLL(so)   # (stays mapped)


def forward(T, E, F, codes):
    """"few 16x32" (features x tokens of a workgroup), "split 3" or "tiles 128x2"."""
    o = (C.c_int * 5)()
    lib().forward(T, F, E, int(codes), o)
    return f"few {o[0] * o[1]}x{16 * o[2]}" if o[0] else f"split {o[3]}" if o[3] else f"tiles {TILES[o[4]]}"


def backward(T, E, F):
    """How dw and dx are computed, and whether x in 8 bits is copied first."""
    o = (C.c_int * 7)()
    lib().backward(T, E, F, o)
    dx = f"dx {TILES[o[4]]}" + (f" split {o[5]}" if o[5] > 1 else "")
    return f"{'one' if o[0] else 'two'} launches, dw {o[1]} ranges {min(o[2], 9)}{' listed apart' if o[6] else ''}, {dx}", "copied" if o[3] else "direct"
