"""The kernel forms that an 8-bit call takes (csrc/dd_routes.hpp, compiled by
the host compiler), so that tests can say which one they mean to reach."""
import ctypes
import functools
import os
import subprocess
import tempfile

from paper_2405_13226_amd import build as B

CUS = 256  # an MI355X
SRC = """
#include "dd_routes.hpp"
extern "C" {
int product(int M, int N, int K, int cus) { return static_cast<int>(dd::gemm_i8_tile(M, N, K, cus)); }
void wgrad(int T, int M, int N, int n, int cus, int *out) {
    const dd::WgradPlan p = dd::wgrad_plan(T, M, N, n, cus);
    out[0] = p.edge; out[1] = p.whole; out[2] = p.heads ? p.shared() : 0; out[3] = p.steps;
    out[4] = p.head; out[5] = p.tails; out[6] = p.most(); out[7] = p.tiles_m * p.tiles_n;
    out[8] = p.heads; out[9] = p.rest();
}
int walk(int wg, int i, int grid, int tiles) { return dd::walk_tile(wg, i, grid, tiles); }
}
"""


@functools.lru_cache(maxsize=None)
def _lib():
    with tempfile.TemporaryDirectory() as d:
        src, so = os.path.join(d, "routes.cpp"), os.path.join(d, "routes.so")
        with open(src, "w") as f:
            f.write(SRC)
        subprocess.run(["g++", *B.CXX_FLAGS, "-shared", "-o", so, src], check=True)
        return ctypes.CDLL(so)


def product(M, N, K):
    """Where an int8 product of these sizes goes."""
    return ("few", "small", "large")[_lib().product(M, N, K, CUS)]


def wgrad(T, M, N, n=1):
    """How n weight gradients run: edge, whole, shared, steps, head, tails,
    most, tiles, heads, rest."""
    out = (ctypes.c_int * 10)()
    _lib().wgrad(T, M, N, n, CUS, out)
    return dict(zip(("edge", "whole", "shared", "steps", "head", "tails", "most", "tiles",
                     "heads", "rest"), out))


def walk(wg, i, grid, tiles):
    """Tile i of a workgroup's walk, as the lanes that hold its place see it."""
    return _lib().walk(wg, i, grid, tiles)
