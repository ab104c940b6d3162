"""Sizes of the input gradient of the expert projection by the launch form that
they reach, and what tells the form: the library's own rule, and how its large
tiles fall to blocks."""
import collections
import ctypes
import os
import subprocess

import numpy as np

from paper_2609_06072_amd import build as b

KERNELS = S16x64, S32x64, S64x64, S32x128, S64x128, TILES, LARGE = range(7)
ONE_PIECE, JOINED, SUMMED = range(3)

SHIM = r"""
#include "%s/ace_internal.hpp"
extern "C" int dx_plan(int dtype, long P, int k, int E, int contraction, int columns, int sums, int* splits) {
  ace::MoeArgs a{};
  a.E = E; a.k = k; a.d_in = contraction; a.d_out = columns; a.pairs = P; a.per_pair = 1;
  const ace::DxPlan p = ace::moe_dx_plan(dtype, a, P, (ace::DxSums)sums);
  *splits = p.splits;
  return (int)p.kernel;
}
"""


def load_rule(tmp):
    """The rule of the built library, behind a C function."""
    src, out = os.path.join(tmp, "dx_plan.hip"), os.path.join(tmp, "dx_plan.so")
    with open(src, "w") as f:
        f.write(SHIM % b.CSRC)
    subprocess.run([b.hipcc(), "-std=c++17", "-fPIC", "-shared", "--offload-host-only", f"--offload-arch={b.ARCH}",
                    "-x", "hip", src, "-x", "none", b.OUT, f"-Wl,-rpath,{os.path.dirname(b.OUT)}", "-o", out],
                   check=True, capture_output=True)
    return ctypes.CDLL(out).dx_plan


def plan(rule, dtype, T, k, E, d_in, d_out, sums):
    """(kernel, splits) for the projection [E, d_out, d_in]."""
    splits = ctypes.c_int()
    kernel = rule(int(dtype == "bf16"), ctypes.c_long(T * k), k, E, d_out, d_in, sums, ctypes.byref(splits))
    return kernel, splits.value


Xcd = collections.namedtuple("Xcd", "rounds parts")


def large_tiles(rows, d_in, splits, step=32):
    """Of an XCD with `step` blocks a set: rounds of whole tiles that its blocks
    take, and the column parts of a tile of the cut round (0: none is cut).
    rows: of each expert."""
    n = int((-(-np.asarray(rows) // 256)).sum()) * -(-d_in // 256) * splits
    per, out = -(-n // 8), set()
    for x in range(8):
        mine = max(0, min(per, n - x * per))
        over = mine % step
        cut = 2 * over <= step and over > 0
        out.add(Xcd(-(-(mine - over if cut else mine) // step), (4 if 4 * over <= step else 2) if cut else 0))
    return out


def routing(kind, T, k, E, seed=1):
    """ids [T, k].  even: in turn.  tails: as many experts as possible end in a tile
    with one row.  random: uneven, one pair in twenty dropped."""
    rng = np.random.default_rng(seed)
    if kind == "even":
        return (np.arange(T * k, dtype=np.int32) % E).reshape(T, k)
    if kind == "tails":
        assert k == 1 and T >= E
        more, last = divmod(T - E, 256)
        n = np.full(E, 1 + more // E * 256)
        n[:more % E] += 256
        n[-1] += last
        return rng.permutation(np.repeat(np.arange(E, dtype=np.int32), n)).reshape(T, 1)
    logits = rng.gumbel(size=(T, E)) - 0.5 * np.log(np.arange(1, E + 1))
    ids = np.argsort(-logits, axis=1)[:, :k].astype(np.int32)
    ids[rng.random((T, k)) < 0.05] = -1
    return np.ascontiguousarray(ids)


def expert_rows(ids, E):
    return np.bincount(ids[ids >= 0], minlength=E)


# T, k, E, d_in, d_out, routing; the bf16 form: kernel, splits, and of large tiles the
# rounds of whole tiles and the column parts of a cut last round, on some XCD
FORMS = [
    # several tiles a block: full and partial ones in turn, the ring runs on
    (4428, 2, 16, 2952, 256, "even", LARGE, 1, 2, 4),
    (3594, 4, 4, 3648, 256, "even", LARGE, 1, 4, 0),
    (4724, 4, 8, 3288, 264, "even", LARGE, 1, 4, 4),
    (7435, 4, 64, 1432, 264, "random", LARGE, 1, 3, 2),
    (4094, 2, 64, 1384, 512, "random", LARGE, 1, 2, 0),
    (3679, 2, 64, 2920, 520, "random", LARGE, 1, 3, 4),
    (16442, 1, 64, 2144, 520, "even", LARGE, 1, 4, 2),
    (9377, 2, 64, 1808, 640, "even", LARGE, 1, 4, 0),
    (2033, 4, 64, 2312, 648, "random", LARGE, 1, 3, 0),
    (8309, 1, 16, 2616, 1024, "even", LARGE, 1, 2, 4),
    # the same where blocks share a contraction, even and ragged
    (5622, 1, 64, 696, 5104, "tails", LARGE, 2, 2, 0),
    (5800, 1, 64, 664, 4880, "tails", LARGE, 2, 2, 4),
    (4742, 1, 64, 480, 4096, "tails", LARGE, 2, 1, 2),
    (42066, 1, 4, 8, 9896, "tails", LARGE, 3, 2, 0),
    (1544, 1, 16, 2240, 5760, "tails", LARGE, 3, 2, 4),
    (3034, 1, 32, 648, 7664, "tails", LARGE, 4, 2, 4),
    (20183, 1, 32, 136, 11776, "tails", LARGE, 4, 2, 0),
    # shares of one round or less
    (10502, 1, 8, 176, 2816, "tails", LARGE, 2, 0, 2),
    (12230, 1, 16, 136, 2272, "tails", LARGE, 2, 0, 2),
    (1042, 1, 2, 2048, 2304, "tails", LARGE, 3, 1, 0),
    (10133, 1, 2, 144, 1656, "tails", LARGE, 3, 0, 2),
    (1172, 1, 8, 1920, 4096, "tails", LARGE, 4, 1, 2),
    (515, 1, 4, 3640, 4608, "tails", LARGE, 4, 1, 4),
    (1997, 1, 1, 1800, 14016, "even", LARGE, 4, 1, 0),
    (3271, 1, 16, 136, 7400, "tails", LARGE, 6, 1, 0),
    (2529, 1, 16, 160, 9160, "tails", LARGE, 7, 1, 0),
    (279, 4, 8, 408, 11976, "random", LARGE, 8, 0, 2),
    (1926, 1, 16, 208, 9216, "tails", LARGE, 8, 1, 0),
    (3269, 1, 32, 136, 8016, "tails", LARGE, 8, 1, 2),
    (2256, 1, 32, 144, 13024, "tails", LARGE, 8, 1, 4),
    # tiles of 128 x 128
    (3208, 1, 32, 200, 1536, "tails", TILES, 3, 0, 0),
    (20738, 1, 256, 8, 1208, "tails", TILES, 3, 0, 0),
    (7901, 1, 2, 16, 13312, "random", TILES, 4, 0, 0),
    (23549, 1, 2, 8, 2040, "even", TILES, 4, 0, 0),
    (67, 1, 2, 2784, 6400, "random", TILES, 5, 0, 0),
    (13019, 1, 200, 8, 1928, "tails", TILES, 5, 0, 0),
    (105, 1, 2, 2672, 9216, "even", TILES, 6, 0, 0),
    (4707, 1, 2, 8, 5024, "random", TILES, 6, 0, 0),
    (4367, 1, 1, 40, 4480, "even", TILES, 7, 0, 0),
    (2042, 2, 4, 8, 4424, "random", TILES, 7, 0, 0),
    (287, 1, 4, 880, 10392, "even", TILES, 8, 0, 0),
    (4914, 1, 32, 8, 8192, "tails", TILES, 8, 0, 0),
]
