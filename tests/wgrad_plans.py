"""The weight gradient's plan (csrc/wgrad_plan.h, plain C++) compiled by itself:
which tiles a call is cut into, and into how many runs of tokens."""
import ctypes
import functools
import os
import subprocess
import tempfile
from typing import NamedTuple

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
CSRC = os.path.join(ROOT, "paper_2507_07114_amd", "csrc")

SOURCE = r"""
#include "wgrad_plan.h"
extern "C" void plan(int bf16, int64_t n, int64_t t, int64_t o, int64_t h, int64_t* out) {
    lossy::WgradPlan g = {};
    lossy::wgrad_plan(n, t, o, h, bf16, &g);
    const int64_t v[] = {g.edge, g.light, g.whole, g.rest, g.runs, g.run_t,
                         (int64_t)lossy::wgrad_part_bytes(g)};
    for (int i = 0; i < 7; ++i) out[i] = v[i];
}
"""


class Plan(NamedTuple):
    edge: int     # of the square tiles
    light: int    # light workgroups
    whole: int    # tiles of one workgroup each
    rest: int     # tiles summed in runs
    runs: int
    run_t: int    # tokens of a run
    part: int     # bytes of the runs' sums

    @property
    def form(self) -> str:
        """"256", "128" or "light", and how its tiles are summed."""
        tiles = "whole" if self.runs == 1 else ("both" if self.whole else "runs")
        return ("light" if self.light else str(self.edge)) + " " + tiles


@functools.lru_cache(maxsize=None)
def _lib():
    with tempfile.TemporaryDirectory() as tmp:
        src, out = os.path.join(tmp, "plan.cpp"), os.path.join(tmp, "plan.so")
        with open(src, "w") as f:
            f.write(SOURCE)
        subprocess.run(["g++", "-std=c++17", "-O1", "-Wall", "-Wextra", "-Werror", "-shared",
                        "-fPIC", f"-I{CSRC}", src, "-o", out], check=True)
        return ctypes.CDLL(out)


def plan(bf16: bool, n: int, t: int, o: int, h: int) -> Plan:
    """Of dy in bf16 or fp32 for n workers' t token places of an [o][h] weight."""
    out = (ctypes.c_int64 * 7)()
    _lib().plan(int(bf16), *(ctypes.c_int64(x) for x in (n, t, o, h)), out)
    return Plan(*out)


# Calls of every form: n, t, o, h, offset, lengths, ld_y - o, ld_q - h, ld_s - groups, and
# the forms that bf16 and fp32 dy take.
CASES = [
    (2, 130, 600, 520, 0, [130, 33], 0, 0, 0, "light whole", "128 whole"),
    (2, 900, 2901, 2905, 3, [899, 161], 3, 7, 1, "light whole", "128 both"),
    (2, 3000, 133, 267, 8, [3000, 300], 1, 5, 0, "128 runs", "128 runs"),
    # 256 x 256 tiles; widths that are multiples of 8 and others take different kernels
    (2, 600, 4096, 4096, 0, [600, 77], 0, 0, 0, "256 whole", "256 whole"),
    (2, 500, 4090, 4091, 3, [0, 499], 3, 5, 1, "256 whole", "256 whole"),
    (2, 1024, 2816, 3000, 8, [1000, 130], 8, 16, 2, "256 both", "256 both"),
    (2, 2000, 3000, 3203, 1, [2000, 673], 1, 3, 0, "256 both", "256 both"),
    (2, 8192, 1024, 2048, 0, [8192, 4099], 0, 0, 0, "256 runs", "256 runs"),
    (2, 8192, 1020, 2045, 5, [5000, -1], 1, 1, 1, "256 runs", "256 runs"),
]
