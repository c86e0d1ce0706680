"""How the linear layer's products are divided (csrc/pp_linear_plan.h itself, compiled for the host)."""
import ctypes
import os
import subprocess

from conftest import ROOT

FORWARD, INPUT, WEIGHT = 0, 1, 2
TYPES = {"f32": 0, "f16": 1, "bf16": 2}
SOURCE = r"""
#include "pp_linear_plan.h"
extern "C" void divide(int call, int type, long long rows, long long n_in, long long n_out, unsigned long long room, long long *out) {
    int shape;
    const pr_plan p = call == 0 ? plan_forward(rows, n_in, n_out, room, &shape) : call == 1 ? plan_input(type, rows, n_in, n_out, room, &shape)
                                                                                : plan_weight(type, rows, n_in, n_out, room, &shape);
    const pr_shape &s = (call == 0 ? FORWARD : call == 1 ? INPUT : WEIGHT)[shape];
    const long long bytes = partial_bytes(p.splits, p.inner, p.outer) + (call == 2 ? sums_bytes(p.splits, p.ni, p.outer) : 0);
    const long long v[] = {s.ti, s.to, p.splits, p.steps, p.per, p.ni, p.no, p.by_piece, bytes, call == 0 ? 1 : planes_of(type)};
    for (int i = 0; i < 10; ++i) out[i] = v[i];
}
"""
FIELDS = ("ti", "to", "pieces", "steps", "per", "ni", "no", "by_piece", "bytes", "planes")


class Plans:
    def __init__(self, folder):
        src, so = os.path.join(folder, "plans.cpp"), os.path.join(folder, "plans.so")
        with open(src, "w") as f:
            f.write(SOURCE)
        subprocess.run(["g++", "-std=c++17", "-O1", "-Wall", "-Wno-unused-function", "-Werror", "-shared", "-fPIC", "-I", os.path.join(ROOT, "include"),
                        "-I", os.path.join(ROOT, "paper_2204_10562_amd", "csrc"), src, "-o", so], check=True)
        self.lib = ctypes.CDLL(so)
        self.lib.divide.argtypes = [ctypes.c_int, ctypes.c_int] + [ctypes.c_longlong] * 3 + [ctypes.c_ulonglong, ctypes.POINTER(ctypes.c_longlong)]

    def divide(self, call, t, rows, n_in, n_out, room=(1 << 64) - 1):
        """The tiles (ti inner results by to outer ones, ni x no of them), pieces and steps of a call, and the bytes of its partial sums."""
        out = (ctypes.c_longlong * len(FIELDS))()
        self.lib.divide(call, TYPES[t], rows, n_in, n_out, room, out)
        return dict(zip(FIELDS, out))
