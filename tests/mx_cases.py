"""Calls of the products with experts in 4 bits, and of their gradient, that together reach every kernel there is for them: what each call takes
is asked of the library's own rule (csrc/mx_plan.h, compiled on its own), on the CPU, so that a rule that moves shows where a test lost its
kernel; the GPU tests run them."""
import ctypes as C
import os
import random
import subprocess

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2604_02715_amd", "csrc")
KERNELS = ("stream", "strip", "wide")
SHIM = """
#include "mx_plan.h"
using namespace fluxmoe;
extern "C" void choose(int grad, uint64_t cap, uint32_t E, uint32_t N, uint32_t K, uint64_t row_stride, uint64_t row_scales_stride, int mx_rows, int rows_vec,
                       int w_words, int row_words, uint32_t* o) {
    const MxCall c{cap, E, N, K, row_stride, row_scales_stride, mx_rows != 0, rows_vec != 0, w_words != 0, row_words != 0};
    const MxChoice k = grad ? mx_choose_grad(c) : mx_choose_product(c);
    o[0] = k.kernel; o[1] = k.rows; o[2] = k.outs; o[3] = k.waves; o[4] = k.vec; o[5] = k.whole;
}
"""


def compile_rule(d):
    """choose(op, cap, E, N, K, row_stride, row_scales_stride, mx, rows_vec, w_words, row_words) -> (op, mx, kernel, rows, outs, waves, vec, whole)"""
    (d / "shim.cpp").write_text(SHIM)
    subprocess.run(["g++", "-std=c++17", "-O1", "-Wall", "-Werror", "-shared", "-fPIC", "-I", CSRC, str(d / "shim.cpp"), "-o", str(d / "shim.so")], check=True)
    so = C.CDLL(str(d / "shim.so"))
    u32, u64 = C.c_uint32, C.c_uint64
    so.choose.argtypes = [C.c_int, u64, u32, u32, u32, u64, u64, C.c_int, C.c_int, C.c_int, C.c_int, C.POINTER(u32)]

    def choose(op, cap, E, N, K, row_stride, row_scales_stride, mx, rows_vec, w_words, row_words):
        o = (u32 * 6)()
        so.choose(op == "grad", cap, E, N, K, row_stride, row_scales_stride, mx, rows_vec, w_words, row_words, o)
        return (op, bool(mx), KERNELS[o[0]], o[1], o[2], o[3], bool(o[4]), bool(o[5]))
    return choose


def rows_of(counts, align=4, ahead=2):
    return ahead + sum(-(-c // align) * align for c in counts)


def taken_by(choose, case):
    """what the case's call takes: tensors begin at aligned addresses, rows `gap` elements further apart than wide, from element `shift` on"""
    width = case["K"] if case["op"] == "product" else case["N"]
    width, size = (width // 2, 1) if case["mx"] else (width, 2)
    stride, blocks = (width + case["gap"]) * size, case["K"] // 32
    scales = blocks + case["scale_gap"] if case["mx"] else 0
    return choose(case["op"], rows_of(case["counts"]), len(case["counts"]), case["N"], case["K"], stride, scales, case["mx"],
                  case["shift"] * size % 16 == 0 and stride % 16 == 0, case["ws_shift"] % 4 == 0 and blocks % 4 == 0, scales % 4 == 0)


def few(E, most, seed):
    """rows of E experts, up to `most` each, every fifth one without"""
    rng = random.Random(seed)
    return [0 if e % 5 == 3 else rng.randrange(1, most + 1) for e in range(E)]


# So many rows: 2 and 13 to an expert on average, 41, 221 and more
TWO, TWELVE, FORTY, MANY = few(300, 4, 1), few(100, 29, 2), [40, 0, 64, 65, 33], [300, 0, 513, 70]
CASES = []


def case(op, takes, counts, N, K, mx=False, gap=0, shift=0, scale_gap=0, ws_shift=0):
    """takes: (kernel, rows, outs, waves, vec, whole)"""
    CASES.append(dict(op=op, takes=takes, counts=counts, N=N, K=K, mx=mx, gap=gap, shift=shift, scale_gap=scale_gap, ws_shift=ws_shift))


def both_scales(op, takes, counts, N, columns, mx=False):
    """with scales as words where K is a multiple of 128, with those of the weights, or the rows, elsewhere, and with the others"""
    for K in columns:
        case(op, takes + (True, K % 128 == 0), counts, N, K, mx)
    K = [K for K in columns if K % 128 == 0][-1]
    case(op, takes + (True, False), counts, N, K, mx, ws_shift=1)
    if mx:
        case(op, takes + (True, False), counts, N, K, mx, scale_gap=3)
        case(op, takes + (True, True), counts, N, K, mx, gap=16, scale_gap=4)


# Rows in 4 bits
both_scales("product", ("stream", 16, 16, 4), [1, 0, 3, 2], 37, (32, 160, 512, 2048, 2080, 4096), True)
both_scales("product", ("stream", 32, 16, 4), [12, 0, 20, 33], 37, (32, 160, 512, 2048, 2080, 4096), True)
both_scales("product", ("stream", 16, 64, 4), TWO, 130, (2080, 2176, 2560), True)
both_scales("product", ("stream", 32, 64, 4), TWELVE, 391, (2080, 2176, 2560), True)
both_scales("product", ("strip", 16, 64, 4), TWO, 521, (32, 160, 256, 288, 1152), True)
both_scales("product", ("strip", 32, 64, 4), TWELVE, 1291, (32, 160, 256, 288, 1152, 2048), True)
both_scales("product", ("strip", 64, 64, 4), FORTY, 301, (32, 160, 256, 288, 1152, 2048, 4128), True)
both_scales("product", ("wide", 256, 256, 8), MANY, 4901, (32, 128, 160, 256, 288, 512, 544, 640, 1056), True)
both_scales("product", ("wide", 256, 256, 8), [600] * 3, 3001, (256, 544, 1152), True)
both_scales("product", ("wide", 256, 256, 8), [257, 2, 255], 8192, (128, 800), True)
for K in (32, 288, 1152):
    case("product", ("stream", 32, 64, 4, False, False), [1, 0, 90, 17], 70, K, True, gap=1)
    case("product", ("stream", 32, 64, 4, False, False), [1, 0, 90, 17], 70, K, True, shift=5, scale_gap=1)

# BF16 rows
both_scales("product", ("stream", 16, 16, 4), [1, 0, 3, 2], 37, (32, 160, 512, 2048, 2080))
both_scales("product", ("stream", 32, 16, 4), [12, 0, 20, 33], 37, (32, 160, 512, 2048, 2080))
both_scales("product", ("stream", 16, 64, 4), TWO, 130, (32, 160, 512, 1056))
both_scales("product", ("stream", 32, 64, 4), TWELVE, 391, (32, 160, 512, 1056))
both_scales("product", ("strip", 16, 32, 4), TWO, 261, (32, 160, 256, 288, 1152))
both_scales("product", ("strip", 32, 64, 4), TWELVE, 1291, (32, 160, 256, 288, 1152))
both_scales("product", ("strip", 64, 32, 4), FORTY, 301, (32, 160, 256, 288, 1152, 2048))
both_scales("product", ("wide", 128, 256, 8), [100, 0, 129, 1], 16391, (32, 128, 160, 544, 640))
both_scales("product", ("wide", 256, 256, 8), MANY, 33001, (32, 128, 160, 544, 640))
for K in (32, 288, 1152):
    case("product", ("stream", 32, 64, 4, False, False), [1, 0, 90, 17], 70, K, gap=1)
    case("product", ("stream", 32, 64, 4, False, False), [1, 0, 90, 17], 70, K, shift=3)
    case("product", ("wide", 128, 256, 8, False, False), MANY, 16391, K, gap=1)

# The gradient: N is what is added up
for N in (8, 40, 264):
    case("grad", ("stream", 16, 256, 8, True, False), [1, 0, 3, 2], N, 800)
    case("grad", ("stream", 16, 256, 4, True, False), TWO, N, 288)
    case("grad", ("stream", 32, 256, 8, True, False), [12, 0, 20, 33], N, 800)
    case("grad", ("stream", 32, 256, 4, True, False), TWELVE, N, 800)
    case("grad", ("stream", 16, 256, 8, False, False), [1, 0, 3, 2], N + 3, 800)
    case("grad", ("stream", 16, 256, 4, False, False), TWO, N, 288, gap=1)
    case("grad", ("stream", 32, 256, 8, False, False), [12, 0, 20, 33], N, 800, shift=1)
    case("grad", ("stream", 32, 256, 4, False, False), TWELVE, N + 1, 800)
for N in (8, 72, 264, 1048):
    case("grad", ("wide", 128, 256, 8, True, False), [100, 0, 129, 1], N, 16416)
    case("grad", ("wide", 128, 256, 8, True, True), [100, 0, 129, 1], N, 16512)
    case("grad", ("wide", 128, 256, 8, True, False), [100, 0, 129, 1], N, 16512, ws_shift=1)
    case("grad", ("wide", 256, 256, 8, True, False), MANY, N, 8224)
    case("grad", ("wide", 256, 256, 8, True, True), MANY, N, 8320)
    case("grad", ("wide", 256, 256, 8, True, False), MANY, N, 8320, ws_shift=3)
    case("grad", ("wide", 256, 256, 8, True, True), MANY, N, 8320, gap=8)
for N in (9, 261, 1031):
    case("grad", ("wide", 128, 256, 8, False, False), [700, 0, 513, 130], N, 3968)
    case("grad", ("wide", 256, 256, 8, False, False), [700, 0, 513, 130], N, 16416)


def name(c):
    kernel, rows, outs, waves, vec, whole = c["takes"]
    return "%s-%s-%s-%dx%d-%dw%s%s-%dx%s-N%d-K%d-%d.%d.%d.%d" % (c["op"], "mx" if c["mx"] else "bf16", kernel, rows, outs, waves, "" if vec else "-anywhere",
                                                               "-words" if whole else "", len(c["counts"]), max(c["counts"]), c["N"], c["K"], c["gap"],
                                                               c["shift"], c["scale_gap"], c["ws_shift"])
