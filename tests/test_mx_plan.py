"""Which kernel a product with experts in 4 bits, or its gradient, takes (host arithmetic, csrc/mx_plan.h, compiled on its own): that the calls of
the GPU tests take what they are there for and leave no kernel out, and what the kernels require of a choice."""
import random

import pytest

import mx_cases as M


@pytest.fixture(scope="module")
def choose(tmp_path_factory):
    return M.compile_rule(tmp_path_factory.mktemp("mx_plan"))


def test_the_cases_take_what_they_are_for(choose):
    for c in M.CASES:
        assert M.taken_by(choose, c) == (c["op"], c["mx"]) + c["takes"], M.name(c)


def random_call(rng):
    """sizes over their whole ranges, experts and their rows also where the rules change over"""
    E = rng.choice([1, 2, 3, 8, 100, 160, 300, 512, 4096, int(2 ** rng.uniform(0, 12))])
    N, K = int(2 ** rng.uniform(0, 20)), 32 * int(2 ** rng.uniform(0, 15))
    cap = int(E * 2 ** rng.uniform(-3, 10)) + 1 if rng.random() < 0.8 else int(2 ** rng.uniform(0, 31))
    op, mx = rng.choice(["product", "product", "grad"]), False
    if op == "product":
        mx = rng.random() < 0.5
    width = (K // 2 if mx else 2 * K) if op == "product" else 2 * N
    far = rng.random() < 0.1
    stride = width + (int(2 ** rng.uniform(0, 34)) if far else 0)
    scales = K // 32 + (int(2 ** rng.uniform(0, 34)) if far and rng.random() < 0.5 else rng.choice([0, 0, 3, 4])) if mx else 0
    return dict(op=op, cap=min(cap, 2 ** 31 - 1), E=E, N=N, K=K, row_stride=stride, row_scales_stride=scales, mx=mx,
                rows_vec=stride % 16 == 0 and rng.random() < 0.8, w_words=K % 128 == 0 and rng.random() < 0.8, row_words=scales % 4 == 0 and rng.random() < 0.8)


def test_no_kernel_is_left_out(choose):
    """every choice that random calls meet is that of a case"""
    rng = random.Random(1)
    met = {choose(**random_call(rng)) for _ in range(200000)}
    covered = {(c["op"], c["mx"]) + c["takes"] for c in M.CASES}
    assert met <= covered, met - covered
    assert covered <= met, covered - met


def test_what_the_kernels_require(choose):
    rng = random.Random(2)
    for _ in range(50000):
        c = random_call(rng)
        op, mx, kernel, rows, outs, waves, vec, whole = choose(**c)
        if whole:
            assert c["w_words"] and (c["row_words"] or not mx) and vec
        if vec:
            assert c["rows_vec"] and (op == "product" or c["N"] % 8 == 0)
        if kernel == "wide":                                 # offsets within a tile in 32 bits, those of rows' scales in 31, less than 2^32 threads
            assert 256 * c["row_stride"] < 2 ** 31 and 256 * c["row_scales_stride"] < 2 ** 31 and (vec or not mx)
            width = c["K"] if op == "grad" else c["N"]
            assert (c["cap"] // 128 + min(c["cap"], c["E"])) * (width // 256 + 8) * 512 < 2 ** 32
            assert op == "product" or c["N"] >= 8
        elif op == "product" and vec:                        # offsets within 64 rows in 31 bits
            assert 64 * c["row_stride"] < 2 ** 31 and 64 * c["row_scales_stride"] < 2 ** 31
        elif op == "product":
            assert (kernel, rows, outs) == ("stream", 32, 64)
