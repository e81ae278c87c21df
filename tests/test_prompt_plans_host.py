"""Host-only: which kernels the planners of w4a16_prompt_attn and w8a8_gemm can pick, and that the GPU tests run each of them."""
import ctypes
import random

import pytest

from paper_2505_22179_amd import binding as B
from tests.test_gpu_prompt_paths import PATHS, PRODUCTS, plan_of
from tests.test_kv8_host import EINVAL, ENULL, EUNSUP

TICKETS = 16384


def test_descriptions_refuse():
    f, out = B.load().w4a16_prompt_attn_plan_describe, (ctypes.c_int * 3)()
    good = (100, 3, 50, 700, 8, 2, 128)
    assert f(*good, out) == 0 and f(*good, None) == ENULL
    for i, value, code in ((0, 0, EINVAL), (1, 0, EINVAL), (2, 0, EINVAL), (3, 0, EINVAL), (4, 9, EINVAL), (5, 0, EINVAL), (6, 0, EINVAL), (6, 96, EUNSUP), (1, 4097, EUNSUP)):
        assert f(*good[:i], value, *good[i + 1:], out) == code, (i, value)
    f, out = B.load_w8a8().w8a8_gemm_plan_describe, (ctypes.c_int * 4)()
    assert f(60, 64, 64, out) == 0 and f(60, 64, 64, None) == ENULL
    for sizes, code in (((0, 64, 64), EINVAL), ((1, 12, 64), EINVAL), ((1, 64, 24), EINVAL), ((1, 64, 65552), EUNSUP), ((2 ** 20 + 1, 64, 64), EUNSUP)):
        assert f(*sizes, out) == code, sizes


def test_every_kernel_of_the_attention_has_its_cases():
    """a plan is a kernel, its tile and D; the sizes that callers have reach no others"""
    rng, picked = random.Random(5), set()
    log = lambda lo, hi: int(round(lo * (hi / lo) ** rng.random()))
    for _ in range(40000):
        Hkv, group, n_seq, D = rng.choice([1, 2, 4, 8, 16]), rng.choice([1, 2, 4, 7, 8, 16]), log(1, 128), rng.choice([64, 128])
        max_q = log(1, 32768)
        picked.add(B.w4a16_prompt_attn_plan_describe(rng.randint(max_q, max(max_q, min(max_q * n_seq, 1 << 21))), n_seq, max_q, max_q + log(1, 200000) - 1, Hkv * group, Hkv, D)[:2] + (D,))
    assert picked == {plan_of(*case)[:2] + (case[3],) for case in PATHS.values()}
    assert picked == {(0, 32, 64), (0, 32, 128), (1, 128, 64), (1, 128, 128), (1, 256, 128), (2, 256, 64), (2, 256, 128)}


@pytest.mark.parametrize("path", PATHS)
def test_the_cases_take_the_kernels_that_they_are_named_for(path):
    lens, Hq, Hkv, D = PATHS[path]
    kind, height, groups = plan_of(lens, Hq, Hkv, D)
    assert path == {0: "few", 1: f"whole {height}", 2: "cut"}[kind] + f", D {D}"
    scratch = B.w4a16_prompt_attn_workspace_bytes(sum(n for n, _ in lens) + 2, len(lens), max(n for n, _ in lens), max(t for _, t in lens), Hq, Hkv, D) - TICKETS
    # whole tiles leave nothing behind; a workgroup of the others up to two pieces: outputs, maximum and sum of each row in fp32
    assert scratch == (0 if kind == 1 else groups * 2 * height * (D + 2) * 4)


def test_every_kernel_of_the_products_has_its_cases():
    rng, picked = random.Random(6), set()
    log = lambda lo, hi: int(round(lo * (hi / lo) ** rng.random()))
    for _ in range(40000):
        kind, tokens, channels, splits = B.w8a8_gemm_plan_describe(log(1, 8192), 8 * log(1, 8192), 16 * log(1, 2048))
        picked.add((kind, tokens, channels, splits > 1))
    cases = {p: B.w8a8_gemm_plan_describe(*sizes) for p, many in PRODUCTS.items() for sizes in many}
    for p, many in PRODUCTS.items():
        for sizes in many:
            kind, tokens, channels, splits = B.w8a8_gemm_plan_describe(*sizes)
            assert p == (kind, tokens, channels, splits > 1), (sizes, splits)
    assert picked == set(cases)
    assert all(len(many) >= 2 for many in PRODUCTS.values())
