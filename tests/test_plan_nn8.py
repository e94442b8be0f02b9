"""Which kernel an 8-bit product takes (CPU): the sizes of the parity tests take the kernels
that they are there for, and those are all kernels that any size takes."""
import ctypes
import os
import random
import subprocess

import pytest

import paper_1807_11091_amd as sa
from nn8_kernel_cases import CASES, case_id, kernel_of


@pytest.mark.parametrize("case", CASES, ids=case_id)
def test_cases_take_their_kernel(case):
    (M, N, K), gated, out, f32, kernel, split = case
    p = sa.product8_plan(M, N, K, gated, out, f32)
    assert (kernel_of(p), p["split"] > 1, p["exact"]) == (kernel, split, int(f32 or "q" in out))
    # parts of k are joined, and blocks of an 8-bit result that lie in several workgroups
    whole = not p["rows"] and p["tile_n"] // (2 if gated else 1) >= sa.BLOCK
    assert p["joined"] == int(split or ("q" in out and not whole))


def forms(gated, out, f32, kernel, split):
    return gated, "q" in out, f32 or "q" in out, kernel, split


def test_cases_cover_every_kernel():
    have = {forms(g, o, f, k, s) for _, g, o, f, k, s in CASES}
    kernels = [16, 32, 64, (128, 64), (128, 128), (256, 128)]
    for gated in (False, True):
        for eight, exact in ((False, False), (True, True)) if gated else ((False, False), (True, True), (False, True)):
            for k in kernels:
                for split in (False, True):
                    assert (gated, eight, exact, k, split) in have
    assert (False, False, False, (256, 256), False) in have
    rng = random.Random(5)
    for _ in range(20000):  # and no other one is reached
        M, N, K = (int(2 ** rng.uniform(0, hi)) for hi in (14, 14, 14))
        gated, out, f32 = rng.choice([(False, "y", False), (False, "y", True), (False, "q", False), (True, "h", False),
                                      (True, "q", False)])
        p = sa.product8_plan(M, N, K, gated, out, f32)
        assert forms(gated, out, f32, kernel_of(p), p["split"] > 1) in have, (M, N, K, gated, out, f32, p)


def test_plan_of_exact_products_and_of_nothing():
    assert sa.product8_plan(8192, 4096, 9830)["exact"] == 0
    exact = sa.product8_plan(8192, 4096, 9830, exact=True)
    assert exact["exact"] == 1 and exact == sa.product8_plan(8192, 4096, 9830, f32=True)
    assert sa.product8_plan(8192, 9830, 4096, True, "h", exact=True)["exact"] == 1
    for sizes in ((0, 5, 5), (5, 0, 5)):
        assert set(sa.product8_plan(*sizes).values()) == {0}
    assert sa.product8_plan(5, 5, 0)["split"] == 1


def test_plan_refuses_what_the_call_refuses():
    for sizes, kw in (((-1, 5, 5), {}), ((5, 5, 1 << 22), {}), ((5, 5, 5), dict(out="")), ((5, 5, 5), dict(gated=True, out="")),
                      ((5, 5, 5), dict(exact=2)), ((5, 5, 5), dict(gated=True, f32=True))):
        with pytest.raises(sa.StructAdmmError):
            sa.product8_plan(*sizes, **kw)
    assert sa.lib().structadmm_linear8_plan(None, None) == -1 and sa.lib().structadmm_glu8_plan(None, None) == -1


def test_info_layout_matches_header(tmp_path):
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    names = [n for n, _ in sa.Product8PlanInfo._fields_]
    lines = ["#include <stdio.h>", "#include <stddef.h>", '#include "structadmm.h"', "int main(void){"]
    lines += [f'printf("%zu\\n", offsetof(sa_product8_plan_info, {n}));' for n in names]
    lines += ['printf("%zu\\n", sizeof(sa_product8_plan_info));', "return 0;}"]
    src, exe = str(tmp_path / "l.c"), str(tmp_path / "l")
    with open(src, "w") as f:
        f.write("\n".join(lines))
    subprocess.check_call(["gcc", "-D__HIP_PLATFORM_AMD__", "-I", os.path.join(root, "include"), "-I", "/opt/rocm/include",
                           src, "-o", exe])
    got = [int(v) for v in subprocess.check_output([exe]).decode().split()]
    assert got == [getattr(sa.Product8PlanInfo, n).offset for n in names] + [ctypes.sizeof(sa.Product8PlanInfo)]
