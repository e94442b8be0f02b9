"""Sizes that take each kernel of the 8-bit products, ragged in every direction.  Not a test
module: test_plan_nn8 holds the plan to them on the CPU, test_parity_nn8_kernels runs them."""

# (M, N, K), gated, outputs, binary32 Y, kernel (rows of M of k_rows8, or k_tile8's tile), k in parts
CASES = [
    ((1, 110, 94), False, "y", False, 16, False),
    ((1, 102, 6147), False, "y", False, 16, True),
    ((19, 107, 98), False, "y", False, 32, False),
    ((18, 103, 6238), False, "y", False, 32, True),
    ((50, 111, 100), False, "y", False, 64, False),
    ((45, 102, 3532), False, "y", False, 64, True),
    ((273, 130, 109), False, "y", False, (128, 64), False),
    ((262, 132, 1251), False, "y", False, (128, 64), True),
    ((5644, 642, 94), False, "y", False, (128, 128), False),
    ((374, 1304, 10379), False, "y", False, (128, 128), True),
    ((5630, 730, 641), False, "y", False, (256, 128), False),
    ((1353, 280, 10299), False, "y", False, (256, 128), True),
    ((1838, 6907, 3619), False, "y", False, (256, 256), False),  # fewer tiles than workgroups, results below 48 MB
    ((5851, 2073, 3356), False, "y", False, (256, 256), False),
    ((4100, 6208, 2500), False, "y", False, (256, 256), False),  # more, results of 48 MB and more
    ((4100, 6199, 2507), False, "y", False, (256, 256), False),
    ((9, 100, 2250), False, "y", True, 16, False),
    ((3, 100, 2100), False, "y", True, 16, True),
    ((18, 4757, 1032), False, "y", True, 32, False),
    ((18, 109, 3265), False, "y", True, 32, True),
    ((4, 101, 94), False, "y", True, 64, False),
    ((33, 101, 6699), False, "y", True, 64, True),
    ((381, 148, 94), False, "y", True, (128, 64), False),
    ((264, 133, 447), False, "y", True, (128, 64), True),
    ((6006, 2285, 105), False, "y", True, (128, 128), False),
    ((315, 4103, 4749), False, "y", True, (128, 128), True),
    ((1929, 2052, 1326), False, "y", True, (256, 128), False),
    ((1024, 4100, 2500), False, "y", True, (256, 128), False),
    ((2048, 4096, 2600), False, "y", True, (256, 128), False),
    ((2770, 308, 4197), False, "y", True, (256, 128), True),
    ((1, 109, 92), False, "q", False, 16, False),
    ((1, 104, 1071), False, "q", False, 16, True),
    ((31, 103, 98), False, "q", False, 32, False),
    ((17, 103, 1246), False, "q", False, 32, True),
    ((46, 107, 101), False, "q", False, 64, False),
    ((34, 103, 1225), False, "q", False, 64, True),
    ((265, 133, 92), False, "q", False, (128, 64), False),
    ((316, 135, 392), False, "q", False, (128, 64), True),
    ((7373, 1795, 93), False, "yq", False, (128, 128), False),
    ((4202, 150, 3835), False, "q", False, (128, 128), True),
    ((6609, 577, 1336), False, "q", False, (256, 128), False),
    ((1024, 4100, 2500), False, "yq", False, (256, 128), False),
    ((2048, 2050, 1300), False, "yq", True, (256, 128), False),
    ((2809, 345, 4302), False, "q", False, (256, 128), True),
    ((1, 105, 99), True, "h", False, 16, False),
    ((1, 104, 5172), True, "h", False, 16, True),
    ((18, 104, 113), True, "h", False, 32, False),
    ((22, 102, 3451), True, "h", False, 32, True),
    ((36, 102, 95), True, "h", False, 64, False),
    ((36, 103, 3263), True, "h", False, 64, True),
    ((267, 83, 109), True, "h", False, (128, 64), False),
    ((265, 65, 1330), True, "h", False, (128, 64), True),
    ((4219, 472, 93), True, "h", False, (128, 128), False),
    ((1046, 195, 6279), True, "h", False, (128, 128), True),
    ((138, 11507, 845), True, "h", False, (256, 128), False),
    ((130, 2817, 6091), True, "h", False, (256, 128), True),
    ((1, 106, 100), True, "q", False, 16, False),
    ((1, 103, 1062), True, "q", False, 16, True),
    ((18, 105, 121), True, "q", False, 32, False),
    ((21, 102, 1114), True, "q", False, 32, True),
    ((50, 108, 102), True, "q", False, 64, False),
    ((39, 101, 1041), True, "q", False, 64, True),
    ((335, 69, 94), True, "q", False, (128, 64), False),
    ((269, 71, 409), True, "q", False, (128, 64), True),
    ((6722, 531, 261), True, "q", False, (128, 128), False),
    ((385, 843, 4372), True, "hq", False, (128, 128), True),
    ((1699, 534, 91), True, "hq", False, (256, 128), False),
    ((2048, 4100, 1300), True, "hq", False, (256, 128), False),
    ((1428, 395, 11290), True, "q", False, (256, 128), True),
]


def kernel_of(plan):
    """A plan's kernel as CASES name it."""
    return plan["rows"] or (plan["tile_n"], plan["tile_m"])


def case_id(c):
    (M, N, K), gated, out, f32, kernel, split = c
    name = f"rows{kernel}" if isinstance(kernel, int) else "tile%dx%d" % kernel
    return f"{M}x{N}x{K}-{'gated' if gated else 'plain'}-{out}{'32' if f32 else ''}-{name}{'-split' if split else ''}"
