"""Shapes of attention of trees, one for each way that the plan takes them: which launches, which forms of a workgroup, whether the sequences'
keys are cut, and what joins the parts.  Test infrastructure."""
from __future__ import annotations

import os
import shutil
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))

# batch, nodes, q heads, kv heads, d, prefix, pages of a sequence, page, type, quantised
CASES = [
    (2, 5, 1, 1, 96, 0, 0, 16, "bf16", False), (1, 32, 12, 3, 128, 0, 0, 4, "bf16", True), (141, 6, 32, 8, 80, 0, 0, 16, "fp16", False),
    (1, 4, 17, 1, 128, 0, 320, 4, "fp16", False), (1, 41, 7, 1, 96, 0, 19, 64, "bf16", True), (5, 5, 45, 3, 128, 0, 280, 4, "bf16", False),
    (92, 19, 6, 1, 80, 2, 1, 4, "fp16", False), (12, 45, 16, 8, 128, 2, 1, 4, "fp16", True), (2, 52, 80, 16, 80, 0, 1, 4, "bf16", False),
    (67, 38, 3, 1, 128, 0, 1, 4, "bf16", True), (1, 24, 9, 1, 80, 0, 260, 4, "fp16", False), (2, 15, 9, 1, 128, 0, 22, 64, "fp16", True),
    (5, 52, 4, 1, 80, 0, 297, 4, "bf16", False), (45, 31, 8, 1, 128, 1, 1, 4, "bf16", False), (3, 54, 54, 3, 80, 4, 1, 4, "fp16", True),
    (4, 57, 36, 3, 128, 0, 1, 4, "fp16", False), (60, 27, 5, 1, 80, 0, 1, 4, "bf16", True), (1, 18, 1, 1, 128, 0, 18, 64, "bf16", False),
    (5, 2, 27, 3, 80, 0, 152, 8, "fp16", True), (21, 5, 10, 1, 128, 0, 129, 8, "fp16", False), (172, 18, 2, 1, 80, 1, 1, 4, "bf16", False),
    (55, 17, 8, 8, 128, 2, 1, 4, "bf16", True), (153, 10, 4, 2, 80, 0, 1, 4, "fp16", False), (17, 3, 96, 16, 128, 0, 1, 4, "fp16", True),
    (1, 2, 1, 1, 128, 0, 161, 4, "bf16", False), (1, 10, 26, 2, 128, 0, 33, 16, "bf16", True), (3, 11, 32, 16, 80, 0, 9, 64, "fp16", False),
    (37, 2, 8, 8, 128, 2, 0, 32, "fp16", False), (213, 3, 3, 3, 80, 1, 0, 4, "bf16", True), (20, 2, 16, 16, 128, 0, 1, 4, "bf16", False),
    (81, 2, 4, 4, 80, 0, 1, 4, "fp16", True), (1, 2, 1, 1, 128, 4, 0, 16, "fp16", False), (1, 2, 1, 1, 80, 2, 0, 4, "bf16", True),
    (1, 2, 1, 1, 128, 0, 1, 4, "bf16", False), (1, 2, 1, 1, 80, 0, 1, 4, "fp16", True), (2, 3, 14, 1, 128, 567, 0, 32, "fp16", False),
    (28, 3, 4, 1, 80, 778, 0, 8, "bf16", True), (34, 4, 48, 8, 128, 1, 0, 64, "bf16", False), (1, 6, 11, 1, 96, 4, 144, 8, "fp16", False),
    (4, 14, 5, 1, 128, 103, 258, 4, "fp16", True), (1, 40, 28, 4, 80, 17, 81, 16, "bf16", False), (162, 5, 30, 2, 128, 2865, 9, 16, "bf16", False),
    (25, 8, 144, 16, 96, 2284, 6, 16, "fp16", True), (4, 9, 2, 1, 128, 2, 320, 4, "fp16", False), (7, 13, 3, 1, 80, 6, 24, 64, "bf16", True),
    (4, 9, 32, 16, 128, 4, 300, 4, "bf16", False), (140, 19, 2, 2, 112, 1109, 1, 16, "fp16", False), (269, 22, 1, 1, 128, 1224, 7, 4, "fp16", True),
    (12, 3, 2, 1, 80, 285, 30, 4, "bf16", False), (5, 13, 4, 1, 128, 275, 140, 4, "bf16", True), (6, 9, 20, 4, 80, 420, 3, 8, "fp16", False),
    (210, 3, 4, 4, 128, 871, 17, 4, "fp16", False), (35, 2, 16, 16, 80, 2800, 1, 16, "bf16", True), (36, 4, 1, 1, 128, 532, 0, 16, "bf16", False),
    (15, 2, 10, 2, 80, 873, 0, 4, "fp16", True), (116, 5, 17, 1, 128, 1, 0, 64, "fp16", False), (2, 37, 2, 1, 80, 1, 302, 4, "bf16", False),
    (2, 23, 8, 2, 128, 9, 263, 4, "bf16", True), (17, 17, 4, 1, 96, 26, 304, 4, "fp16", False), (35, 8, 72, 8, 128, 2772, 21, 4, "fp16", False),
    (69, 11, 24, 4, 80, 3139, 1, 16, "bf16", True), (1, 49, 3, 1, 128, 3, 113, 16, "bf16", False), (1, 35, 8, 2, 80, 82, 79, 16, "fp16", True),
    (4, 44, 6, 2, 128, 178, 158, 8, "fp16", False), (41, 32, 48, 8, 80, 4607, 1, 32, "bf16", False), (106, 14, 36, 3, 128, 4191, 1, 64, "bf16", True),
    (3, 3, 15, 1, 80, 15, 40, 32, "fp16", False), (4, 2, 38, 2, 128, 2, 83, 16, "fp16", True), (58, 4, 5, 1, 80, 6, 22, 64, "bf16", False),
    (138, 2, 18, 2, 128, 1099, 2, 16, "bf16", False), (38, 6, 32, 8, 96, 1124, 1, 8, "fp16", True), (3, 3, 16, 1, 128, 194, 12, 16, "fp16", False),
    (16, 9, 2, 2, 80, 939, 5, 8, "bf16", True), (8, 47, 3, 1, 128, 410, 1, 4, "bf16", False), (208, 2, 16, 16, 80, 178, 1, 8, "fp16", False),
    (354, 2, 8, 8, 128, 377, 1, 64, "fp16", True), (3, 6, 1, 1, 96, 519, 0, 4, "bf16", False), (3, 7, 16, 8, 128, 1134, 0, 64, "bf16", True),
    (16, 2, 32, 16, 128, 5840, 0, 4, "fp16", False), (1, 4, 5, 1, 128, 8, 131, 8, "fp16", False), (1, 41, 8, 8, 96, 5, 41, 32, "bf16", True),
    (2, 2, 256, 16, 128, 27, 399, 4, "bf16", False), (3, 6, 1, 1, 80, 3, 6, 64, "fp16", False), (3, 2, 48, 8, 128, 459, 10, 32, "fp16", True),
    (4, 8, 32, 16, 96, 469, 1, 16, "bf16", False), (57, 1, 16, 16, 128, 601, 10, 32, "bf16", False), (61, 1, 16, 16, 96, 3318, 3, 64, "fp16", True),
    (2, 2, 1, 1, 128, 543, 0, 64, "fp16", False), (1, 1, 2, 1, 80, 834, 0, 4, "bf16", True), (1, 2, 1, 1, 128, 501, 5, 4, "bf16", False),
    (1, 2, 1, 1, 112, 734, 20, 8, "fp16", True), (7, 3, 6, 1, 256, 0, 0, 32, "fp16", False), (4, 59, 4, 2, 208, 0, 0, 64, "bf16", True),
    (439, 9, 2, 1, 256, 0, 0, 64, "bf16", False), (1, 6, 3, 1, 192, 0, 9, 64, "fp16", False), (1, 11, 24, 4, 256, 0, 142, 8, "fp16", True),
    (60, 2, 9, 1, 192, 0, 18, 32, "bf16", False), (135, 3, 6, 1, 256, 1, 1, 4, "bf16", False), (10, 49, 8, 2, 192, 1, 1, 4, "fp16", True),
    (138, 3, 6, 1, 256, 0, 1, 4, "fp16", False), (17, 3, 48, 8, 192, 0, 1, 4, "bf16", True), (1, 2, 1, 1, 256, 0, 70, 8, "bf16", False),
    (6, 3, 16, 2, 192, 0, 33, 16, "fp16", True), (45, 3, 8, 4, 256, 0, 133, 4, "fp16", False), (2, 2, 4, 1, 192, 1, 0, 8, "bf16", False),
    (1, 2, 3, 1, 256, 1, 0, 4, "bf16", True), (1, 2, 2, 2, 208, 0, 1, 4, "fp16", False), (1, 2, 1, 1, 256, 0, 1, 4, "fp16", True),
    (1, 7, 3, 1, 256, 206, 0, 4, "bf16", False), (6, 52, 1, 1, 256, 464, 0, 16, "bf16", True), (111, 2, 19, 1, 192, 1, 0, 8, "fp16", False),
    (1, 2, 9, 1, 256, 44, 198, 4, "fp16", False), (1, 2, 144, 16, 192, 3, 72, 16, "bf16", True), (62, 17, 1, 1, 256, 168, 20, 32, "bf16", False),
    (101, 10, 6, 3, 208, 2147, 1, 32, "fp16", False), (132, 19, 2, 2, 256, 2377, 45, 8, "fp16", True), (2, 9, 1, 1, 208, 188, 4, 4, "bf16", False),
    (12, 4, 6, 2, 256, 116, 9, 32, "bf16", True), (21, 13, 4, 4, 192, 1, 12, 16, "fp16", False), (439, 2, 2, 2, 256, 332, 5, 8, "fp16", False),
    (95, 2, 4, 4, 192, 1429, 1, 64, "bf16", True), (1, 2, 1, 1, 256, 241, 0, 4, "bf16", False), (3, 2, 1, 1, 208, 445, 0, 4, "fp16", True),
    (1, 2, 1, 1, 256, 151, 13, 8, "fp16", False), (1, 2, 1, 1, 256, 339, 15, 4, "bf16", True), (4, 2, 8, 2, 64, 0, 0, 8, "bf16", False),
    (44, 5, 38, 2, 48, 0, 0, 8, "fp16", True), (1, 27, 3, 1, 64, 0, 41, 32, "fp16", False), (2, 4, 136, 8, 48, 0, 264, 4, "bf16", True),
    (26, 43, 9, 3, 64, 1, 1, 4, "bf16", False), (128, 9, 9, 1, 48, 1, 1, 4, "fp16", True), (29, 5, 51, 3, 64, 0, 1, 4, "fp16", False),
    (76, 9, 11, 1, 48, 0, 1, 4, "bf16", True), (1, 13, 2, 1, 64, 0, 72, 16, "bf16", False), (43, 3, 9, 1, 48, 0, 77, 16, "fp16", True),
    (2, 20, 1, 1, 64, 11, 259, 4, "fp16", False), (1, 5, 7, 1, 48, 2, 138, 8, "bf16", True), (37, 3, 48, 8, 64, 0, 1, 4, "bf16", False),
    (17, 11, 32, 16, 48, 0, 1, 4, "fp16", True), (1, 2, 1, 1, 64, 0, 44, 16, "fp16", False), (35, 2, 15, 1, 48, 0, 17, 32, "bf16", True),
    (87, 4, 10, 1, 64, 1, 0, 4, "bf16", False), (27, 4, 16, 16, 48, 1, 0, 64, "fp16", True), (320, 2, 1, 1, 64, 0, 1, 4, "fp16", False),
    (381, 2, 1, 1, 48, 0, 1, 4, "bf16", True), (1, 3, 1, 1, 64, 1, 0, 8, "bf16", False), (1, 6, 2, 1, 48, 1, 0, 64, "fp16", True),
    (2, 2, 1, 1, 64, 0, 1, 4, "fp16", False), (2, 2, 1, 1, 48, 0, 1, 4, "bf16", True), (10, 3, 3, 1, 64, 1165, 0, 8, "bf16", False),
    (138, 19, 3, 1, 48, 1, 0, 8, "fp16", True), (1, 10, 7, 1, 64, 2, 39, 32, "fp16", False), (4, 11, 24, 4, 48, 142, 140, 8, "bf16", True),
    (151, 9, 15, 1, 64, 2169, 1, 16, "bf16", False), (65, 16, 20, 2, 48, 2151, 1, 32, "fp16", True), (3, 11, 2, 1, 64, 177, 17, 64, "fp16", False),
    (8, 17, 8, 4, 48, 324, 39, 32, "bf16", True), (131, 2, 18, 2, 64, 1508, 1, 8, "bf16", False), (67, 13, 8, 4, 48, 1089, 10, 4, "fp16", True),
    (2, 2, 20, 1, 64, 1, 196, 4, "fp16", False), (5, 24, 9, 1, 48, 122, 163, 4, "bf16", True), (155, 2, 4, 4, 64, 1738, 8, 8, "bf16", False),
    (588, 2, 1, 1, 48, 2480, 1, 64, "fp16", True), (1, 2, 13, 1, 64, 1291, 0, 8, "fp16", False), (2, 32, 16, 16, 64, 13090, 0, 32, "bf16", True),
    (1, 3, 6, 1, 64, 2, 25, 64, "bf16", False), (2, 32, 16, 16, 64, 2, 31, 64, "fp16", True), (5, 2, 2, 1, 64, 2, 58, 16, "fp16", False),
    (4, 16, 16, 16, 48, 116, 189, 4, "bf16", True), (50, 1, 16, 16, 64, 5082, 4, 8, "bf16", False), (55, 1, 16, 16, 48, 9641, 1, 32, "fp16", True),
    (2, 2, 1, 1, 64, 2779, 0, 16, "fp16", False), (2, 3, 1, 1, 48, 892, 0, 4, "bf16", True), (1, 2, 1, 1, 64, 951, 1, 64, "bf16", False),
    (1, 2, 1, 1, 48, 813, 2, 64, "fp16", True),
]


def name(case):
    return "x".join(str(x) for x in case[:8]) + f"_{case[8]}_{'e4m3' if case[9] else 'same'}"


def pages_of(case):
    """Pages of the case's cache."""
    return -(-case[5] // case[7]) + case[0] * case[6] + 2


def build_driver(folder):
    """tests/tree_plan_driver.cpp: the plan alone, host code."""
    if shutil.which("hipcc") is None:
        pytest.skip("no hipcc")
    exe = os.path.join(str(folder), "plan")
    r = subprocess.run(["hipcc", "-x", "hip", "--cuda-host-only", "-std=c++17", "-O1", "-Wall", "-Wextra", "-I", os.path.join(ROOT, "include"),
                        "-I", os.path.join(ROOT, "paper_2601_12698_amd", "csrc"), os.path.join(ROOT, "tests", "tree_plan_driver.cpp"), "-o", exe],
                       stdout=subprocess.PIPE, stderr=subprocess.STDOUT, text=True, timeout=600)
    assert r.returncode == 0, r.stdout[-4000:]
    return exe


def plans_of(driver, cases):
    """For each case what the driver says of it, None where there is nothing to do or the shape is refused."""
    lines = "".join(f"{b} {n} {hq} {hk} {d} {page} {pages_of(c)} {prefix} {width} {int(dtype == 'fp16')} {int(quantised)}\n"
                    for c in cases for b, n, hq, hk, d, prefix, width, page, dtype, quantised in (c,))
    r = subprocess.run([driver], input=lines, stdout=subprocess.PIPE, stderr=subprocess.STDOUT, text=True, timeout=300)
    assert r.returncode == 0, r.stdout[-4000:]
    got = [line.split() for line in r.stdout.splitlines()]
    assert len(got) == len(cases)
    return [f[1:] if len(f) == 8 else None for f in got]


def ways_of(driver, cases):
    """The same without the number of splits and the order of the sequences."""
    return [p and (int(p[0]), *p[1:4], p[6]) for p in plans_of(driver, cases)]


# without keys of their own, and with lists and lengths that are not there, in more workgroups than the chip has places
WITHOUT_OWN = [(20, 3, 80, 16, 256, 2, 0, 32, "fp16", True), (60, 20, 64, 16, 64, 40, 0, 16, "bf16", False), (40, 10, 240, 16, 128, 5, 0, 8, "fp16", False),
               (40, 24, 224, 16, 112, 100, 0, 4, "bf16", True), (50, 9, 16, 16, 192, 33, 0, 64, "bf16", True)]
