"""Which kernel an 8-bit product takes, from the library's own rules built for the host, and sizes for each of them."""
import ctypes
import os
import subprocess

from tests import host_lib as H

SM_COUNT = 148

# rows, features, k of products that go to each kernel, whatever the type, alignment or mask: tiles of 16, 32, 64 and 128 rows by how many blocks share k, ...
FEW = {
    (16, 1): (300, 264, 300), (16, 2): (17, 1000, 1155), (16, 8): (9, 140, 8200),
    (32, 1): (25, 12507, 300), (32, 2): (736, 140, 1036), (32, 4): (20, 2400, 2300), (32, 8): (17, 1033, 4256),
    (64, 1): (60, 15000, 260), (64, 2): (33, 9120, 1247), (64, 4): (256, 1152, 4608), (64, 8): (377, 200, 6800),
    (128, 2): (73, 8520, 6000), (128, 4): (655, 705, 3144), (128, 8): (752, 200, 15600),
}
ONE = [(1100, 1501, 1000), (1100, 1504, 520)]
PAIR = [(2304, 4100, 300), (4099, 2049, 1152)]
# ... to tiles of one SM without a mask and of a pair with one, and the other way round
MASKED_TO_PAIR = (4096, 1152, 4608)
MASKED_TO_ONE = (2304, 1152, 520)


def load(folder):
    from paper_2509_11628_b200 import build
    cuda = os.path.join(os.path.dirname(os.path.dirname(os.path.realpath(build._nvcc()))), "include")
    so = os.path.join(str(folder), "libmatmul8_plan.so")
    subprocess.check_call(["g++", "-std=c++17", "-O1", "-fPIC", "-shared", "-I", cuda, "-I", os.path.join(H.ROOT, "include"), "-I", build.CSRC, "-o", so,
                           os.path.join(build.CSRC, "speca_matmul8_plan.cpp"), os.path.join(H.ROOT, "tests", "c_abi", "matmul8_plan.cpp")])
    return ctypes.CDLL(so)


def plan(lib, m, n, k, dtype="bf16", eight=False, vectors=True, masked=False, sm_count=SM_COUNT):
    """("few", rows of a tile, shares of k), ("one",) or ("pair",)."""
    got = [ctypes.c_int(-1) for _ in range(3)]
    lib.host_plan_matmul8(m, n, k, 1 if dtype == "bf16" else 0, int(eight), int(vectors), int(masked), sm_count, *(ctypes.byref(x) for x in got))
    kernel, rows, ranks = (x.value for x in got)
    return ("few", rows, ranks) if kernel == 0 else ("one",) if kernel == 1 else ("pair",)
