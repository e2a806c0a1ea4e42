"""The rules that pick a kernel for attention over caches in 8 bits, held against measured times (B200, us); needs no GPU."""
import ctypes
import os
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module")
def rules(tmp_path_factory):
    at = tmp_path_factory.mktemp("rules")
    (at / "rules.cpp").write_text("""
#include "lagkv_quant_rules.h"
extern "C" int unit(long long heads, int D, int int8, int rows, long long S, int capped) {
    return lagkv::quant_unit_rows(heads, D, int8 != 0, rows, S, capped != 0);
}
extern "C" int cluster(long long units, long long S, int a, int b, int c) {
    const int fits[3] = {a, b, c};
    return lagkv::quant_cluster_ctas(units, S, fits);
}
""")
    subprocess.run([os.environ.get("CXX", "g++"), "-std=c++17", "-O1", "-shared", "-fPIC", f"-I{ROOT}/paper_2504_04704_b200/csrc", "-o", str(at / "rules.so"),
                    str(at / "rules.cpp")], check=True)
    lib = ctypes.CDLL(str(at / "rules.so"))
    lib.unit.argtypes = [ctypes.c_longlong, ctypes.c_int, ctypes.c_int, ctypes.c_int, ctypes.c_longlong, ctypes.c_int]
    lib.cluster.argtypes = [ctypes.c_longlong] * 2 + [ctypes.c_int] * 3
    return lib


# (KV heads of all sequences, channels, int8, query rows to a KV head, rows, capped): time with units of 8, 16, 32, 128 and 256 query rows
UNITS = [
    ((8, 128, 1, 16, 256, 0), (9.46, 10.62, 11.72, 14.10)),
    ((8, 64, 0, 16, 256, 0), (9.18, 10.47, 11.96, 12.88)),
    ((128, 128, 1, 16, 8192, 0), (87.40, 60.83, 81.77, 106.19)),
    ((128, 64, 1, 16, 8192, 0), (60.76, 43.32, 58.12, 96.04)),
    ((24, 128, 1, 20, 16411, 0), (52.88, 46.97, 40.30, 53.70)),
    ((24, 64, 1, 20, 16411, 1), (41.83, 39.25, 36.22, 88.20)),
    ((24, 64, 1, 35, 16411, 0), (55.70, 43.87, 45.45, 44.36)),
    ((24, 64, 1, 35, 16411, 1), (63.52, 52.85, 58.28, 88.49)),
    ((24, 64, 0, 35, 16411, 0), (53.14, 44.40, 43.86, 44.65)),
    ((24, 64, 0, 35, 16411, 1), (60.84, 53.64, 56.73, 89.50)),
    ((24, 96, 1, 35, 16411, 0), (67.72, 54.34, 53.58, 50.54)),
    ((24, 96, 1, 35, 16411, 1), (75.69, 63.36, 66.42, 95.12)),
    ((24, 128, 1, 35, 16411, 0), (80.80, 63.60, 64.84, 53.26)),
    ((24, 128, 1, 35, 16411, 1), (88.93, 72.56, 78.16, 96.68)),
    ((24, 128, 0, 40, 16411, 1), (80.18, 68.96, 75.62, 97.16)),
    ((8, 128, 0, 48, 32768, 1), (64.61, 49.81, 54.76, 76.26)),
    ((24, 128, 1, 64, 16411, 1), (135.63, 94.06, 78.74, 95.68)),
    ((128, 128, 1, 64, 8192, 0), (325.19, 219.98, 173.05, 117.38)),
    ((128, 128, 1, 64, 8192, 1), (350.28, 241.48, 194.24, 234.41)),
    ((512, 128, 1, 35, 512, 0), (90.29, 77.97, 80.22, 50.51)),
    ((512, 64, 1, 16, 512, 0), (32.65, 27.37, 35.36, 39.76)),
    ((128, 256, 0, 24, 8192, 0), (268.36, 178.86)),
    ((24, 256, 1, 64, 16411, 1), (239.75, 163.90)),
    ((16, 128, 1, 256, 131072, 0), (None, None, None, 346.0, 335.7)),
    ((64, 128, 1, 192, 32768, 0), (None, None, None, 353.4, 336.5)),
    ((8, 128, 1, 256, 32768, 0), (None, None, 145.22, 64.4, 71.1)),
    ((1, 128, 1, 192, 131072, 0), (None, None, None, 69.5, 95.2)),
    ((2, 96, 1, 256, 400000, 0), (None, None, None, 163.0, 179.6)),
    ((128, 64, 1, 256, 16384, 0), (None, None, None, 326.8, 320.9)),
]


@pytest.mark.parametrize("call,times", UNITS, ids=[" ".join(map(str, c)) for c, _ in UNITS])
def test_units(rules, call, times):
    """The unit of each call is the quickest measured, or within 3 % of it."""
    took = times[(8, 16, 32, 128, 256).index(rules.unit(*call))]
    assert took is not None and took <= 1.03 * min(t for t in times if t)


def test_no_unit_that_is_not_built(rules):
    """256 rows in int8 only, 256 channels in units of 8 and 16 only."""
    for heads in (1, 24, 512, 1 << 20):
        for D in (64, 96, 128, 256):
            for int8 in (0, 1):
                for rows in (1, 8, 9, 33, 128, 129, 4096):
                    for S in (1, 500, 16384, 1 << 20, (1 << 31) - 65537):
                        for capped in (0, 1):
                            got = rules.unit(heads, D, int8, rows, S, capped)
                            assert got in ((8, 16) if D == 256 else (8, 16, 32, 128, 256) if int8 and rows > 128 else (8, 16, 32, 128))


def test_the_calls_of_the_gpu_tests_reach_every_unit(rules):
    """The sizes that tests/test_gpu_quant_edges.py and tests/test_gpu_quant_attention.py count on."""
    room, wide = 40000, 1600000
    for D in (64, 96, 128):
        for int8 in (0, 1):
            reached = {rules.unit(6, D, int8, rows, room, 0) for rows in (8, 16, 28, 80)}
            assert reached == {8, 16, 32, 128}, (D, int8)
            assert rules.unit(4, D, int8, 256, room, 1) == 128
        for heads in (2, 4, 6, 10, 28):
            for capped in (0, 1):
                assert rules.unit(heads, D, 1, 160, -(-wide // heads), capped) == 256


# (KV heads of all sequences, rows), one token of 4 query heads to a KV head: time without and in clusters of 4, 8, 16
CLUSTERS = [
    ((8, 256), (7.89, 6.16, 6.24, 7.54)),
    ((8, 640), (8.63, 7.03, 6.26, 7.61)),
    ((8, 1216), (9.07, 8.06, 7.35, 7.87)),
    ((8, 2048), (9.41, 9.33, 7.55, 8.10)),
    ((8, 4096), (11.07, 12.95, 9.59, 9.40)),
    ((8, 8192), (12.93, 20.10, 13.42, 11.98)),
    ((8, 20000), (17.30, 41.26, 23.92, 19.85)),
    ((1, 1216), (8.50, 8.03, 7.25, 6.76)),
    ((4, 640), (8.30, 6.77, 6.27, 7.02)),
    ((4, 1216), (8.69, 8.05, 7.29, 6.76)),
    ((4, 4096), (9.97, 12.93, 9.32, 8.26)),
    ((8, 2560), (10.09, 10.15, 8.32, 9.08)),
    ((32, 256), (8.54, 6.51, 7.02, 20.35)),
    ((32, 2048), (11.89, 9.71, 8.80, 22.14)),
    ((32, 4096), (13.98, 13.48, 11.66, 25.74)),
    ((64, 256), (9.11, 7.06, 12.93, None)),
    ((64, 1216), (12.54, 9.87, 15.73, None)),
    ((64, 2560), (15.05, 12.89, 18.92, None)),
]


@pytest.mark.parametrize("call,times", CLUSTERS, ids=[" ".join(map(str, c)) for c, _ in CLUSTERS])
def test_clusters(rules, call, times):
    """The form of each call is the quickest measured, or within 3 % of it."""
    took = times[(1, 4, 8, 16).index(rules.cluster(*call, 64, 32, 8))]
    assert took is not None and took <= 1.03 * min(t for t in times if t)


def test_clusters_that_do_not_fit_are_not_taken(rules):
    """A device or context that runs fewer clusters of a size at once gets another size, or the form without."""
    assert rules.cluster(8, 4096, 64, 32, 8) == 16
    assert rules.cluster(8, 4096, 64, 32, 7) == 8
    assert rules.cluster(8, 4096, 64, 32, 0) == 8
    assert rules.cluster(8, 4096, 64, 7, 7) == 1                   # 4 CTAs would have too many rows each
    assert rules.cluster(8, 1216, 64, 0, 0) == 4
    assert rules.cluster(8, 1216, 7, 7, 7) == 1 and rules.cluster(1, 1, 0, 0, 0) == 1
