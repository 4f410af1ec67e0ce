"""Which shapes the microscaled 4-bit products take (csrc/mx4_rule.hpp, host code), and that the GPU tests reach all of them."""
import os
import shutil
import subprocess

import pytest

import test_gpu_mx4_shapes as G

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
MAT = ["small", "tile32", "tile64", "tile64w", "tile128"]
FFN = ["thin", "small", "tall"]


@pytest.fixture(scope="module")
def rule(tmp_path_factory):
    if shutil.which("g++") is None:
        pytest.skip("g++ not found")
    d = tmp_path_factory.mktemp("rule")
    src, exe = d / "rule.cpp", d / "rule"
    # (the layouts alone: the plan's device code is for hipcc)
    (d / "expert_plan.hpp").write_text('#pragma once\n#include <stddef.h>\nnamespace dymoe { static inline size_t expert_plan_bytes(size_t P, size_t tiles) '
                                       '{ return (8 + (2 * P + 3) / 4 * 4 + 16 * tiles) * 4; } }\n')
    for name in ("mx4_layout.hpp", "mx4_rule.hpp"):
        shutil.copy(os.path.join(ROOT, "paper_2603_19172_amd", "csrc", name), d / name)
    src.write_text('#include <cstdio>\n#include <cstdlib>\n#include "mx4_rule.hpp"\n'
                   'int main(int n, char** a) { long v[6]; for (int i = 0; i + 1 < n; i++) v[i] = atol(a[i + 1]); '
                   'if (n == 7) { auto c = dymoe::mx4_ffn_choice(v[0], v[1], v[2], v[3], v[4], v[5]); '
                   'std::printf("%d %d %d %d\\n", (int)c.shape, c.up_waves, c.down_waves, c.splits); return 0; } '
                   'auto c = dymoe::mx4_mat_choice(v[0], v[1], v[2], v[3], v[4]); std::printf("%d %d %d\\n", (int)c.shape, (int)c.fuse, c.waves); }\n')
    subprocess.run(["g++", "-std=c++17", "-O1", "-Wall", "-Werror", "-fsanitize=address,undefined", "-fno-sanitize-recover=all", "-I", str(d),
                    str(src), "-o", str(exe)], check=True)

    def ask(*v):
        out = subprocess.run([str(exe)] + [str(int(i)) for i in v], check=True, capture_output=True, text=True).stdout
        return tuple(int(i) for i in out.split())
    return ask


@pytest.fixture(scope="module")
def product(rule):
    def ask(T, N, K, coded=0, num_cu=256):
        shape, fuse, waves = rule(T, N, K, coded, num_cu)
        return MAT[shape], bool(fuse), waves
    return ask


@pytest.fixture(scope="module")
def experts(rule):
    def ask(T, H, F, E, k, num_cu=256):
        v = rule(T, H, F, E, k, num_cu)
        return (FFN[v[0]], *v[1:])
    return ask


def test_the_gpu_tests_take_the_shapes_they_name(product, experts):
    for shape, T, N, K in G.PRODUCTS:
        assert product(T, N, K)[0] == product(T, N, K, coded=1)[0] == shape, (shape, T, N, K)
    assert {p[0] for p in G.PRODUCTS} == set(MAT)
    small = [product(*p[1:]) for p in G.PRODUCTS if p[0] == "small"] + [product(*s) for s in G.G.SIZES]
    assert {(s[1], s[2]) for s in small if s[0] == "small"} >= {(True, 8), (False, 8), (False, 4)}
    for T, H, F, E, k, splits in G.TALL:
        assert experts(T, H, F, E, k) == ("tall", 0, 0, splits), (T, H, F, E, k)
    assert {t[-1] for t in G.TALL} == {1, 2, 4}
    for T, H, F, E, k, up, down in G.STRIPS:
        assert experts(T, H, F, E, k) == ("small", up, down, 1), (T, H, F, E, k, experts(T, H, F, E, k))
    assert {s[5] for s in G.STRIPS} == {1, 2, 4} and {s[6] for s in G.STRIPS} == {1, 2, 4, 8}
    for c in G.THIN:
        assert experts(*c)[0] == "thin", c
    # last tiles of every number of fragments
    for shape, rows in (("tile64", 64), ("tile64w", 64), ("tile128", 128)):
        assert {(p[1] % rows + 31) // 32 for p in G.PRODUCTS if p[0] == shape} >= set(range(1, rows // 32))


def test_both_sides_of_each_line(product, experts):
    assert product(1, 4096, 4096) == ("small", True, 8) and product(1, 4096, 4096, coded=1) == ("small", False, 8)
    assert product(4, 4096, 4096)[1] and not product(5, 4096, 4096)[1] and product(32, 4096, 512)[1] and not product(33, 64, 64)[1]
    assert product(8, 12768, 4096) == ("small", False, 8) and product(8, 12800, 4096) == ("small", False, 4)
    assert product(32, 1 << 24, 512)[0] == "small" and product(33, 6144, 2048)[0] == "small" and product(33, 6145, 2048)[0] == "tile32"
    assert product(33, 4096, 2049)[0] == "small" and product(33, 4097, 2049)[0] == "tile32"
    assert product(64, 16384, 512)[0] == "tile32" and product(64, 16385, 512)[0] == "tile64" and product(64, 65536, 512)[0] == "tile64"
    assert product(64, 65537, 512)[0] == "tile128" and product(128, 32769, 512)[0] == "tile64w"
    assert product(128, 65280, 512)[0] == "tile64w" and product(128, 65281, 512)[0] == "tile128"
    assert experts(2, 4096, 14336, 8, 2)[0] == "thin" and experts(3, 4096, 14336, 8, 2)[0] == "small"
    assert experts(4, 2048, 768, 128, 8)[0] == "thin" and experts(5, 2048, 768, 128, 8)[0] == "small" and experts(1, 128, 128, 128, 65)[0] == "small"
    assert experts(1, 131072, 768, 8, 2)[0] == "small" and experts(1, 2048, 131072, 8, 1)[0] == "small"
    assert experts(80, 4096, 14336, 8, 2)[0] == "small" and experts(81, 4096, 14336, 8, 2)[0] == "tall" and experts(32, 256, 256, 1, 1)[0] == "small"
    assert experts(1, 4096, 14336, 8, 3)[0] == "thin" and experts(8192, 4096, 14336, 8, 1)[3] == 1


@pytest.mark.parametrize("num_cu", [1, 7, 32, 256, 304])
def test_any_chip_and_any_size_has_a_shape(product, experts, num_cu):
    for T, N, K in ((1, 1, 1), (1 << 24, 1, 1), (1, 1 << 24, 131072), (1 << 24, 4096, 131072), (300, 70, 129)):
        for coded in (0, 1):
            assert product(T, N, K, coded, num_cu)[0] in MAT
    for T, H, F, E, k in ((1, 1, 1, 1, 1), (1 << 22, 64, 64, 8, 8), (1000, 131072, 131072, 1024, 10), (64, 64, 131072, 1, 1)):
        shape, up, down, splits = experts(T, H, F, E, k, num_cu)
        assert shape in FFN and up in (0, 1, 2, 4) and down in (0, 1, 2, 4, 8) and splits in (1, 2, 4)


def test_rows_and_their_codes_are_summed_alike(product):
    for T, N, K in ((1, 12769, 4096), (1, 14336, 4096), (4, 13001, 4096), (5, 13001, 4096), (32, 12800, 512), (33, 12800, 512), (1, 4096, 14336), (8, 12800, 4096)):
        (shape, fuse, waves), coded = product(T, N, K), product(T, N, K, coded=1)
        assert coded == (shape, False, waves) and (waves == 8 or not fuse), (T, N, K)
