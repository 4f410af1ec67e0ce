"""Which shapes the 8-bit integer products take (csrc/int8_rule.hpp, host code), and that the GPU tests reach all of them."""
import os
import shutil
import subprocess

import pytest

import test_gpu_int8_shapes as G

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
MAT = ["thin", "small32", "small64", "split4", "split2", "one", "two"]
FFN = ["thin", "small", "grouped"]


@pytest.fixture(scope="module")
def rule(tmp_path_factory):
    if shutil.which("g++") is None:
        pytest.skip("g++ not found")
    d = tmp_path_factory.mktemp("rule")
    src, exe = d / "rule.cpp", d / "rule"
    src.write_text('#include <cstdio>\n#include <cstdlib>\n#include "int8_rule.hpp"\n'
                   'int main(int n, char** a) { long v[6]; for (int i = 0; i < 5; i++) v[i] = atol(a[i + 1]); '
                   'if (n == 6) { std::printf("%d 0\\n", (int)dymoe::i8_ffn_choice(v[0], v[1], v[2], v[3], v[4])); return 0; } '
                   'auto c = dymoe::i8_mat_choice(v[0], v[1], v[2], v[3], v[4]); std::printf("%d %d\\n", (int)c.shape, (int)c.fuse); }\n')
    subprocess.run(["g++", "-std=c++17", "-O1", "-Wall", "-Werror", "-fsanitize=address,undefined", "-fno-sanitize-recover=all",
                    "-I", os.path.join(ROOT, "paper_2603_19172_amd", "csrc"), str(src), "-o", str(exe)], check=True)

    def ask(*v):
        out = subprocess.run([str(exe)] + [str(int(i)) for i in v], check=True, capture_output=True, text=True).stdout
        return tuple(int(i) for i in out.split())
    return ask


@pytest.fixture(scope="module")
def product(rule):
    """product(T, N, K): the shape and whether its workgroups quantise the rows"""
    def ask(T, N, K, coded=0, num_cu=256):
        shape, fuse = rule(T, N, K, coded, num_cu, 0)
        return MAT[shape], bool(fuse)
    return ask


@pytest.fixture(scope="module")
def experts(rule):
    return lambda *v: FFN[rule(*v)[0]]


def test_the_gpu_tests_take_the_shapes_they_name(product, experts):
    for shape, T, N, K in G.PRODUCTS:
        assert product(T, N, K)[0] == product(T, N, K, coded=1)[0] == shape
    assert {p[0] for p in G.PRODUCTS} == set(MAT)
    for T, H, F in G.EXPERTS + G.LONG_ROWS:
        assert experts(T, H, F, len(G.LOADS) if T == 700 else 2, 2) == "grouped"
    assert min(G.LOADS) <= 160 < max(G.LOADS) and sum(G.LOADS) <= 1400
    # a last tile of each number of fragments, of tall tiles and of wide ones
    assert {(n % 128 + 31) // 32 for n in G.LOADS if n > 160} >= {1, 2, 3}
    assert {(n + 31) // 32 for n in G.LOADS if n <= 160} == {1, 2, 3, 4, 5}
    for T, E in G.SILU_T:
        assert experts(T, 128, 1, E, 1) == ("thin" if T <= 2 else "small" if T <= 20 * E or T <= 32 else "grouped")


def test_both_sides_of_each_line(product, experts):
    assert product(1, 4096, 4096) == ("thin", True) and product(4, 4096, 4096) == ("thin", False) and product(1, 4096, 4096, coded=1) == ("thin", False)
    assert product(8, 1 << 24, 128)[0] == "thin" and product(9, 1 << 24, 128)[0] == "one"
    assert product(16, 49152, 128)[0] == "thin" and product(16, 49153, 128)[0] != "thin" and product(17, 64, 128)[0] == "small32"
    assert product(32, 10240, 512)[0] == "small32" and product(33, 10240, 512)[0] == "small64" and product(33, 10241, 512)[0] == "split2"
    assert product(128, 32768, 1024)[0] == "split4" and product(128, 32769, 1024)[0] == "split2" and product(128, 32768, 896)[0] == "split2"
    assert product(128, 40960, 1024)[0] == "split2" and product(128, 40961, 1024)[0] == "one"
    assert product(2048, 8192, 2048)[0] == "two" and product(2048, 8192, 1920)[0] == "one" and product(2048, 7936, 2048)[0] == "one"
    assert experts(2, 4096, 14336, 8, 2) == "thin" and experts(3, 4096, 14336, 8, 2) == "small" and experts(1, 4096, 14336, 8, 5) == "small"
    assert experts(32, 2048, 768, 8, 8) == "small" and experts(33, 2048, 768, 8, 4) == "small" and experts(41, 2048, 768, 8, 4) == "grouped"
    assert experts(80, 4096, 14336, 8, 2) == "small" and experts(81, 4096, 14336, 8, 2) == "grouped"


@pytest.mark.parametrize("num_cu", [1, 7, 32, 256, 304])
def test_any_chip_and_any_size_has_a_shape(product, num_cu):
    for T, N, K in ((1, 1, 1), (1 << 24, 1, 1), (1, 1 << 24, 131072), (1 << 24, 4096, 131072), (300, 70, 129)):
        for coded in (0, 1):
            assert product(T, N, K, coded, num_cu)[0] in MAT
