"""Workspaces of the microscaled 4-bit calls: a program that holds that of its largest batch has enough for every smaller one, and the experts' holds
all parts of the pairs' outputs that the rule cuts a call into (csrc/mx4_layout.hpp, mx4_rule.hpp, host code)."""
import os
import random
import shutil
import subprocess

import pytest
import torch

from paper_2603_19172_amd import binding as B

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))

# H, F, E, k
LAYERS = [(2048, 768, 128, 8), (4096, 14336, 8, 2), (264, 1000, 2, 1), (300, 8300, 2, 1), (1030, 3100, 3, 2), (33, 131072, 1, 1), (256, 4096, 1024, 10),
          (131072, 4096, 2, 2)]


@pytest.mark.parametrize("H,F,E,k", LAYERS)
def test_a_larger_batch_has_no_smaller_workspace(H, F, E, k):
    edges = sorted({t for e in (32, 64, 128, 256, 512, 1024, 1536, 2048, 3000, 4096, 8192, 1 << 14, 1 << 16) for p in (e, e * 4, e // k, e * 20)
                    for t in (p - 1, p, p + 1) if t > 0} | set(range(0, 600)))
    nb = [B.moe_ffn_mx4_workspace_bytes(t, H, F, E, k) for t in edges]
    assert all(a <= b for a, b in zip(nb, nb[1:])), [(t, a, b) for t, a, b in zip(edges, nb, nb[1:]) if a > b][:5]


def test_the_other_calls_workspaces_grow_too():
    for f in (lambda t: B.matmul_mx4_workspace_bytes(t, 700, 4096), lambda t: B.route_balance_workspace_bytes(t, 130)):
        nb = [f(t) for t in range(0, 5000)]
        assert all(a <= b for a, b in zip(nb, nb[1:]))


@pytest.fixture(scope="module")
def ask(tmp_path_factory):
    if shutil.which("g++") is None:
        pytest.skip("g++ not found")
    d = tmp_path_factory.mktemp("layout")
    (d / "expert_plan.hpp").write_text('#pragma once\n#include <stddef.h>\nnamespace dymoe { static inline size_t expert_plan_bytes(size_t P, size_t tiles) '
                                       '{ return (8 + (2 * P + 3) / 4 * 4 + 16 * tiles) * 4; } }\n')
    for name in ("mx4_layout.hpp", "mx4_rule.hpp"):
        shutil.copy(os.path.join(ROOT, "paper_2603_19172_amd", "csrc", name), d / name)
    (d / "ask.cpp").write_text('#include <cstdio>\n#include "mx4_rule.hpp"\n'
                               'int main() { long T, H, F, E, k, cu; while (std::scanf("%ld %ld %ld %ld %ld %ld", &T, &H, &F, &E, &k, &cu) == 6) { '
                               'auto L = dymoe::mx4_ffn_layout(T, H, F, E, k); auto c = dymoe::mx4_ffn_choice(T, H, F, E, k, cu); '
                               'std::printf("%d %zu\\n", c.splits, L.plan - L.part); } }\n')
    subprocess.run(["g++", "-std=c++17", "-O1", "-Wall", "-Werror", "-fsanitize=address,undefined", "-fno-sanitize-recover=all", "-I", str(d),
                    str(d / "ask.cpp"), "-o", str(d / "ask")], check=True)

    def ask(cases):
        text = "\n".join(" ".join(str(v) for v in c) for c in cases)
        out = subprocess.run([str(d / "ask")], input=text, check=True, capture_output=True, text=True).stdout
        return [tuple(int(v) for v in line.split()) for line in out.splitlines()]
    return ask


def test_every_part_has_its_place(ask):
    rng = random.Random(7)
    cases = []
    for H, F, E, k in LAYERS:
        for T in [1, 33, 81, 128, 129, 512, 1024, 1025, 4096, 8192, 8193, 16384] + [int(2 ** rng.uniform(0, 15)) for _ in range(60)]:
            cases += [(T, H, F, E, k, cu) for cu in (1, 32, 256, 304)]
    seen = set()
    for (T, H, F, E, k, cu), (splits, held) in zip(cases, ask(cases)):
        seen.add(splits)
        assert held >= splits * T * k * (-(-H // 8) * 8) * 4, (T, H, F, E, k, cu)
    assert seen == {1, 2, 4}
    # and little more where the rule never cuts: 128 experts' down projection has tiles for every compute unit
    (splits, held), = ask([(1024, 2048, 768, 128, 8, 256)])
    assert splits == 1 and held == 1024 * 8 * 2048 * 4


@pytest.mark.gpu
@pytest.mark.parametrize("T,H,F,E,k", [(150, 300, 8300, 2, 1), (400, 264, 2100, 2, 1), (90, 2048, 768, 16, 8)])
def test_smaller_batches_in_the_largest_ones_workspace(T, H, F, E, k):
    """The batch of T tokens and smaller ones give the same bits in the workspace of T tokens, nothing behind it touched."""
    import test_gpu_mx4 as G
    ctx = B.Context(0)
    ex, _ = G.make_experts(ctx, 3, E, H, F)
    nb = B.moe_ffn_mx4_workspace_bytes(T, H, F, E, k)
    buf = torch.full((nb + 256,), 255, dtype=torch.uint8, device=G.DEV)
    for t in (T, T - 1, T // 2, 33, 5, 1):
        x = G.randn(t, t, H)
        idx, gate = G.choices(t, t, E, k)
        assert torch.equal(ctx.moe_ffn_mx4(x, idx, gate, ex.table, F, workspace=buf[:nb]), ctx.moe_ffn_mx4(x, idx, gate, ex.table, F))
        assert (buf[nb:] == 255).all()
    ctx.close()
