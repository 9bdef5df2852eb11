"""Which form of tree attention a batch takes (csrc/tree_plan.hpp), compiled for the host and looked at without a GPU."""
import os
import shutil
import subprocess

import pytest

import tree_shapes
from paper_2508_07101_amd import build as lib_build

CXX = shutil.which("g++") or shutil.which("c++")
pytestmark = pytest.mark.skipif(CXX is None, reason="no host compiler")


def _plans(tmp_path, shapes):
    src = tmp_path / "plan.cpp"
    src.write_text(r'''
#include <cstdio>
#include "tree_plan.hpp"
using namespace cusa;
int main() {
    int chosen, len, batch, G, g, nodes;
    while (std::scanf("%d %d %d %d %d %d", &chosen, &len, &batch, &G, &g, &nodes) == 6) {
        const TreePlan p = plan_tree(chosen ? TREE_CHOSEN : TREE_FULL, len, batch, G, g, nodes);
        std::printf("%d %d %d\n", p.rows, p.m_tiles, p.n_splits);
    }
    return 0;
}
''')
    exe = tmp_path / "plan"
    subprocess.check_call([CXX, "-std=c++17", "-O1", "-Wall", "-Werror", "-I", lib_build.CSRC, "-o", str(exe), str(src)])
    asked = "\n".join(f"{int(s['budget'] > 0)} {tree_shapes.bound(s)} {len(s['n'])} {s['G']} {s['H'] // s['G']} {max(s['n'])}" for s in shapes)
    return [tuple(map(int, line.split())) for line in subprocess.run([str(exe)], input=asked, capture_output=True, text=True, check=True).stdout.splitlines()]


def test_the_shapes_that_are_tested_take_the_forms_that_they_are_there_for(tmp_path):
    names = list(tree_shapes.SHAPES)
    for name, (rows, m_tiles, n_splits) in zip(names, _plans(tmp_path, [tree_shapes.SHAPES[n] for n in names])):
        s = tree_shapes.SHAPES[name]
        own = [n * s["H"] // s["G"] for n in s["n"]]
        assert rows == s["rows"], name
        if name.startswith("128"):
            assert all(64 < r <= 128 for r in own)
        elif rows == 256:                              # the first workgroup of each tree has the form of eight waves
            assert all(r > 128 for r in own), name
        else:
            assert m_tiles == 2 and all(128 < r <= 256 for r in own), name
        assert m_tiles == (max(own) + rows - 1) // rows
        if name in ("pieces", "long lists"):
            assert n_splits > 1, name
        if name in ("steps", "lists", "wide trees"):
            assert n_splits == 1, name


def test_the_widest_form_of_the_weights_tests(tmp_path):
    """test_gpu_tree_weights.py: 20 sequences under 64 nodes, 64 query heads over 16, of 104 to 5064 tokens."""
    shapes = [dict(H=64, G=16, before=[before] * 20, n=[64] * 20, budget=0) for before in (40, 64, 300, 1100, 5000)]
    assert all(rows == 256 for rows, _, _ in _plans(tmp_path, shapes))
