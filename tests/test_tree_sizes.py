"""Workspace sizes of ecokv_decode_tree for calls that have nothing to do: nobody
continues a prompt, or there are no layers.  The queries run in a process of their own:
a division by zero ends it."""
import json
import os
import subprocess
import sys

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))

QUERIES = r"""
import json
import paper_2609_06663_amd as P
out = []
for L, fan in ((1, [0, 0]), (0, [0, 3]), (0, [0, 0]), (3, [0, 0, 0])):
    for Hq, Hkv in ((8, 8), (28, 4), (64, 1)):
        for D in (64, 128):
            s = P.Shape(L, Hq, Hkv, D, 4, [1000 * i for i in range(len(fan))])
            for mc, mt in ((0, 0), (100, 10), (6553, 700), (2 ** 31 - 1, 2 ** 31 - 65)):
                for nodes in (1, 4, 16, 64):
                    out.append(P.ecokv_decode_tree_workspace_size(s, fan, mc, mt, nodes))
print(json.dumps(out))
"""

CONTINUATIONS = r"""
import torch
import paper_2609_06663_amd as P
from paper_2609_06663_amd.pipeline import Continuations, EvictionPass
ep = EvictionPass(P.Shape(0, 8, 8, 128, 4, [0, 1000]), [100], device="cpu")
co = Continuations(ep, [2], 10, P.Rope(0), 16, 4)
print(co.workspace.numel())
"""


def run(code):
    r = subprocess.run([sys.executable, "-c", code], cwd=ROOT, capture_output=True, text=True, timeout=300)
    assert r.returncode == 0, (r.returncode, r.stderr[-500:])
    return json.loads(r.stdout)


def test_sizes_of_calls_that_have_nothing_to_do():
    sizes = run(QUERIES)
    assert len(sizes) == 4 * 3 * 2 * 4 * 4 and not any(sizes)


def test_continuations_of_no_layers():
    assert run(CONTINUATIONS) == 256


@pytest.mark.parametrize("nodes", [1, 16])
def test_a_prompt_that_nobody_continues_beside_one_that_is(nodes):
    import paper_2609_06663_amd as P
    s = P.Shape(1, 8, 8, 64, 4, [0, 1000, 2000])
    assert P.ecokv_decode_tree_workspace_size(s, [0, 0, 2], 100, 10, nodes) > 0
