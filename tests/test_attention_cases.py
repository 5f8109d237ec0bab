"""Every kernel that cache_attention() chooses from, undivided and in parts, has a case that is compared with 64 bits (no GPU needed)."""
import ctypes
import itertools
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.abspath(__file__)))
import attention_cases as cases   # noqa: E402

import paper_2410_03355_b200 as lt   # noqa: E402
from paper_2410_03355_b200 import cache as binding   # noqa: E402

TYPES = {"bf16": torch.bfloat16, "f32": torch.float32}


def path(c):
    class View:   # a cache of which only the sizes are looked at
        struct = binding._CacheStruct(1 << 20, 1 << 20, 1 << 20, 1 << 20, 1000, c["H"], c["S"], c["D"])
        _at = ctypes.addressof(struct)
    B, width = len(c["lengths"]), c["room"] // c["S"]
    need = lt.cache_attention_workspace_bytes(B, c["R"], c["H"] * c["G"], View, width, dtype=TYPES[c["dtype"]])
    return cases.path_of(c["dtype"], B, c["R"], c["H"], c["G"], c["D"], c["S"], width, need)


def test_every_kernel_has_a_case():
    have = {path(c) for c in cases.CASES}
    want = {("few", rows, DP, t, parts) for rows, DP, t, parts in itertools.product((8, 16), (64, 128), ("bf16", "f32"), (False, True))}
    want |= {("mid", 64, DP, "bf16", parts) for DP, parts in itertools.product((64, 128), (False, True))}
    want |= {("wide", rows, DP, t, parts) for rows, DP, t, parts in itertools.product((64, 128), (64, 128), ("bf16", "f32"), (False, True))}
    assert want - have == set()
    assert have - want == set()


def test_names_are_different():
    names = [cases.name_of(c) for c in cases.CASES]
    assert len(set(names)) == len(names)
