"""CPU-side checks of the rule that chooses kernels and splits for attention over the 8-bit cache, called by its C++ name."""
import ctypes
import os
import random
import re
import subprocess

import pytest

import paper_2510_26527_amd as psd


class Plan(ctypes.Structure):
    _fields_ = [("rows", ctypes.c_int), ("splits", ctypes.c_int), ("range", ctypes.c_int)]


@pytest.fixture(scope="module")
def rules():
    if not os.path.exists(psd.LIB_PATH):
        from paper_2510_26527_amd import build
        build.build()
    syms = subprocess.run(["nm", "-D", "--defined-only", psd.LIB_PATH], check=True, capture_output=True, text=True).stdout.split()

    def find(name, restype):
        f = getattr(psd.lib(), next(s for s in syms if re.match(rf"_ZN3psd{len(name)}{name}E", s)))
        f.restype, f.argtypes = restype, [ctypes.c_int] * 6
        return f
    return find("kv8_attn_plan", Plan), find("kv8_attn_max_splits", ctypes.c_int)


def test_splits_cover_the_keys_and_stay_within_what_workspaces_are_sized_for(rules):
    plan, most = rules
    rng = random.Random(1)
    for _ in range(4000):
        h_kv, group, d = rng.choice([1, 2, 4, 8, 32]), rng.choice([1, 4, 7, 8]), rng.choice([64, 128])
        B, R = rng.choice([1, 2, 5, 16, 64, 200]), rng.choice([1, 2, 9, 16, 33, 128, 500, 2000])
        top = R + rng.choice([0, 1, 63, 64, 1000, 5000, 40000, 200000])
        bound = most(B, R, h_kv * group, h_kv, d, top)
        for n in {R, top, R + (top - R) // 2, R + (top - R) // 7}:
            p, blocks = plan(B, R, h_kv * group, h_kv, d, n), (n + 63) // 64
            assert 1 <= p.splits <= bound <= 1024 and p.rows in (16, 64, 128)
            assert (p.splits - 1) * p.range < blocks <= p.splits * p.range          # every split has keys, and none is left out
            assert psd.psd_kv8_attention_workspace_bytes(B, R, h_kv * group, h_kv, d, n) == (
                0 if p.splits == 1 else sum((x + 255) // 256 * 256 for x in (B * R * h_kv * group * p.splits * d * 4, B * R * h_kv * group * p.splits * 8)))


@pytest.mark.parametrize("rows,B,R,h_q,h_kv,d,n", [
    (16, 1, 1, 32, 8, 128, 5000), (16, 1, 9, 32, 8, 128, 4009), (16, 1, 200, 2, 2, 64, 200),
    (64, 3, 250, 12, 6, 64, 350), (64, 2, 170, 32, 16, 128, 240), (128, 3, 130, 64, 64, 64, 203), (128, 5, 70, 64, 64, 128, 160), (128, 2, 150, 90, 90, 128, 448),
    (128, 1, 140, 256, 1, 64, 320), (128, 2, 560, 32, 32, 64, 560), (16, 1, 100, 16, 4, 128, 4100), (128, 1, 100, 32, 8, 128, 4100), (16, 9, 12, 32, 8, 128, 2012), (64, 9, 12, 32, 8, 128, 4012), (64, 5, 3, 416, 52, 64, 65),
    (16, 4, 5, 32, 8, 128, 16005), (64, 4, 5, 32, 8, 128, 32005),
    (64, 17, 20, 16, 16, 128, 68), (64, 6, 40, 32, 32, 64, 1240), (64, 2, 150, 32, 8, 128, 448), (64, 2, 20, 130, 130, 64, 448),
    (64, 1, 140, 64, 1, 64, 320), (16, 1, 9, 32, 8, 128, 17009), (64, 1, 9, 32, 8, 128, 25009), (64, 2, 620, 8, 4, 64, 620), (128, 1, 2001, 32, 32, 128, 2001)])
def test_which_kernel_takes_which_rows(rules, rows, B, R, h_q, h_kv, d, n):
    """Among them the shapes with which the GPU tests mean to reach the blocks of 64 and of 128 rows."""
    assert rules[0](B, R, h_q, h_kv, d, n).rows == rows
