"""The division of work of the attention of new tokens on a paged cache, replayed on the CPU: every block of keys of every tile
is taken exactly once, and what the last kernel needs to find the pieces agrees with who made them."""
import ctypes
import os
import random
import subprocess

import pytest

HERE = os.path.dirname(os.path.abspath(__file__))
SRC = os.path.join(HERE, "extend_plan_check.cpp")
HDR = os.path.join(HERE, "..", "paper_2603_17484_amd", "csrc", "extend_plan.hpp")
LIB = os.path.join(HERE, "libextend_plan_check.so")


@pytest.fixture(scope="module")
def chk():
    if not os.path.exists(LIB) or os.path.getmtime(LIB) < max(os.path.getmtime(SRC), os.path.getmtime(HDR)):
        subprocess.run(["g++", "-O2", "-std=c++17", "-shared", "-fPIC", SRC, "-o", LIB], check=True)
    return ctypes.CDLL(LIB)


def check(chk, blocks, workgroups, each=None):
    each = each or [1] * len(blocks)
    msg = ctypes.create_string_buffer(256)
    ints = ctypes.c_int * len(blocks)
    rc = chk.plan_check(ints(*blocks), ints(*each), len(blocks), workgroups, msg, 256)
    assert rc == 0, f"{msg.value.decode()}: {workgroups} workgroups, {blocks[:20]} {each[:20]}"


@pytest.mark.parametrize("workgroups", [1, 2, 7, 256, 512])
def test_every_block_once(chk, workgroups):
    rng = random.Random(workgroups)
    check(chk, [1], workgroups)
    check(chk, [513] * 4, workgroups)
    check(chk, [1] * 2000, workgroups)
    for _ in range(400):
        most = rng.choice([1, 3, 5, 9, 70, 2000])
        blocks = [rng.randint(1, most) for _ in range(rng.choice([1, 2, 5, 40, 700]))]
        check(chk, blocks, workgroups)
        check(chk, blocks, workgroups, [rng.choice([2, 3, 4, 6, 8, 9]) for _ in blocks])


def test_every_short_line(chk):
    """All tiles of up to 8 blocks, three at a time, on a few workgroups: each way in which ends of stretches can meet tiles."""
    for a in range(1, 9):
        for b in range(1, 9):
            for c in range(1, 9):
                for w in (2, 3, 4, 6, 9):
                    check(chk, [a, b, c], w)
                    check(chk, [a, b, c], w, [9, 2, 8])
                    check(chk, [a, b, c], w, [3, 6, 2])


def test_sequences_out_of_range_are_clamped(chk):
    big = 2 ** 31 - 1
    values = [-big - 1, -7, -1, 0, 1, 5, 63, 64, 100, big]
    for start in values:
        for end in values:
            for pos in values:
                for tokens, max_new, cap in ((1, 1, 16), (64, 3, 16), (100, 100, 64), (5, 200, 1 << 30), (5, big, big)):
                    assert chk.seq_check(start, end, pos, tokens, max_new, cap), (start, end, pos, tokens, max_new, cap)
