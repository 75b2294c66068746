"""The division of work of calls with lists of routed rows, segments of long tiles among it, replayed on the CPU."""
import ctypes
import os
import random
import subprocess

import pytest

HERE = os.path.dirname(os.path.abspath(__file__))
SRC = os.path.join(HERE, "extend_segments_check.cpp")
HDR = os.path.join(HERE, "..", "paper_2603_17484_amd", "csrc", "extend_plan.hpp")
LIB = os.path.join(HERE, "libextend_segments_check.so")


@pytest.fixture(scope="module")
def chk():
    if not os.path.exists(LIB) or os.path.getmtime(LIB) < max(os.path.getmtime(SRC), os.path.getmtime(HDR)):
        subprocess.run(["g++", "-O2", "-std=c++17", "-shared", "-fPIC", SRC, "-o", LIB], check=True)
    return ctypes.CDLL(LIB)


def check(chk, new, cached, heads, kv, W, f, fp8=False, do_local=True, workgroups=256):
    """-> segments, the longest work of a workgroup over an even share."""
    msg = ctypes.create_string_buffer(256)
    ints = ctypes.c_int * len(new)
    out = (ctypes.c_int * 3)()
    rc = chk.segments_check(ints(*new), ints(*cached), len(new), kv, heads // kv, W, int(100 * f), int(fp8), int(do_local), workgroups, out, msg, 256)
    assert rc == 0, f"{msg.value.decode()}: {new} behind {cached}, {heads}/{kv} heads, window {W}, {f} routed, fp8 {fp8}"
    return out[0], out[1] / max(out[2], 1)


# whose segments, rounded down, left almost all of the line to a few workgroups, or were as many as there are workgroups and dropped
UNEVEN = [([128], [65536], 28, 4, 512, 0.2), ([128], [32768], 28, 4, 512, 0.5), ([64], [32768], 32, 8, 512, 1.0), ([256], [131072], 12, 1, 512, 0.5), ([96], [65536], 28, 4, 64, 0.2),
          ([313], [17548], 12, 1, 100, 1.0), ([252], [22548], 28, 4, 100, 1.0), ([191], [33548], 12, 1, 1024, 1.0)]


@pytest.mark.parametrize("case", UNEVEN)
def test_short_chunks_behind_long_caches(chk, case):
    for fp8 in (False, True):
        assert check(chk, *case, fp8=fp8)[0] > 0


@pytest.mark.parametrize("heads,kv", [(28, 4), (32, 8), (12, 1), (16, 16), (16, 1), (8, 2)])
def test_nobody_has_more_than_a_share(chk, heads, kv):
    segments = 0
    for new in (9, 40, 64, 96, 128, 191, 256, 500, 777, 2048):
        for cached in (0, 63, 500, 4096, 16000, 32768, 65537, 131072):
            for W in (0, 64, 100, 512, 1024, 4096):
                for f in (0.1, 0.2, 0.5, 1.0):
                    segments += check(chk, [new], [cached], heads, kv, W, f, new % 2 == 0)[0] > 0
    assert segments > 200


def test_several_sequences_and_one_branch_alone(chk):
    rng = random.Random(4)
    for _ in range(3000):
        B = rng.choice([1, 2, 3, 7, 30])
        most = rng.choice([1, 30, 300, 2000])
        far = rng.choice([1, 1000, 30000, 200000])
        heads, kv = rng.choice([(28, 4), (32, 8), (12, 1), (4, 2), (1, 1)])
        new, cached = [rng.randint(0, most) for _ in range(B)], [rng.randint(0, far) for _ in range(B)]
        check(chk, new, cached, heads, kv, rng.choice([0, 30, 100, 1024, 9000]), rng.choice([0.0, 0.1, 0.5, 1.0]), rng.random() < 0.5, rng.random() < 0.7, rng.choice([1, 8, 256]))
