"""Which form of the group-scaled products a shape is launched in, asked of the launchers' own plans (host arithmetic, no GPU), and that the shapes
that the GPU tests run take them all."""
import ctypes as C
import os
import random
import subprocess
import sys

import pytest

from tests import gs4_shapes as S

SOURCE = os.path.join(os.path.dirname(os.path.abspath(__file__)), "native", "gs4_plan.cpp")
SMS = 148


@pytest.fixture(scope="module")
def plan(tmp_path_factory):
    lib = str(tmp_path_factory.mktemp("native") / "gs4_plan.so")
    subprocess.check_call(["g++", "-std=c++17", "-O2", "-Wall", "-Wextra", "-Werror", "-shared", "-fPIC", SOURCE, "-o", lib])
    lib = C.CDLL(lib)
    sizes = [C.c_int64] + [C.c_int] * 10
    lib.gs4_is_many.argtypes = sizes
    lib.gs4_few.argtypes = lib.gs4_many.argtypes = sizes + [C.POINTER(C.c_int64)]

    def of(shape, sms=SMS):
        a = tuple(shape) + (sms,)
        if lib.gs4_is_many(*a):
            out = (C.c_int64 * len(S.MANY))()
            lib.gs4_many(*a, out)
            return "many", dict(zip(S.MANY, out))
        out = (C.c_int64 * len(S.FEW))()
        lib.gs4_few(*a, out)
        return "few", dict(zip(S.FEW, out))
    return of


def test_plans_are_sound(plan):
    """Everything a kernel relies on, over the whole range of sizes and for devices of other numbers of SMs: shared memory, shares that add up, places for every row."""
    rng = random.Random(1)
    shapes = [S.any_shape(rng) for _ in range(4000)] + list(S.SHAPES)
    shapes += [(8, 1, 1 << 20, 1 << 20, 32, 1, S.BF16, 0, 1, 1), (4, 1, 1, 1 << 20, 32, 1, S.F32, 0, 1, 0), (1, 1, 1, 1, 32, 0, S.F16, 0, 1, 0),
               (24 * 4096, 4096, 64, 1 << 20, 32, 1, S.F16, 1, 0, 0), (1, 4096, 1 << 20, 32, 64, 0, S.F32, 1, 0, 1), (12 * 200, 200, 40, 1 << 20, 32, 1, S.F32, 1, 1, 1)]
    for shape in shapes:
        R, E, M, K, group, zero, x_type, experts, in_order, x_vec = shape
        tiles, units = -(-M // 32), -(-K // 128)
        for sms in (16, 64, SMS, 200):
            kind, p = plan(shape, sms)
            if kind == "many":
                assert p["bn"] in ((16, 32, 64) if x_type == S.F32 else (16, 32, 64, 128, 192, 256)) and p["split"] in (1, 2, 4)
                assert p["units"] * p["split"] >= units and p["mtiles"] * 4 >= tiles
                assert p["ntiles"] == -(-R // p["bn"]) + (min(E, R) if experts else 0)
                continue
            cols = p["tokens"] * p["parts"]
            block = 2048 + (80 if zero else 64) * (1 if group % 128 == 0 else 2 if group % 64 == 0 else 4)
            sums = 1 if group % 128 == 0 else 2 if group % 64 == 0 else 4
            assert p["parts"] == (2 if x_type == S.F32 else 1) and cols <= 8 * p["nt"] and (experts or p["tokens"] >= R) and p["nt"] <= (2 if experts else 1)
            assert p["wr"] * p["wk"] == 8 and p["split"] in (1, 2, 4, 8) and p["per"] % p["wr"] == 0 and p["per"] > 0
            assert p["groups"] * p["per"] >= tiles > (p["groups"] - 1) * p["per"]
            assert p["slice"] % 128 == 0 and p["slice"] * p["split"] >= units * 128 and 128 <= p["slab"] <= p["slice"] and p["slab"] % 128 == 0
            assert not p["alone"] or (p["wk"] == 1 and p["split"] == 1 and p["slab"] == p["slice"])
            assert not p["single"] or (p["alone"] and p["per"] == p["wr"] and 16 * 36 * 4 <= 2 * block)
            # ring; x and factors of a stage; sums: of each row block, or of a warp where it stores them itself, or none where they are in its ring
            red = 0 if p["single"] else p["wr"] * p["wk"] * 8 * p["nt"] * 36 * 4 * (1 if p["alone"] else p["per"] // p["wr"])
            ring = 8 * 2 * (2 if p["nt"] == 1 else 1) * block
            factors = 0 if x_type == S.F16 else p["slab"] // 128 * sums * 8 * p["nt"] * 4
            assert ring + cols * (p["slab"] * 2 + 64) + factors + red == p["smem"] <= 226 * 1024
            # passes: what any spread of R rows over E matrices can need
            most = max(sum(-(-n // p["tokens"]) for n in spread) for spread in ([R], [1] * (min(E, R) - 1) + [R - min(E, R) + 1])) if experts else 1
            assert p["grid"] >= most * p["groups"] * p["split"]


def test_plans_of_a_device_whose_sms_are_not_known(tmp_path):
    """Counted as one: seven eighths of that, which clusters are given, were none, and the division by them ended the process.  (So in a process of its own.)"""
    lib = str(tmp_path / "gs4_plan.so")
    subprocess.check_call(["g++", "-std=c++17", "-O2", "-shared", "-fPIC", SOURCE, "-o", lib])
    code = """
import ctypes as C, sys
lib = C.CDLL(sys.argv[1])
lib.gs4_few.argtypes = [C.c_int64] + [C.c_int] * 10 + [C.POINTER(C.c_int64)]
out = (C.c_int64 * %d)()
for experts, E in ((0, 1), (1, 5)):
    for sms in (1, 2):
        lib.gs4_few(8, E, 4096, 4096, 64, 1, 1, experts, 1, 1, sms, out)
        print(out[0], out[3])
""" % len(S.FEW)
    done = subprocess.run([sys.executable, "-c", code, lib], capture_output=True, text=True, timeout=60)
    assert done.returncode == 0 and len(done.stdout.split()) == 8


def test_the_tested_shapes_take_every_form(plan):
    """Every pair of features that turns up among shapes of the whole range is one that a shape of the GPU tests has: an estimate that is fitted anew cannot drop one silently."""
    covered = set()
    for shape in S.SHAPES:
        kind, p = plan(shape)
        covered |= S.pairs(kind, S.features(kind, p, shape))
    rng = random.Random(2)
    seen = {}
    for _ in range(20000):
        shape = S.any_shape(rng)
        kind, p = plan(shape)
        for pair in S.pairs(kind, S.features(kind, p, shape)):
            seen.setdefault(pair, []).append(shape)
    missing = {pair: shapes[0] for pair, shapes in seen.items() if len(shapes) >= 3 and pair not in covered}
    assert not missing, missing
    assert {f for _, *two in covered for f in two} >= {"single", "alone", "rounds", "an idle rank", "stages2", "stages3", "split2", "split4", "split8", "wr1", "wr2", "wr4", "wr8",
                                                       "experts of 16 columns", "tiles of 64", "tiles of 128", "tiles of 192", "tiles of 256", "tensor copies", "single values"}
