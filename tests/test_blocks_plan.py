"""The tile plan of the linear layers on 8-bit operands and by expert (csrc/blocks_plan.h, compiled for the host): whatever the shape, the tiles
cover the result, the stages fit, and there are as many as the kernel's barriers need to stay in step."""
import ctypes as C
import os
import random
import subprocess

import pytest

HERE = os.path.dirname(os.path.abspath(__file__))


@pytest.fixture(scope="module")
def plan(tmp_path_factory):
    out = tmp_path_factory.mktemp("plan") / "libblocks_host.so"
    subprocess.run(["g++", "-std=c++17", "-O1", "-shared", "-fPIC", "-x", "c++", os.path.join(HERE, "blocks_plan_host_shim.cc"), "-o", str(out)], check=True)
    lib = C.CDLL(str(out))

    def call(rows, n, nkb, experts=0, f8=True, sms=148):
        o = (C.c_longlong * 15)()
        lib.blocks_plan_host(rows, n, nkb, experts, int(f8), sms, o)
        return dict(zip(("bm", "bn", "pair", "tiles_n", "stages", "tiles", "kps", "unit_stages", "smem", "turns", "units", "most_units", "ks", "few", "few_smem"), o))
    return call


def shapes():
    rnd = random.Random(3)
    out = [(r, n, nkb, e) for r in (1, 8, 40, 64, 65, 16, 17, 127, 128, 129, 300, 100000, 1 << 30) for n in (1, 7, 64, 257, 9500, 1 << 20) for nkb in (1, 2, 3, 65, 1000)
           for e in (0, 1, 2, 64, 1024)]
    return out + [(int(2 ** rnd.uniform(0, 15)), int(2 ** rnd.uniform(0, 15)), int(2 ** rnd.uniform(0, 8)), rnd.choice([0, 0, 1, 3, 8, 100])) for _ in range(3000)]


def test_every_plan_is_one_the_kernel_can_run(plan):
    for rows, n, nkb, e in shapes():
        for sms, f8 in ((148, True), (148, False), (132, True), (7, False)):
            if not f8 and e == 0:
                continue
            p = plan(rows, n, nkb, e, f8, sms)
            bm, bn, kps, stages, pair = p["bm"], p["bn"], p["kps"], p["stages"], p["pair"]
            assert 16 <= bm <= 128 and bm % 16 == 0 and 16 <= bn <= 256 and bn % 16 == 0 and (not pair or bn % 32 == 0 and bn > 128), p
            assert p["tiles_n"] * bn >= n > (p["tiles_n"] - 1) * bn
            tile = bm * (2 if pair else 1)
            if p["few"]:        # operands exchanged: half an SM's shared and tensor memory, a stage's accumulator each, the others' sums in the first CTA's stages
                block = (bm + bn) * 128
                assert bm in (16, 32, 64) and bn <= 128 and not pair and p["ks"] in (1, 2, 4, 8) and nkb >= p["ks"], p
                assert 1 <= stages <= 8 and stages * bm <= 256 and stages * block <= p["few_smem"] and (stages - 1) * block + 16384 <= p["few_smem"], p
                assert (p["ks"] - 1) * bm * 512 <= p["few_smem"], p
            else:
                assert 1 <= p["units"] <= p["most_units"] and p["units"] * p["unit_stages"] <= stages <= 12 and not (p["turns"] and stages % 2), p
                assert p["units"] == 2 or bn <= 64, p                # (the wider tiles' kernels count on two)
                block = (bm + (128 if pair else bn)) * 128
                assert stages * kps * block <= p["smem"] and (stages * kps - 1) * block + 16384 <= p["smem"]   # (the MMA reads 128 rows of any block)
                # a shared K: narrow tiles, work for each CTA, and the others' sums fit the first one's stages
                assert p["ks"] in (1, 2, 4) and (p["ks"] == 1 or bn <= 64 and nkb >= 8 * p["ks"] and (p["ks"] - 1) * 32768 <= p["smem"]), p
            if e == 0:
                assert p["tiles"] == -(-rows // tile) * p["tiles_n"]
            else:       # however the rows are spread over the experts
                assert p["tiles"] >= (rows // tile + min(rows, e) - (1 if rows % tile == 0 else 0)) * p["tiles_n"]


def kernel_of(p):
    return ("few", p["bm"], p["ks"]) if p["few"] else (("pair",) if p["pair"] else ("wide",) if p["bn"] > 128 else ("middle",) if p["bn"] > 64 else ("narrow", p["ks"]))


def test_the_gpu_tests_reach_every_kernel(plan):
    """Over the shapes of test_gpu_linear_blocks.py: operands exchanged at every height, alone and with a shared K, and every width of the others."""
    import test_gpu_linear_blocks as T
    seen = {(True,) + kernel_of(plan(m, n, -(-k // 128))) for m, n, k in T.SCALED} | {(True,) + kernel_of(plan(m, n, 65)) for m, n in T.LONG_K}
    shapes = [(c, n, k) for c in T.COUNTS for n, k in ((96, 136), (257, 1040), (2048, 64))] + T.EVERY
    for counts, n, k in shapes:
        seen.add((False,) + kernel_of(plan(sum(counts), n, -(-k // 64), len(counts), False)))
        seen.add((True,) + kernel_of(plan(sum(counts), n, -(-k // 128), len(counts), True)))
    seen |= {(False,) + kernel_of(plan(m, n // 2, 129, 2, False)) for m, n in T.LONG_K}
    missing = [(f8,) + k for f8 in (False, True) for k in
               [("pair",), ("wide",), ("middle",)] + [("narrow", ks) for ks in (1, 2, 4)] + [("few", h, ks) for h in (16, 32, 64) for ks in (1, 2, 4)] + [("few", 16, 8)]
               if (f8,) + k not in seen]
    assert not missing


def test_the_boxes_tests_have_several_wide_tiles_a_block(plan):
    import test_gpu_linear_blocks as T
    for m, n, k in T.BOXES:
        for p in (plan(m, n, -(-k // 128)), plan(m - 33, n, -(-k // 64), 3, False)):
            assert p["bn"] == 256 and p["tiles"] > 148 // (2 if p["pair"] else 1), (m, n, k, p)
