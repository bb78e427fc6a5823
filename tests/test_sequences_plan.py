"""The plan of attention over several sequences (csrc/sequences_plan.h, compiled for the host): every visible key lies in a block of its item, every block in
one share, quotients are exact, and the parts fit the scratch memory."""
import ctypes as C
import os
import random
import subprocess

import pytest

HERE = os.path.dirname(os.path.abspath(__file__))


@pytest.fixture(scope="module")
def lib(tmp_path_factory):
    out = tmp_path_factory.mktemp("plan") / "libsequences_plan.so"
    subprocess.run(["g++", "-std=c++17", "-O1", "-shared", "-fPIC", "-x", "c++", os.path.join(HERE, "sequences_plan_host_shim.cc"), "-o", str(out)], check=True)
    lib = C.CDLL(str(out))
    for f in (lib.seq_share_host, lib.seq_scratch_host, lib.seq_parts_end_host):
        f.restype = C.c_int64
    lib.seq_share_host.argtypes = [C.c_int64, C.c_int, C.c_int]
    lib.seq_shares_host.argtypes = [C.c_int64, C.c_int]
    lib.seq_owner_host.argtypes = [C.c_int64, C.c_int, C.c_int64]
    lib.seq_quotient_host.argtypes, lib.seq_quotient_host.restype = [C.c_int, C.c_uint32], C.c_uint32
    lib.seq_mode_host.argtypes = [C.c_int64] + [C.c_int] * 4
    lib.seq_whole_host.argtypes = [C.c_int64, C.c_int, C.c_int64, C.c_int, C.c_int]
    return lib


def test_heads_of_a_tile(lib):
    for hq, hkv in [(1, 1), (8, 1), (15, 5), (6, 2), (64, 1), (65, 1), (70, 1), (128, 1), (200, 2), (65536, 1), (96, 32)]:
        o = (C.c_int * 4)()
        lib.seq_fold_host(hq, hkv, o)
        group, fold, per, tokens = o
        assert group == hq // hkv and 1 <= fold <= 64 and (per - 1) * fold < group <= per * fold and tokens >= 2 and fold * tokens <= 128


def test_blocks_hold_every_key_that_is_seen_and_none_twice(lib):
    rnd = random.Random(1)
    for _ in range(3000):
        nq, nk = rnd.choice([1, 2, 37, 130, 300]), rnd.choice([0, 1, 63, 64, 65, 128, 200, 700])
        causal = rnd.random() < 0.8
        window = rnd.choice([0, 0, 1, 5, 64, 100, 5000]) if causal else 0
        prefix = min(nk, rnd.choice([0, 0, 1, 64, 65, 150])) if causal else 0
        bn, tokens = rnd.choice([64, 128]), rnd.choice([2, 16, 50, 84, 128, 256])
        first = rnd.randrange((nq + tokens - 1) // tokens) * tokens
        out = (C.c_int * 64)()
        n = lib.seq_blocks_host(nq, nk, prefix, first, tokens, bn, int(causal), window, out, 64)
        blocks = list(out[:n])
        assert 1 <= n <= 64 and len(set(blocks)) == n and blocks == sorted(blocks)
        seen = set()
        for i in range(first, min(nq, first + tokens)):
            p = nk - nq + i
            for j in range(nk):
                ok = not causal or (j <= p and (window == 0 or p - j < window)) or j < prefix
                if ok:
                    seen.add(j)
                if i in (first, nq - 1):
                    s = (C.c_int * 2)()
                    lib.seq_seen_host(p, nk, prefix, int(causal), window, s)
                    assert ok == (j < s[1] and (j >= s[0] or j < prefix)), (p, j)
        assert seen <= {b * bn + x for b in blocks for x in range(bn)}
        assert all(b * bn < max(nk, 1) for b in blocks)              # no block lies behind the last key (but the first, where there is none)


def test_every_tick_has_one_share(lib):
    rnd = random.Random(2)
    totals = [1, 2, 147, 148, 149, 296, 1000, 2 ** 31 - 1, 2 ** 31, 2 ** 32 - 1, 2 ** 32, 2 ** 32 + 1, 2 ** 45 + 12345] + [int(2 ** rnd.uniform(0, 50)) for _ in range(300)]
    for total in totals:
        most = rnd.choice([1, 2, 148, 160, 296, 320])
        n = lib.seq_shares_host(total, most)
        assert n == min(total, most)
        ends = [lib.seq_share_host(total, most, c) for c in range(n + 1)]
        assert ends[0] == 0 and ends[-1] == total and all(0 < b - a <= (total + n - 1) // n for a, b in zip(ends, ends[1:]))
        for c in range(n):
            for at in (ends[c], ends[c + 1] - 1, (ends[c] + ends[c + 1]) // 2):
                if at < ends[c + 1]:
                    assert lib.seq_owner_host(total, most, at) == c, (total, most, at)


def test_quotients_by_the_page_size_are_exact(lib):
    rnd = random.Random(3)
    for d in [8, 16, 24, 32, 40, 64, 72, 128, 256, 1000, 1 << 20, (1 << 20) - 8, 104, 8 * 131071]:
        for x in [0, 1, d - 1, d, d + 1, 2 * d - 1, 2 ** 30, 2 ** 31 - 1, 2 ** 31 - 1 - (2 ** 31 - 1) % d, (2 ** 31 - 1) // d * d - 1] + [rnd.randrange(2 ** 31) for _ in range(500)]:
            assert lib.seq_quotient_host(d, x) == x // d, (d, x)


def test_parts_fit_the_scratch_memory_and_tiles_the_sms(lib):
    for hd in range(8, 257, 8):
        for sms in (1, 74, 132, 148, 160, 400):
            for mode in ((2,) if hd > 128 else (0, 1)):
                assert lib.seq_parts_end_host(mode, hd, sms) <= lib.seq_scratch_host(hd)
        for tq, seqs in ((1, 1), (900, 1), (901, 1), (10000, 7), (64, 64)):
            mode = lib.seq_mode_host(tq, seqs, 16, 1, hd)
            assert (mode == 2) == (hd > 128)
            nbox, bn = (hd + 63) // 64, lib.seq_bn_host(mode)
            stages = (lib.seq_smem_host(mode) - 1024 - (2 if mode == 0 else 1) * nbox * 128 * 128) // (nbox * bn * 128)
            assert stages >= 3 and lib.seq_smem_host(mode) * (2 if mode == 1 else 1) <= 225 * 1024


def test_whole_items_where_cutting_would_gain_nothing(lib):
    assert lib.seq_whole_host(960 * 4, 296, 960, 4, 6) == 1            # many short ones
    assert lib.seq_whole_host(8 * 27, 296, 8, 27, 6) == 0              # a token over a long cache: its keys over the chip
    assert lib.seq_whole_host(10 ** 6, 148, 1000, 1000, 5) == 0        # seven and a bit long ones a share: cut
    assert lib.seq_whole_host(148 * 30, 148, 148, 30, 5) == 1          # one each


def test_short_sequences_are_never_cut(lib):
    """What a call without scratch memory counts on: up to 512 keys every item stays whole, however many there are and of whatever lengths."""
    rnd = random.Random(4)
    for mode, join in ((0, 5), (1, 9), (2, 9)):
        assert lib.seq_always_whole_host(mode, 1) and lib.seq_always_whole_host(mode, 512) and not lib.seq_always_whole_host(mode, 1000)
        w, most = lib.seq_ticks_host(mode), w_blocks(lib, mode)
        for _ in range(2000):
            items = rnd.choice([1, 2, 7, 100, 147, 148, 149, 300, 1000, 50000])
            longest = w + rnd.randint(1, most)
            total = rnd.randint(longest + (items - 1) * (w + 1), items * longest) if items > 1 else longest
            assert lib.seq_whole_host(total, 296 if mode == 1 else 148, items, longest, join)


def w_blocks(lib, mode):
    return 512 // lib.seq_bn_host(mode)
