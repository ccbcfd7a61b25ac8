"""How finch_attend deals a batch out to workgroups (host only): every tile of rows is there once for each of its splits, and what a
problem gets does not suffer from the others of its batch."""
import ctypes
import random

import pytest

import paper_2408_00167_amd as F

FEW, SOME, MANY = 0, 1, 2
BASE = 1 << 40


def batch(shapes, G=4, d=128):
    """[(n_que, c, m, causal)], one problem each, on addresses that nobody reads."""
    arr = (F.finch_attention * len(shapes))()
    for i, (n, c, m, causal) in enumerate(shapes):
        a, at = arr[i], BASE + i * (1 << 36)
        a.q, a.out, a.k_cache, a.v_cache, a.k_chunk, a.v_chunk = (at + (j << 33) for j in range(6))
        a.q_row = a.out_row = G * d
        a.q_head = a.out_head = a.cache_row = a.chunk_row = d
        a.n_que, a.c, a.m, a.causal = n, c, m, causal
    return arr


def plan(shapes, kernel, G=4, d=128, dtype=F.FINCH_BF16, cu=256, pieces=True):
    lib, cfg, arr = F.load_library(), F.finch_config(dtype, d, G, 0), batch(shapes, G, d)
    said = (ctypes.c_int64 * 8)()
    st = lib.finch_debug_attend_plan(ctypes.byref(cfg), cu, arr, len(shapes), kernel, said, None)
    assert st == F.FINCH_OK
    got = dict(zip(("workgroups", "span", "splits", "slots", "joined", "bytes", "rows_lo", "rows_hi"), said))
    if pieces:
        out = (ctypes.c_int32 * (5 * max(1, got["workgroups"])))()
        assert lib.finch_debug_attend_plan(ctypes.byref(cfg), cu, arr, len(shapes), kernel, said, out) == F.FINCH_OK
        got["pieces"] = [tuple(out[5 * w:5 * w + 5]) for w in range(got["workgroups"])]
    return got


def geometry(kernel, dtype):
    """rows and keys of a tile"""
    return (16, 16) if dtype == F.FINCH_F32 else {FEW: (16, 32), SOME: (32, 32), MANY: (256, 64)}[kernel]


def keys_of(shape, kt):
    return -(-shape[1] // kt) + -(-shape[2] // kt)


def check(shapes, G=4, d=128, dtype=F.FINCH_BF16, cu=256):
    """Every problem goes to one kernel, and that one has each of its tiles of rows once for each split; returns per kernel its plan."""
    plans, taken = {}, set()
    for kernel in (FEW, SOME, MANY):
        got = plans[kernel] = plan(shapes, kernel, G, d, dtype, cu)
        mine = {p: -(-s[0] * G // geometry(kernel, dtype)[0]) for p, s in enumerate(shapes)
                if s[0] and got["workgroups"] and got["rows_lo"] <= s[0] * G <= got["rows_hi"]}
        assert not taken & set(mine)
        taken |= set(mine)
        got["problems"] = set(mine)
        seen, slots = {}, set()
        for p, rt, split, splits, slot in got["pieces"]:
            if rt < mine.get(p, 0):  # (the others have nothing to do)
                seen.setdefault((p, rt), []).append(split)
                assert 0 <= split < splits <= got["splits"]
                if splits > 1:
                    assert 0 <= slot and slot + splits <= got["slots"] and (slot + split) not in slots
                    slots.add(slot + split)
                # no split has more tiles of keys than `span`, or than there are splits for
                assert -(-keys_of(shapes[p], geometry(kernel, dtype)[1]) // got["span"]) <= splits
        assert set(seen) == {(p, rt) for p, n in mine.items() for rt in range(n)}
        for (p, rt), splits in seen.items():
            assert sorted(splits) == list(range(len(splits))), (kernel, p, rt)
        assert got["slots"] <= 8192 and got["slots"] * geometry(kernel, dtype)[0] * (d + 2) * 4 <= 64 << 20
    assert taken == {p for p, s in enumerate(shapes) if s[0]}
    return plans


def request(n, c, heads=8):
    return [(n, c, n, 1)] * heads


@pytest.mark.parametrize("dtype,d,G", [(F.FINCH_BF16, 128, 4), (F.FINCH_BF16, 64, 1), (F.FINCH_F32, 64, 3)])
@pytest.mark.parametrize("seed", range(6))
def test_every_tile_of_rows_is_there_once(dtype, d, G, seed):
    rng = random.Random(seed)
    shapes = []
    for _ in range(rng.choice([1, 3, 20, 150, 400])):
        n = rng.choice([0, 1, 1, 1, 3, 8, 40, rng.randint(1, 700)])
        c = rng.choice([0, 100, 1000, rng.randint(0, 20000), 130000 if rng.random() < 0.1 else 50])
        shapes += [(n, c, rng.choice([n, n + 30, 0]), rng.randint(0, 1))] * rng.choice([1, 2, 8])
    check(shapes, G, d, dtype, cu=rng.choice([256, 304, 20]))


def test_alike_problems_are_one_run_in_the_batch_s_order():
    """Problem fastest, then tiles of rows from the last one down, then splits."""
    got = check(request(4096, 1364))[MANY]
    assert got["splits"] == 1 and got["bytes"] == 0
    assert [x[:2] for x in got["pieces"]] == [(p, rt) for rt in reversed(range(64)) for p in range(8)]
    got = check(request(1, 1408))[FEW]
    assert got["splits"] == 12 and [x[:3] for x in got["pieces"]] == [(p, 0, s) for s in range(12) for p in range(8)]


def test_one_run_where_all_workgroups_are_on_the_chip_at_once():
    """Nothing is looked up then: problems come in the batch's order, with the most splits and tiles of rows of any."""
    got = check([(1, c, 1, 1) for c in (4331, 4464, 7414, 3751) for _ in range(5)], G=3)[FEW]
    assert got["splits"] == 24 and [x[:3] for x in got["pieces"]] == [(p, 0, s) for s in range(24) for p in range(20)]
    got = check([(n, 9, n, 1) for n in (387, 348, 264) for _ in range(8)], d=64)[MANY]
    assert [x[:2] for x in got["pieces"]] == [(p, rt) for rt in reversed(range(7)) for p in range(24)]
    # nor where none of them has nothing to do
    got = check([(1, c, 1, 1) for c in (6, 40, 6, 60) * 200], G=1)[FEW]
    assert [x[0] for x in got["pieces"]] == list(range(800))


@pytest.mark.parametrize("others", [8, 64, 128, 512, 1016])
@pytest.mark.parametrize("first", [True, False])
def test_many_rows_on_a_long_cache_keep_their_splits_beside_tokens(others, first):
    long, tokens = request(128, 131000), [(1, 1000, 1, 1)] * others
    alone, got = plan(long, MANY), check(long + tokens if first else tokens + long)
    assert alone["splits"] == 17 and {k: got[MANY][k] for k in ("workgroups", "span", "splits", "slots")} == {k: alone[k] for k in ("workgroups", "span", "splits", "slots")}
    assert got[FEW]["splits"] == plan(tokens, FEW)["splits"] and got[FEW]["workgroups"] == plan(tokens, FEW)["workgroups"]


@pytest.mark.parametrize("at", [0, 500, 1016])
def test_a_long_cache_keeps_splits_beside_short_ones(at):
    """Eight problems of 131000 keys among 1016 of 1000: the longest workgroup has not much more than a compute unit's share."""
    shapes = [(1, 1000, 1, 1)] * 1016
    shapes[at:at] = request(1, 131000)
    got = check(shapes)[FEW]
    work = sum(keys_of(s, 32) for s in shapes)
    assert got["splits"] >= 50 and got["span"] <= 1.1 * work / 1024


def test_little_problems_go_along_with_many_rows():
    """Prompts of 58 rows beside long ones, a few rows beside a chunk; not where their caches would make their workgroups long, nor as many of
    them as make a launch worth while."""
    packed = [x for n in (2048, 1128, 1781, 58, 268) for x in [(n, 0, n, 1)] * 32]
    got = check(packed, G=1)
    assert got[MANY]["problems"] == set(range(160)) and got[MANY]["workgroups"] == 32 * (8 + 5 + 7 + 1 + 2)
    chunk = request(4096, 1364)
    assert check(chunk + request(1, 100))[FEW]["problems"] == set() and check(request(12, 100) + chunk)[SOME]["problems"] == set()
    assert len(check(chunk + request(1, 1364))[FEW]["problems"]) == 8
    assert len(check(chunk + request(1, 1000, 1024))[FEW]["problems"]) == 1024
    assert len(check(chunk + request(16, 13000))[SOME]["problems"]) == 8


def test_a_launch_has_no_workgroups_for_other_kernels_problems():
    chunk, tokens = request(4096, 1364), request(1, 1000, 1024)
    got = check(chunk + tokens)
    assert got[MANY]["workgroups"] == 512
    assert got[FEW]["workgroups"] == plan(tokens, FEW)["workgroups"]


@pytest.mark.parametrize("long", [(1, 13000), (1, 100000), (8, 13000), (10, 131000), (128, 6000), (128, 13000), (128, 131000), (40, 60000)])
def test_the_longest_workgroup_beside_a_chunk(long):
    """Beside a chunk of 4096 rows no workgroup has more keys than the chunk's own longest one (86 tiles of 64), or a compute unit's
    share of all the work where that is more."""
    shapes = request(4096, 1364) + request(*long)
    got = check(shapes)
    for kernel, p in got.items():
        rows, kt = geometry(kernel, F.FINCH_BF16)
        work = sum(-(-4 * shapes[i][0] // rows) * keys_of(shapes[i], kt) for i in p["problems"])
        longest = max((-(-keys_of(shapes[x[0]], kt) // x[3]) for x in p["pieces"]), default=0)
        assert longest * kt <= max(86 * 64, 1.1 * kt * work / 256), (kernel, longest)
    # and they are not the last to start
    first = {}
    for w, x in enumerate(got[MANY]["pieces"]):
        first.setdefault(x[0], w)
    if 4 * long[0] > 64 and long[1] > 6000:
        assert max(first[p] for p in range(8, 16)) < 512


def test_no_batch_is_too_wide_for_one_launch():
    """One problem of 1024 tiles of rows beside 4095 of one tile: 5119 workgroups, and no more."""
    shapes = [(16384, 0, 16384, 1)] + [(1, 0, 1, 1)] * 4095
    got = plan(shapes, SOME, G=1, d=128, dtype=F.FINCH_F32)
    assert got["workgroups"] >= 1024 + 4095 and got["workgroups"] < 1 << 14
    wide = plan([(1 << 22, 0, 1, 0)] * 64, MANY, pieces=False)  # more workgroups than a launch has: it takes several
    assert wide["workgroups"] == 64 * (1 << 16)
    lib, cfg, said = F.load_library(), F.finch_config(F.FINCH_F32, 64, 1, 0), (ctypes.c_int64 * 8)()
    shapes = [(1 << 24, 0, 1, 0)] * 1025  # 2^20 tiles of rows each
    assert lib.finch_debug_attend_plan(ctypes.byref(cfg), 256, batch(shapes, 1, 64), 1024, SOME, said, None) == F.FINCH_OK
    assert lib.finch_debug_attend_plan(ctypes.byref(cfg), 256, batch(shapes, 1, 64), 1025, SOME, said, None) == F.FINCH_ERR_CAPACITY


def test_more_groups_than_runs_are_put_together():
    """200 requests of different length, in turn of few and of many rows: neighbours that are near share a run, with little idle work."""
    rng = random.Random(3)
    shapes = []
    for i in range(200):
        shapes += request(rng.randint(100, 900) if i % 2 else 1, rng.randint(500, 4000))
    got = check(shapes)
    tiles = sum(-(-4 * s[0] // 256) for p, s in enumerate(shapes) if p in got[MANY]["problems"])
    assert got[MANY]["workgroups"] <= 5 * tiles
