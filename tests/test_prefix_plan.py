"""How attention behind shared prefixes is cut into CTAs and where its parts lie: the plan itself, compiled for the host. CPU only."""
import ctypes
import random
import shutil
import subprocess

import pytest

from paper_2609_10018_gb300 import build

PROGRAM = """
#include "prefix_parts.h"
using namespace elasto;
extern "C" void plan(const long long* z, long long* p) {
  PrefixSizes s{z[0], z[1], (int)z[2], (int)z[3], (int)z[4], (int)z[5], (int)z[6], (int)z[7], z[8], z[9], (int)z[10]};
  const PrefixPlan r = prefix_plan(s);
  const long long v[] = {r.hg, r.nsub, r.qpt, r.pair, r.split, (long long)r.items, r.many, r.blocks, r.own_split, r.prefix_parts(), r.parts(), r.fused};
  for (int i = 0; i < 12; ++i) p[i] = v[i];
}
extern "C" int from(int tiles, int rank, int split) { return split_from(tiles, rank, split); }
extern "C" long long sums(int part, int h, long long row, long long rho, int hs, int quads) { return PrefixParts{nullptr, nullptr, rho, hs, quads}.sums_at(part, h, row); }
extern "C" long long stat(int part, int h, long long row, long long rho, int hs, int quads) { return PrefixParts{nullptr, nullptr, rho, hs, quads}.stat_at(part, h, row); }
extern "C" int most_parts() { return kMaxParts; }
// A walk whose tile `missing` does not come: the tiles met, those worked on as bits; whether all came.
extern "C" int walk(int t0, int t1, int keys, int least, int missing, int* meets, long long* worked) {
  *meets = 0, *worked = 0;
  return walk_tiles(t0, t1, keys, least, [&](int i) { return t0 + i != missing; }, [&](int, int, bool) { ++*meets; },
                    [&](int i, int t) { *worked |= i == t - t0 ? 1LL << t : 1LL << 63; });
}
"""
FIELDS = ("hg", "nsub", "qpt", "pair", "split", "items", "many", "blocks", "own_split", "prefix_parts", "parts", "fused")


@pytest.fixture(scope="module")
def rule(tmp_path_factory):
    cxx = shutil.which("g++")
    if cxx is None:
        pytest.skip("no g++")
    d = tmp_path_factory.mktemp("prefix_plan")
    (d / "rule.cpp").write_text(PROGRAM)
    subprocess.run([cxx, "-std=c++17", "-shared", "-fPIC", "-I", build.CSRC, str(d / "rule.cpp"), "-o", str(d / "rule.so")], check=True)
    lib = ctypes.CDLL(str(d / "rule.so"))
    lib.sums.restype = lib.stat.restype = ctypes.c_longlong
    for f in (lib.sums, lib.stat):
        f.argtypes = [ctypes.c_int, ctypes.c_int, ctypes.c_longlong, ctypes.c_longlong, ctypes.c_int, ctypes.c_int]
    return lib


def _plan(rule, **z):
    z = dict(rows=64, most=64, batch=64, max_queries=1, prefixes=1, group=4, heads_kv=8, head_dim=128, max_prefix=8192, max_keys=1024, sms=152) | z
    out = (ctypes.c_longlong * 12)()
    rule.plan((ctypes.c_longlong * 11)(*z.values()), out)
    return dict(zip(FIELDS, out))


def _sizes(n):
    r = random.Random(7)
    log = lambda a, b: int(round(a * (b / a) ** r.random()))  # noqa: E731
    for _ in range(n):
        batch, queries = log(1, 600), log(1, 300)
        rows = r.choice([batch * queries, log(1, batch * queries)])
        yield dict(rows=rows, most=rows + r.choice([0, log(1, 5000)]), batch=batch, max_queries=queries, prefixes=r.choice([1, 1, 2, 9, 70]),
                   group=r.choice([1, 2, 3, 7, 8, 31, 32, 33, 40, 128]), heads_kv=r.choice([1, 3, 8, 32]), head_dim=r.choice([8, 64, 80, 128]),
                   max_prefix=log(1, 1 << 30), max_keys=r.choice([0, log(1, 1 << 20), 1 << 30]), sms=r.choice([16, 76, 148, 152]))


def test_plans_stay_within_their_limits(rule):
    for z in _sizes(400):
        p = _plan(rule, **z)
        assert 1 <= p["hg"] <= 32 and p["hg"] * p["nsub"] >= z["group"] and p["hg"] * (p["nsub"] - 1) < z["group"], z
        assert p["qpt"] == 128 // p["hg"] >= 4
        tiles = -(-z["max_prefix"] // 128)
        assert 1 <= p["split"] <= min(64, tiles) and p["parts"] <= rule.most_parts(), (z, p)
        rows = 64 if p["many"] else 16
        assert p["blocks"] == -(-z["max_queries"] * z["group"] // rows)
        assert p["own_split"] == 1 or z["max_keys"] >= 32 * p["own_split"], (z, p)


def test_rows_joined_at_once_have_one_part(rule):
    seen = 0
    for z in _sizes(2000):
        p = _plan(rule, **z)
        if p["fused"]:
            seen += 1
            assert p["prefix_parts"] == p["own_split"] == 1 and not p["many"]
    assert seen > 0
    # (the sizes of the GPU's test of it)
    assert _plan(rule, rows=81, most=83, batch=11, max_queries=9, prefixes=8, group=16, heads_kv=13, max_prefix=200, max_keys=60)["fused"]


def test_items_suffice_however_the_rows_fall_to_the_prefixes(rule):
    r = random.Random(3)
    for z in _sizes(400):
        p = _plan(rule, **z)
        step = p["qpt"] * (1 if p["pair"] else 2)
        for _ in range(5):
            cuts = sorted(r.randint(0, z["most"]) for _ in range(z["prefixes"] - 1))
            shares = [b - a for a, b in zip([0] + cuts, cuts + [z["most"]])]
            assert sum(-(-n // step) for n in shares) <= p["items"], (z, p, shares)


@pytest.mark.parametrize("split", [1, 2, 3, 7, 64])
def test_every_tile_has_one_cta(rule, split):
    for tiles in (0, 1, 2, 63, 64, 65, 1000, 1 << 23, 1 << 26):  # (2^30 keys in blocks of 16)
        edges = [rule.__getattr__("from")(tiles, k, split) for k in range(split + 1)]
        assert edges[0] == 0 and edges[-1] == tiles and edges == sorted(edges)
        assert max(b - a for a, b in zip(edges, edges[1:])) <= -(-tiles // split)


def test_parts_do_not_overlap(rule):
    parts, hs, rho, quads = 3, 5, 96, 6
    seen = set()
    for p in range(parts):
        for h in range(hs):
            for row in range(rho):
                for q in range(quads):
                    seen |= {rule.sums(p, h, row, rho, hs, quads) + 128 * q + i for i in range(4)}
    assert seen == set(range(parts * hs * rho * quads * 4))
    seen = {rule.stat(p, h, row, rho, hs, quads) for p in range(parts) for h in range(hs) for row in range(rho)}
    assert seen == set(range(0, 2 * parts * hs * rho, 2))


def test_every_form_has_a_case(rule):
    """What the tests on the GPU rely on to reach each form: blocks of 64 rows, in one and several CTAs; parts of one, a few and
    more than eight."""
    room = dict(batch=6, prefixes=3, group=2, heads_kv=2, max_prefix=300)
    few, more = (_plan(rule, rows=600, most=600, max_queries=600, max_keys=k, **room) for k in (130, 1100))
    assert few["many"] and few["own_split"] == 1 and more["many"] and more["own_split"] > 1
    many = _plan(rule, rows=3400, most=3400, max_queries=3400, max_keys=130, **room)
    assert many["many"] and many["parts"] == 2 and 3400 * 4 * 6 > 40000
    parts = _plan(rule, rows=150, most=150, batch=320, max_queries=128, prefixes=2, group=1, heads_kv=1, max_prefix=20000, max_keys=69)
    assert not parts["many"] and not parts["fused"] and parts["parts"] > 8 and 128 * 320 > 40000


@pytest.mark.parametrize("least", [0, 1, 63, 64, 100, 128, 500, 640])
def test_a_warp_that_gives_up_meets_the_others(rule, least):
    """Warps wait for each tile by themselves, and for one another at tiles that rows see in part. However far a warp comes
    before it gives up, it has to meet the others as often as they do."""
    for t0, t1 in ((0, 1), (0, 10), (3, 9), (4, 4)):
        meets, worked = ctypes.c_int(), ctypes.c_longlong()
        all_meets = [t for t in range(t0, t1) if least < 64 * (t + 1)]
        for missing in range(t0, t1 + 1):
            ok = rule.walk(t0, t1, 64, least, missing, ctypes.byref(meets), ctypes.byref(worked))
            assert ok == (missing == t1) and meets.value == len(all_meets), (t0, t1, missing)
            assert worked.value == sum(1 << t for t in range(t0, missing))  # (nothing from the tile on that did not come)


def test_forms_of_the_test_of_infinite_values(rule):
    """Sizes of test_infinite_values_behind_scores_of_minus_infinity: several parts and few rows, many rows, a join inside."""
    room = dict(batch=3, prefixes=2, max_prefix=140, max_keys=20)
    for queries, group, heads_kv in ((1, 2, 2), (4, 2, 2), (5, 7, 4)):
        p = _plan(rule, rows=3 * queries, most=3 * queries, max_queries=queries, group=group, heads_kv=heads_kv, **room)
        assert not p["fused"] and not p["many"] and p["parts"] > 2, p
    for queries in (1, 4):
        most = 3 * queries + 7000
        p = _plan(rule, rows=most, most=most, max_queries=7000, group=2, heads_kv=2, **room)
        assert p["many"] and 7000 * 4 * 3 > 40000 and not p["fused"], p
    p = _plan(rule, rows=12, most=12, max_queries=4, group=32, heads_kv=52, **room)
    assert p["fused"], p


def test_a_workspace_has_only_the_parts_that_are_written(rule):
    """Where the kernel of the own keys joins its rows, and where there are no own keys, the prefix's parts are all."""
    seen = set()
    for z in _sizes(2000):
        p = _plan(rule, **z)
        own = 0 if p["fused"] or z["max_keys"] == 0 else p["own_split"]
        assert p["parts"] == p["prefix_parts"] + own, (z, p)
        seen.add((bool(p["fused"]), z["max_keys"] == 0))
    assert seen == {(False, False), (True, False), (False, True)}
