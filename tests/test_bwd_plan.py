"""Host logic of the backward launch against brute force on the CPU: every key tile and every query tile is owned exactly once,
and the parts of its stream hold, without gap or overlap, exactly the tiles with a visible (query, key) pair."""
import random

import pytest

import paper_2603_24517_b200 as lib
from paper_2603_24517_b200 import build as lib_build

TILE = 128


@pytest.fixture(scope="module", autouse=True)
def _built():
    lib_build.build()


def drawn(rng):
    """Sizes of up to a few thousand items."""
    if rng.random() < 0.3:  # many short ones: several runs
        hkv = rng.choice([5, 8, 10, 16])
        return rng.randint(4, 18), hkv * rng.choice([1, 1, 2, 3]), hkv, rng.randint(65, 640), rng.randint(65, 640), rng.random() < 0.6
    hkv = rng.choice([1, 2, 3, 5, 8, 16])
    group = rng.choice([1, 1, 1, 2, 3, 4, 8, 16, 32])
    B = rng.choice([1, 1, 2, 3, 7, 13])
    Sq, Sk = (int(2 ** rng.uniform(0, rng.choice([7, 11, 15]))) for _ in range(2))
    if rng.random() < 0.3:
        Sk = Sq
    while B * hkv * (group * (Sq // TILE + 1) + Sk // TILE + 1) > 1500:
        B, Sq, Sk = (B + 1) // 2, Sq // 2 + 1, Sk // 2 + 1
    return B, hkv * group, hkv, Sq, Sk, rng.random() < 0.6


FIXED = [
    (13, 10, 10, 512, 512, True), (13, 10, 10, 512, 512, False),       # three runs of 44, 43, 43 units
    (9, 40, 20, 300, 400, True), (5, 26, 26, 700, 129, True),          # several runs, ragged
    (1, 1, 1, 128, 1 << 17, False), (1, 1, 1, 1 << 17, 128, True),     # cut into 32 parts, and rows without keys
    (1, 4, 1, 65, 9000, True), (2, 32, 8, 1, 4097, True), (1, 32, 2, 9, 9, True), (1, 2, 2, 4000, 300, True),
]


def check(B, Hq, Hkv, Sq, Sk, causal):
    plan = lib.attn_bwd_plan(B, Hq, Hkv, Sq, Sk, 128, causal)
    items = [lib.attn_bwd_plan_item(B, Hq, Hkv, Sq, Sk, 128, causal, w) for w in range(plan["n_items"])]
    pack, q_heads, group = plan["pack_log2"], plan["q_heads"], plan["q_heads"] // Hkv
    assert q_heads << pack == Hq and (pack == 0 or q_heads == Hkv)
    rows = Sq << pack
    n_qt, n_kt = -(-rows // TILE), -(-Sk // TILE)
    assert (plan["n_q_tiles"], plan["n_k_tiles"]) == (n_qt, n_kt)

    def sees(qt, kt):  # the tile's last row sees most
        last_row = (min(rows, (qt + 1) * TILE) - 1) >> pack
        return not causal or kt * TILE <= last_row + Sk - Sq

    parts = {}
    for it in items:
        assert it["row0"] % TILE == 0 and it["t0"] >= 0 and it["n"] >= 0
        parts.setdefault((it["keys"], it["b"], it["head"], it["row0"] // TILE), []).append(it)
    want = {(1, b, h, t) for b in range(B) for h in range(Hkv) for t in range(n_kt)} | \
           {(0, b, h, t) for b in range(B) for h in range(q_heads) for t in range(n_qt)}
    assert set(parts) == want
    stream = {(1, t): [q for q in range(n_qt) if sees(q, t)] for t in range(n_kt)}
    stream.update({(0, t): [k for k in range(n_kt) if sees(t, k)] for t in range(n_qt)})
    for (keys, b, h, tile), its in parts.items():
        tiles = stream[keys, tile]
        length = len(tiles) * (group if keys else 1)
        assert sorted(it["split"] for it in its) == list(range(plan["key_splits"] if keys else plan["query_splits"]))
        at = 0
        for it in sorted(its, key=lambda it: it["split"]):
            assert it["t0"] == at
            at += it["n"]
            assert it["per_head"] == len(tiles) and (not tiles or tiles == list(range(it["first"], it["first"] + it["per_head"])))
        assert at == length
    return plan


@pytest.mark.parametrize("sizes", FIXED)
def test_every_tile_once(sizes):
    check(*sizes)


def test_every_tile_once_in_drawn_problems():
    rng = random.Random(7)
    plans = []
    for _ in range(600):
        sizes = drawn(rng)
        plans.append((sizes, check(*sizes)))
    units = lambda s: s[0] * s[2]  # noqa: E731
    several = [p for s, p in plans if p["run"] < units(s)]
    assert len(several) > 20 and any(0 < p["run_extra"] * p["run"] < units(s) for s, p in plans)
    for what in ("key_splits", "query_splits"):
        assert sum(p[what] > 1 for _, p in plans) > 20
    assert sum(p["pack_log2"] > 0 for _, p in plans) > 20


def test_unequal_runs():
    plan = lib.attn_bwd_plan(13, 10, 10, 512, 512, 128, True)
    assert (plan["run"], plan["run_extra"]) == (44, 1) and plan["n_items"] == 130 * 8


def test_argument_errors():
    cdll = lib.load_library()
    assert cdll.attn_bwd_plan(1, 1, 1, 1, 1, 128, 0, None) == 1 and cdll.attn_bwd_plan_item(1, 1, 1, 1, 1, 128, 0, 0, None) == 1
    for bad in ((0, 1, 1, 1, 1, 128, 0), (1, 3, 2, 1, 1, 128, 0), (1, 1, 1, 1, 1, 64, 0)):
        for call in (lambda: lib.attn_bwd_plan(*bad), lambda: lib.attn_bwd_plan_item(*bad, 0)):
            with pytest.raises(lib.AttnError):
                call()
    n = lib.attn_bwd_plan(1, 2, 1, 300, 300, 128, True)["n_items"]
    for w in (-1, n):
        with pytest.raises(lib.AttnError):
            lib.attn_bwd_plan_item(1, 2, 1, 300, 300, 128, True, w)
