"""How csrc/attn_bwd_plan.h cuts a call of attn_bwd() into items and deals them to workgroups, compiled without HIP: every piece of every tile once,
whatever the sizes."""
import ctypes
import os
import random
import subprocess

import pytest

import paper_2603_24517_amd as A

HERE = os.path.dirname(os.path.abspath(__file__))
SHIM = os.path.join(HERE, "bwd_plan_shim.cpp")
NAMES = ("groups", "xcd_groups", "together", "keys_tiles", "keys_splits", "keys_window", "keys_items", "rows_tiles", "rows_splits", "rows_window", "rows_items",
         "bytes")


@pytest.fixture(scope="module")
def lib(tmp_path_factory):
    so = str(tmp_path_factory.mktemp("bwd_plan") / "plan.so")
    subprocess.run(["g++", "-std=c++17", "-O2", "-Wall", "-Werror", "-shared", "-fPIC", "-o", so, SHIM], check=True)
    lib = ctypes.CDLL(so)
    lib.plan_seconds.restype = ctypes.c_double
    return lib


def _call(B, Hq, Hkv, Sq, Skv, causal):
    return (ctypes.c_int * 6)(B, Hq, Hkv, Sq, Skv, int(causal))


@pytest.fixture(scope="module")
def plan(lib):
    def plan(*call):
        out = (ctypes.c_longlong * 12)()
        rc = lib.plan_of(_call(*call), out)
        return dict(zip(NAMES, out)) if rc == A.ATTN_OK else rc
    return plan


HEADS = [(1, 1), (2, 1), (4, 4), (16, 16), (32, 8), (32, 4), (64, 8), (12, 2), (6, 2), (3, 1), (10, 5)]
# B, Hq, Hkv, Sq, Skv, causal: one token; tile borders; rows without a key; few items, which are cut; groups that divide among 8 XCDs and groups that do
# not; inputs that no cache holds, whose two kinds of items are dealt side by side; windows that are all groups and windows that are not
CALLS = [(1, 1, 1, 1, 1, True), (3, 2, 2, 1, 600, False), (1, 2, 1, 300, 40, True), (1, 2, 2, 300, 1, True), (1, 4, 4, 512, 512, False),
         (24, 16, 16, 200, 200, True), (1, 32, 8, 1111, 1111, True), (1, 32, 8, 512, 8192, True), (8, 16, 16, 4096, 4096, False),
         (2, 32, 8, 16384, 16384, True), (512, 8, 4, 62, 62, True), (96, 16, 16, 200, 200, True), (208, 12, 4, 90, 200, False),
         (96, 16, 16, 300, 300, True), (27, 24, 24, 642, 642, False), (11, 32, 8, 4096, 4096, True), (97, 8, 8, 1000, 1000, False),
         (11, 12, 12, 2000, 2000, True), (13 * 61, 8, 8, 200, 200, True), (70000, 2, 1, 1, 1, True)]


@pytest.mark.parametrize("call", CALLS, ids=str)
def test_every_item_is_dealt_once(lib, call):
    assert lib.deal_check(_call(*call)) == 0


def test_calls_reach_every_order(plan):
    plans = [plan(*c) for c in CALLS]
    assert any(p["together"] for p in plans) and any(p["xcd_groups"] == 0 for p in plans)
    assert any(p["keys_splits"] > 1 for p in plans) and any(p["rows_splits"] > 1 for p in plans)
    assert any(0 < p["keys_window"] < p["xcd_groups"] for p in plans) and any(p["keys_window"] == p["xcd_groups"] for p in plans)


@pytest.mark.parametrize("seed", range(8))
def test_every_item_of_drawn_calls_is_dealt_once(lib, plan, seed):
    rng = random.Random(seed)
    for _ in range(150):
        Hq, Hkv = rng.choice(HEADS)
        Sq = int(2 ** rng.uniform(0, 13))
        Skv = Sq if rng.random() < 0.5 else int(2 ** rng.uniform(0, 13))
        B = int(2 ** rng.uniform(0, min(10.0, max(0.0, 22 - (Sq + Skv).bit_length() - Hq.bit_length()))))
        call = (B, Hq, Hkv, Sq, Skv, rng.random() < 0.6)
        assert lib.deal_check(_call(*call)) == 0, call


@pytest.fixture(scope="module")
def checked(tmp_path_factory):
    """The plan in a program that ends where signed arithmetic overflows."""
    exe = str(tmp_path_factory.mktemp("bwd_plan") / "plan")
    subprocess.run(["g++", "-std=c++17", "-O1", "-Wall", "-DPLAN_MAIN", "-fsanitize=undefined", "-fno-sanitize-recover=all", "-o", exe, SHIM], check=True)

    def run(calls):
        text = "".join(" ".join(str(int(x)) for x in c) + "\n" for c in calls)
        out = subprocess.run([exe], input=text, capture_output=True, text=True, timeout=60)
        assert out.returncode == 0, out.stderr
        return [int(x) for x in out.stdout.split()]
    return run


def _within_limits(B, Hq, Hkv, Sq, Skv, causal):
    G = Hq // Hkv
    p = 4 if G % 4 == 0 else 2 if G % 2 == 0 else 1
    return (Sq + Skv < 2 ** 31 - 1024 and Hq <= 32768 and B * Hkv * -(-Skv // 128) < 2 ** 23 and B * Hq // p * -(-Sq // (128 // p)) < 2 ** 23)


EDGES = [1, 2, 31, 32, 33, 127, 128, 129, 2 ** 15, 2 ** 16 - 1, 2 ** 23 - 1, 2 ** 23, 2 ** 25, 2 ** 29, 2 ** 30, 2 ** 31 - 1026, 2 ** 31 - 1]


@pytest.mark.parametrize("causal", [False, True])
def test_sizes_at_the_limits(checked, causal):
    """All products of the largest arguments: refused or planned as the header says, without a signed overflow on the way."""
    heads = [(1, 1), (2, 1), (4, 1), (32768, 1), (32768, 32768), (3, 3), (32, 8)]
    calls = [(B, *h, Sq, Skv, causal) for B in EDGES for h in heads for Sq in EDGES for Skv in EDGES]
    got = checked(calls)
    for c, rc in zip(calls, got):
        assert rc == (A.ATTN_OK if _within_limits(*c) else A.ATTN_E_UNSUPPORTED), (c, rc)


@pytest.mark.parametrize("xcd_groups,S", [(g, S) for g in (5, 7, 11, 13, 62, 97, 101, 2 * 53, 3 * 37, 131, 997, 131071) for S in (64, 300, 1000, 4096)
                                          if g < 1000 or S == 64])       # (more items than a call may have)
def test_windows_of_group_counts_without_divisors(plan, lib, xcd_groups, S):
    """An XCD's 64 places are not asked to take more than twice their items at a time because its groups divide badly, nor to look for divisors."""
    call = (xcd_groups, 8, 8, S, S, False)
    p = plan(*call)
    assert p["xcd_groups"] == xcd_groups
    tiles = -(-S // 128)
    per_group = 2 * tiles if p["together"] else tiles
    if p["together"] or xcd_groups * tiles > 4 * 64:
        wanted = -(-64 // per_group)
        assert wanted <= p["keys_window"] <= max(wanted, 2 * wanted - 1) or xcd_groups < 2 * wanted, p
        assert p["rows_window"] == p["keys_window"]
    assert lib.deal_check(_call(*call)) == 0
    assert lib.plan_seconds(_call(*call)) < 100e-6       # (the search for a divisor took 500 us and more of the longest here)
