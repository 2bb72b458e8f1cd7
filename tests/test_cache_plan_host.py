"""How attention on caches is launched (compiled for the host; no GPU)."""
import os
import subprocess
from typing import NamedTuple

import pytest

import paper_2605_08123_amd as ska

from . import test_gpu_cache as small
from . import test_gpu_cache_ends as ends
from . import test_gpu_cache_rows as rows

HERE = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(HERE)
CSRC = os.path.join(ROOT, "paper_2605_08123_amd", "csrc")
ALL = 1 << 20
F32, BF16, E4M3, INT8 = 0, 1, 2, 3


def build(tmp_path, name):
    exe = str(tmp_path / name)
    subprocess.run(["g++", "-std=c++17", "-O1", "-Wall", "-I", CSRC, "-I", os.path.join(ROOT, "include"), "-o", exe, os.path.join(HERE, name + ".cpp")], check=True)
    return exe


def test_joins_within_32_bits_of_threads(tmp_path):
    """cache_joins.cpp: every launch of a join has fewer than 2^32 threads."""
    run = subprocess.run([build(tmp_path, "cache_joins")], capture_output=True, text=True)
    print(run.stdout)
    assert run.returncode == 0, run.stdout


class Plan(NamedTuple):
    both: int         # an item's workgroups take the prefix too
    nq: int           # blocks of 16 rows of a workgroup
    own_parts: int
    front_parts: int  # 0: the prefix has no workgroups
    last_first: int
    own_wgs: int
    front_wgs: int


@pytest.fixture(scope="session")
def plans(tmp_path_factory):
    """Plans of problems (B, Hq, Hk, Lq, Lp, Lk, d, W, causal, dtype, store); Lp 0: no prefix."""
    exe = build(tmp_path_factory.mktemp("plans"), "cache_plans")

    def ask(problems):
        run = subprocess.run([exe], input="\n".join(" ".join(str(int(x)) for x in p) for p in problems), capture_output=True, text=True, check=True)
        return [Plan(*(int(x) for x in line.split()[:7])) for line in run.stdout.splitlines()]
    return ask


@pytest.mark.parametrize("dtype,store", [(BF16, BF16), (BF16, E4M3), (BF16, INT8), (F32, INT8)])
def test_large_problems_behind_a_prefix_take_64_rows(dtype, store, plans):
    """Rounds of workgroups count: half as many of twice the rows take less time."""
    sizes = [(16, 8, 2, 2048, 16384, 4096), (64, 8, 2, 128, 65536, 256), (16, 8, 2, 512, 16384, 1024), (16, 8, 2, 400, 300, 400), (2, 16, 2, 700, 2000, 3000)]
    for p in plans([(*s, 64, ALL, 1, dtype, store) for s in sizes]):
        assert p.nq == 4 and not p.both
    for p in plans([(*s, 128, ALL, 1, dtype, store) for s in sizes]):
        assert p.nq == 2
    # a few rows of many items, short walks: 32
    for p in plans([(64, 8, 4, 4, 8000, 300, 64, ALL, 1, dtype, store), (16, 8, 2, 1, 1800, 30, 64, ALL, 1, dtype, store)]):
        assert p.nq == 2


@pytest.mark.parametrize("dtype,store,d", [(BF16, BF16, 32), (BF16, BF16, 64), (BF16, E4M3, 32), (BF16, INT8, 64), (F32, E4M3, 32), (F32, INT8, 64)])
def test_blocks_of_64_rows_up_to_the_headers_limit(dtype, store, d):
    """Own and prefix's blocks of 64 rows, fewer than 2^23 - 8 together, are taken (of 32 rows there would be more)."""
    need = lambda Hk: ska.ska_prefix_attn_workspace_bytes(1, 4 * Hk, Hk, 1 << 24, 64, 64, d, ALL, True, dtype, store)   # noqa: E731
    for Hk in (1, 2, 3):   # 2 Hk 2^20 blocks
        assert need(Hk) > 0, Hk
    assert need(4) == 0


def code(kind):
    """dtype, store of the C ABI of ("e4m3", torch.bfloat16) and the like."""
    dtype = F32 if kind[1] == small.F32 else BF16
    return dtype, {"same": dtype, "e4m3": E4M3, "int8": INT8}[kind[0]]


def cache(shape, kind):
    return (*shape[:4], 0, *shape[4:8], *code(kind))


def prefix(shape, kind):
    return (*shape[:9], *code(kind))


def test_which_workgroups_the_gpu_tests_reach(plans):
    """The tests of 64 rows take them, in one part and in several, blocks in either order; those of small problems the other two forms."""
    one = plans([cache(s, k) for s in rows.ROWS for k in rows.CODES])
    assert all(p.nq == 4 and p.own_parts == 1 for p in one) and {p.last_first for p in one} == {0, 1}
    several = plans([cache(s, k) for s, k in rows.PARTS])
    assert all(p.nq == 4 and p.own_parts > 1 for p in several) and {p.last_first for p in several} == {0, 1}
    one = plans([prefix(s, k) for s in rows.PREFIX for k in rows.KINDS[1:]])
    assert all(p.nq == 4 and p.front_parts == p.own_parts == 1 for p in one)
    assert all(p.nq == 4 and p.front_parts > 1 for p in plans([prefix(s, k) for s, k in rows.PREFIX_PARTS]))
    one = plans([prefix(s, k) for s in small.PREFIX for k in rows.KINDS])
    assert {p.both for p in one} == {0, 1} and all(p.nq == (1 if p.both else 2) for p in one) and any(p.front_parts > 1 for p in one)
    one = plans([cache(s, k) for s in small.ATTN for k in rows.CODES])
    assert all(p.nq == 2 for p in one) and any(p.own_parts > 1 for p in one)
    Lq, Lk, d = ends.CLIMB[-1]
    one = plans([cache((1, 2, 1, Lq, Lk, d, ALL, 1), k) for k in rows.CODES] + [prefix((1, 2, 1, Lq, 1, Lk, d, ALL, 1), ("same", small.BF16))])
    assert all(p.nq == 4 for p in one)
