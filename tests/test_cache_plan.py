"""How the calls on a cache that grows and shrinks are cut into parts (host code): the limits that the kernels rely on.  No GPU needed."""
import os
import subprocess

import pytest

from paper_2503_18893_amd import build as xbuild

FIELDS = ("mode", "H_kv", "H_q", "d_h", "L", "k", "batch", "dtype", "N", "c")
TREE, WEIGHTS, BLOCKS = 0, 1, 2


@pytest.fixture(scope="module")
def plan_of(tmp_path_factory):
    objs = [os.path.join(xbuild.OBJ_DIR, src.replace(".hip", ".o")) for src in xbuild.SOURCES]
    if not all(os.path.exists(o) for o in objs):
        xbuild.build_library()
    exe = str(tmp_path_factory.mktemp("plan") / "probe")
    src = os.path.join(os.path.dirname(os.path.abspath(__file__)), "cache_plan_probe.cpp")
    subprocess.run([xbuild._hipcc(), *xbuild.HIPCC_FLAGS, "-x", "hip", src, "-x", "none", *objs, "-o", exe], check=True, capture_output=True)

    def run(shapes):
        base = dict(mode=TREE, H_kv=8, H_q=32, d_h=128, L=1, k=1, batch=1, dtype=1, N=1, c=0)
        text = "\n".join(" ".join(str({**base, **s}[f]) for f in FIELDS) for s in shapes)
        out = subprocess.run([exe], input=text, capture_output=True, text=True, check=True).stdout.splitlines()
        assert len(out) == len(shapes)
        return [{n: int(v) for n, v in (kv.split("=") for kv in line.split())} for line in out]
    return run


def test_parts_leave_one_for_every_sequence_and_fit_the_merge(plan_of):
    shapes = [dict(mode=m, H_kv=h, H_q=h * r, L=L, batch=b, N=n if m == TREE else 1, dtype=t)
              for m in (TREE, WEIGHTS) for h in (1, 4, 8) for r in (1, 7, 16) for L in (1, 63, 4097, 1 << 20) for b in (1, 3, 64, 1000)
              for n in (1, 9, 64, 1024) for t in (0, 1) if b * h * n <= 65535]
    for s, p in zip(shapes, plan_of(shapes)):
        assert p["status"] == 0 and s["batch"] <= p["parts"] <= s["batch"] + p["max_parts"] - 1, (s, p)
        rows = s["N"] * s["H_q"] // s["H_kv"]
        assert p["rows"] == 16 or rows > p["rows"] // 2, (s, p)   # no tile is empty by half for no reason
        assert p["round"] % 64 == 0 and (p["round"] == 128 or not p["mfma"] or p["rows"] > 64), (s, p)
        assert p["total"] >= p["parts"] * s["N"] * s["H_q"] * (128 + 2) * 4, (s, p)


def test_blocks_of_a_part_fit_their_list(plan_of):
    shapes = [dict(mode=BLOCKS, L=L, k=k, batch=b, N=n, c=c) for L in (1, 1000, 200_000, 1 << 20) for k in (1, 999, 100_000, 1 << 20) if k <= L
              for b in (1, 16) for n in (1, 200) for c in (1, 2, 3, 7, 16, 24, 64, 129, 5000)]
    seen = 0
    for s, p in zip(shapes, plan_of(shapes)):
        if p["status"] == -2:
            assert s["k"] > 256 * (p["part_blocks"] - 128), (s, p)  # more blocks than 256 parts hold
            continue
        assert p["status"] == 0 and 1 <= p["parts"] <= p["max_parts"], (s, p)
        tokens = min(p["k_ch"] * s["c"], s["L"])
        chunk = -(-(-(-tokens // p["parts"])) // p["round"]) * p["round"]  # (the most: fewer tokens are visible to most queries)
        assert (chunk - 1) // s["c"] + 2 <= p["part_blocks"] + 2, (s, p)
        assert p["k_ch"] == min(-(-s["k"] // s["c"]), p["n_c"])
        seen += p["parts"] > 1
    assert seen


@pytest.mark.parametrize("dtype,d_h", [(1, 128), (1, 64), (0, 128), (0, 33)])
def test_queries_of_any_type_have_the_same_number_of_blocks(plan_of, dtype, d_h):
    most = 491520
    shapes = [dict(mode=BLOCKS, L=600_000, k=k, dtype=dtype, d_h=d_h, N=1, c=c, batch=b)
              for k, c, b in ((most, 1, 1), (most + 1, 1, 1), (507_904, 1, 1), (600_000, 1, 2), (600_000, 2, 2))]
    assert [p["status"] for p in plan_of(shapes)] == [0, -2, -2, -2, 0]


def rounds_of_a_part(lengths, p):
    """The smallest part, in rounds, with which all sequences' parts are at most p["parts"]."""
    r = [-(-n // p["round"]) for n in lengths]
    return next(m for m in range(1, max(r) + 1) if sum(-(-x // m) for x in r) <= p["parts"])


def test_the_cases_of_many_tiles_have_many_tiles(plan_of):
    """tests/test_gpu_cache_tiles.py means to run the loops over a part's tiles, with every number of rows."""
    import test_gpu_cache_tiles as tiles
    shapes = [dict(mode=TREE, H_kv=h, H_q=h * r, d_h=d, L=max(n), batch=len(n), N=N, dtype=int(t == "bf16")) for t, h, r, d, n, N, _, _ in tiles.TREES.values()]
    for name, p in zip(tiles.TREES, plan_of(shapes)):
        _, _, _, _, lengths, N, rows, rounds = tiles.TREES[name]
        assert p["rows"] == rows, (name, p)
        assert rounds_of_a_part([n + N for n in lengths], p) >= rounds, (name, p)
    shapes = [dict(mode=BLOCKS, H_kv=h, H_q=h * r, d_h=d, L=L, k=k, batch=b, N=N, c=24, dtype=int(t == "bf16")) for t, h, r, d, b, N, L, k, _ in tiles.BLOCKS.values()]
    for name, p in zip(tiles.BLOCKS, plan_of(shapes)):
        k, parts = tiles.BLOCKS[name][-2:]
        assert p["parts"] == parts and k / parts / p["round"] >= 5, (name, p)
