"""The entry points for models of many matrices are exported, bound, and refuse what can be seen to be wrong without a device."""
import ctypes as C
import os
import re

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
NAMES = ["adapter_grad", "adapter_matmul", "expert_grad", "expert_matmul", "group_rows"]


def _lib():
    path = os.path.join(ROOT, "paper_2002_00655_amd", "libdpaps.so")
    if not os.path.exists(path):
        from paper_2002_00655_amd import build
        build.build(verbose=False)
    return C.CDLL(path)


def test_declared_exported_and_bound():
    text = re.sub(r"/\*.*?\*/", "", open(os.path.join(ROOT, "include", "dpaps.h")).read(), flags=re.S)
    declared = re.findall(r"^\s*int\s+((?:group|expert|adapter)_\w+)\s*\(", text, flags=re.M)
    lib, src = _lib(), open(os.path.join(ROOT, "paper_2002_00655_amd", "ps.py")).read()
    assert sorted(declared) == NAMES
    for name in NAMES:
        assert hasattr(lib, name) and f"_lib.{name}(" in src and f'"{name}"' in src, name


def test_null_handles_are_refused():
    lib, i32, i64, f = _lib(), C.c_int32, C.c_int64, C.c_float
    assert lib.group_rows(None, i32(1), None, i32(0), i64(0), i64(-1), None, None, None) == -1
    assert lib.expert_matmul(None, i32(-1), i64(0), i32(1), i32(1), i32(1), i32(0), None, None, i64(0), None, i32(0), i64(1), i32(1), None, i32(0), i64(1), i32(1),
                             None) == -1
    assert lib.expert_grad(None, i32(1), i32(1), i32(1), None, None, i64(0), None, i64(1), i32(1), None, i64(1), i32(1), i32(0), None, i32(0), None) == -1
    assert lib.adapter_matmul(None, i32(-1), i64(0), i32(1), i32(1), i64(0), i64(0), i32(1), i32(1), f(1), None, None, i64(0), None, i32(0), i64(1), None, i32(0), i64(1),
                              None) == -1
    assert lib.adapter_grad(None, i32(-1), i64(0), i32(1), i32(1), i64(0), i64(0), i32(1), i32(1), f(1), None, None, i64(0), None, i64(1), None, i64(1), i32(0), None,
                            i32(0), i64(1), None, None, None) == -1


def test_tiles_of_groups():
    """Numbers of tiles (see csrc/groups.h): group e's tiles from floor(start_e / BM) + e on; no two groups share a number, and a number's group is the last
    one that starts at or before it."""
    import random
    rng = random.Random(0)
    for _ in range(300):
        G, BM = rng.randint(1, 70), rng.choice([1, 2, 16, 64, 128])
        sizes = [rng.choice([0, 0, 1, rng.randint(0, 3 * BM), BM, 2 * BM]) for _ in range(G + 1)]
        start = [sum(sizes[:e]) for e in range(G + 2)]
        n, seen = start[-1], []
        for tile in range(n // BM + G + 1):
            e = max(e for e in range(G + 1) if start[e] // BM + e <= tile)
            first = start[e] + (tile - start[e] // BM - e) * BM
            rows = max(0, min(BM, start[e + 1] - first))
            seen += [(e, first + r) for r in range(rows)]
        assert seen == [(e, p) for e in range(G + 1) for p in range(start[e], start[e + 1])]


def test_runs_of_tiles():
    """Every tile is dealt to one workgroup (see tile_place in csrc/products.h), for any number of rows and columns of tiles."""
    def run_of(tiles):
        run = 32
        while run > 1 and tiles < 64 * run:
            run //= 2
        return run
    for rows in (1, 2, 3, 7, 8, 9, 63, 130, 321):
        for cols in (1, 2, 7, 8, 9, 16, 17):
            tiles, run, seen = rows * cols, run_of(rows * cols), set()
            grid = -(-tiles // (8 * run)) * 8 * run
            for block in range(grid):
                turn = block // 8
                at = (turn // run * 8 + block % 8) * run + turn % run
                if at >= tiles:
                    continue
                band = at // (rows * 8)
                r, width = at - band * rows * 8, min(8, cols - band * 8)
                seen.add((r // width, band * 8 + r % width))
            assert seen == {(r, c) for r in range(rows) for c in range(cols)}, (rows, cols)


def test_quotients():
    """The quotient by a multiplication (Quotient in csrc/products.h) is exact for numbers below 2^29."""
    import random
    rng = random.Random(1)
    for by in [1, 2, 3, 5, 7, 8, 12, 63, 64, 65, 1000, 4097, 65535, 65536, 10 ** 6, 2 ** 28 + 1, 2 ** 29 - 1]:
        low = 0
        while (1 << low) < by:
            low += 1
        shift = 29 + low
        m = ((1 << shift) + by - 1) // by
        assert m < 2 ** 32 or by == 1
        for q in [0, 1, by - 1, by, by + 1, 2 ** 29 - 1] + [rng.randrange(2 ** 29) for _ in range(2000)]:
            if 0 <= q < 2 ** 29 and by > 1:
                assert q * m >> shift == q // by and q * m < 2 ** 64, (q, by)
