"""CPU: what the calls of models of many matrices launch, with a stand-in for the HIP runtime (tests/_hip_launches.hip): the numbers of the server that
low-rank products read, how much scratch laid matrices take, how many workgroups a call has."""
import os
import subprocess
import sys

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
PACKAGE = os.path.join(ROOT, "paper_2002_00655_amd")

PROGRAM = r"""
import ctypes as C, sys
stub, lib = C.CDLL(sys.argv[1], C.RTLD_GLOBAL), C.CDLL(sys.argv[2])
i32, i64, f, vp = C.c_int32, C.c_int64, C.c_float, C.c_void_p
for name in ("launch_groups", "launch_reads_from", "launch_reads_to"):
    getattr(stub, name).restype = i64
stub.launch_name.restype = C.c_char_p
lib.ps_last_error.restype = C.c_char_p
at = lambda x: vp(x << 32)                           # tensors: addresses, on 16 bytes
F32, BF16, F16 = 0, 1, 2
def server(keys, values):
    h = vp()
    assert lib.ps_create(i64(keys), i32(values), i32(1), C.byref(h)) == 0
    stub.launch_clear()
    return h
def launches():
    n = stub.launch_count()
    got = [(stub.launch_name(i).decode(), stub.launch_groups(i), stub.launch_reads_from(i), stub.launch_reads_to(i)) for i in range(n)]
    stub.launch_clear()
    return got
def adapter_matmul(h, n, rows, dim, first_a, first_b, adapters, rank, kind, out_kind=None):
    return lib.adapter_matmul(h, i32(-1), i64(0), i32(rows), i32(dim), i64(first_a), i64(first_b), i32(adapters), i32(rank), f(1), at(1), at(2), i64(n), at(3), i32(kind),
                              i64(dim), at(4), i32(kind if out_kind is None else out_kind), i64(rows), None)
def adapter_grad(h, n, rows, dim, first_a, first_b, adapters, rank, kind, dx=True):
    return lib.adapter_grad(h, i32(-1), i64(0), i32(rows), i32(dim), i64(first_a), i64(first_b), i32(adapters), i32(rank), f(1), at(1), at(2), i64(n), at(3), i64(dim),
                            at(4), i64(rows), i32(kind), at(5) if dx else None, i32(kind), i64(dim), at(6), at(7), None)
def expert_matmul(h, n, experts, rows, dim, kind, turned=0, x_pairs=1, out_pairs=1):
    return lib.expert_matmul(h, i32(-1), i64(0), i32(experts), i32(rows), i32(dim), i32(turned), at(1), at(2), i64(n), at(3), i32(kind), i64(rows if turned else dim),
                             i32(x_pairs), at(4), i32(kind), i64(dim if turned else rows), i32(out_pairs), None)
exec(sys.argv[3])
"""


@pytest.fixture(scope="module")
def run(tmp_path_factory):
    so = str(tmp_path_factory.mktemp("launches") / "launches.so")
    subprocess.check_call(["hipcc", "--offload-arch=gfx950", "--offload-host-only", "-O1", "-std=c++17", "-shared", "-fPIC", "-Wno-unused-command-line-argument",
                           "-I", os.path.join(ROOT, "include"), "-I", os.path.join(PACKAGE, "csrc"), os.path.join(ROOT, "tests", "_hip_launches.hip"), "-o", so])
    lib = os.path.join(PACKAGE, "libdpaps.so")
    if not os.path.exists(lib):
        from paper_2002_00655_amd import build
        build.build(verbose=False)

    def program(steps):
        r = subprocess.run([sys.executable, "-c", PROGRAM, so, lib, steps], capture_output=True, text=True, timeout=120)
        assert r.returncode == 0, r.stderr[-2000:]
    return program


def test_products_with_adapters_read_their_keys_only(run):
    """Nothing behind the last adapter's matrices, whatever the rank: the last key of the server may be theirs."""
    run("""
laid = 0
for rank in range(1, 65):
    for rows, dim, n, adapters in ((1024, 1024, 8192, 16), (72, 1000, 13000, 5), (1000, 72, 13000, 20), (512, 512, 300, 7), (96, 128, 5, 3), (1024, 1024, 2000, 200)):
        for kind in (F32, BF16, F16):
            for b_last in (True, False):
                L, W = max(rows, dim), adapters * rank
                keys = rows + 2 * W
                h = server(keys, L)
                first_a, first_b = (rows, rows + W) if b_last else (rows + W, rows)
                assert adapter_matmul(h, n, rows, dim, first_a, first_b, adapters, rank, kind) == 0
                for dx in (True, False):
                    assert adapter_grad(h, n, rows, dim, first_a, first_b, adapters, rank, kind, dx) == 0
                got = launches()
                laid += sum("k_laid" in name for name, *_ in got) if rank % 8 else 0
                products = [l for l in got if "k_expert" in l[0] or "k_adapter" in l[0]]
                assert products
                for name, _, first, end in products:
                    assert 0 <= first < end <= keys * L, (rank, rows, dim, n, kind, name, end, keys * L)
                lib.ps_destroy(h)
assert laid > 0
""")


def test_laid_adapters_are_bounded(run):
    """Matrices are laid up to a GiB: a call of many adapters goes by tiles where its laid matrices would be more, and a gradient that is not asked for dx lays none."""
    run("""
room = 1.25                                          # what a server's scratch is larger than it has to be
def up(x, by): return -(-x // by) * by
for rows, rank, adapters, n in ((1024, 4, 32767, 64 * 32767), (1024, 64, 8000, 64 * 8000), (1024, 16, 200, 20000), (64, 4, 32767, 64 * 32767), (256, 33, 2000, 400000)):
    dim = 1024
    h = server(rows + 2 * adapters * rank, 1024)
    for grad in (False, True):
        K, N = (rows, dim) if grad else (dim, rows)
        laid = 2 * up(K, 32) * up(N, 256) + 2 * adapters * up(rank, 32) * up(N, 256)
        numbers = (10 if grad else 4) * up(rank, 8) * n + 4 * n
        most = room * (numbers + min(laid, 1 << 30) + (1 << 29 if grad else 0) + 4096) + 4096
        stub.refuse_allocations_from(i64(int(most) + 1))
        args = (h, n, rows, dim, rows, rows + adapters * rank, adapters, rank, BF16)
        if grad:
            assert adapter_grad(*args, dx=False) == 0
            got = launches()
            assert not any("k_lay" in l[0] or "k_laid" in l[0] for l in got)
            assert adapter_grad(*args) == 0, (rows, rank, adapters, lib.ps_last_error(h))
        else:
            assert adapter_matmul(*args) == 0, (rows, rank, adapters, lib.ps_last_error(h))
        assert any("k_laid" in l[0] for l in launches()) == (laid <= 1 << 30), (rows, rank, adapters, grad)
        stub.refuse_allocations_from(i64(1 << 62))
    lib.ps_destroy(h)
""")


def test_few_rows_of_many_groups(run):
    """Calls within the limit that the header states, workgroups of 64 x 64 numbers (32 x 16 of 32 columns and fewer) and one more row of them for each group, are taken."""
    run("""
import random
rng = random.Random(3)
def log_int(lo, hi): return int(round(lo * (hi / lo) ** rng.random()))
cases = [(1, 65536, 4096, 1), (1, 65536, 1024, 8), (3, 5000, 65536, 1), (64, 65536, 16384, 2), (40, 65536, 40, 1024), (1, 65536, 16383, 1)]
cases += [(log_int(1, 3000), log_int(1, 65536), log_int(1, 65536), log_int(1, 32)) for _ in range(300)]
taken = 0
for n, experts, rows, dim in cases:
    if experts * rows > 1 << 31: continue
    h = server(experts * rows, dim)
    for turned in (0, 1):
        N = dim if turned else rows
        groups = (n // 64 + experts + 1) * -(-N // 64) if N > 32 else (n // 32 + experts + 1) * -(-N // 16)
        for kind in (F32, BF16, F16):
            rc = expert_matmul(h, n, experts, rows, dim, kind, turned)
            got = [l for l in launches() if "k_expert" in l[0] or "k_laid" in l[0]]
            if groups < 1 << 24:
                assert rc == 0, (n, experts, rows, dim, turned, kind, lib.ps_last_error(h))
                taken += 1
            if rc == 0: assert len(got) == 1 and got[0][1] < (1 << 24) + 256, (got, n, experts, rows, dim)
            else: assert rc == -9 and not got
    lib.ps_destroy(h)
assert taken > 500, taken
""")


def test_sums_over_pairs_of_any_size(run):
    """Products summed over pairs have the limit of the products, which come first."""
    run("""
for n, K, N, pairs in ((1 << 25, 8, 1024, 2), (1 << 26, 8, 1024, 4), ((1 << 21) + 6, 8, 1024, 2), (6, 8, 5, 3)):
    h = server(K, 1024)
    assert expert_matmul(h, n, 1, K, N, BF16, turned=1, out_pairs=pairs) == 0, (n, lib.ps_last_error(h))
    got = [l for l in launches() if "k_pair_sums" in l[0]]
    assert len(got) == 1 and got[0][1] < 1 << 24
    lib.ps_destroy(h)
""")
