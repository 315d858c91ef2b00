"""CPU: the device code of products of grouped rows itself (csrc/groups.h, products.h, experts.h), compiled for the host: which rows a tile has, which tile a
workgroup has, quotients by a multiplication, and what the loaders read and bring into LDS - with pages that cannot be read around what they may."""
import os
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))

MODEL = r"""
#include "_lanes_on_cpu.h"
#include "experts.h"
#include <algorithm>
#include <random>

static std::mt19937_64 rng(1);
static int below(int64_t n) { return (int)(rng() % (uint64_t)n); }
#define CHECK(x) do { if (!(x)) { printf("%s:%d: %s\n", __FILE__, __LINE__, #x); exit(1); } } while (0)

// ---- the rows of a tile ----------------------------------------------------------------------------------------------
static RowTile tile_of(const RowGroups &g, int tile, int BM) {
    static RowTile t[64];
    wave([&](int l) { t[l] = row_tile(g, tile, BM); });
    for (int l = 1; l < 64; ++l) CHECK(memcmp(&t[0], &t[l], sizeof(RowTile)) == 0);
    return t[0];
}
static void tiles_of(int G, int BM, int kind, int most_tiles) {
    std::vector<int32_t> offsets(1, 0);
    int64_t n = 0;
    for (int e = 0; e < G; ++e) {
        const int size = kind == 0 ? below(3) : kind == 1 ? (below(4) ? 0 : below(3 * BM + 1)) : kind == 2 ? (below(2) ? BM : 2 * BM) : (e == G / 2 ? 5 * BM + 1 : 0);
        offsets.push_back((int32_t)(n += size));
    }
    n += kind % 2 ? below(2 * BM) : 0;                                   // rows of no group
    RowGroups g;
    g.offsets = offsets.data(); g.groups = G; g.n = (int32_t)n;
    const int64_t tiles = row_tiles(n, G, BM);
    const auto check = [&](int tile) {
        // the last group, or the rows of none, whose first tile has this number or one before
        int e = 0;
        for (int lo = 0, hi = G; lo <= hi;) {
            const int mid = (lo + hi) / 2;
            if (offsets[mid] / BM + mid <= tile) { e = mid; lo = mid + 1; } else hi = mid - 1;
        }
        const int64_t s = offsets[e], end = e < G ? offsets[e + 1] : n, first = s + (int64_t)(tile - s / BM - e) * BM;
        const RowTile t = tile_of(g, tile, BM);
        CHECK(t.group == e && t.start == s && t.end == end);
        CHECK(t.rows == std::max<int64_t>(0, std::min<int64_t>(BM, end - first)));
        if (t.rows) CHECK(t.first == first);
        return t.rows;
    };
    if (tiles <= most_tiles) {
        int64_t rows = 0;
        for (int tile = 0; tile < tiles; ++tile) rows += check(tile);
        CHECK(rows == n);
    } else for (int i = 0; i < most_tiles; ++i) check(i < 70 ? i : i < 140 ? (int)(tiles - 1 - (i - 70)) : below(tiles));
}
// offsets that are none: whatever a tile has lies among the n rows
static void tiles_of_any(int G, int BM) {
    const int n = below(5 * BM * G) + 1;
    std::vector<int32_t> offsets;
    for (int e = 0; e <= G; ++e) offsets.push_back(below(3) ? below(n + 1) : (int32_t)rng());
    RowGroups g;
    g.offsets = offsets.data(); g.groups = G; g.n = n;
    for (int i = 0; i < 60; ++i) {
        const RowTile t = tile_of(g, below(row_tiles(n, G, BM)), BM);
        CHECK(t.group >= 0 && t.group <= G && t.rows >= 0 && t.rows <= BM);
        if (t.rows) CHECK(t.first >= 0 && t.first + t.rows <= n);
    }
}

// ---- which tile a workgroup has --------------------------------------------------------------------------------------
static void places(int rows, int cols) {
    std::vector<int> seen((size_t)rows * cols, 0);
    for (unsigned b = 0; b < die_grid((int64_t)rows * cols); ++b) {
        blockIdx.x = b;
        const TilePlace p = tile_place(rows, cols);
        if (p.row < 0) continue;
        CHECK(p.row < rows && p.col >= 0 && p.col < cols);
        ++seen[(size_t)p.row * cols + p.col];
    }
    for (int s : seen) CHECK(s == 1);
}

static void quotients() {
    for (int64_t by : {1, 2, 3, 5, 7, 8, 12, 63, 64, 65, 1000, 4097, 65535, 65536, 1000000, (1 << 28) + 1, (1 << 29) - 1}) {
        const Quotient f((int32_t)by);
        for (int i = 0; i < 3000; ++i) {
            const int64_t k = (below(1 << 29) / by) * by + (i % 3) - 1, q = i < 3 ? (i == 0 ? 0 : i == 1 ? (1 << 29) - 1 : by) : k;
            if (q >= 0 && q < (1 << 29)) CHECK(f((int)q) == q / by);
        }
    }
}

// ---- what is read, and what of it stands in LDS ----------------------------------------------------------------------
constexpr int SLACK = 256;                                               // numbers behind the last key (ps_create)
struct Store {
    float *val; int64_t keys, L;
    Store(int64_t k, int64_t l) : val(fenced<float>(k * l + SLACK)), keys(k), L(l) {
        for (int64_t i = 0; i < k * l; ++i) val[i] = (float)(below(255) - 127);      // (exact in 16 bits)
        for (int i = 0; i < SLACK; ++i) val[k * l + i] = __builtin_nanf("");
    }
    ~Store() { unfence(val, (keys * L + SLACK) * 4); }
};
template <class CT> using Tile = std::vector<Vec<CT, unit_of<CT>()>>;
// number k of a tile's line, of the step in LDS
template <class CT> static double in_lds(const Tile<CT> &t, int line, int k) { return (double)(float)t[unit_place(line, k / unit_of<CT>())][k % unit_of<CT>()]; }
template <class F> static void every_step(int K, int step, F f) {
    for (int s = 0; s * step < K; ++s) f(s, s < K / step);
}
// C, K numbers of N columns, each a key, the last one the store's last
template <class CT, class T> static void key_columns(int N, int K, int L) {
    Store st(N + 2, L);
    typedef KeyColumns<CT, T::COLS, T::THREADS> C;
    for (int c0 = 0; c0 < N; c0 += T::COLS) {
        const float *w = st.val + 2 * (int64_t)L;
        every_step(K, step_of<CT>(), [&](int s, bool full) {
            Tile<CT> lds(T::COLS * UNITS);
            for (threadIdx.x = 0; threadIdx.x < T::THREADS; ++threadIdx.x) {
                C c;
                c.init(w + (int64_t)c0 * L, L, N - c0);
                if (full) c.template load<false>(s, K); else c.template load<true>(s, K);
                c.put(lds.data());
            }
            for (int c = 0; c < T::COLS && c0 + c < N; ++c)
                for (int k = 0; k < step_of<CT>(); ++k) {
                    const int at = s * step_of<CT>() + k;
                    CHECK(in_lds<CT>(lds, c, k) == (at < K ? (double)w[(int64_t)(c0 + c) * L + at] : 0.0));
                }
        });
    }
}
// the same of a matrix whose K keys are the numbers of a sum
template <class CT, class T> static void key_rows(int N, int K, int L) {
    Store st(K + 2, L);
    typedef KeyRows<CT, T::COLS, T::THREADS> C;
    for (int c0 = 0; c0 < N; c0 += T::COLS) {
        const float *w = st.val + 2 * (int64_t)L;
        every_step(K, step_of<CT>(), [&](int s, bool full) {
            Tile<CT> lds(T::COLS * UNITS);
            for (threadIdx.x = 0; threadIdx.x < T::THREADS; ++threadIdx.x) {
                C c;
                c.init(w + c0, L);
                if (full) c.template load<false>(s, K); else c.template load<true>(s, K);
                c.put(lds.data());
            }
            for (int c = 0; c < T::COLS && c0 + c < N; ++c)
                for (int k = 0; k < step_of<CT>(); ++k) {
                    const int at = s * step_of<CT>() + k;
                    CHECK(in_lds<CT>(lds, c, k) == (at < K ? (double)w[(int64_t)at * L + c0 + c] : 0.0));
                }
        });
    }
}
// rows of a tensor, which has nothing behind its last number
template <class ST, class CT, class T> static void rows_of_tensor(int n, int K, int stride) {
    const size_t count = (size_t)(n - 1) * stride + K;
    ST *x = fenced<ST>(count);
    for (size_t i = 0; i < count; ++i) x[i] = (ST)(float)(below(255) - 127);
    std::vector<int> row(std::max(T::ROWS, 1024));
    for (int &r : row) r = below(n);
    row[0] = n - 1;
    every_step(K, step_of<CT>(), [&](int s, bool full) {
        Tile<CT> lds(T::ROWS * UNITS);
        for (threadIdx.x = 0; threadIdx.x < T::THREADS; ++threadIdx.x) {
            KMajor<ST, CT, T::ROWS, T::THREADS> m;
            m.init([&](int r) { return x + (int64_t)row[r] * stride; });
            if (full) m.template load<false>(s, K); else m.template load<true>(s, K);
            m.put(lds.data());
        }
        for (int r = 0; r < T::ROWS; ++r)
            for (int k = 0; k < step_of<CT>(); ++k) {
                const int at = s * step_of<CT>() + k;
                CHECK(in_lds<CT>(lds, r, k) == (at < K ? (double)(float)x[(int64_t)row[r] * stride + at] : 0.0));
            }
    });
    // ... and its columns, K of them, for sums over rows
    const int rows = std::min(n, 200);
    for (int c0 = 0; c0 < K; c0 += T::COLS)
        every_step(rows, step_of<CT>(), [&](int s, bool full) {
            Tile<CT> lds(T::COLS * UNITS);
            for (threadIdx.x = 0; threadIdx.x < T::THREADS; ++threadIdx.x) {
                ChosenRows<ST, CT, T::COLS, T::THREADS> c;
                const auto of = [&](int i) { return x + c0 + (int64_t)row[i] * stride; };
                if (full) c.template load<false>(s, rows, K - c0, of); else c.template load<true>(s, rows, K - c0, of);
                c.put(lds.data());
            }
            for (int c = 0; c < T::COLS && c0 + c < K; ++c)
                for (int k = 0; k < step_of<CT>(); ++k) {
                    const int at = s * step_of<CT>() + k;
                    CHECK(in_lds<CT>(lds, c, k) == (at < rows ? (double)(float)x[(int64_t)row[at] * stride + c0 + c] : 0.0));
                }
        });
    unfence(x, count * sizeof(ST));
}
// the kernel for few rows: its reads only
template <class CT, class XT, bool TURNED, int MT> static void few_rows(int N, int K, int L) {
    typedef FewRows<CT, XT, TURNED, MT> F;
    Store st((TURNED ? K : N) + 2, L);
    const size_t count = (size_t)5 * K;
    XT *x = fenced<XT>(count);
    for (size_t i = 0; i < count; ++i) x[i] = (XT)1.0f;
    for (int c0 = 0; c0 < N; c0 += F::COLS)
        for (threadIdx.x = 0; threadIdx.x < F::THREADS; ++threadIdx.x) {
            F f;
            f.run(st.val + 2 * (int64_t)L, L, K, c0, N, [&](int r) { return x + (r < 5 ? r : 4) * (int64_t)K; });
        }
    unfence(x, count * sizeof(XT));
}
template <class CT> static void loaders(int N, int K, int L) {
    if (K <= L) { key_columns<CT, Tile64>(N, K, L); key_columns<CT, Tile128>(N, K, L); key_columns<CT, Narrow>(N, K, L); }
    if (N <= L) { key_rows<CT, Tile64>(N, K, L); key_rows<CT, Tile128>(N, K, L); key_rows<CT, Narrow>(N, K, L); }
}

int main(int argc, char **argv) {
    const std::string what = argv[1];
    if (what == "tiles") {
        for (int G : {1, 2, 7, 63, 64, 65, 127, 128, 129, 1000, 4095, 4096, 4097, 65535, 65536})
            for (int BM : {16, 64, 128, 256})
                for (int kind = 0; kind < 4; ++kind) tiles_of(G, BM, kind, G <= 129 ? 300 : 150);
        for (int i = 0; i < 80; ++i) tiles_of_any(i % 4 ? 1 + below(200) : 4000 + below(200), i % 2 ? 16 : 128);
    } else if (what == "places") {
        for (int rows : {1, 2, 3, 7, 8, 9, 63, 130, 321, 5000})
            for (int cols : {1, 2, 7, 8, 9, 16, 17, 40}) places(rows, cols);
    } else if (what == "quotients") quotients();
    else if (what == "loaders") {
        const int sizes[][3] = {{1, 1, 1}, {3, 7, 7}, {40, 33, 40}, {65, 64, 65}, {33, 130, 130}, {129, 100, 129}, {200, 31, 200}, {64, 128, 128}, {24, 256, 256}};
        for (const auto &s : sizes) { loaders<float>(s[0], s[1], s[2]); loaders<bf16_t>(s[0], s[1], s[2]); loaders<f16_t>(s[0], s[1], s[2]); }
    } else if (what == "tensors") {
        const int sizes[][3] = {{1, 1, 1}, {5, 7, 9}, {70, 40, 40}, {130, 65, 72}, {300, 130, 130}};
        for (const auto &s : sizes) {
            rows_of_tensor<float, float, Tile64>(s[0], s[1], s[2]);
            rows_of_tensor<bf16_t, bf16_t, Tile64>(s[0], s[1], s[2]);
            rows_of_tensor<f16_t, f16_t, Tile128>(s[0], s[1], s[2]);
            rows_of_tensor<bf16_t, float, Tile128>(s[0], s[1], s[2]);
            rows_of_tensor<f16_t, float, Narrow>(s[0], s[1], s[2]);
            rows_of_tensor<float, float, Low>(s[0], s[1], s[2]);
        }
    } else {
        const int sizes[][3] = {{1, 1, 1}, {3, 7, 7}, {5, 20, 20}, {16, 33, 40}, {17, 64, 65}, {33, 130, 130}, {40, 512, 512}, {24, 1000, 1000}};
        for (const auto &s : sizes) {
            few_rows<float, float, false, 1>(s[0], s[1], s[2]); few_rows<bf16_t, bf16_t, false, 1>(s[0], s[1], s[2]); few_rows<float, bf16_t, false, 2>(s[0], s[1], s[2]);
            if (s[0] > s[2]) continue;
            few_rows<float, float, true, 1>(s[0], s[1], s[2]); few_rows<f16_t, f16_t, true, 1>(s[0], s[1], s[2]); few_rows<float, f16_t, true, 1>(s[0], s[1], s[2]);
        }
    }
    puts("fine");
}
"""


@pytest.fixture(scope="module")
def model(tmp_path_factory):
    d = tmp_path_factory.mktemp("groups")
    (d / "model.cpp").write_text(MODEL)
    rocm = os.environ.get("ROCM_PATH", "/opt/rocm")
    subprocess.check_call([os.path.join(rocm, "llvm", "bin", "clang++"), "-std=c++17", "-O0", "-w", "-D__HIP_PLATFORM_AMD__", "-I", os.path.join(rocm, "include"),
                           "-I", os.path.join(ROOT, "tests"), "-I", os.path.join(ROOT, "include"), "-I", os.path.join(ROOT, "paper_2002_00655_amd", "csrc"),
                           str(d / "model.cpp"), "-o", str(d / "model")])
    return str(d / "model")


@pytest.mark.parametrize("what", ["tiles", "places", "quotients", "loaders", "tensors", "few"])
def test_device_code(model, what):
    r = subprocess.run([model, what], capture_output=True, text=True, timeout=120)
    assert r.returncode == 0 and r.stdout.strip() == "fine", (r.returncode, r.stdout[-500:], r.stderr[-500:])
