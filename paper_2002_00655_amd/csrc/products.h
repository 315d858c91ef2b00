// Tiles of products of rows with matrices of the server, on the matrix cores.
//
// A tile is sum_k R[k][r] C[k][c]: R, the tile's rows (of a call's tensors), C its columns (of the server's matrices, or of tensors).  Both come into LDS as
// units of 16 bytes, numbers that follow each other in k, of the type CT that the matrix instruction takes: 8 units of a row or column are a step, and lie in one
// line of 128 bytes.  What lies in memory in that order is read so (KMajor); what lies the other way - neighbouring columns together - is read as blocks of
// a unit's numbers in k by four columns and turned in registers (NMajor).  The server's numbers of 32 bits are rounded to CT on the way.
#pragma once
#include "elements.h"

template <class T, int W> struct LooseOf { typedef T type __attribute__((ext_vector_type(W), aligned(sizeof(T)))); };
template <class T, int W> using Loose = typename LooseOf<T, W>::type;          // W neighbouring elements that start on any one

typedef float floatx16 __attribute__((ext_vector_type(16)));

template <class CT> constexpr int unit_of() { return 16 / (int)sizeof(CT); }   // numbers of a unit
constexpr int UNITS = 8;                                                       // units of a step
template <class CT> constexpr int step_of() { return UNITS * unit_of<CT>(); }  // numbers of a step

// Where unit u of row r lies in a tile in LDS.  Turned within the line by the row, so that neither eight neighbouring rows' same units (the
// matrix instruction's reads) nor those of every fourth row (what NMajor writes) share banks.
__device__ __forceinline__ int unit_place(int r, int u) { return r * UNITS + (u ^ ((r ^ (r >> 3)) & 7)); }

template <class CT, class ST, int W> __device__ __forceinline__ Vec<CT, W> as_type(Vec<ST, W> v) {
    if constexpr (std::is_same<CT, ST>::value) return v;
    else return __builtin_convertvector(v, Vec<CT, W>);
}

// The W elements at p of which `left` exist, the others zero.
template <class ST, int W> __device__ __forceinline__ Vec<ST, W> load_some(const ST *p, int left) {
    if (left >= W) return *reinterpret_cast<const Loose<ST, W> *>(p);
    Vec<ST, W> v = {};
#pragma unroll
    for (int i = 0; i < W; ++i)
        if (i < left) v[i] = p[i];
    return v;
}

// ROWS rows whose numbers follow each other in k.
template <class ST, class CT, int ROWS, int THREADS> struct KMajor {
    static constexpr int KU = unit_of<CT>(), N = ROWS * UNITS / THREADS;
    static_assert(N * THREADS == ROWS * UNITS && THREADS % UNITS == 0);
    const ST *row[N];                                                          // NULL: a row of zeros
    Vec<ST, KU> raw[N];
    template <class F> __device__ __forceinline__ void init(F row_of) {
#pragma unroll
        for (int i = 0; i < N; ++i) row[i] = row_of((i * THREADS + (int)threadIdx.x) / UNITS);
    }
    __device__ __forceinline__ void load(int step, int K) {
        const int k = step * step_of<CT>() + ((int)threadIdx.x % UNITS) * KU;
#pragma unroll
        for (int i = 0; i < N; ++i) {
            raw[i] = Vec<ST, KU>{};
            if (row[i] && k < K) raw[i] = load_some<ST, KU>(row[i] + k, K - k);
        }
    }
    __device__ __forceinline__ void put(Vec<CT, KU> *lds) const {
#pragma unroll
        for (int i = 0; i < N; ++i) lds[unit_place((i * THREADS + (int)threadIdx.x) / UNITS, (int)threadIdx.x % UNITS)] = as_type<CT, ST, KU>(raw[i]);
    }
};

// COLS columns that follow each other, for every k.
template <class ST, class CT, int COLS, int THREADS> struct NMajor {
    static constexpr int KU = unit_of<CT>(), BLOCKS = COLS / 4 * UNITS, N = BLOCKS < THREADS ? 1 : BLOCKS / THREADS;
    static constexpr bool ALL = N * THREADS == BLOCKS;                         // else only the first threads have one
    static_assert(ALL || BLOCKS < THREADS);
    Vec<ST, 4> raw[N][KU];
    // row_of(k): where the columns are for this k (below K); cols: those that there are
    template <class F> __device__ __forceinline__ void load(int step, int K, int cols, F row_of) {
#pragma unroll
        for (int b = 0; b < N; ++b) {
            const int at = b * THREADS + (int)threadIdx.x, c = at % (COLS / 4) * 4, k = step * step_of<CT>() + at / (COLS / 4) * KU;
#pragma unroll
            for (int i = 0; i < KU; ++i) {
                raw[b][i] = Vec<ST, 4>{};
                if (k + i < K && c < cols && (ALL || at < BLOCKS)) raw[b][i] = load_some<ST, 4>(row_of(k + i) + c, cols - c);
            }
        }
    }
    __device__ __forceinline__ void put(Vec<CT, KU> *lds) const {
#pragma unroll
        for (int b = 0; b < N; ++b) {
            const int at = b * THREADS + (int)threadIdx.x, c = at % (COLS / 4) * 4, u = at / (COLS / 4);
            if (!ALL && at >= BLOCKS) return;
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                Vec<ST, KU> v;
#pragma unroll
                for (int i = 0; i < KU; ++i) v[i] = raw[b][i][j];
                lds[unit_place(c + j, u)] = as_type<CT, ST, KU>(v);
            }
        }
    }
};

template <class CT> __device__ __forceinline__ floatx16 mfma_unit(Vec<CT, unit_of<CT>()> a, Vec<CT, unit_of<CT>()> b, floatx16 c) {
    if constexpr (sizeof(CT) == 4) {
        // (the instruction takes two k; which two does not matter, as long as both sides take the same)
#pragma unroll
        for (int j = 0; j < 4; ++j) c = __builtin_amdgcn_mfma_f32_32x32x2f32(a[j], b[j], c, 0, 0, 0);
        return c;
    } else if constexpr (std::is_same<CT, bf16_t>::value) return __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, b, c, 0, 0, 0);
    else return __builtin_amdgcn_mfma_f32_32x32x16_f16(a, b, c, 0, 0, 0);
}

// A wavefront's part of a tile, 32 MC columns by 32 MR rows from (c0, r0) on: one step's products.  Lane l holds in acc[i][j][4 q + e] the column
// c0 + 32 i + 8 q + 4 (l / 32) + e of row r0 + 32 j + l % 32.
template <class CT, int MC, int MR>
__device__ __forceinline__ void step_products(const Vec<CT, unit_of<CT>()> *cols, const Vec<CT, unit_of<CT>()> *rows, int c0, int r0, int units, floatx16 (&acc)[MC][MR]) {
    const int l32 = threadIdx.x & 31, h = (threadIdx.x & 63) >> 5;
#pragma unroll
    for (int s = 0; s < UNITS / 2; ++s) {
        if (2 * s >= units) break;
        Vec<CT, unit_of<CT>()> a[MC], b[MR];
#pragma unroll
        for (int i = 0; i < MC; ++i) a[i] = cols[unit_place(c0 + 32 * i + l32, 2 * s + h)];
#pragma unroll
        for (int j = 0; j < MR; ++j) b[j] = rows[unit_place(r0 + 32 * j + l32, 2 * s + h)];
#pragma unroll
        for (int i = 0; i < MC; ++i)
#pragma unroll
            for (int j = 0; j < MR; ++j) acc[i][j] = mfma_unit<CT>(a[i], b[j], acc[i][j]);
    }
}

// The instruction for 16 columns by 16 rows, as many units as there are lanes.
typedef float floatx4 __attribute__((ext_vector_type(4)));
template <class CT> __device__ __forceinline__ floatx4 mfma_small(Vec<CT, unit_of<CT>()> a, Vec<CT, unit_of<CT>()> b, floatx4 c) {
    if constexpr (sizeof(CT) == 4) {
#pragma unroll
        for (int j = 0; j < 4; ++j) c = __builtin_amdgcn_mfma_f32_16x16x4f32(a[j], b[j], c, 0, 0, 0);
        return c;
    } else if constexpr (std::is_same<CT, bf16_t>::value) return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0);
    else return __builtin_amdgcn_mfma_f32_16x16x32_f16(a, b, c, 0, 0, 0);
}

// A quotient by a number that is known before the launch: of q < 2^29.
struct Quotient {
    uint32_t by = 1, m = 1;
    int shift = 0;
    __host__ Quotient(int32_t d = 1) : by((uint32_t)d) {
        int l = 0;
        while (l < 31 && (1u << l) < by) ++l;
        shift = 29 + l;
        m = (uint32_t)((((uint64_t)1 << shift) + by - 1) / by);
    }
    __device__ __forceinline__ int operator()(int q) const { return by == 1 ? q : (int)((uint64_t)(uint32_t)q * m >> shift); }
};

// Four neighbouring numbers of a result, of which `left` exist.
template <class T> __device__ __forceinline__ void put_some(T *p, Vec<float, 4> v, int left) {
    if (left >= 4) *reinterpret_cast<Loose<T, 4> *>(p) = as_type<T, float, 4>(v);
    else
#pragma unroll
        for (int i = 0; i < 4; ++i)
            if (i < left) p[i] = (T)v[i];
}
__device__ __forceinline__ void put_typed(void *to, int32_t type, int64_t at, Vec<float, 4> v, int left) {
    if (type == PS_F32) put_some(reinterpret_cast<float *>(to) + at, v, left);
    else if (type == PS_BF16) put_some(reinterpret_cast<bf16_t *>(to) + at, v, left);
    else put_some(reinterpret_cast<f16_t *>(to) + at, v, left);
}

// A tile's form: WC x WR wavefronts of 32 MC columns by 32 MR rows each.
template <int MC_, int MR_, int WC_, int WR_> struct Form {
    static constexpr int MC = MC_, MR = MR_, WC = WC_, WR = WR_, COLS = 32 * MC * WC, ROWS = 32 * MR * WR, THREADS = 64 * WC * WR;
};
typedef Form<1, 1, 2, 2> Tile64;
typedef Form<2, 2, 2, 2> Tile128;
typedef Form<1, 1, 1, 4> Narrow;                                     // 32 columns, 128 rows
typedef Form<1, 1, 4, 1> Low;                                        // 128 columns, 32 rows
