// Products of grouped rows: what their kernels are given, for the calls made of them.  Products in tiles: expert.hip; by way of laid matrices: laid.hip; with adapters:
// adapter.hip; sums over a group's rows: outer.hip.
#pragma once
#include "groups.h"
#include "products.h"

// out_q = scale * M x_q per row q of a group, M the group's matrix in the server, or its transpose; zero for rows of no group
struct ExpertArgs {
    RowGroups g;
    const void *x; int64_t x_stride; int32_t x_type; Quotient x_shared;       // row q is row q / x_shared of x; order == NULL there: place p
    const float *w; int64_t L, each;                                         // matrix e's rows are the L numbers from w + (e * each + r) * L on
    int32_t K, N, turned;                                                    // turned: M is the transpose: the sum goes over the K rows
    float scale;
    void *out; int64_t out_stride; int32_t out_type, by_place;               // by_place: the row at place p goes to row p of out
    int32_t precise;                                                         // products of numbers of 32 bits
    int32_t *group_of;                                                       // not NULL: the group of the row at place p
    void *also; int64_t also_stride; int32_t also_type;                      // not NULL: the result once more, in another type
    int32_t zero_from;                                                       // the columns from here on, up to N, have no key: they are written as zeros; 0: none
    __host__ __device__ int32_t columns() const { return zero_from ? zero_from : N; }      // that may be read; one at least in every workgroup's columns
};
// count: one, or two of the same groups, columns and types in one launch
int dpaps_expert_product(dpaps_ps *ps, const ExpertArgs *a, int count, hipStream_t st);

// out_e[i][j] = sum over group e's rows of left[i] right[j]
struct OuterArgs {
    RowGroups g;
    const void *left; int64_t left_stride; int32_t left_type, left_by_place; Quotient left_shared;
    const void *right; int64_t right_stride; int32_t right_type; Quotient right_shared;
    int32_t rows, cols;
    void *out; int32_t out_type;
};
// count: one, or two of the same groups and types in the same launches.  part: scratch of dpaps_outer_bytes(...) bytes
size_t dpaps_outer_bytes(const dpaps_ps *ps, const OuterArgs *a, int count);
int dpaps_outer_sums(dpaps_ps *ps, const OuterArgs *a, int count, float *part, hipStream_t st);
int dpaps_too_large(dpaps_ps *ps, const char *what);

// The row number that stands at a place; -1, and the handle's error, where there is no such row.
__device__ __forceinline__ int row_at(const RowGroups &g, int place, int32_t *err) {
    const int q = g.order[place];
    if (q >= 0 && q < g.n) return q;
    atomicExch(err, PS_EKEY);
    return -1;
}

// out_p = M x_p + sum_r low[place of p][r] B_e[r], with a matrix M for all rows (or its transpose), low: fp32, of rows of a group, scaled already
struct AdapterArgs {
    RowGroups g;
    const void *x; int64_t x_stride; int32_t x_type;
    const float *w; int64_t L;
    int32_t K, N, turned;
    const float *low; int64_t low_stride; int32_t rank;
    const int32_t *group_of;                                                 // the group of the row at place p
    const float *b;                                                          // group e's rank rows from b + e * rank * L on
    void *out; int64_t out_stride; int32_t out_type;
};

// Products by way of laid matrices (laid.hip): the server's numbers rounded to 16 bits once, before the product, and put into the order of its loads.
// out_q = M x_q, M the group's matrix (laid: matrix e from e * w_size on; zero for rows of no group), or, with `low`, M x_q + B_e' low_p of one matrix M for all rows,
// low_p: the low-rank numbers of the row at place p, `rank` of them and zeros up to a multiple of eight, B_e: the laid matrix of its group.
struct LaidArgs {
    RowGroups g;
    const void *x; int64_t x_stride; Quotient x_shared;
    int32_t K, N;
    const void *w; int64_t w_size;                                           // elements of a laid matrix
    const void *low, *b; int64_t b_size; int32_t rank, low_stride;           // low: NULL, a matrix for each group
    void *out; int64_t out_stride; int32_t out_type;
};
// What is laid: M_e's number of column c and place k of the sum is value c of key k (turned) or value k of key c, of keys from w + e * each * L on.
struct LayArgs {
    const float *w; int64_t L, each;
    int32_t K, N, turned;
    void *to; int64_t size;
};
int64_t dpaps_laid_size(int32_t K, int32_t N);                               // elements of a laid matrix: N as a multiple of 256, K of 32
constexpr int64_t LAID_MOST = (int64_t)1 << 29;                              // elements that a call lays, at most: a GiB; beyond that its products go by tiles
bool dpaps_laid_fits(const void *x, int64_t x_stride, int32_t K);
// `each`: of the matrices of all groups that have rows (each.each: how many keys one has), and, if `one` is there, of a single one, in the same launch
int dpaps_lay(dpaps_ps *ps, const RowGroups &g, int32_t type, const LayArgs &each, const LayArgs *one, hipStream_t st);
int dpaps_laid_product(dpaps_ps *ps, int32_t type, const LaidArgs &a, hipStream_t st);

// Few rows: MT tiles of 16 rows by the columns of a workgroup, whose wavefronts share the sum over k.  Both operands come straight from memory into the registers
// that the matrix instruction reads, and nothing but the wavefronts' sums sees LDS: what counts is that all of the matrix is on its way at once.
//   M as it is:  16 columns; lane l has column l % 16, and of a step's 4 units the one l / 16
//   turned:      64 columns; lane l has the four columns from 4 (l % 16) on, for the numbers of unit l / 16: operand j is column 4 i + j of lane i
// Of M as it is four wavefronts share the sum (the low-rank numbers of 16,384 rows of 16 adapters, K 512: 16.6 us, by eight 22.5; 128 rows of 16 experts x 256: 7.8 and 7.9), of turned
// ones, of which there are a quarter as many workgroups, eight (333 rows of 5 experts, 400 x 100, 32 bits: 7.5 us, by four 8.6).
// out[row][column] of wavefront w in sums, [w][16 MT][columns].
template <class CT, class XT, bool TURNED, int MT> struct FewRows {
    static constexpr int KU = unit_of<XT>(), COLS = TURNED ? 64 : 16, OPS = TURNED ? 4 : 1, WAVES = TURNED ? 8 : 4, THREADS = 64 * WAVES, STEP = 4 * KU;
    static constexpr int AHEAD = TURNED ? (KU == 8 ? 2 : 4) : (KU == 8 ? 4 : 8);
    static constexpr int SUMS = WAVES * 16 * MT * COLS;
    floatx4 acc[OPS][MT];
    // The unit that a lane has of 16-bit products with M as it is: four numbers from k on and the four 16 further, on both sides, so that the lanes of a column
    // read neighbours.
    template <class ST> __device__ static __forceinline__ Vec<ST, 8> halves(const ST *p, int k, int K) {
        Vec<ST, 4> lo = {}, hi = {};
        if (k < K) lo = load_some<ST, 4>(p + k, K - k);
        if (k + 16 < K) hi = load_some<ST, 4>(p + k + 16, K - k - 16);
        return __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7);
    }
    // w: where the matrix starts; c0: its first column here; N: the columns that it has; x_of(r): where row r < 16 MT of the tile is (any row where there is none)
    template <class F> __device__ __forceinline__ void run(const float *w, int64_t L, int K, int c0, int N, F x_of) {
        const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, l16 = lane & 15, g = lane >> 4;
        const int steps = (K + STEP - 1) / STEP, s0 = steps * wave / WAVES, s1 = steps * (wave + 1) / WAVES;
        const float *mine = TURNED ? w + c0 + 4 * l16 : w + (int64_t)(c0 + l16 < N ? c0 + l16 : N - 1) * L;
        const int cols = N - c0 - 4 * l16;
#pragma unroll
        for (int j = 0; j < OPS; ++j)
#pragma unroll
            for (int m = 0; m < MT; ++m) acc[j][m] = floatx4{0.0f, 0.0f, 0.0f, 0.0f};
        const XT *x[MT];
#pragma unroll
        for (int m = 0; m < MT; ++m) x[m] = x_of(16 * m + l16);
        for (int s = s0; s < s1; s += AHEAD) {
            Vec<float, KU> wv[AHEAD][OPS];
            Vec<XT, KU> xv[AHEAD][MT];
#pragma unroll
            for (int u = 0; u < AHEAD; ++u) {
                const int k = (s + u) * STEP + g * KU, left = s + u < s1 ? K - k : 0;
                if constexpr (TURNED) {
                    Vec<float, 4> rows[KU];
#pragma unroll
                    for (int i = 0; i < KU; ++i) {
                        rows[i] = Vec<float, 4>{};
                        if (i < left && cols > 0) rows[i] = load_some<float, 4>(mine + (int64_t)(k + i) * L, cols);
                    }
#pragma unroll
                    for (int j = 0; j < 4; ++j)
#pragma unroll
                        for (int i = 0; i < KU; ++i) wv[u][j][i] = rows[i][j];
                } else if constexpr (sizeof(CT) == 4) {
                    wv[u][0] = Vec<float, KU>{};
                    if (left > 0) wv[u][0] = load_some<float, KU>(mine + k, left);
                } else wv[u][0] = halves<float>(mine, (s + u) * STEP + 4 * g, s + u < s1 ? K : 0);
#pragma unroll
                for (int m = 0; m < MT; ++m) {
                    if constexpr (TURNED || sizeof(CT) == 4) {
                        xv[u][m] = Vec<XT, KU>{};
                        if (left > 0) xv[u][m] = load_some<XT, KU>(x[m] + k, left);
                    } else xv[u][m] = halves<XT>(x[m], (s + u) * STEP + 4 * g, s + u < s1 ? K : 0);
                }
            }
#pragma unroll
            for (int u = 0; u < AHEAD; ++u)
#pragma unroll
                for (int j = 0; j < OPS; ++j)
#pragma unroll
                    for (int m = 0; m < MT; ++m) acc[j][m] = mfma_small<CT, KU>(as_type<CT, float, KU>(wv[u][j]), as_type<CT, XT, KU>(xv[u][m]), acc[j][m]);
        }
    }
    __device__ __forceinline__ void put(float *sums) const {
        const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, l16 = lane & 15, g = lane >> 4;
#pragma unroll
        for (int m = 0; m < MT; ++m) {
            float *to = sums + ((wave * MT + m) * 16 + l16) * COLS + (TURNED ? 16 : 4) * g;
            if constexpr (TURNED) {
#pragma unroll
                for (int i = 0; i < 4; ++i) *reinterpret_cast<Vec<float, 4> *>(to + 4 * i) = Vec<float, 4>{acc[0][m][i], acc[1][m][i], acc[2][m][i], acc[3][m][i]};
            } else *reinterpret_cast<Vec<float, 4> *>(to) = acc[0][m];
        }
    }
    // the sum of all wavefronts, of four neighbouring columns: piece p of 16 MT COLS / 4, its row and its first column
    static constexpr int PIECES = 16 * MT * COLS / 4;
    __device__ static __forceinline__ int row_of(int p) { return p / (COLS / 4); }
    __device__ static __forceinline__ int col_of(int p) { return p % (COLS / 4) * 4; }
    __device__ static __forceinline__ Vec<float, 4> sum(const float *sums, int p) {
        Vec<float, 4> v = *reinterpret_cast<const Vec<float, 4> *>(sums + p * 4);
#pragma unroll
        for (int w = 1; w < WAVES; ++w) v = v + *reinterpret_cast<const Vec<float, 4> *>(sums + w * 16 * MT * COLS + p * 4);
        return v;
    }
};
