// Matrices orthogonalised by Newton-Schulz products, and the step of weight matrices in the server that uses it.
//
// X_0 = D / (|D|_F + eps), then a number of times
//   A = X X',   P = a I + b A + c A^2,   X <- P X          (a, b, c below; X: n x m with n <= m, transposed if need be)
// which brings every singular value s to p(p(...p(s))), p(s) = a s + b s^3 + c s^5: near 1 after five steps, unless it
// was very small.
//
// All products are of fp16 numbers on the matrix cores with sums in 32 bits.  Numbers are held
//   as pairs   the sum of two fp16 numbers, high + low: 11 bits each and a sign between them, an error of 2^-23 of the number at most;
//              a product is high high + high low + low high (what is left out is 2^-22 of it at most, 2^-24 as a rule): three instructions;
//   single     as one fp16 number: an error of 2^-11 at most, an eighth of what rounding to bf16 costs.
// Pairs throughout for results of 32 bits and of fp16, where one launch does it all, and where A is at most 64 x 64: the error of one of a few numbers of P
// is that of all columns of X, so single ones cost up to twice or, of 4 x 376, three times the rounding of a bf16 result (of 65 to 128 rows 1.2 times).
// Of other bf16 results all numbers are single, except X where all but the last two steps multiply it by P: there an error of X goes into all directions
// alike, and every step that is left raises the weak ones by 3.4 (an error of A or P moves strong directions a little, and is not raised).  Five steps of
// matrices with one to 32 singular values 10^2 to 10^6 times all others, the roundings simulated in 64 bits: the result is off by up to 0.0039 of its norm
// (its own rounding: 0.0017), with X single in the last three steps by 0.014, with X as pairs in all by 0.0037; ten steps 0.008, with X as pairs in the
// first two alone 4.5.  (Products of bf16 numbers: 0.3 to 1.)  Errors of the sums, in 32 bits, are raised as well: 2^-21 3.4445^steps of the norm at most.
// It costs two instructions instead of one in three of fifteen products: two of 4096 x 4096 3.88 ms, with X as pairs in two steps 3.65; pairs throughout,
// as for a result of 32 bits, 9.33 ms.
// fp16 holds few magnitudes, so every number is scaled by a power of two: the spectral norms of X, A and P are at most 1.21,
// 1.46 and 3.45 whatever D is (p of [0, 1.21] stays below 1.21), and so is every element; scaled they fill the
// upper end of the type, and what is lost at the lower end is 2^-39 or less of each element - of X_0's norm, where |D| is not far below eps; where it is, X_0 is
// as small as |D| / eps, and its elements have so many digits less: of 600 x 600, |D| a millionth of eps, 2^-39 is 0.0007 of the norm.
// All three products have the form sum_k L[i][k] R[j][k] with both operands' rows contiguous in k: A = X X' and
// A^2 = A A' (A is symmetric) as they are, P X with X transposed - so X is written both ways.  Of the symmetric ones only the tiles on and below
// the diagonal are computed; a tile is written to its mirror place as well.
#include "elements.h"
#include "token_ids.h"

#include <cmath>
#include <type_traits>

namespace {

constexpr float NS_A = 3.4445f, NS_B = -4.7750f, NS_C = 2.0315f;
constexpr float X_SCALE = 16384.0f, G_SCALE = 16384.0f, P_SCALE = 8192.0f;

typedef f16_t half8 __attribute__((ext_vector_type(8)));
typedef f16_t half4 __attribute__((ext_vector_type(4)));
typedef float floatx4 __attribute__((ext_vector_type(4)));
typedef float floatx16 __attribute__((ext_vector_type(16)));

inline size_t up256(size_t x) { return (x + 255) / 256 * 256; }

// Two numbers as high and low parts, each rounded to the nearest: two conversions, and two fused subtractions, which are exact
typedef f16_t half2 __attribute__((ext_vector_type(2)));
typedef float floatx2 __attribute__((ext_vector_type(2)));
struct Parts { half2 hi, lo; };
template <bool PAIR> __device__ __forceinline__ Parts parts_of(float a, float b) {
    Parts p;
    p.hi = __builtin_convertvector(floatx2{a, b}, half2);
    if constexpr (PAIR) p.lo = __builtin_convertvector(floatx2{__builtin_fmaf((float)p.hi[0], -1.0f, a), __builtin_fmaf((float)p.hi[1], -1.0f, b)}, half2);
    return p;
}

// A matrix in scratch lies as the matrix instruction takes it: 32 rows and 16 numbers of each are a block, in which lane l of a wavefront
// finds its eight numbers, of row l % 32 from number 8 (l / 32) on, at 16 l bytes (pairs: the 64 lanes' high parts, then their
// low parts); the blocks of the same rows follow one another.  So operands come into registers in whole lines, and never see LDS.
// The eight numbers of row r from k on (k a multiple of 8), K numbers a row:
template <bool PAIR> __device__ __forceinline__ int64_t place8(int r, int k, int K) {
    return ((int64_t)(r >> 5) * (K >> 4) + (k >> 4)) * (PAIR ? 1024 : 512) + ((k & 8) * 4 + (r & 31)) * 8;
}

// ---- the norm, and the momentum -------------------------------------------------------------------------------------
constexpr int NORM_BLOCKS = 256;             // workgroups per matrix at most

struct MuonIn {
    const void *in; int64_t ld; int32_t type;    // batch * rows rows
    int32_t rows, cols;
    // of a step: where the momentum is in the store (else NULL)
    float *val; int64_t L; int64_t first; float mu; int32_t nesterov;
    float *d;                                    // of a step: the matrices to be orthogonalised, batch * rows x cols
    double *squares;                             // batch x NORM_BLOCKS: sums of squares
    int32_t blocks;
    float eps;
};
// The sum of a workgroup's 256 numbers, in a fixed order; the same in all threads.
__device__ __forceinline__ double sum_of_256(double x) {
    __shared__ double lds[4];
    for (int d = 32; d > 0; d >>= 1) x += __shfl_xor(x, d);
    if ((threadIdx.x & 63) == 0) lds[threadIdx.x >> 6] = x;
    __syncthreads();
    return (lds[0] + lds[1]) + (lds[2] + lds[3]);
}

// Of matrix blockIdx.y: sums of squares in 64 bits (no number of 32 bits overflows there); of a step, first M <- mu M + G, and
// what is orthogonalised, D = G + mu M (Nesterov) or M.  V numbers of a row at a time, P = cols / V such pieces a row; a thread
// goes through every (256 blocks)th piece of the matrix, AHEAD of them together.
// Memory bounds a step: eight matrices of 2048 x 512, a bf16 gradient, 118 MB read and written in 24 us, 4.9 TB/s.  Two of 4096 x 4096 in bf16 are 67 MB in
// 29 us, 2.3 TB/s, half of a copy's rate: what a thread has on its way, four pieces of 8 bytes, and at most 256 workgroups a matrix bound that.
template <class T, int V, bool STEP>
__global__ __launch_bounds__(256) void k_muon_norm(MuonIn a, uint32_t P, double inv_P, const int32_t *err) {
    constexpr int AHEAD = STEP ? 2 : 4;
    if (STEP && *(volatile const int32_t *)err) return;
    const int64_t row0 = (int64_t)blockIdx.y * a.rows, pieces = (int64_t)a.rows * P, step = (int64_t)a.blocks * 256;
    const T *in = reinterpret_cast<const T *>(a.in);
    double s = 0.0;
    for (int64_t at = (int64_t)blockIdx.x * 256 + threadIdx.x; at < pieces; at += step * AHEAD) {
        Vec<float, V> x[AHEAD], m[AHEAD];
        int64_t row[AHEAD];
        int c[AHEAD];
#pragma unroll
        for (int u = 0; u < AHEAD; ++u) {
            const int64_t q = at + u * step < pieces ? at + u * step : 0, r = quotient(q, P, inv_P);
            row[u] = row0 + r;
            c[u] = (int)(q - r * P) * V;
            x[u] = load_vec<T, V>(in + row[u] * a.ld + c[u]);
            if constexpr (STEP) m[u] = load_vec<float, V>(a.val + (a.first + row[u]) * a.L + a.cols + c[u]);
        }
#pragma unroll
        for (int u = 0; u < AHEAD; ++u) {
            if (at + u * step >= pieces) break;
            if constexpr (STEP) {
                const Vec<float, V> moment = a.mu * m[u] + x[u];
                store_vec<float, V>(a.val + (a.first + row[u]) * a.L + a.cols + c[u], moment);
                x[u] = a.nesterov ? x[u] + a.mu * moment : moment;
                store_vec<float, V>(a.d + row[u] * a.cols + c[u], x[u]);
            }
            if constexpr (V == 1) s += (double)x[u] * (double)x[u];
            else
#pragma unroll
                for (int e = 0; e < V; ++e) s += (double)x[u][e] * (double)x[u][e];
        }
    }
    s = sum_of_256(s);
    if (threadIdx.x == 0) a.squares[(int64_t)blockIdx.y * NORM_BLOCKS + blockIdx.x] = s;
}

// A matrix's numbers become X_0, scaled.  In 64 bits where the sum of squares is far from 1, so that neither a norm above the largest 32-bit number nor
// one near the smallest loses anything (everywhere, 3 of the 49 us of 16 matrices of 100 x 100).  An infinity or NaN anywhere in the matrix makes all of X
// NaN, as the division and the products would; a matrix of zeros stays one, also where eps is 0.
struct Scale {
    bool usual;
    float f;
    double wide;
    __device__ __forceinline__ Scale(double square, float eps) : usual(square >= 1e-30 && square <= 1e30), f(0.0f), wide(0.0) {
        if (usual) f = X_SCALE / (sqrtf((float)square) + eps);
        else if (square != 0.0) wide = square <= 1.7e308 ? (double)X_SCALE / (sqrt(square) + (double)eps) : __builtin_nan("");
    }
    template <int N> __device__ __forceinline__ void apply(float (&v)[N]) const {
        if (usual) {
#pragma unroll
            for (int i = 0; i < N; ++i) v[i] *= f;
        } else {
#pragma unroll
            for (int i = 0; i < N; ++i) v[i] = (float)((double)v[i] * wide);
        }
    }
};

// X_0 both ways, zero where the padded matrices go on.
template <bool PAIR>
__device__ __forceinline__ void put8(f16_t *to, int r, int k, int K, const float (&v)[8]) {
    half8 hi, lo;
#pragma unroll
    for (int i = 0; i < 8; i += 2) {
        const Parts p = parts_of<PAIR>(v[i], v[i + 1]);
        hi[i] = p.hi[0]; hi[i + 1] = p.hi[1];
        if constexpr (PAIR) { lo[i] = p.lo[0]; lo[i + 1] = p.lo[1]; }
    }
    f16_t *p = to + place8<PAIR>(r, k, K);
    *reinterpret_cast<half8 *>(p) = hi;
    if constexpr (PAIR) *reinterpret_cast<half8 *>(p + 512) = lo;
}
// PAIR: X as pairs, as X transposed always is.  A workgroup turns 64 x 64 in LDS.  Memory bounds it: two of 4096 x 4096 in bf16, 268 MB read and written,
// 62 us, 4.3 TB/s; eight of 2048 x 512, 101 MB, 16 us (some of it in the die's caches).
template <class T, bool PAIR>
__global__ __launch_bounds__(256) void k_muon_scale(MuonIn a, bool tall, int np, int mp, f16_t *x, f16_t *xt) {
    __shared__ float tile[64][65];
    const int64_t b = blockIdx.z;
    const int i0 = blockIdx.y * 64, j0 = blockIdx.x * 64;                     // of X
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int r0 = tall ? j0 : i0, c0 = (tall ? i0 : j0) + lane;              // of the matrix itself
    float v[16];
#pragma unroll
    for (int u = 0; u < 16; ++u) {
        const int r = r0 + wave + 4 * u;
        v[u] = r < a.rows && c0 < a.cols ? (float)reinterpret_cast<const T *>(a.in)[(b * a.rows + r) * a.ld + c0] : 0.0f;
    }
    const double square = sum_of_256((int)threadIdx.x < a.blocks ? a.squares[b * NORM_BLOCKS + threadIdx.x] : 0.0);
    Scale(square, a.eps).apply(v);
#pragma unroll
    for (int u = 0; u < 16; ++u) {
        if (tall) tile[lane][wave + 4 * u] = v[u]; else tile[wave + 4 * u][lane] = v[u];
    }
    __syncthreads();
    x += b * (int64_t)np * mp * (PAIR ? 2 : 1);
    xt += b * (int64_t)np * mp * 2;
#pragma unroll
    for (int u = 0; u < 2; ++u) {
        const int r = u * 32 + (lane & 31), k = wave * 16 + (lane >> 5) * 8;
        float y[8], w[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) { y[i] = tile[r][k + i]; w[i] = tile[k + i][r]; }
        put8<PAIR>(x, i0 + r, j0 + k, mp, y);
        put8<true>(xt, j0 + r, i0 + k, np, w);
    }
}

// ---- the products ---------------------------------------------------------------------------------------------------
constexpr int GJ = 4;                            // columns of a band
constexpr uint32_t DIES = 8;                     // compute dies, each with a cache of its own
constexpr int CHAIN = 12;                        // blocks of k whose products one chain of matrix instructions adds (a multiple of DEPTH and KB)
// The numbers of the left and the right operand: single ones, or pairs in the right one, or in both.
enum MuonKind { SINGLE, RIGHT_SPLIT, SPLIT };
constexpr int left_parts(int kind) { return kind == SPLIT ? 2 : 1; }
constexpr int right_parts(int kind) { return kind == SINGLE ? 1 : 2; }
constexpr int products_of(int kind) { return left_parts(kind) + right_parts(kind) - 1; }
enum MuonProduct { MUON_GRAM, MUON_POLY, MUON_APPLY, MUON_LAST, MUON_STEP };       // LAST, STEP: APPLY with the result put where it belongs
struct MuonArgs {
    const f16_t *lhs, *rhs;                      // rows of K numbers
    int64_t lhs_size, rhs_size, out_size, out_t_size;   // of one matrix, in elements as they are stored
    int32_t K, tiles_i, tiles_j, tiles, tile0;   // tiles: of one matrix; tile0: the first one of the launch
    int32_t shares; float *part;                 // workgroups that share a tile's sum over k, and where they put their sums
    f16_t *out; int32_t out_ld;                  // GRAM: A, POLY: P, APPLY: X
    f16_t *out_t; int32_t out_t_ld, out_t_pair;  // APPLY: X transposed; out_t_pair: as pairs, for RIGHT_SPLIT
    // LAST: the result
    void *to; int64_t to_ld; int32_t to_type, to_vec, tall, n, m;   // to_vec: eight numbers of a row can be written together
    float *val; int64_t L, first; float keep, step;    // of a step: W <- keep W - step X
};

template <bool PAIR> __device__ __forceinline__ void get8(const f16_t *m, int r, int k, int K, float (&v)[8]) {
    const f16_t *p = m + place8<PAIR>(r, k, K);
    const half8 hi = *reinterpret_cast<const half8 *>(p);
    half8 lo = {};
    if constexpr (PAIR) lo = *reinterpret_cast<const half8 *>(p + 512);
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] = PAIR ? (float)hi[e] + (float)lo[e] : (float)hi[e];
}
// Eight neighbouring numbers of a row of the result, of which `left` are its: what is there already (of a step), and what is written.
__device__ __forceinline__ void get_weights(const MuonArgs &a, int64_t row, int col, float (&w)[8], int left) {
    const float *p = a.val + (a.first + row) * a.L + col;
    if (a.to_vec && left >= 8) {
        const Vec<float, 8> x = load_vec<float, 8>(p);
#pragma unroll
        for (int e = 0; e < 8; ++e) w[e] = x[e];
    } else {
#pragma unroll
        for (int e = 0; e < 8; ++e) w[e] = e < left ? p[e] : 0.0f;
    }
}
template <class T> __device__ __forceinline__ void put_numbers(T *p, const float (&v)[8], int left, bool vec) {
    if (vec && left >= 8) {
        Vec<float, 8> x;
#pragma unroll
        for (int e = 0; e < 8; ++e) x[e] = v[e];
        store_vec<T, 8>(p, x);
    } else {
#pragma unroll
        for (int e = 0; e < 8; ++e)
            if (e < left) p[e] = (T)v[e];
    }
}
__device__ __forceinline__ void put_result(const MuonArgs &a, int64_t row, int col, const float (&v)[8], int left) {
    if (a.to_type == PS_F32) put_numbers(reinterpret_cast<float *>(a.to) + row * a.to_ld + col, v, left, a.to_vec);
    else if (a.to_type == PS_BF16) put_numbers(reinterpret_cast<bf16_t *>(a.to) + row * a.to_ld + col, v, left, a.to_vec);
    else put_numbers(reinterpret_cast<f16_t *>(a.to) + row * a.to_ld + col, v, left, a.to_vec);
}
// Which tile a workgroup has, and which share of the sum over k.  Workgroups go to the compute dies in turn: each die gets
// neighbouring tiles, in bands of four rows or columns, whose operands its cache then holds (32 tiles at a time: 4 and 8 blocks of rows).
struct Place { int64_t b; int ti, tj, share, slot; };
template <int MODE>
__device__ __forceinline__ Place place_of(const MuonArgs &a, uint32_t block, uint32_t all) {
    const uint32_t die = block % DIES, at = die * (all / DIES) + (die < all % DIES ? die : all % DIES) + block / DIES;
    Place p;
    p.share = (int)(at % (uint32_t)a.shares);
    p.slot = (int)(at / (uint32_t)a.shares);
    p.b = (a.tile0 + p.slot) / a.tiles;
    const int tile = (a.tile0 + p.slot) % a.tiles;
    if constexpr (MODE == MUON_GRAM || MODE == MUON_POLY) {
        // on and below the diagonal: bands of four rows; in a band the columns before the diagonal one by one, then its triangle
        const auto row_of = [](int t) {
            int i = (int)((sqrtf(8.0f * (float)t + 1.0f) - 1.0f) * 0.5f);
            while ((i + 1) * (i + 2) / 2 <= t) ++i;
            while (i * (i + 1) / 2 > t) --i;
            return i;
        };
        const int first = row_of(tile) & ~3, r = tile - first * (first + 1) / 2, rows = a.tiles_i - first < 4 ? a.tiles_i - first : 4;
        if (r < first * rows) {
            p.ti = first + r % rows;
            p.tj = r / rows;
        } else {
            const int t = r - first * rows, i = row_of(t);
            p.ti = first + i;
            p.tj = first + t - i * (i + 1) / 2;
        }
    } else {
        const int first = tile / (GJ * a.tiles_i) * GJ, r = tile - first * a.tiles_i, columns = a.tiles_j - first < GJ ? a.tiles_j - first : GJ;
        p.ti = r / columns;
        p.tj = first + r % columns;
    }
    return p;
}

// The sums leave by way of LDS, 64 x 64 at a time, so that rows of the result and rows of its mirror image are both written in whole
// lines.  SUMS_LD: a row of 64 sums there: 32 rows' pieces of 16 bytes lie in all banks.
constexpr int SUMS_LD = 68;
// From LDS, where KS wavefronts have put their shares of the sums, to where they belong: rows gi .., columns gj .. of matrix p.b.  group: of the KS wavefronts.
template <int KS, int KIND, int MODE>
__device__ __forceinline__ void write_tile(const MuonArgs &a, const Place &p, int gi, int gj, const float *sums, int group) {
    constexpr float FACTOR = MODE == MUON_GRAM ? G_SCALE / (X_SCALE * X_SCALE) : MODE == MUON_APPLY ? 1.0f / P_SCALE : MODE >= MUON_LAST ? 1.0f / (P_SCALE * X_SCALE) : 1.0f;
    const int lane = threadIdx.x & 63, l32 = lane & 31, h = lane >> 5;
    const bool turned = MODE >= MUON_LAST && a.tall;
                const auto sum = [&](int w) {
                    float v = sums[w];
#pragma unroll
                    for (int k = 1; k < KS; ++k) v += sums[k * (64 * SUMS_LD) + w];
                    return v * FACTOR;
                };
                if constexpr (MODE >= MUON_LAST) {
                    // eight rows at a time, eight lanes a row; of a step the weights of all of them first
                    const int R0 = (turned ? gj : gi) + group * 8 + (lane >> 3), c = (lane & 7) * 8, C = (turned ? gi : gj) + c;
                    const int height = turned ? a.m : a.n, left = (turned ? a.n : a.m) - C;
                    const auto at = [&](int q) { return (q * KS * 8 + group * 8 + (lane >> 3)) * SUMS_LD + c; };
                    if constexpr (MODE == MUON_STEP) {
                        float w[8 / KS][8];
#pragma unroll
                        for (int q = 0; q < 8 / KS; ++q)
                            if (R0 + q * KS * 8 < height) get_weights(a, p.b * height + R0 + q * KS * 8, C, w[q], left);
#pragma unroll
                        for (int q = 0; q < 8 / KS; ++q) {
                            float v[8];
#pragma unroll
                            for (int e = 0; e < 8; ++e) v[e] = a.keep * w[q][e] - a.step * sum(at(q) + e);
                            if (R0 + q * KS * 8 < height) put_numbers(a.val + (a.first + p.b * height + R0 + q * KS * 8) * a.L + C, v, left, a.to_vec);
                        }
                    } else {
#pragma unroll 1
                        for (int q = 0; q < 8 / KS; ++q) {
                            float v[8];
#pragma unroll
                            for (int e = 0; e < 8; ++e) v[e] = sum(at(q) + e);
                            if (R0 + q * KS * 8 < height) put_result(a, p.b * height + R0 + q * KS * 8, C, v, left);
                        }
                    }
                } else {
                    const bool columns = MODE == MUON_APPLY || p.ti != p.tj;
                    for (int way = 0; way < (columns ? 2 : 1); ++way) {
#pragma unroll 2
                        for (int q = group; q < 8; q += KS) {
                            const int r = (q & 1) * 32 + l32, c = (q >> 1) * 16 + h * 8;   // row r of what is written, numbers c .. c + 7
                            float v[8];
#pragma unroll
                            for (int e = 0; e < 8; ++e) v[e] = sum(way ? (c + e) * SUMS_LD + r : r * SUMS_LD + c + e);
                            const int R = (way ? gj : gi) + r, C = (way ? gi : gj) + c;
                            if constexpr (MODE == MUON_POLY) {                    // (A is symmetric: it is read as the result is written)
                                float g[8];
                                get8<KIND == SPLIT>(a.lhs + p.b * a.lhs_size, R, C, a.K, g);
#pragma unroll
                                for (int e = 0; e < 8; ++e)
                                    v[e] = v[e] * (NS_C * P_SCALE / (G_SCALE * G_SCALE)) + g[e] * (NS_B * P_SCALE / G_SCALE) + (R == C + e ? NS_A * P_SCALE : 0.0f);
                            }
                            f16_t *const to = MODE == MUON_APPLY && way ? a.out_t + p.b * a.out_t_size : a.out + p.b * a.out_size;
                            const int ld = MODE == MUON_APPLY && way ? a.out_t_ld : a.out_ld;
                            if (KIND == RIGHT_SPLIT && way && a.out_t_pair) put8<true>(to, R, C, ld, v);
                            else put8<KIND == SPLIT>(to, R, C, ld, v);
                        }
                    }
                }
}
// The numbers of the matrix instruction: x has 32 x 32 pieces, of which a lane has column lane % 32, rows 8 g + 4 (lane / 32) + 0..3 for
// g = 0..3; from row i0, column j0 on.  mine: where this wavefront puts them, sums: the first one's place.
template <int FI, int FJ, int KS, int KIND, int MODE>
__device__ __forceinline__ void put_tile(const MuonArgs &a, const Place &p, const floatx16 (&x)[FI][FJ], int i0, int j0, float *mine, const float *sums, int group) {
    const int lane = threadIdx.x & 63, l32 = lane & 31, h = lane >> 5;
    const bool turned = MODE >= MUON_LAST && a.tall;                           // X is the transposed matrix
#pragma unroll
    for (int si = 0; si < FI / 2; ++si)
#pragma unroll
        for (int sj = 0; sj < FJ / 2; ++sj) {
#pragma unroll
            for (int fi = 0; fi < 2; ++fi)
#pragma unroll
                for (int fj = 0; fj < 2; ++fj) {
                    const floatx16 v = x[2 * si + fi][2 * sj + fj];
                    if (turned) {
#pragma unroll
                        for (int g = 0; g < 4; ++g)
                            *reinterpret_cast<floatx4 *>(&mine[(fj * 32 + l32) * SUMS_LD + fi * 32 + 8 * g + 4 * h]) = floatx4{v[4 * g], v[4 * g + 1], v[4 * g + 2], v[4 * g + 3]};
                    } else {
#pragma unroll
                        for (int e = 0; e < 16; ++e) mine[(fi * 32 + 8 * (e >> 2) + 4 * h + (e & 3)) * SUMS_LD + fj * 32 + l32] = v[e];
                    }
                }
            if constexpr (KS > 1) __syncthreads();
            else asm volatile("" ::: "memory");                                // (a wavefront's accesses to LDS stay in order)
            write_tile<KS, KIND, MODE>(a, p, i0 + si * 64, j0 + sj * 64, sums, group);
            asm volatile("" ::: "memory");
        }
}

// The sums of a wavefront: C[i][j] += sum_k L[i][k] R[j][k], 32 x 32 pieces (v_mfma_f32_32x32x16_f16).
// The matrix instruction does not round its sums to the nearest: a chain of them loses up to a unit in the last place at each link, always the
// same way.  (One row of 5,000 in a chain of 313: an error of 72 units of 2^-24.)  So with pairs the chains are cut, and their sums
// added by ordinary additions.  (The sums of at most 16 blocks of k in k_muon_one and of the polynomial in k_muon_poly_apply are one chain.)
template <int FI, int FJ, int KIND> struct Sums {
    static constexpr int L = left_parts(KIND), R = right_parts(KIND);
    floatx16 acc[FI][FJ], total[KIND == SPLIT ? FI : 1][KIND == SPLIT ? FJ : 1];
    __device__ __forceinline__ void clear() {
#pragma unroll
        for (int i = 0; i < FI; ++i)
#pragma unroll
            for (int j = 0; j < FJ; ++j) {
                acc[i][j] = floatx16{};
                if constexpr (KIND == SPLIT) total[i][j] = floatx16{};
            }
    }
    __device__ __forceinline__ void add(const half8 (&l)[FI][L], const half8 (&r)[FJ][R]) {
#pragma unroll
        for (int e = products_of(KIND) - 1; e >= 0; --e)                      // low high and high low, as there are parts, then high high
#pragma unroll
            for (int i = 0; i < FI; ++i)
#pragma unroll
                for (int j = 0; j < FJ; ++j)
                    acc[i][j] = __builtin_amdgcn_mfma_f32_32x32x16_f16(l[i][e == 2 ? L - 1 : 0], r[j][e == 1 ? R - 1 : 0], acc[i][j], 0, 0, 0);
    }
    __device__ __forceinline__ void cut() {
        if constexpr (KIND == SPLIT) {
#pragma unroll
            for (int i = 0; i < FI; ++i)
#pragma unroll
                for (int j = 0; j < FJ; ++j) { total[i][j] = total[i][j] + acc[i][j]; acc[i][j] = floatx16{}; }
        }
    }
    __device__ __forceinline__ const floatx16 (&all() const)[FI][FJ] {
        if constexpr (KIND == SPLIT) return total;
        else return acc;
    }
};

// Few or small tiles: 64 x 64 per workgroup, and its four wavefronts share the sum over k, a block in turn.  Operands come straight
// from memory, DEPTH blocks ahead; nobody waits for anybody before the end.  Latency bounds it: launch, first operands, a meeting, the way out.  A A' of
// 1024 x 1024 in pairs, 136 tiles, 14 us (3.4 GFLOP of instructions), of 128 x 128 5.7; P X of 128 x 384 5.2.  Eight wavefronts a tile: 3 to 5 % slower.
template <int KIND, int MODE>
__global__ __launch_bounds__(256) __attribute__((amdgpu_waves_per_eu(2))) void k_muon_small(MuonArgs a, const int32_t *err) {
    constexpr int KS = 4, L = left_parts(KIND), R = right_parts(KIND), DEPTH = KIND == SPLIT ? 3 : 4;
    __shared__ __attribute__((aligned(16))) float lds[KS][64 * SUMS_LD];
    const int lane = threadIdx.x & 63, group = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6);
    const Place p = place_of<MODE>(a, blockIdx.x, gridDim.x);
    const int i0 = p.ti * 64, j0 = p.tj * 64, blocks = a.K >> 4, turns = blocks / KS;             // (sides are multiples of 64)
    const int first = turns * p.share / a.shares, cnt = turns * (p.share + 1) / a.shares - first, block0 = first * KS + group;
    const f16_t *l = a.lhs + p.b * a.lhs_size + ((int64_t)(i0 >> 5) * blocks + block0) * (512 * L);
    const f16_t *r = a.rhs + p.b * a.rhs_size + ((int64_t)(j0 >> 5) * blocks + block0) * (512 * R);
    const int64_t rows32 = (int64_t)blocks * 512;                              // elements to the next 32 rows, of a part
    half8 lf[DEPTH][2][L], rf[DEPTH][2][R];
    const auto load = [&](half8 (&x)[2][L], half8 (&y)[2][R], int t) {
#pragma unroll
        for (int f = 0; f < 2; ++f) {
#pragma unroll
            for (int e = 0; e < L; ++e) x[f][e] = *reinterpret_cast<const half8 *>(l + (int64_t)t * (KS * 512 * L) + f * (rows32 * L) + e * 512 + lane * 8);
#pragma unroll
            for (int e = 0; e < R; ++e) y[f][e] = *reinterpret_cast<const half8 *>(r + (int64_t)t * (KS * 512 * R) + f * (rows32 * R) + e * 512 + lane * 8);
        }
    };
    Sums<2, 2, KIND> s;
    s.clear();
#pragma unroll
    for (int d = 0; d < DEPTH; ++d)
        if (d < cnt) load(lf[d], rf[d], d);
    for (int c0 = 0; c0 < cnt; c0 += CHAIN) {
        const int c1 = c0 + CHAIN < cnt ? c0 + CHAIN : cnt;
        for (int t0 = c0; t0 < c1; t0 += DEPTH) {
#pragma unroll
            for (int d = 0; d < DEPTH; ++d) {
                const int t = t0 + d;
                if (t < c1) {
                    s.add(lf[d], rf[d]);
                    if (t + DEPTH < cnt) load(lf[d], rf[d], t + DEPTH);
                }
            }
        }
        s.cut();
    }
    if (MODE == MUON_STEP && *(volatile const int32_t *)err) return;  // (set before this launch: the same for all)
    if (MODE == MUON_GRAM && a.shares > 1) {
        // a share of the sums: 64 x 64, row by row
        float *to = a.part + (int64_t)(p.slot * a.shares + p.share) * 4096;
#pragma unroll
        for (int fi = 0; fi < 2; ++fi)
#pragma unroll
            for (int fj = 0; fj < 2; ++fj)
#pragma unroll
                for (int e = 0; e < 16; ++e) lds[group][(fi * 32 + 8 * (e >> 2) + 4 * (lane >> 5) + (e & 3)) * SUMS_LD + fj * 32 + (lane & 31)] = s.all()[fi][fj][e];
        __syncthreads();
        for (int q = group; q < 16; q += KS) {
            const int at = (q * 4 + (lane >> 4)) * SUMS_LD + (lane & 15) * 4;
            floatx4 v = *reinterpret_cast<const floatx4 *>(&lds[0][at]);
#pragma unroll
            for (int k = 1; k < KS; ++k) v += *reinterpret_cast<const floatx4 *>(&lds[k][at]);
            *reinterpret_cast<floatx4 *>(to + q * 256 + lane * 4) = v;
        }
        return;
    }
    put_tile<2, 2, KS, KIND, MODE>(a, p, s.all(), i0, j0, lds[group], lds[0], group);
}

// The shares of a small tile's sums added: each wavefront every fourth share, and then the four.
template <int KIND>
__global__ __launch_bounds__(256) void k_muon_join_small(MuonArgs a, int32_t shares) {
    constexpr int KS = 4;
    __shared__ __attribute__((aligned(16))) float lds[KS][64 * SUMS_LD];
    const Place p = place_of<MUON_GRAM>(a, blockIdx.x, gridDim.x);             // (a.shares is 1 here)
    const int lane = threadIdx.x & 63, group = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6);
    floatx4 x[16];
#pragma unroll
    for (int q = 0; q < 16; ++q) x[q] = floatx4{};
    for (int k = group; k < shares; k += KS) {
        const float *from = a.part + (int64_t)(p.slot * shares + k) * 4096 + lane * 4;
#pragma unroll
        for (int q = 0; q < 16; ++q) x[q] += *reinterpret_cast<const floatx4 *>(from + q * 256);
    }
#pragma unroll
    for (int q = 0; q < 16; ++q) *reinterpret_cast<floatx4 *>(&lds[group][(q * 4 + (lane >> 4)) * SUMS_LD + (lane & 15) * 4]) = x[q];
    __syncthreads();
    write_tile<KS, KIND, MUON_GRAM>(a, p, p.ti * 64, p.tj * 64, lds[0], group);
}

// Thin matrices, A of 64 N x 64 N: the polynomial and P X in one launch.  A workgroup has 64 x 64 of P X; it works out the 64 rows of P that this takes by itself
// - a wavefront 32 columns of P, or 32 x 32 -, into LDS, and goes on as k_muon_small, with its part of X on the way meanwhile.  Calls in 32 bits, this way and
// with a launch for each: 10 x 300 60 us and 77, 127 x 333 81 and 92, 128 x 1024 96 and 108, 64 x 4096 89 and 106, 16 of 128 x 1024 125 and 135; where
// there is work for all compute units P's rows worked out m / 64 times cost what the launch saves: 128 x 20000 204 and 202, 256 of 64 x 1024 331 and 325.
template <int KIND, int MODE, int N>
__global__ __launch_bounds__(256) __attribute__((amdgpu_waves_per_eu(2))) void k_muon_poly_apply(MuonArgs a, const int32_t *err) {
    constexpr int KS = 4, L = left_parts(KIND), R = right_parts(KIND), BLOCKS = 4 * N;
    __shared__ __attribute__((aligned(16))) float lds[KS][64 * SUMS_LD];      // P's rows first, then the sums
    static_assert(64 * 64 * N * L * 2 <= sizeof(lds));
    f16_t *const rows = reinterpret_cast<f16_t *>(&lds[0][0]);
    const int lane = threadIdx.x & 63, group = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6), l32 = lane & 31, h = lane >> 5;
    const Place p = place_of<MODE>(a, blockIdx.x, gridDim.x);
    const f16_t *const A = a.lhs + p.b * a.lhs_size, *const x = a.rhs + p.b * a.rhs_size;
    half8 rf[N][2][R];
#pragma unroll
    for (int t = 0; t < N; ++t)
#pragma unroll
        for (int f = 0; f < 2; ++f)
#pragma unroll
            for (int e = 0; e < R; ++e) rf[t][f][e] = *reinterpret_cast<const half8 *>(x + ((int64_t)(p.tj * 2 + f) * BLOCKS + group + KS * t) * (512 * R) + e * 512 + lane * 8);
    // columns 32 c .. of P, rows 32 (r + i) .. of the workgroup's: the matrix instruction gives them with rows and columns exchanged
    const int c = N == 2 ? group : group & 1, r = N == 2 ? 0 : group >> 1;
    floatx16 sum[N];
#pragma unroll
    for (int i = 0; i < N; ++i) sum[i] = floatx16{};
#pragma unroll
    for (int b = 0; b < BLOCKS; ++b) {
        half8 lf[L], af[N][L];
#pragma unroll
        for (int e = 0; e < L; ++e) {
            lf[e] = *reinterpret_cast<const half8 *>(A + (c * BLOCKS + b) * (512 * L) + e * 512 + lane * 8);
#pragma unroll
            for (int i = 0; i < N; ++i) af[i][e] = *reinterpret_cast<const half8 *>(A + ((p.ti * 2 + r + i) * BLOCKS + b) * (512 * L) + e * 512 + lane * 8);
        }
#pragma unroll
        for (int e = 2 * (L - 1); e >= 0; --e)
#pragma unroll
            for (int i = 0; i < N; ++i) sum[i] = __builtin_amdgcn_mfma_f32_32x32x16_f16(lf[e == 2 ? L - 1 : 0], af[i][e == 1 ? L - 1 : 0], sum[i], 0, 0, 0);
    }
#pragma unroll
    for (int i = 0; i < N; ++i)
#pragma unroll
        for (int g = 0; g < 4; ++g) {
            const int row = (r + i) * 32 + l32, I = p.ti * 64 + row, k = c * 32 + 8 * g + 4 * h;
            const f16_t *from = A + place8<L == 2>(I, k & ~7, 64 * N) + (k & 4);
            const half4 hi = *reinterpret_cast<const half4 *>(from);
            half4 lo = {};
            if constexpr (L == 2) lo = *reinterpret_cast<const half4 *>(from + 512);
            float v[4];
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const float was = L == 2 ? (float)hi[e] + (float)lo[e] : (float)hi[e];
                v[e] = sum[i][4 * g + e] * (NS_C * P_SCALE / (G_SCALE * G_SCALE)) + was * (NS_B * P_SCALE / G_SCALE) + (I == k + e ? NS_A * P_SCALE : 0.0f);
            }
            const Parts p0 = parts_of<L == 2>(v[0], v[1]), p1 = parts_of<L == 2>(v[2], v[3]);
            f16_t *to = rows + place8<L == 2>(row, k & ~7, 64 * N) + (k & 4);
            *reinterpret_cast<half4 *>(to) = __builtin_shufflevector(p0.hi, p1.hi, 0, 1, 2, 3);
            if constexpr (L == 2) *reinterpret_cast<half4 *>(to + 512) = __builtin_shufflevector(p0.lo, p1.lo, 0, 1, 2, 3);
        }
    __syncthreads();
    Sums<2, 2, KIND> s;
    s.clear();
#pragma unroll
    for (int t = 0; t < N; ++t) {
        half8 lf[2][L];
#pragma unroll
        for (int f = 0; f < 2; ++f)
#pragma unroll
            for (int e = 0; e < L; ++e) lf[f][e] = *reinterpret_cast<const half8 *>(rows + (f * BLOCKS + group + KS * t) * (512 * L) + e * 512 + lane * 8);
        s.add(lf, rf[t]);
    }
    s.cut();
    if (MODE == MUON_STEP && *(volatile const int32_t *)err) return;  // (set before this launch: the same for all)
    __syncthreads();                                                          // (P has been read: its place is used again)
    put_tile<2, 2, KS, KIND, MODE>(a, p, s.all(), p.ti * 64, p.tj * 64, lds[group], lds[0], group);
}

// until at most N of this wavefront's loads are on their way and all it has asked of LDS is there, then until all wavefronts are so far
template <int N> __device__ __forceinline__ void wait_and_meet() {
    asm volatile("" ::: "memory");
    __builtin_amdgcn_s_waitcnt(0x0070 | (N & 15) | ((N >> 4) << 14));
    __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");
}

// The order of a turn's instructions: after a product a read of LDS, as long as there are any, and the loads spread over the products - a
// wavefront that has a vector unit to itself keeps its matrix pipe fed.
template <int PRODUCTS, int READS, int LOADS, int I = 0> __device__ __forceinline__ void interleave() {
    constexpr int R = (I + 1) * READS / PRODUCTS - I * READS / PRODUCTS, L = (I + 1) * LOADS / PRODUCTS - I * LOADS / PRODUCTS;
    __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);
    if constexpr (R > 0) __builtin_amdgcn_sched_group_barrier(0x100, R, 0);
    if constexpr (L > 0) __builtin_amdgcn_sched_group_barrier(0x020, L, 0);
    if constexpr (I + 1 < PRODUCTS) interleave<PRODUCTS, READS, LOADS, I + 1>();
}

// Larger ones: 64 FI x 64 FI per workgroup, a quarter per wavefront, operands by way of LDS, so that a line is read from the die's cache by
// one wavefront and used by two.  A stage has KB blocks of k; STAGES of them are in LDS or on their way there, straight from memory.  A wavefront
// asks for the next block's operands before it multiplies the ones it has, also across the meeting of the wavefronts at which a
// stage is given up and the next one is known to be there.
// The matrix units bound the large ones (a library's product of 8192 x 8192 fp16 numbers: 1,071 TFLOP/s).  Two of 4096 x 4096, tiles of 256: P X 275 GFLOP in
// 252 us, 1,091 TFLOP/s, with pairs on the right 550 in 452, 1,216; X X' 146 in 164 with its rest and the join, 890.  Tiles of 128, pairs: P X of 1024 x 1024
// by 4096, 25.8 GFLOP in 33 us: 23 of them at 1,120 TFLOP/s, the rest launch, first operands and the way out; X X' 13.5 in 28 with the join.
// (Operands straight from memory into registers are slower: the die's cache bounds it then.)
constexpr int stage_pieces(int FI, int KB, int kind) { return 2 * FI * KB * (left_parts(kind) + right_parts(kind)); }   // of 1,024 bytes
template <int FI, int KB, int STAGES, int KIND, int MODE>
__global__ __launch_bounds__(256) __attribute__((amdgpu_waves_per_eu(STAGES * stage_pieces(FI, KB, KIND) <= 80 ? 2 : 1))) void k_muon_large(MuonArgs a, const int32_t *err) {
    constexpr int L = left_parts(KIND), R = right_parts(KIND), T = 64 * FI, U = KB == 1 ? 2 : KB, OWN = FI / 2;
    constexpr int PER_L = KB * L, PER_R = KB * R, ML = OWN * PER_L, MR = OWN * PER_R, MINE = ML + MR, RIGHT = 4 * ML, STAGE = 4 * MINE * 1024;
    static_assert(STAGES >= 3 && U % 2 == 0 && FI % 2 == 0);
    extern __shared__ __attribute__((aligned(16))) unsigned char lds_bytes[];
    unsigned char *const lds = lds_bytes;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6);
    const Place p = place_of<MODE>(a, blockIdx.x, gridDim.x);
    const int blocks = a.K >> 4, turns = blocks / U, first = (int)((int64_t)turns * p.share / a.shares), cnt = (int)((int64_t)turns * (p.share + 1) / a.shares) - first;
    // A stage in LDS: of each operand's 2 FI times 32 rows, KB blocks with their parts, 1,024 bytes each.  This wavefront fetches those of OWN times 32 rows
    // of either operand.
    const char *left[OWN], *right[OWN];
#pragma unroll
    for (int i = 0; i < OWN; ++i) {
        const int rows = wave * OWN + i;
        left[i] = reinterpret_cast<const char *>(a.lhs + p.b * a.lhs_size + ((int64_t)(p.ti * (2 * FI) + rows) * blocks + first * U) * (512 * L));
        right[i] = reinterpret_cast<const char *>(a.rhs + p.b * a.rhs_size + ((int64_t)(p.tj * (2 * FI) + rows) * blocks + first * U) * (512 * R));
    }
    const uint32_t lane16 = lane * 16;
    const int last = cnt * (U / KB) - 1;
    // a KB-th of stage t, into its slot; behind the last stage that one once more, into a slot that nobody reads, so that all turns are alike
    const auto fetch = [&](int slot, int t, int kb) {
        const int64_t at = t < last ? t : last;
#pragma unroll
        for (int i = kb * MINE / KB; i < (kb + 1) * MINE / KB; ++i) {
            const int j = i < ML ? i : i - ML;
            const char *from = i < ML ? left[j / PER_L % OWN] + at * (PER_L * 1024) + j % PER_L * 1024 : right[j / PER_R % OWN] + at * (PER_R * 1024) + j % PER_R * 1024;
            __builtin_amdgcn_global_load_lds((const __attribute__((address_space(1))) void *)(from + lane16),
                                             (__attribute__((address_space(3))) void *)(lds + slot * STAGE + (i < ML ? wave * ML + j : RIGHT + wave * MR + j) * 1024), 16, 0, 0);
        }
    };
    const int wi = wave >> 1, wj = wave & 1;
    half8 lf[2][FI][L], rf[2][FI][R];
    const auto read = [&](half8 (&x)[FI][L], half8 (&y)[FI][R], int slot, int kb) {
        const unsigned char *at = lds + slot * STAGE + lane * 16;
#pragma unroll
        for (int f = 0; f < FI; ++f)
#pragma unroll
            for (int e = 0; e < L; ++e) x[f][e] = *reinterpret_cast<const half8 *>(at + ((wi * FI + f) * PER_L + kb * L + e) * 1024);
#pragma unroll
        for (int f = 0; f < FI; ++f)
#pragma unroll
            for (int e = 0; e < R; ++e) y[f][e] = *reinterpret_cast<const half8 *>(at + (RIGHT + (wj * FI + f) * PER_R + kb * R + e) * 1024);
    };
    Sums<FI, FI, KIND> s;
    s.clear();
#pragma unroll
    for (int t = 0; t < STAGES - 1; ++t)
#pragma unroll
        for (int kb = 0; kb < KB; ++kb) fetch(t, t, kb);
    wait_and_meet<(STAGES - 2) * MINE>();
    read(lf[0], rf[0], 0, 0);
    int slot = 0, into = STAGES - 1, stage = 0;                               // where this stage is, and stage + STAGES - 1 goes
    for (int c0 = 0; c0 < cnt; c0 += CHAIN / U) {
        const int c1 = c0 + CHAIN / U < cnt ? c0 + CHAIN / U : cnt;
        for (int t = c0; t < c1; ++t) {
#pragma unroll
            for (int kb = 0; kb < U; ++kb) {
                const bool end = (kb + 1) % KB == 0;                          // of the stage: it has been read, and the next one is there
                if (end) wait_and_meet<(STAGES - 3) * MINE + (KB - 1) * MINE / KB>();
                const int next = !end ? slot : slot + 1 == STAGES ? 0 : slot + 1;
                read(lf[(kb + 1) & 1], rf[(kb + 1) & 1], next, (kb + 1) % KB);
                fetch(into, stage + STAGES - 1, kb % KB);
                s.add(lf[kb & 1], rf[kb & 1]);
                interleave<FI * FI * products_of(KIND), FI * (L + R), MINE / KB>();
                if (end) { into = slot; slot = next; ++stage; }
            }
        }
        s.cut();
    }
    wait_and_meet<0>();                                                       // (nothing is on its way to LDS, and all stages have been read)
    if (MODE == MUON_STEP && *(volatile const int32_t *)err) return;  // (set before this launch: the same for all)
    if (a.shares > 1) {
        // a share of the sums: 16 bytes per lane at a time, as they are
        floatx4 *to = reinterpret_cast<floatx4 *>(a.part) + ((int64_t)(p.slot * a.shares + p.share) * 4 + wave) * (FI * FI * 4 * 64) + lane;
#pragma unroll
        for (int i = 0; i < FI; ++i)
#pragma unroll
            for (int j = 0; j < FI; ++j)
#pragma unroll
                for (int g = 0; g < 4; ++g) {
                    const floatx16 v = s.all()[i][j];
                    to[((i * FI + j) * 4 + g) * 64] = floatx4{v[4 * g], v[4 * g + 1], v[4 * g + 2], v[4 * g + 3]};
                }
        return;
    }
    float *const mine = reinterpret_cast<float *>(lds) + wave * (64 * SUMS_LD);
    put_tile<FI, FI, 1, KIND, MODE>(a, p, s.all(), p.ti * T + wi * FI * 32, p.tj * T + wj * FI * 32, mine, mine, 0);
}

// The shares of the sums added: a workgroup for 64 x 64 of a tile, each wavefront every fourth share, and then the four.  36 tiles of 128 x 128 in seven
// shares: 17 MB in 7 us; without shares the product takes 74 us instead of 21.
template <int FI, int KIND, int MODE>
__global__ __launch_bounds__(256) void k_muon_join(MuonArgs a, int32_t shares) {
    constexpr int KS = 4, PARTS = FI * FI;
    __shared__ __attribute__((aligned(16))) float lds[KS][64 * SUMS_LD];
    const Place p = place_of<MODE>(a, blockIdx.x / PARTS, gridDim.x / PARTS);  // (a.shares is 1 here)
    const int part = blockIdx.x % PARTS, wave = part & 3, si = (part >> 2) / (FI / 2), sj = (part >> 2) % (FI / 2);
    const int lane = threadIdx.x & 63, group = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6);
    floatx16 x[2][2];
#pragma unroll
    for (int i = 0; i < 2; ++i)
#pragma unroll
        for (int j = 0; j < 2; ++j) x[i][j] = floatx16{};
    for (int k = group; k < shares; k += KS) {
        const floatx4 *from = reinterpret_cast<const floatx4 *>(a.part) + ((int64_t)(p.slot * shares + k) * 4 + wave) * (FI * FI * 4 * 64) + lane;
#pragma unroll
        for (int i = 0; i < 2; ++i)
#pragma unroll
            for (int j = 0; j < 2; ++j)
#pragma unroll
                for (int g = 0; g < 4; ++g) {
                    const floatx4 v = from[(((2 * si + i) * FI + 2 * sj + j) * 4 + g) * 64];
#pragma unroll
                    for (int e = 0; e < 4; ++e) x[i][j][4 * g + e] += v[e];
                }
    }
    put_tile<2, 2, KS, KIND, MODE>(a, p, x, p.ti * 64 * FI + ((wave >> 1) * FI + 2 * si) * 32, p.tj * 64 * FI + ((wave & 1) * FI + 2 * sj) * 32, lds[group], lds[0], group);
}

// ---- matrices of up to 128 x 128 or 64 x 256: all steps in one launch ----------------------------------------------------
// A workgroup of eight wavefronts has a matrix; of its frame, sides of multiples of 64, a wavefront has 64 x 32, as the sums of the
// matrix instruction lie: two pieces of 32 x 32.  X stays in registers as 32-bit numbers; LDS has one operand of X - its rows for A = X X', then
// its columns for P X - and A, then P.  The norm and, of a step, momentum and weights are read and written as they lie in registers.
// What several launches per step cost - 5 us each for a few microseconds of products - is what this saves.  32 bits, this way and by tiles: 64 x 256 39 us
// and 74, 10 x 200 29 and 74, 16 of 100 x 100 45 and 83, 300 of 128 x 128 103 and 246; bf16 results, which have single numbers by tiles: 64 x 256 42 and 61,
// 16 of 100 x 100 48 and 69.  What is left is a chain of four meetings a step, with a product of up to 16 blocks of k, or a change of parts in LDS,
// between two of them.  Larger thin matrices in slices of 128 or 256 columns, with a launch per step that adds the slices' A, are slower than
// by tiles: 128 x 1024 156 us instead of 96.
constexpr int ONE_SIDE = 128, ONE_THREADS = 512;
inline bool one_fits(int32_t n, int32_t m) { return m <= ONE_SIDE || (n <= 64 && m <= 256); }

// The 4 x 4 numbers of 16 bits of four lanes transposed: rows 0, 1 and rows 2, 3 of a lane's column become, of lane q, row q of the four columns.
__device__ __forceinline__ void turn_quad(uint32_t &r01, uint32_t &r23) {
    const auto other = [](uint32_t x, auto perm) { return (uint32_t)__builtin_amdgcn_mov_dpp((int)x, decltype(perm)::value, 0xf, 0xf, true); };
    const std::integral_constant<int, 0xB1> by_one{};                         // lanes 1 0 3 2
    const std::integral_constant<int, 0x4E> by_two{};                         // lanes 2 3 0 1
    const bool high = threadIdx.x & 2;
    const uint32_t got = other(high ? r01 : r23, by_two), a0 = high ? got : r01, a1 = high ? r23 : got;    // of columns q % 2 and q % 2 + 2
    const uint32_t select = threadIdx.x & 1 ? 0x03020706u : 0x05040100u;
    r01 = __builtin_amdgcn_perm(other(a0, by_one), a0, select);
    r23 = __builtin_amdgcn_perm(other(a1, by_one), a1, select);
}

struct MuonOne { MuonIn in; MuonArgs out; int32_t n, m, nq, mq, steps; };     // nq, mq: the frame

template <class T, bool STEP>
__global__ __launch_bounds__(ONE_THREADS) void k_muon_one(MuonOne a, const int32_t *err) {
    constexpr int S = 2;
    extern __shared__ __attribute__((aligned(16))) f16_t one_lds[];
    __shared__ double squares[ONE_THREADS / 64];
    if (STEP && *(volatile const int32_t *)err) return;                       // (set before this launch: the same for all)
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6), l32 = lane & 31, h = lane >> 5;
    const int nq = a.nq, mq = a.mq, across = nq == 64 ? 8 : 4, i0 = wave / across * 64, j0 = wave % across * 32;
    const bool tall = a.out.tall, has_x = i0 < nq && j0 < mq, has_a = i0 < nq && j0 < nq;
    f16_t *const r1 = one_lds, *const r2 = one_lds + nq * mq * S;
    const int64_t row0 = (int64_t)blockIdx.x * a.in.rows;
    const MuonIn &in = a.in;
    // piece f, sum e: row i0 + 32 f + 8 (e / 4) + 4 h + e % 4, column j0 + l32 of X
    const auto row_of = [&](int f, int e) { return i0 + 32 * f + 8 * (e >> 2) + 4 * h + (e & 3); };
    float v0[32];
    double s = 0.0;
#pragma unroll
    for (int f = 0; f < 2; ++f)
#pragma unroll
        for (int e = 0; e < 16; ++e) {
            const int i = row_of(f, e), j = j0 + l32;
            float v = 0.0f;
            if (has_x && i < a.n && j < a.m) {
                const int64_t row = row0 + (tall ? j : i), col = tall ? i : j;
                v = (float)reinterpret_cast<const T *>(in.in)[row * in.ld + col];
                if constexpr (STEP) {
                    float *m = in.val + (in.first + row) * in.L + in.cols + col;
                    const float moment = in.mu * *m + v;
                    *m = moment;
                    v = in.nesterov ? v + in.mu * moment : moment;
                }
            }
            v0[f * 16 + e] = v;
            s += (double)v * (double)v;
        }
    for (int d = 32; d > 0; d >>= 1) s += __shfl_xor(s, d);
    if (lane == 0) squares[wave] = s;
    __syncthreads();
    s = 0.0;
#pragma unroll
    for (int w = 0; w < ONE_THREADS / 64; ++w) s += squares[w];
    Scale(s, in.eps).apply(v0);                                               // (zero outside the matrix, or all NaN)
    floatx16 x[2];
#pragma unroll
    for (int i = 0; i < 32; ++i) x[i >> 4][i & 15] = v0[i];

    // the numbers as parts: pair (f, 2 g + e): rows 4 g + 2 e and the next one of piece f
    const auto split = [&](Parts (&q)[2][8], const floatx16 (&v)[2], float factor) {
#pragma unroll
        for (int f = 0; f < 2; ++f)
#pragma unroll
            for (int e = 0; e < 8; ++e) q[f][e] = parts_of<true>(v[f][2 * e] * factor, v[f][2 * e + 1] * factor);
    };
    // into m of K numbers a row: rows and columns exchanged, four rows' numbers are neighbours; and as they are
    const auto put_columns = [&](f16_t *m, int K, const Parts (&q)[2][8]) {
#pragma unroll
        for (int f = 0; f < 2; ++f)
#pragma unroll
            for (int g = 0; g < 4; ++g) {
                const int i = row_of(f, 4 * g), j = j0 + l32;
                f16_t *p = m + place8<true>(j, i & ~7, K) + (i & 4);
                *reinterpret_cast<half4 *>(p) = __builtin_shufflevector(q[f][2 * g].hi, q[f][2 * g + 1].hi, 0, 1, 2, 3);
                *reinterpret_cast<half4 *>(p + 512) = __builtin_shufflevector(q[f][2 * g].lo, q[f][2 * g + 1].lo, 0, 1, 2, 3);
            }
    };
    const auto put_rows = [&](f16_t *m, int K, const Parts (&q)[2][8]) {
#pragma unroll
        for (int f = 0; f < 2; ++f)
#pragma unroll
            for (int g = 0; g < 4; ++g) {
                const int i = row_of(f, 4 * g) + (lane & 3), j = j0 + (l32 & ~3);
                f16_t *p = m + place8<true>(i, j & ~7, K) + (j & 4);
                uint32_t a = __builtin_bit_cast(uint32_t, q[f][2 * g].hi), b = __builtin_bit_cast(uint32_t, q[f][2 * g + 1].hi);
                turn_quad(a, b);
                *reinterpret_cast<uint2 *>(p) = uint2{a, b};
                a = __builtin_bit_cast(uint32_t, q[f][2 * g].lo);
                b = __builtin_bit_cast(uint32_t, q[f][2 * g + 1].lo);
                turn_quad(a, b);
                *reinterpret_cast<uint2 *>(p + 512) = uint2{a, b};
            }
    };
    // this wavefront's sums over the first `used` blocks of k, 16 at most (so that chains are short: see Sums), of rows of K numbers of l and r
    const auto product = [&](const f16_t *l, const f16_t *r, int K, int used, floatx16 (&sum)[2]) {
        const int blocks = K >> 4;
        const f16_t *pl = l + (i0 >> 5) * blocks * (512 * S) + lane * 8, *pr = r + (j0 >> 5) * blocks * (512 * S) + lane * 8;
        sum[0] = floatx16{};
        sum[1] = floatx16{};
        for (int k = 0; k < used; ++k) {
            half8 lf[2][S], rf[S];
#pragma unroll
            for (int e = 0; e < S; ++e) {
                lf[0][e] = *reinterpret_cast<const half8 *>(pl + k * (512 * S) + e * 512);
                lf[1][e] = *reinterpret_cast<const half8 *>(pl + (blocks + k) * (512 * S) + e * 512);
                rf[e] = *reinterpret_cast<const half8 *>(pr + k * (512 * S) + e * 512);
            }
#pragma unroll
            for (int e = 2; e >= 0; --e)
#pragma unroll
                for (int f = 0; f < 2; ++f) sum[f] = __builtin_amdgcn_mfma_f32_32x32x16_f16(lf[f][e == 2 ? S - 1 : 0], rf[e == 1 ? S - 1 : 0], sum[f], 0, 0, 0);
        }
    };
    const int used_n = (a.n + 15) >> 4, used_m = (a.m + 15) >> 4;
    float x_factor = 1.0f;                                                    // x holds this times the scaled X
    for (int step = 0; step < a.steps; ++step) {
        floatx16 g[2], q[2];
        Parts parts[2][8], more[2][8];
        if (has_x) {
            split(parts, x, x_factor);
            put_rows(r1, mq, parts);
        }
        __syncthreads();
        if (has_a) {
            product(r1, r1, mq, used_m, g);
            split(more, g, G_SCALE / (X_SCALE * X_SCALE));
            put_columns(r2, nq, more);                                        // (A is symmetric)
        }
        __syncthreads();
        if (has_x) put_columns(r1, nq, parts);
        if (has_a) product(r2, r2, nq, used_n, q);
        __syncthreads();
        if (has_a) {
#pragma unroll
            for (int f = 0; f < 2; ++f)
#pragma unroll
                for (int e = 0; e < 16; ++e)
                    q[f][e] = q[f][e] * (NS_C * P_SCALE / (G_SCALE * G_SCALE)) +
                              (g[f][e] * (NS_B * P_SCALE / (X_SCALE * X_SCALE)) + (row_of(f, e) == j0 + l32 ? NS_A * P_SCALE : 0.0f));
            split(more, q, 1.0f);
            put_columns(r2, nq, more);
        }
        __syncthreads();
        if (has_x) product(r2, r1, nq, used_n, x);
        x_factor = 1.0f / P_SCALE;
        __syncthreads();
    }
#pragma unroll
    for (int f = 0; f < 2; ++f)
#pragma unroll
        for (int e = 0; e < 16; ++e) {
            const int i = row_of(f, e), j = j0 + l32;
            if (has_x && i < a.n && j < a.m) {
                const float v = x[f][e] * (x_factor / X_SCALE);
                const int64_t row = row0 + (tall ? j : i), col = tall ? i : j;
                if constexpr (STEP) {
                    float *w = a.out.val + (a.out.first + row) * a.out.L + col;
                    *w = a.out.keep * *w - a.out.step * v;
                } else if (a.out.to_type == PS_BF16) reinterpret_cast<bf16_t *>(a.out.to)[row * a.out.to_ld + col] = (bf16_t)v;
                else if (a.out.to_type == PS_F32) reinterpret_cast<float *>(a.out.to)[row * a.out.to_ld + col] = v;
                else reinterpret_cast<f16_t *>(a.out.to)[row * a.out.to_ld + col] = (f16_t)v;
            }
        }
}

// ---- host -----------------------------------------------------------------------------------------------------------
// Sides count as multiples of the tile's, 64, 128 or 256.  Tiles of 128 read a line of an operand half as often, tiles of 256 a quarter
// as often, but few of them leave compute units idle, and they fill up more.  Whole calls, tiles of 64 and of 128: 32 bits, 300 x 300 111 us and 151,
// 1024 x 1024 202 and 261, two of them 292 and 320, 1500 x 2000 516 and 448, four of 1024 x 1024 458 and 431, 1024 x 4096 429 and 372, 4096 x 4096 5,086
// and 4,486; 32 of 300 x 300, which become 320 and 384, 199 and 292; bf16 results, 300 of 200 x 200 520 and 500, 100 of 300 x 700 545 and 671, 26 of
// 1000 x 1010 1,535 and 1,133 - the line is at 2.9 million numbers, unless the larger tile makes them a quarter more.  Tiles of 128 and of 256 for bf16
// results: it is the rounds of the compute units that the 256s fill which count - seven tenths of them in P X, half of one in X X' -, and sides above 2048.
// P X fills 0.77 to 1 of its rounds: 4096 x 4096 1,970 and 1,847, two of them 3,667 and 3,379, two of 3584 x 3584 2,609 and 2,376, four of 2560 x 2560 1,971
// and 1,850, 5000 x 5000 3,593 and 3,205, 8192 x 8192 13,593 and 11,882; 0.70 to 0.75: 4864 x 4864 3,001 and 2,980, 4352 x 8704 4,070 and 3,973, three of
// 2816 x 2816 1,876 and 1,918; 0.56 to 0.66: 4352 x 4352 2,295 and 2,593, two of 3328 x 3328 2,060 and 2,150, three of 2560 x 2560 1,487 and 1,716.  X X' fills
// less than half of a round: 3584 x 7168 2,305 and 2,510, 2000 x 8000 921 and 1,578.  Short sums: eight of 2048 x 2048 2,063 and 2,136 (16 of them 4,156
// and 3,988), 16 of 1536 x 1536 1,888 and 2,163, 64 of 1024 x 1024 2,629 and 2,780.  And no more than a fiftieth more numbers: 4200 x 4200 by tiles of 256 is 4352 x 4352.
struct MuonPlan {
    int32_t batch, n, m, tile, np, mp, blocks;
    bool tall, split, one;
    size_t off_d, off_x, off_xt[2], off_g, off_p, off_part, bytes;
};
inline int64_t half_of(int64_t t) { return t * (t + 1) / 2; }
// Of single numbers, the first steps, which read X as pairs: all but two, what the last ones raise an error of X by, and two at least.
inline int pair_steps(int32_t steps) { return steps > 4 ? steps - 2 : 2; }
constexpr int PAIR_SIDE = 64;                    // pairs throughout where A is at most so large
constexpr int MOST_SHARES = 8, TURNS_AT_LEAST = 2, SMALL_SHARES = 16, SMALL_TURNS = 4;
// Workgroups that share a tile's sum over k, where there are fewer tiles than compute units.
int shares_of(const dpaps_ps *ps, int64_t tiles, int32_t K) {
    int64_t s = ps->num_cu / tiles;
    if (s > MOST_SHARES) s = MOST_SHARES;
    if (s > K / 64 / TURNS_AT_LEAST) s = K / 64 / TURNS_AT_LEAST;
    return s < 2 ? 1 : (int)s;
}
// The same for tiles of 64, a long sum: at least SMALL_TURNS blocks of k for each wavefront.  A share more costs the join, 3 us, and saves a part of the sum's
// time: 10 x 4096 in 32 bits 101 us instead of 211, 128 x 1024 106 instead of 117; 128 x 512, with two shares, 102 instead of 97
// (with the polynomial in a launch of its own).
int small_shares(const dpaps_ps *ps, int64_t tiles, int32_t K) {
    const int64_t by_K = K / 64 / SMALL_TURNS, most = ps->num_cu / tiles;
    if (by_K < 4) return 1;
    const int64_t s = by_K < most ? by_K : most;
    return s < 2 ? 1 : s > SMALL_SHARES ? SMALL_SHARES : (int)s;
}
MuonPlan muon_plan(const dpaps_ps *ps, int32_t batch, int32_t rows, int32_t cols, bool split, bool step) {
    MuonPlan p{};
    p.batch = batch; p.tall = rows > cols; p.split = split;
    p.n = p.tall ? cols : rows; p.m = p.tall ? rows : cols;
    p.one = one_fits(p.n, p.m);
    if (p.one) {                                  // (no scratch)
        p.np = (int32_t)(ceil_div64(p.n, 64) * 64); p.mp = (int32_t)(ceil_div64(p.m, 64) * 64);
        return p;
    }
    const auto padded = [&](int64_t t) { return ceil_div64(p.n, t) * t * ceil_div64(p.m, t) * t * batch; };
    p.tile = padded(64) >= (int64_t)11264 * ps->num_cu && 4 * padded(128) <= 5 * padded(64) ? 128 : 64;
    const int64_t whole = ceil_div64(p.n, 256) * ceil_div64(p.m, 256) * batch, cus = ps->num_cu;
    if (!split && p.n > 2048 && 50 * padded(256) <= 51 * padded(128) && 2 * half_of(ceil_div64(p.n, 256)) * batch >= cus &&
        10 * whole >= 7 * ceil_div64(whole, cus) * cus)
        p.tile = 256;
    p.np = (int32_t)(ceil_div64(p.n, p.tile) * p.tile); p.mp = (int32_t)(ceil_div64(p.m, p.tile) * p.tile);
    const int64_t blocks = ceil_div64((int64_t)rows * cols, 1024);
    p.blocks = (int32_t)(blocks < NORM_BLOCKS ? blocks : NORM_BLOCKS);
    const size_t size = split ? 4 : 2, nm = (size_t)batch * p.np * p.mp, nn = (size_t)batch * p.np * p.np * size;
    p.off_d = up256((size_t)batch * NORM_BLOCKS * sizeof(double));
    p.off_x = p.off_d + (step ? up256((size_t)batch * rows * cols * sizeof(float)) : 0);
    p.off_xt[0] = p.off_x + up256(nm * size);
    p.off_xt[1] = p.off_xt[0] + up256(nm * 4);
    p.off_g = p.off_xt[1] + up256(nm * 4);
    p.off_p = p.off_g + up256(nn);
    p.off_part = p.off_p + up256(nn);
    // (shares times tiles are at most as many as the compute units)
    p.bytes = p.off_part + (size_t)ps->num_cu * p.tile * p.tile * sizeof(float);
    return p;
}

template <int FI, int KB, int STAGES, int KIND, int MODE>
int large(dpaps_ps *ps, const MuonArgs &a, int64_t tiles, hipStream_t st) {
    static LdsAllowed allowed;
    constexpr int STAGED = STAGES * stage_pieces(FI, KB, KIND) * 1024, SUMMED = 4 * 64 * SUMS_LD * 4, LDS = STAGED > SUMMED ? STAGED : SUMMED;
    static_assert(LDS <= 160 * 1024);
    const int rc = dpaps_allow_lds(ps, allowed, reinterpret_cast<const void *>(&k_muon_large<FI, KB, STAGES, KIND, MODE>), LDS);
    if (rc) return rc;
    k_muon_large<FI, KB, STAGES, KIND, MODE><<<(unsigned)(tiles * a.shares), 256, LDS, st>>>(a, ps->err);
    PS_HIP(ps, hipGetLastError());
    return PS_OK;
}
// Tiles tile0 .. tile0 + tiles - 1, fewer than compute units: with shared sums, if that can be.
template <int FI, int KB, int KIND, int MODE>
int large_rest(dpaps_ps *ps, MuonArgs a, int64_t tiles, hipStream_t st) {
    const int32_t shares = shares_of(ps, tiles, a.K);
    a.shares = shares;
    const int rc = large<FI, KB, 4, KIND, MODE>(ps, a, tiles, st);
    if (rc || shares == 1) return rc;
    a.shares = 1;
    k_muon_join<FI, KIND, MODE><<<(unsigned)(FI * FI * tiles), 256, 0, st>>>(a, shares);
    PS_HIP(ps, hipGetLastError());
    return PS_OK;
}
// X X' or A A', of which half of the tiles is computed
template <int TILE, int KIND, int MODE>
int half_product(dpaps_ps *ps, MuonArgs a, int32_t batch, hipStream_t st) {
    a.tiles = (int32_t)half_of(a.tiles_i);
    a.shares = 1;
    const int64_t tiles = (int64_t)a.tiles * batch, cus = ps->num_cu;
    if constexpr (TILE == 64) {
        if constexpr (MODE == MUON_GRAM) a.shares = small_shares(ps, tiles, a.K);
        k_muon_small<KIND, MODE><<<(unsigned)(tiles * a.shares), 256, 0, st>>>(a, ps->err);
        PS_HIP(ps, hipGetLastError());
        if constexpr (MODE == MUON_GRAM) {
            const int32_t shares = a.shares;
            a.shares = 1;
            if (shares > 1) k_muon_join_small<KIND><<<(unsigned)tiles, 256, 0, st>>>(a, shares);
            PS_HIP(ps, hipGetLastError());
        }
        return PS_OK;
    } else if constexpr (TILE == 256) {
        // as many tiles as make full rounds of the compute units, and the rest with shared sums
        const int64_t rest = tiles > cus && tiles % cus <= cus / 2 ? tiles % cus : 0;
        const int rc = large<4, 2, 4, KIND, MODE>(ps, a, tiles - rest, st);
        if (rc || rest == 0) return rc;
        a.tile0 = (int32_t)(tiles - rest);
        return large_rest<4, 2, KIND, MODE>(ps, a, rest, st);
    } else {
        constexpr int KB = KIND == SPLIT ? 2 : 4;                             // so 128 KB of LDS; half of that where two workgroups share a compute unit
        if (tiles > cus) return large<2, KB / 2, 4, KIND, MODE>(ps, a, tiles, st);
        if (a.K <= 1024 && tiles < cus) {                                     // (with a short sum, tiles of 64)
            a.tiles_i *= 2;
            return half_product<64, KIND, MODE>(ps, a, batch, st);
        }
        return large_rest<2, KB, KIND, MODE>(ps, a, tiles, st);
    }
}
// P X
template <int TILE, int KIND, int MODE>
int whole_product(dpaps_ps *ps, MuonArgs a, int32_t batch, hipStream_t st) {
    a.tiles = a.tiles_i * a.tiles_j;
    a.shares = 1;
    const int64_t tiles = (int64_t)a.tiles * batch;
    if constexpr (TILE == 64) {
        k_muon_small<KIND, MODE><<<(unsigned)tiles, 256, 0, st>>>(a, ps->err);
        PS_HIP(ps, hipGetLastError());
        return PS_OK;
    } else if constexpr (TILE == 256) {
        return large<4, 2, KIND == RIGHT_SPLIT ? 3 : 4, KIND, MODE>(ps, a, tiles, st);
    } else {
        // (96 to 128 KB of LDS; 64 or 72 where two workgroups share a compute unit)
        constexpr int KB = KIND == SINGLE ? 4 : 2;
        if (tiles > ps->num_cu) return large<2, KIND == RIGHT_SPLIT ? KB : KB / 2, KIND == RIGHT_SPLIT ? 3 : 4, KIND, MODE>(ps, a, tiles, st);
        return large<2, KB, 4, KIND, MODE>(ps, a, tiles, st);
    }
}

// the polynomial and P X of thin matrices
template <int KIND, int MODE>
int poly_apply(dpaps_ps *ps, MuonArgs a, int32_t batch, hipStream_t st) {
    a.tiles = a.tiles_i * a.tiles_j;
    a.shares = 1;
    const unsigned grid = (unsigned)((int64_t)a.tiles * batch);
    if (a.tiles_i == 2) k_muon_poly_apply<KIND, MODE, 2><<<grid, 256, 0, st>>>(a, ps->err);
    else if constexpr (KIND == SPLIT) k_muon_poly_apply<KIND, MODE, 1><<<grid, 256, 0, st>>>(a, ps->err);     // (see PAIR_SIDE)
    PS_HIP(ps, hipGetLastError());
    return PS_OK;
}

template <int TILE, bool PAIR>
int iterate(dpaps_ps *ps, const MuonPlan &p, MuonIn in, MuonArgs last, int32_t steps, hipStream_t st) {
    constexpr int KIND = PAIR ? SPLIT : SINGLE;
    char *ws = (char *)ps->ws;
    f16_t *x = (f16_t *)(ws + p.off_x), *xt = (f16_t *)(ws + p.off_xt[0]), *xt_next = (f16_t *)(ws + p.off_xt[1]), *g = (f16_t *)(ws + p.off_g), *q = (f16_t *)(ws + p.off_p);
    const int64_t S = PAIR ? 2 : 1, nm = (int64_t)p.np * p.mp, nn = (int64_t)p.np * p.np * S;
    const dim3 grid((unsigned)(p.mp / 64), (unsigned)(p.np / 64), (unsigned)p.batch);
    if (in.type == PS_F32) k_muon_scale<float, PAIR><<<grid, 256, 0, st>>>(in, p.tall, p.np, p.mp, x, xt);
    else if (in.type == PS_BF16) k_muon_scale<bf16_t, PAIR><<<grid, 256, 0, st>>>(in, p.tall, p.np, p.mp, x, xt);
    else k_muon_scale<f16_t, PAIR><<<grid, 256, 0, st>>>(in, p.tall, p.np, p.mp, x, xt);
    PS_HIP(ps, hipGetLastError());
    const bool thin = TILE == 64 && p.np <= 128;
    for (int s = 0; s < steps; ++s) {
        MuonArgs a{};
        a.tiles_i = p.np / TILE; a.tiles_j = p.mp / TILE;
        a.part = (float *)(ws + p.off_part);
        a.lhs = a.rhs = x; a.lhs_size = a.rhs_size = nm * S; a.K = p.mp; a.out = g; a.out_ld = p.np; a.out_size = nn;
        int rc = half_product<TILE, KIND, MUON_GRAM>(ps, a, p.batch, st);
        if (rc) return rc;
        if (!thin) {
            a.lhs = a.rhs = g; a.lhs_size = a.rhs_size = nn; a.out = q;
            a.K = p.np;
            rc = half_product<TILE, KIND, MUON_POLY>(ps, a, p.batch, st);
            if (rc) return rc;
        }
        const bool end = s + 1 == steps, pairs = !PAIR && s < pair_steps(steps);
        MuonArgs b = end ? last : a;
        b.tiles_i = a.tiles_i; b.tiles_j = a.tiles_j; b.K = p.np;
        // (X transposed is read by other workgroups while it is written: into the other place; X itself is not)
        b.lhs = thin ? g : q; b.lhs_size = nn; b.rhs = xt; b.rhs_size = nm * 2;
        b.out = x; b.out_ld = p.mp; b.out_size = nm * S;
        b.out_t = xt_next; b.out_t_ld = p.np; b.out_t_size = nm * 2; b.out_t_pair = s + 1 < pair_steps(steps);
        const auto apply = [&](auto kind, auto mode) {
            if constexpr (TILE == 64)
                if (thin) return poly_apply<decltype(kind)::value, decltype(mode)::value>(ps, b, p.batch, st);
            return whole_product<TILE, decltype(kind)::value, decltype(mode)::value>(ps, b, p.batch, st);
        };
        const std::integral_constant<int, MUON_APPLY> more{};
        const std::integral_constant<int, MUON_LAST> result{};
        if constexpr (PAIR) {
            const std::integral_constant<int, SPLIT> split{};
            rc = !end ? apply(split, more) : last.val ? apply(split, std::integral_constant<int, MUON_STEP>{}) : apply(split, result);
        } else if (pairs) {
            const std::integral_constant<int, RIGHT_SPLIT> right{};
            rc = end ? apply(right, result) : apply(right, more);
        } else {
            const std::integral_constant<int, SINGLE> single{};
            rc = end ? apply(single, result) : apply(single, more);
        }
        if (rc) return rc;
        f16_t *const t = xt; xt = xt_next; xt_next = t;
    }
    return PS_OK;
}

template <class T>
int norm_of(dpaps_ps *ps, const MuonPlan &p, const MuonIn &in, hipStream_t st) {
    const dim3 grid((unsigned)p.blocks, (unsigned)p.batch);
    const bool four = rows_allow(in.in, in.type, in.cols, in.ld, 4) &&
                      (!in.val || (rows_allow(in.val + in.first * in.L + in.cols, PS_F32, in.cols, in.L, 4) && rows_allow(in.d, PS_F32, in.cols, in.cols, 4)));
    const uint32_t P = (uint32_t)(four ? in.cols / 4 : in.cols);
    if (in.val) {
        if (four) k_muon_norm<T, 4, true><<<grid, 256, 0, st>>>(in, P, 1.0 / P, ps->err);
        else k_muon_norm<T, 1, true><<<grid, 256, 0, st>>>(in, P, 1.0 / P, ps->err);
    } else {
        if (four) k_muon_norm<T, 4, false><<<grid, 256, 0, st>>>(in, P, 1.0 / P, ps->err);
        else k_muon_norm<T, 1, false><<<grid, 256, 0, st>>>(in, P, 1.0 / P, ps->err);
    }
    PS_HIP(ps, hipGetLastError());
    return PS_OK;
}

template <class T, bool STEP>
int one_of(dpaps_ps *ps, const MuonOne &a, int32_t batch, hipStream_t st) {
    static LdsAllowed allowed;
    constexpr size_t MOST = (size_t)2 * ONE_SIDE * ONE_SIDE * 4;
    const int rc = dpaps_allow_lds(ps, allowed, reinterpret_cast<const void *>(&k_muon_one<T, STEP>), MOST);
    if (rc) return rc;
    k_muon_one<T, STEP><<<(unsigned)batch, ONE_THREADS, (size_t)a.nq * (a.nq + a.mq) * 4, st>>>(a, ps->err);
    PS_HIP(ps, hipGetLastError());
    return PS_OK;
}
template <class T>
int one_launch(dpaps_ps *ps, const MuonPlan &p, const MuonIn &in, const MuonArgs &last, int32_t steps, hipStream_t st) {
    const MuonOne a{in, last, p.n, p.m, p.np, p.mp, steps};
    return in.val ? one_of<T, true>(ps, a, p.batch, st) : one_of<T, false>(ps, a, p.batch, st);
}

int orthogonalize(dpaps_ps *ps, const MuonPlan &p, MuonIn in, MuonArgs last, int32_t steps, hipStream_t st) {
    last.n = p.n; last.m = p.m; last.tall = p.tall;
    if (p.one) {
        if (in.type == PS_F32) return one_launch<float>(ps, p, in, last, steps, st);
        return in.type == PS_BF16 ? one_launch<bf16_t>(ps, p, in, last, steps, st) : one_launch<f16_t>(ps, p, in, last, steps, st);
    }
    char *ws = (char *)ps->ws;
    in.squares = (double *)ws;
    in.blocks = p.blocks;
    if (in.val) in.d = (float *)(ws + p.off_d);
    int rc;
    if (in.type == PS_F32) rc = norm_of<float>(ps, p, in, st);
    else if (in.type == PS_BF16) rc = norm_of<bf16_t>(ps, p, in, st);
    else rc = norm_of<f16_t>(ps, p, in, st);
    if (rc) return rc;
    if (in.val) { in.in = in.d; in.ld = in.cols; in.type = PS_F32; }
    if (p.split) return p.tile == 128 ? iterate<128, true>(ps, p, in, last, steps, st) : iterate<64, true>(ps, p, in, last, steps, st);
    if (p.tile == 256) return iterate<256, false>(ps, p, in, last, steps, st);
    return p.tile == 128 ? iterate<128, false>(ps, p, in, last, steps, st) : iterate<64, false>(ps, p, in, last, steps, st);
}

bool sizes_allowed(int32_t batch, int32_t rows, int32_t cols) { return rows <= PS_MUON_MAX_SIDE && cols <= PS_MUON_MAX_SIDE && batch <= PS_MUON_MAX_BATCH; }

}  // namespace

extern "C" int muon_orthogonalize(ps_handle ps, int32_t batch, int32_t rows, int32_t cols, const void *in, int32_t in_type, int64_t in_ld, void *out,
                                  int32_t out_type, int64_t out_ld, int32_t steps, float eps, void *stream) {
    if (!ps || batch < 0 || rows < 0 || cols < 0 || !is_element_type(in_type) || !is_element_type(out_type) || steps < 1 || steps > 100 || !(eps >= 0.0f)) return PS_EINVAL;
    if (batch == 0 || rows == 0 || cols == 0) return PS_OK;
    if (!in || !out || in_ld < cols || out_ld < cols) return PS_EINVAL;
    if (!sizes_allowed(batch, rows, cols)) return PS_ELIMIT;
    const MuonPlan p = muon_plan(ps, batch, rows, cols, out_type != PS_BF16 || (rows < cols ? rows : cols) <= PAIR_SIDE, false);
    const int rc = dpaps_ws_reserve(ps, p.bytes);
    if (rc) return rc;
    MuonIn a{};
    a.in = in; a.ld = in_ld; a.type = in_type; a.rows = rows; a.cols = cols; a.eps = eps;
    MuonArgs last{};
    last.to = out; last.to_ld = out_ld; last.to_type = out_type; last.to_vec = rows_allow(out, out_type, 8, out_ld, 8);
    return orthogonalize(ps, p, a, last, steps, (hipStream_t)stream);
}

extern "C" int muon_step(ps_handle ps, int32_t worker, int64_t first_key, int32_t batch, int32_t rows, int32_t dim, const void *grad, int32_t grad_type,
                         int64_t grad_ld, float lr, float momentum, int32_t nesterov, float weight_decay, int32_t steps, float eps, void *stream) {
    if (!ps || batch < 0 || rows < 0 || dim <= 0 || dim > ps->L / 2 || !is_element_type(grad_type) || steps < 1 || steps > 100 || !(eps >= 0.0f)) return PS_EINVAL;
    const int64_t keys = (int64_t)batch * rows;
    if (first_key < 0 || keys > ps->K || first_key > ps->K - keys) return PS_EINVAL;
    if (worker < -1 || worker >= ps->W) return PS_EWORKER;
    if (keys == 0) return PS_OK;
    if (!grad || grad_ld < dim) return PS_EINVAL;
    if (!sizes_allowed(batch, rows, dim)) return PS_ELIMIT;
    // (of numbers of 32 bits the products are, too, whatever the gradient's type)
    const MuonPlan p = muon_plan(ps, batch, rows, dim, true, true);
    int rc = dpaps_ws_reserve(ps, p.bytes);
    if (rc) return rc;
    hipStream_t st = (hipStream_t)stream;
    MuonIn a{};
    a.in = grad; a.ld = grad_ld; a.type = grad_type; a.rows = rows; a.cols = dim; a.eps = eps;
    a.val = ps->val; a.L = ps->L; a.first = first_key; a.mu = momentum; a.nesterov = nesterov != 0;
    MuonArgs last{};
    last.val = ps->val; last.L = ps->L; last.first = first_key; last.to_vec = ps->L % 4 == 0;
    last.keep = (float)(1.0 - (double)lr * weight_decay);
    last.step = (float)(lr * sqrt(rows > dim ? (double)rows / dim : 1.0));
    rc = orthogonalize(ps, p, a, last, steps, st);
    if (rc) return rc;
    TokenIds t;                                   // the keys first_key, first_key + 1, ...
    t.n = keys; t.first = first_key; t.count = keys;
    return dpaps_route_tokens(ps, worker, t, true, true, st);
}
