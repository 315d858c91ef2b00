// Matrices orthogonalised by Newton-Schulz products, and the step of weight matrices in the server that uses it.
//
// X_0 = D / (|D|_F + eps), then a number of times
//   A = X X',   P = a I + b A + c A^2,   X <- P X          (a, b, c below; X: n x m with n <= m, transposed if need be)
// which brings every singular value s to p(p(...p(s))), p(s) = a s + b s^3 + c s^5: near 1 after five steps, unless it
// was very small.
//
// All products are of fp16 numbers on the matrix cores with sums in 32 bits.  Numbers are held
//   SPLIT    as the sum of two fp16 numbers, high + low: 22 bits and a sign each way, an error of 2^-24 of the number, so what a float has;
//            a product is high high + high low + low high (what is left out is 2^-24 of it): three instructions;
//   single   as one fp16 number, where the result is rounded to bf16: an error of 2^-12, an eighth of what that rounding costs.
// fp16 holds few magnitudes, so every number is scaled by a power of two: the spectral norms of X, A and P are at most 1.21,
// 1.46 and 3.45 whatever D is (p of [0, 1.21] stays below 1.21), and so is every element; scaled they fill the
// upper end of the type, and what is lost at the lower end is 2^-39 of the norm or less.
// All three products have the form sum_k L[i][k] R[j][k] with both operands' rows contiguous in k: A = X X' and
// A^2 = A A' (A is symmetric) as they are, P X with X transposed - so X is written both ways.  Of the symmetric ones only the tiles on and below
// the diagonal are computed; a tile is written to its mirror place as well.
#include "elements.h"
#include "token_ids.h"

#include <cmath>

namespace {

constexpr float NS_A = 3.4445f, NS_B = -4.7750f, NS_C = 2.0315f;
constexpr float X_SCALE = 16384.0f, G_SCALE = 16384.0f, P_SCALE = 8192.0f;

typedef f16_t half8 __attribute__((ext_vector_type(8)));
typedef f16_t half4 __attribute__((ext_vector_type(4)));
typedef float floatx16 __attribute__((ext_vector_type(16)));
typedef float floatx4 __attribute__((ext_vector_type(4)));

inline size_t up256(size_t x) { return (x + 255) / 256 * 256; }

// A matrix in scratch: element (r, k) of a row of ld elements.  SPLIT: 8 high parts, then their 8 low parts, and so on.
template <bool SPLIT> __device__ __forceinline__ int64_t place(int64_t r, int k, int ld) {
    return SPLIT ? r * (2 * (int64_t)ld) + (k >> 3) * 16 + (k & 7) : r * (int64_t)ld + k;
}

// ---- the norm, and the momentum -------------------------------------------------------------------------------------
constexpr int NORM_BLOCKS = 128;             // workgroups per matrix at most

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
__device__ __forceinline__ float element(const MuonIn &a, int64_t row, int col) {
    const int64_t i = row * a.ld + col;
    if (a.type == PS_F32) return reinterpret_cast<const float *>(a.in)[i];
    return a.type == PS_BF16 ? (float)reinterpret_cast<const bf16_t *>(a.in)[i] : (float)reinterpret_cast<const f16_t *>(a.in)[i];
}

// The sum of a workgroup's 256 numbers, in a fixed order; the same in all threads.
__device__ __forceinline__ double sum_of_256(double x) {
    __shared__ double lds[4];
    for (int d = 32; d > 0; d >>= 1) x += __shfl_xor(x, d);
    if ((threadIdx.x & 63) == 0) lds[threadIdx.x >> 6] = x;
    __syncthreads();
    return (lds[0] + lds[1]) + (lds[2] + lds[3]);
}

// Of matrix blockIdx.y: sums of squares in 64 bits (no number of 32 bits overflows there); of a step, first M <- mu M + G, and
// what is orthogonalised, D = G + mu M (Nesterov) or M.
__global__ __launch_bounds__(256) void k_muon_norm(MuonIn a, const int32_t *err) {
    if (a.val && *(volatile const int32_t *)err) return;
    const int64_t row0 = (int64_t)blockIdx.y * a.rows;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    double s = 0.0;
    for (int r = blockIdx.x * 4 + wave; r < a.rows; r += a.blocks * 4) {
        for (int c = lane; c < a.cols; c += 64) {
            float x = element(a, row0 + r, c);
            if (a.val) {
                float *m = a.val + (a.first + row0 + r) * a.L + a.cols + c;
                const float moment = a.mu * *m + x;
                *m = moment;
                x = a.nesterov ? x + a.mu * moment : moment;
                a.d[(row0 + r) * a.cols + c] = x;
            }
            s += (double)x * (double)x;
        }
    }
    s = sum_of_256(s);
    if (threadIdx.x == 0) a.squares[(int64_t)blockIdx.y * NORM_BLOCKS + blockIdx.x] = s;
}

// X_0 both ways, zero where the padded matrices go on.  A norm that is no number, or infinite, makes all of the matrix NaN, as the division would.
template <bool SPLIT>
__device__ __forceinline__ void put8(f16_t *to, int64_t r, int k, int ld, const float (&v)[8]) {
    half8 hi, lo;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        hi[i] = (f16_t)v[i];
        lo[i] = (f16_t)(v[i] - (float)hi[i]);
    }
    f16_t *p = to + place<SPLIT>(r, k, ld);
    *reinterpret_cast<half8 *>(p) = hi;
    if constexpr (SPLIT) *reinterpret_cast<half8 *>(p + 8) = lo;
}
template <bool SPLIT>
__global__ __launch_bounds__(256) void k_muon_scale(MuonIn a, bool tall, int np, int mp, f16_t *x, f16_t *xt) {
    __shared__ float tile[64][65];
    const int64_t b = blockIdx.z;
    const double square = sum_of_256((int)threadIdx.x < a.blocks ? a.squares[b * NORM_BLOCKS + threadIdx.x] : 0.0);
    const float norm = (float)sqrt(square);
    const float f = norm <= 3.0e38f ? X_SCALE / (norm + a.eps) : __builtin_nanf("");
    const int i0 = blockIdx.y * 64, j0 = blockIdx.x * 64;                     // of X
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int r0 = tall ? j0 : i0, c0 = tall ? i0 : j0;                       // of the matrix itself
    for (int r = wave; r < 64; r += 4) {
        const int rr = r0 + r, cc = c0 + lane;
        const float v = rr < a.rows && cc < a.cols ? f * element(a, b * a.rows + rr, cc) : 0.0f;
        if (tall) tile[lane][r] = v; else tile[r][lane] = v;
    }
    __syncthreads();
    x += b * (int64_t)np * mp * (SPLIT ? 2 : 1);
    xt += b * (int64_t)np * mp * (SPLIT ? 2 : 1);
    for (int q = threadIdx.x; q < 512; q += 256) {
        const int r = q >> 3, k = (q & 7) * 8;
        float v[8], w[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) { v[i] = tile[r][k + i]; w[i] = tile[k + i][r]; }
        put8<SPLIT>(x, i0 + r, j0 + k, mp, v);
        put8<SPLIT>(xt, j0 + r, i0 + k, np, w);
    }
}

// ---- the products ---------------------------------------------------------------------------------------------------
constexpr int CHAIN = 8;                         // stages whose products one chain of matrix instructions adds (numbers of 24 bits)
enum MuonProduct { MUON_GRAM, MUON_POLY, MUON_APPLY, MUON_LAST };
struct MuonArgs {
    const f16_t *lhs, *rhs;                      // rows of K numbers
    int64_t lhs_size, rhs_size, out_size;        // of one matrix, in elements as they are stored
    int32_t K, tiles_i, tiles_j;
    f16_t *out; int32_t out_ld;                  // GRAM: A, POLY: P, APPLY: X
    f16_t *out_t; int32_t out_t_ld;              // APPLY: X transposed
    // LAST: the result
    void *to; int64_t to_ld; int32_t to_type, tall, n, m;
    float *val; int64_t L, first; float keep, step;    // of a step: W <- keep W - step X
};

// C[i][j] = sum_k L[i][k] R[j][k], a tile of TILE x TILE per workgroup of four wavefronts, each a quarter of it in 32 x 32 pieces
// (v_mfma_f32_32x32x16_f16).  128 bytes of each row go through LDS at a time, straight from memory, two stages: the next
// one is on its way while this one is multiplied.  A row's eight pieces of 16 bytes are exchanged by the row's number, so that
// the 8 lanes that LDS serves together read different banks.
template <int TILE, bool SPLIT, int MODE>
__global__ __launch_bounds__(256) void k_muon_product(MuonArgs a, const int32_t *err) {
    constexpr int W = TILE / 2, F = W / 32, STAGE = TILE * 128, LOADS = TILE * 8 / 256, BK = SPLIT ? 32 : 64, S = SPLIT ? 2 : 1;
    __shared__ __attribute__((aligned(16))) unsigned char lds[2][2][STAGE];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6);
    const int64_t b = blockIdx.y;
    int ti, tj;
    if constexpr (MODE == MUON_GRAM || MODE == MUON_POLY) {                   // on and below the diagonal, row by row
        ti = (int)((sqrtf(8.0f * (float)blockIdx.x + 1.0f) - 1.0f) * 0.5f);
        while ((ti + 1) * (ti + 2) / 2 <= (int)blockIdx.x) ++ti;
        while (ti * (ti + 1) / 2 > (int)blockIdx.x) --ti;
        tj = (int)blockIdx.x - ti * (ti + 1) / 2;
    } else {
        ti = (int)blockIdx.x % a.tiles_i;
        tj = (int)blockIdx.x / a.tiles_i;
    }
    const int64_t row_bytes = (int64_t)a.K * S * 2;
    const char *lhs = reinterpret_cast<const char *>(a.lhs + b * a.lhs_size) + (int64_t)ti * TILE * row_bytes;
    const char *rhs = reinterpret_cast<const char *>(a.rhs + b * a.rhs_size) + (int64_t)tj * TILE * row_bytes;
    // piece q of a stage: row q / 8, its place q % 8 in LDS holds the row's piece (q % 8) ^ (row % 8)
    int64_t from[LOADS];
#pragma unroll
    for (int i = 0; i < LOADS; ++i) {
        const int q = (i * 4 + wave) * 64 + lane, row = q >> 3;
        from[i] = row * row_bytes + (((q & 7) ^ (row & 7)) << 4);
    }
    const auto load = [&](int stage, int kt) {
#pragma unroll
        for (int i = 0; i < LOADS; ++i) {
            const int at = (i * 4 + wave) * 1024;
            __builtin_amdgcn_global_load_lds((const __attribute__((address_space(1))) void *)(lhs + from[i] + (int64_t)kt * 128),
                                             (__attribute__((address_space(3))) void *)(&lds[stage][0][at]), 16, 0, 0);
            __builtin_amdgcn_global_load_lds((const __attribute__((address_space(1))) void *)(rhs + from[i] + (int64_t)kt * 128),
                                             (__attribute__((address_space(3))) void *)(&lds[stage][1][at]), 16, 0, 0);
        }
    };
    const int wi = (wave >> 1) * W, wj = (wave & 1) * W, l32 = lane & 31, h = lane >> 5;
    const auto piece = [&](int stage, int side, int row, int c) {
        return *reinterpret_cast<const half8 *>(&lds[stage][side][row * 128 + ((c ^ (row & 7)) << 4)]);
    };
    floatx16 acc[F][F];
#pragma unroll
    for (int i = 0; i < F; ++i)
#pragma unroll
        for (int j = 0; j < F; ++j) acc[i][j] = floatx16{};
    // The matrix instruction does not round its sums to the nearest: a chain of them loses up to a unit in the last place at each link, always the
    // same way.  (One row of 5,000 in a chain of 313: an error of 72 units of 2^-24.)  So with numbers of 24 bits the chains are cut
    // and their sums added by ordinary additions.
    floatx16 total[SPLIT ? F : 1][SPLIT ? F : 1];
    if constexpr (SPLIT) {
#pragma unroll
        for (int i = 0; i < F; ++i)
#pragma unroll
            for (int j = 0; j < F; ++j) total[i][j] = floatx16{};
    }
    const int kts = a.K / BK;
    load(0, 0);
    for (int kt = 0; kt < kts; ++kt) {
        __builtin_amdgcn_s_waitcnt(0x0f70);                                    // vmcnt(0): this wavefront's part of the stage is there
        __syncthreads();                                                       // and so are the others'; the other stage has been read
        if (kt + 1 < kts) load((kt + 1) & 1, kt + 1);
        const int st = kt & 1;
#pragma unroll
        for (int s = 0; s < BK / 16; ++s) {
            half8 l[F][S], r[F][S];
#pragma unroll
            for (int f = 0; f < F; ++f)
#pragma unroll
                for (int e = 0; e < S; ++e) {
                    const int c = SPLIT ? 4 * s + 2 * h + e : 2 * s + h;
                    l[f][e] = piece(st, 0, wi + f * 32 + l32, c);
                    r[f][e] = piece(st, 1, wj + f * 32 + l32, c);
                }
#pragma unroll
            for (int i = 0; i < F; ++i)
#pragma unroll
                for (int j = 0; j < F; ++j) {
                    if constexpr (SPLIT) {
                        acc[i][j] = __builtin_amdgcn_mfma_f32_32x32x16_f16(l[i][1], r[j][0], acc[i][j], 0, 0, 0);
                        acc[i][j] = __builtin_amdgcn_mfma_f32_32x32x16_f16(l[i][0], r[j][1], acc[i][j], 0, 0, 0);
                    }
                    acc[i][j] = __builtin_amdgcn_mfma_f32_32x32x16_f16(l[i][0], r[j][0], acc[i][j], 0, 0, 0);
                }
        }
        if constexpr (SPLIT) {
            if ((kt & (CHAIN - 1)) == CHAIN - 1) {
#pragma unroll
                for (int i = 0; i < F; ++i)
#pragma unroll
                    for (int j = 0; j < F; ++j) { total[i][j] = total[i][j] + acc[i][j]; acc[i][j] = floatx16{}; }
            }
        }
    }
    if constexpr (SPLIT) {
#pragma unroll
        for (int i = 0; i < F; ++i)
#pragma unroll
            for (int j = 0; j < F; ++j) acc[i][j] = total[i][j] + acc[i][j];
    }
    // the result: of a 32 x 32 piece a lane has column lane % 32, rows 8 g + 4 (lane / 32) + 0..3 for g = 0..3
    if (MODE == MUON_LAST && a.val && *(volatile const int32_t *)err) return;
#pragma unroll
    for (int fi = 0; fi < F; ++fi)
#pragma unroll
        for (int fj = 0; fj < F; ++fj)
#pragma unroll
            for (int g = 0; g < 4; ++g) {
                const int i = ti * TILE + wi + fi * 32 + 8 * g + 4 * h, j = tj * TILE + wj + fj * 32 + l32;
                float v[4];
#pragma unroll
                for (int e = 0; e < 4; ++e) v[e] = acc[fi][fj][g * 4 + e];
                if constexpr (MODE == MUON_LAST) {
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        if (i + e >= a.n || j >= a.m) continue;
                        const float x = v[e] * (1.0f / (P_SCALE * X_SCALE));
                        const int64_t row = b * (a.tall ? a.m : a.n) + (a.tall ? j : i + e), col = a.tall ? i + e : j;
                        if (a.val) {
                            float *w = a.val + (a.first + row) * a.L + col;
                            *w = a.keep * *w - a.step * x;
                        } else if (a.to_type == PS_F32) reinterpret_cast<float *>(a.to)[row * a.to_ld + col] = x;
                        else if (a.to_type == PS_BF16) reinterpret_cast<bf16_t *>(a.to)[row * a.to_ld + col] = (bf16_t)x;
                        else reinterpret_cast<f16_t *>(a.to)[row * a.to_ld + col] = (f16_t)x;
                    }
                } else {
                    f16_t *out = a.out + b * a.out_size;
                    if constexpr (MODE == MUON_GRAM) {
#pragma unroll
                        for (int e = 0; e < 4; ++e) v[e] *= G_SCALE / (X_SCALE * X_SCALE);
                    }
                    if constexpr (MODE == MUON_APPLY) {
#pragma unroll
                        for (int e = 0; e < 4; ++e) v[e] *= 1.0f / P_SCALE;
                    }
                    if constexpr (MODE == MUON_POLY) {
                        // A at these places (it is symmetric: four in a row)
                        const f16_t *p = a.lhs + b * a.lhs_size + place<SPLIT>(j, i, a.K);
                        const half4 hi = *reinterpret_cast<const half4 *>(p);
                        half4 lo = {};
                        if constexpr (SPLIT) lo = *reinterpret_cast<const half4 *>(p + 8);
#pragma unroll
                        for (int e = 0; e < 4; ++e) {
                            const float g1 = SPLIT ? (float)hi[e] + (float)lo[e] : (float)hi[e];
                            v[e] = v[e] * (NS_C * P_SCALE / (G_SCALE * G_SCALE)) + g1 * (NS_B * P_SCALE / G_SCALE) + (i + e == j ? NS_A * P_SCALE : 0.0f);
                        }
                    }
                    half4 hi, lo;
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        hi[e] = (f16_t)v[e];
                        lo[e] = (f16_t)(v[e] - (float)hi[e]);
                        f16_t *p = out + place<SPLIT>(i + e, j, a.out_ld);
                        p[0] = hi[e];
                        if constexpr (SPLIT) p[8] = lo[e];
                    }
                    f16_t *t = nullptr;                                       // the mirror place, or X transposed
                    if constexpr (MODE == MUON_APPLY) t = a.out_t + b * a.out_size + place<SPLIT>(j, i, a.out_t_ld);
                    else if (ti != tj) t = out + place<SPLIT>(j, i, a.out_ld);
                    if (t) {
                        *reinterpret_cast<half4 *>(t) = hi;
                        if constexpr (SPLIT) *reinterpret_cast<half4 *>(t + 8) = lo;
                    }
                }
            }
}

// ---- host -----------------------------------------------------------------------------------------------------------
struct MuonPlan {
    int32_t batch, n, m, tile, np, mp, blocks;
    bool tall, split;
    size_t off_d, off_x, off_xt[2], off_g, off_p, bytes;
};
MuonPlan muon_plan(int32_t batch, int32_t rows, int32_t cols, bool split, bool step) {
    MuonPlan p{};
    p.batch = batch; p.tall = rows > cols; p.split = split;
    p.n = p.tall ? cols : rows; p.m = p.tall ? rows : cols;
    p.tile = 64;
    if (ceil_div64(p.n, 128) * ceil_div64(p.n, 128) * batch >= 128) p.tile = 128;
    p.np = (int32_t)(ceil_div64(p.n, p.tile) * p.tile); p.mp = (int32_t)(ceil_div64(p.m, p.tile) * p.tile);
    p.blocks = (int32_t)(ceil_div64(rows, 4) < NORM_BLOCKS ? ceil_div64(rows, 4) : NORM_BLOCKS);
    const size_t size = split ? 4 : 2, nm = (size_t)batch * p.np * p.mp * size, nn = (size_t)batch * p.np * p.np * size;
    p.off_d = up256((size_t)batch * NORM_BLOCKS * sizeof(double));
    p.off_x = p.off_d + (step ? up256((size_t)batch * rows * cols * sizeof(float)) : 0);
    p.off_xt[0] = p.off_x + up256(nm);
    p.off_xt[1] = p.off_xt[0] + up256(nm);
    p.off_g = p.off_xt[1] + up256(nm);
    p.off_p = p.off_g + up256(nn);
    p.bytes = p.off_p + up256(nn);
    return p;
}

template <int TILE, bool SPLIT, int MODE>
int product(dpaps_ps *ps, const MuonArgs &a, int32_t batch, hipStream_t st) {
    const int64_t tiles = MODE == MUON_GRAM || MODE == MUON_POLY ? (int64_t)a.tiles_i * (a.tiles_i + 1) / 2 : (int64_t)a.tiles_i * a.tiles_j;
    k_muon_product<TILE, SPLIT, MODE><<<dim3((unsigned)tiles, (unsigned)batch), 256, 0, st>>>(a, ps->err);
    PS_HIP(ps, hipGetLastError());
    return PS_OK;
}

template <int TILE, bool SPLIT>
int iterate(dpaps_ps *ps, const MuonPlan &p, MuonIn in, MuonArgs last, int32_t steps, hipStream_t st) {
    char *ws = (char *)ps->ws;
    f16_t *x = (f16_t *)(ws + p.off_x), *xt = (f16_t *)(ws + p.off_xt[0]), *xt_next = (f16_t *)(ws + p.off_xt[1]), *g = (f16_t *)(ws + p.off_g), *q = (f16_t *)(ws + p.off_p);
    const int64_t S = SPLIT ? 2 : 1, nm = (int64_t)p.np * p.mp * S, nn = (int64_t)p.np * p.np * S;
    k_muon_scale<SPLIT><<<dim3((unsigned)(p.mp / 64), (unsigned)(p.np / 64), (unsigned)p.batch), 256, 0, st>>>(in, p.tall, p.np, p.mp, x, xt);
    PS_HIP(ps, hipGetLastError());
    for (int s = 0; s < steps; ++s) {
        MuonArgs a{};
        a.tiles_i = p.np / TILE; a.tiles_j = p.mp / TILE;
        a.lhs = a.rhs = x; a.lhs_size = a.rhs_size = nm; a.K = p.mp; a.out = g; a.out_ld = p.np; a.out_size = nn;
        int rc = product<TILE, SPLIT, MUON_GRAM>(ps, a, p.batch, st);
        if (rc) return rc;
        a.lhs = a.rhs = g; a.lhs_size = a.rhs_size = nn; a.K = p.np; a.out = q;
        rc = product<TILE, SPLIT, MUON_POLY>(ps, a, p.batch, st);
        if (rc) return rc;
        MuonArgs b = s + 1 == steps ? last : a;
        b.tiles_i = a.tiles_i; b.tiles_j = a.tiles_j; b.K = p.np;
        b.lhs = q; b.lhs_size = nn; b.rhs = xt; b.rhs_size = nm;
        if (s + 1 == steps) rc = product<TILE, SPLIT, MUON_LAST>(ps, b, p.batch, st);
        else {
            // (X transposed is read by other workgroups while it is written: into the other place; X itself is not)
            b.out = x; b.out_ld = p.mp; b.out_t = xt_next; b.out_t_ld = p.np; b.out_size = nm;
            rc = product<TILE, SPLIT, MUON_APPLY>(ps, b, p.batch, st);
        }
        if (rc) return rc;
        f16_t *const t = xt; xt = xt_next; xt_next = t;
    }
    return PS_OK;
}

int orthogonalize(dpaps_ps *ps, const MuonPlan &p, MuonIn in, MuonArgs last, int32_t steps, hipStream_t st) {
    char *ws = (char *)ps->ws;
    in.squares = (double *)ws;
    in.blocks = p.blocks;
    if (in.val) in.d = (float *)(ws + p.off_d);
    k_muon_norm<<<dim3((unsigned)p.blocks, (unsigned)p.batch), 256, 0, st>>>(in, ps->err);
    PS_HIP(ps, hipGetLastError());
    if (in.val) { in.in = in.d; in.ld = in.cols; in.type = PS_F32; }
    last.n = p.n; last.m = p.m; last.tall = p.tall;
    if (p.split) return p.tile == 128 ? iterate<128, true>(ps, p, in, last, steps, st) : iterate<64, true>(ps, p, in, last, steps, st);
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
    const MuonPlan p = muon_plan(batch, rows, cols, out_type != PS_BF16, false);
    const int rc = dpaps_ws_reserve(ps, p.bytes);
    if (rc) return rc;
    MuonIn a{};
    a.in = in; a.ld = in_ld; a.type = in_type; a.rows = rows; a.cols = cols; a.eps = eps;
    MuonArgs last{};
    last.to = out; last.to_ld = out_ld; last.to_type = out_type;
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
    const MuonPlan p = muon_plan(batch, rows, dim, true, true);
    int rc = dpaps_ws_reserve(ps, p.bytes);
    if (rc) return rc;
    hipStream_t st = (hipStream_t)stream;
    MuonIn a{};
    a.in = grad; a.ld = grad_ld; a.type = grad_type; a.rows = rows; a.cols = dim; a.eps = eps;
    a.val = ps->val; a.L = ps->L; a.first = first_key; a.mu = momentum; a.nesterov = nesterov != 0;
    MuonArgs last{};
    last.val = ps->val; last.L = ps->L; last.first = first_key;
    last.keep = (float)(1.0 - (double)lr * weight_decay);
    last.step = (float)(lr * sqrt(rows > dim ? (double)rows / dim : 1.0));
    rc = orthogonalize(ps, p, a, last, steps, st);
    if (rc) return rc;
    TokenIds t;                                   // the keys first_key, first_key + 1, ...
    t.n = keys; t.first = first_key; t.count = keys;
    return dpaps_route_tokens(ps, worker, t, true, true, st);
}
