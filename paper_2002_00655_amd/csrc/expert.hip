// Products of grouped rows with matrices that lie in the server, and the matrices' gradients.
//
//   product    y_q = W_g(q) x_q,   or W'_g(q) x_q,        W_e: the rows of expert e, keys of the server
//   gradient   dW_e = sum over e's rows of dy_q x_q'
// Rows are taken in the groups' order, in tiles of rows of one group; where they lie stays as it is: they are read, and results are written, through that order.
// Products are of numbers of the rows' 16-bit type, with sums in 32 bits, where rows and results both have 16 bits: the server's numbers of 32 bits are rounded to it, which
// puts as much error on a result as its own rounding does (2^-9 or 2^-12 of each term at most, on average over the terms).  Else of numbers of 32 bits.
#include "experts.h"

namespace {

constexpr int BR = 128, BC = 128, TILE_THREADS = 256;

__device__ __forceinline__ int row_at(const RowGroups &g, int place, int32_t *err) {
    const int q = g.order[place];
    if (q >= 0 && q < g.n) return q;
    atomicExch(err, PS_EKEY);
    return -1;
}

template <class CT, class XT, bool TURNED>
__global__ __launch_bounds__(TILE_THREADS) void k_expert(ExpertArgs a, int32_t col_tiles, int32_t *err) {
    constexpr int KU = unit_of<CT>();
    __shared__ Vec<CT, KU> lds[2][(BR + BC) * UNITS];
    __shared__ int at[BR];                                           // the rows' numbers; -1: none
    __shared__ int off;
    look_for_all(err, &off);
    const RowTile t = row_tile(a.g, (int)(blockIdx.x / (uint32_t)col_tiles), BR);
    const int c0 = (int)(blockIdx.x % (uint32_t)col_tiles) * BC, tid = threadIdx.x;
    __syncthreads();
    if (off || t.rows == 0) return;
    if (tid < BR) at[tid] = tid < t.rows ? row_at(a.g, t.first + tid, err) : -1;
    __syncthreads();
    floatx16 acc[2][2] = {};
    const int wave = tid >> 6, wc = (wave & 1) * 64, wr = (wave >> 1) * 64, cols = a.N - c0;
    if (t.group < a.g.groups) {
        const float *w = a.w + (int64_t)t.group * a.each * a.L;
        KMajor<XT, CT, BR, TILE_THREADS> rows;
        rows.init([&](int r) { return at[r] < 0 ? nullptr : reinterpret_cast<const XT *>(a.x) + a.x_shared(at[r]) * a.x_stride; });
        const int steps = (a.K + step_of<CT>() - 1) / step_of<CT>();
        auto loop = [&](auto load, auto &columns) {
            rows.load(0, a.K);
            load(0);
            rows.put(lds[0]);
            columns.put(lds[0] + BR * UNITS);
            __syncthreads();
            for (int s = 0; s < steps; ++s) {
                if (s + 1 < steps) { rows.load(s + 1, a.K); load(s + 1); }
                step_products<CT, 2, 2>(lds[s & 1] + BR * UNITS, lds[s & 1], wc, wr, UNITS, acc);
                if (s + 1 < steps) { rows.put(lds[(s + 1) & 1]); columns.put(lds[(s + 1) & 1] + BR * UNITS); }
                __syncthreads();
            }
        };
        if constexpr (TURNED) {
            NMajor<float, CT, BC, TILE_THREADS> columns;
            loop([&](int s) { columns.load(s, a.K, cols, [&](int k) { return w + (int64_t)k * a.L + c0; }); }, columns);
        } else {
            KMajor<float, CT, BC, TILE_THREADS> columns;
            columns.init([&](int c) { return c < cols ? w + (int64_t)(c0 + c) * a.L : nullptr; });
            loop([&](int s) { columns.load(s, a.K); }, columns);
        }
    }
    const int l32 = tid & 31, h = (tid & 63) >> 5;
#pragma unroll
    for (int j = 0; j < 2; ++j) {
        const int r = wr + 32 * j + l32;
        if (at[r] < 0) continue;
        const int64_t to = (int64_t)(a.by_place ? t.first + r : at[r]) * a.out_stride;
#pragma unroll
        for (int i = 0; i < 2; ++i)
#pragma unroll
            for (int q = 0; q < 4; ++q) {
                const int c = wc + 32 * i + 8 * q + 4 * h;
                const Vec<float, 4> v = {acc[i][j][4 * q], acc[i][j][4 * q + 1], acc[i][j][4 * q + 2], acc[i][j][4 * q + 3]};
                if (c < cols) put_typed(a.out, a.out_type, to + c0 + c, a.scale * v, cols - c);
            }
    }
}

// Group blockIdx.y's sum of products, a tile of it.  Left and right in the order of the places of the group's rows.
template <class CT, class LT, class RT>
__global__ __launch_bounds__(TILE_THREADS) void k_outer(OuterArgs a, int32_t row_tiles, int32_t col_tiles, int32_t *err) {
    constexpr int KU = unit_of<CT>();
    __shared__ Vec<CT, KU> lds[2][(BR + BC) * UNITS];
    __shared__ int off;
    look_for_all(err, &off);
    const int tid = threadIdx.x, group = (int)(blockIdx.x / (uint32_t)(row_tiles * col_tiles)), tile = (int)(blockIdx.x % (uint32_t)(row_tiles * col_tiles));
    const int r0 = tile / col_tiles * BR, c0 = tile % col_tiles * BC;
    const int first = a.g.start(group), end = a.g.start(group + 1), K = end > first ? end - first : 0;
    __syncthreads();
    if (off) return;
    floatx16 acc[2][2] = {};
    const int wave = tid >> 6, wc = (wave & 1) * 64, wr = (wave >> 1) * 64;
    NMajor<LT, CT, BR, TILE_THREADS> left;
    NMajor<RT, CT, BC, TILE_THREADS> right;
    const int steps = (K + step_of<CT>() - 1) / step_of<CT>();
    // (a row out of range is left out: row 0 would be read in its place, so its number is looked at first)
    const auto number = [&](int p) {
        const int q = row_at(a.g, first + p, err);
        return q < 0 ? 0 : q;
    };
    const auto load = [&](int s) {
        left.load(s, K, a.rows - r0, [&](int p) {
            return reinterpret_cast<const LT *>(a.left) + (int64_t)(a.left_by_place ? first + p : a.left_shared(number(p))) * a.left_stride + r0;
        });
        right.load(s, K, a.cols - c0, [&](int p) { return reinterpret_cast<const RT *>(a.right) + (int64_t)a.right_shared(number(p)) * a.right_stride + c0; });
    };
    if (steps > 0) {
        load(0);
        left.put(lds[0]);
        right.put(lds[0] + BR * UNITS);
        __syncthreads();
    }
    for (int s = 0; s < steps; ++s) {
        if (s + 1 < steps) load(s + 1);
        step_products<CT, 2, 2>(lds[s & 1] + BR * UNITS, lds[s & 1], wc, wr, UNITS, acc);
        if (s + 1 < steps) { left.put(lds[(s + 1) & 1]); right.put(lds[(s + 1) & 1] + BR * UNITS); }
        __syncthreads();
    }
    const int l32 = tid & 31, h = (tid & 63) >> 5;
#pragma unroll
    for (int j = 0; j < 2; ++j) {
        const int r = r0 + wr + 32 * j + l32;
        if (r >= a.rows) continue;
#pragma unroll
        for (int i = 0; i < 2; ++i)
#pragma unroll
            for (int q = 0; q < 4; ++q) {
                const int c = c0 + wc + 32 * i + 8 * q + 4 * h;
                const Vec<float, 4> v = {acc[i][j][4 * q], acc[i][j][4 * q + 1], acc[i][j][4 * q + 2], acc[i][j][4 * q + 3]};
                if (c < a.cols) put_typed(a.out, a.out_type, ((int64_t)group * a.rows + r) * a.cols + c, v, a.cols - c);
            }
    }
}

// out_t = the sum of the rows t b .. t b + b - 1 of `in`, in that order
__global__ __launch_bounds__(256) void k_pair_sums(const float *in, int64_t n, int32_t b, int32_t N, void *out, int32_t out_type, int64_t out_stride, uint32_t P, double inv_P,
                                                   const int32_t *err) {
    if (*(volatile const int32_t *)err) return;
    const int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x, t = quotient(i, P, inv_P);
    if (t >= n) return;
    const int c = (int)(i - t * P) * 4, left = N - c;
    const float *p = in + t * b * N + c;
    Vec<float, 4> v = load_some<float, 4>(p, left);
    for (int j = 1; j < b; ++j) v = v + load_some<float, 4>(p + (int64_t)j * N, left);
    put_typed(out, out_type, t * out_stride + c, v, left);
}

int too_large(dpaps_ps *ps, const char *what) {
    ps->last_error = std::string(what) + ": too large for one launch";
    return PS_ELIMIT;
}

}  // namespace

int dpaps_expert_product(dpaps_ps *ps, const ExpertArgs &a, hipStream_t st) {
    const int32_t col_tiles = (a.N + BC - 1) / BC;
    const int64_t grid = row_tiles(a.g.n, a.g.groups, BR) * col_tiles;
    if (grid >= ((int64_t)1 << 24)) return too_large(ps, "expert_matmul");
#define EXPERT(CT, XT)                                                                                      \
    do {                                                                                                    \
        if (a.turned) k_expert<CT, XT, true><<<(unsigned)grid, TILE_THREADS, 0, st>>>(a, col_tiles, ps->err); \
        else k_expert<CT, XT, false><<<(unsigned)grid, TILE_THREADS, 0, st>>>(a, col_tiles, ps->err);         \
    } while (0)
    if (a.x_type == PS_F32) EXPERT(float, float);
    else if (a.x_type == PS_BF16) {
        if (a.precise) EXPERT(float, bf16_t);
        else EXPERT(bf16_t, bf16_t);
    } else {
        if (a.precise) EXPERT(float, f16_t);
        else EXPERT(f16_t, f16_t);
    }
#undef EXPERT
    PS_HIP(ps, hipGetLastError());
    return PS_OK;
}

int dpaps_outer_sums(dpaps_ps *ps, const OuterArgs &a, hipStream_t st) {
    const int32_t row_tiles = (a.rows + BR - 1) / BR, col_tiles = (a.cols + BC - 1) / BC;
    const int64_t grid = (int64_t)a.g.groups * row_tiles * col_tiles;
    if (grid >= ((int64_t)1 << 24)) return too_large(ps, "expert_grad");
#define OUTER(CT, LT, RT) k_outer<CT, LT, RT><<<(unsigned)grid, TILE_THREADS, 0, st>>>(a, row_tiles, col_tiles, ps->err)
    if (a.left_type == PS_F32) {
        if (a.right_type == PS_F32) OUTER(float, float, float);
        else if (a.right_type == PS_BF16) OUTER(float, float, bf16_t);
        else OUTER(float, float, f16_t);
    } else if (a.left_type == PS_BF16) OUTER(bf16_t, bf16_t, bf16_t);
    else OUTER(f16_t, f16_t, f16_t);
#undef OUTER
    PS_HIP(ps, hipGetLastError());
    return PS_OK;
}

extern "C" int expert_matmul(ps_handle ps, int32_t worker, int64_t first_key, int32_t num_experts, int32_t rows, int32_t dim, int32_t transposed,
                             const int32_t *order, const int32_t *offsets, int64_t n, const void *x, int32_t x_type, int64_t x_stride, int32_t x_pairs, void *out,
                             int32_t out_type, int64_t out_stride, int32_t out_pairs, void *stream) {
    if (!ps || num_experts <= 0 || rows <= 0 || dim <= 0 || dim > ps->L || !is_element_type(x_type) || !is_element_type(out_type)) return PS_EINVAL;
    if (worker < -1 || worker >= ps->W) return PS_EWORKER;
    const int64_t keys = (int64_t)num_experts * rows;
    if (first_key < 0 || keys > ps->K || first_key > ps->K - keys) return PS_EINVAL;
    RowGroups g;
    int rc = dpaps_row_groups(ps, order, offsets, num_experts, n, &g);
    if (rc) return rc;
    if (n == 0) return PS_OK;
    const int32_t K = transposed ? rows : dim, N = transposed ? dim : rows;
    if (x_pairs < 1 || out_pairs < 1 || n % x_pairs || n % out_pairs || !x || !out || x_stride < 0 || out_stride < N) return PS_EINVAL;
    hipStream_t st = (hipStream_t)stream;
    ExpertArgs a{};
    a.g = g; a.x = x; a.x_stride = x_stride; a.x_type = x_type; a.x_shared = Quotient(x_pairs);
    a.w = ps->val + first_key * ps->L; a.L = ps->L; a.each = rows; a.K = K; a.N = N; a.turned = transposed != 0;
    a.scale = 1.0f; a.precise = x_type == PS_F32 || out_type == PS_F32;
    a.out = out; a.out_stride = out_stride; a.out_type = out_type;
    if (out_pairs > 1) {
        rc = dpaps_ws_reserve(ps, (size_t)n * N * sizeof(float));
        if (rc) return rc;
        a.out = ps->ws; a.out_stride = N; a.out_type = PS_F32;
    }
    rc = dpaps_expert_product(ps, a, st);
    if (rc) return rc;
    if (out_pairs > 1) {
        const uint32_t P = (uint32_t)((N + 3) / 4);
        const int64_t blocks = ceil_div64(n / out_pairs * P, 256);
        if (blocks >= ((int64_t)1 << 24)) return too_large(ps, "expert_matmul");
        k_pair_sums<<<(unsigned)blocks, 256, 0, st>>>((const float *)ps->ws, n / out_pairs, out_pairs, N, out, out_type, out_stride, P, 1.0 / P, ps->err);
        PS_HIP(ps, hipGetLastError());
    }
    GroupKeys k;
    k.first_a = first_key; k.each = rows;
    return dpaps_route_groups(ps, worker, g, k, st);
}

extern "C" int expert_grad(ps_handle ps, int32_t num_experts, int32_t rows, int32_t dim, const int32_t *order, const int32_t *offsets, int64_t n,
                           const void *left, int64_t left_stride, int32_t left_pairs, const void *right, int64_t right_stride, int32_t right_pairs, int32_t type,
                           void *out, int32_t out_type, void *stream) {
    if (!ps || num_experts <= 0 || rows <= 0 || dim <= 0 || !is_element_type(type) || !is_element_type(out_type) || !out) return PS_EINVAL;
    RowGroups g;
    const int rc = dpaps_row_groups(ps, order, offsets, num_experts, n, &g);
    if (rc) return rc;
    if (left_pairs < 1 || right_pairs < 1 || n % left_pairs || n % right_pairs || (n > 0 && (!left || !right || left_stride < 0 || right_stride < 0))) return PS_EINVAL;
    OuterArgs a{};
    a.g = g; a.left = left; a.left_stride = left_stride; a.left_type = type; a.left_shared = Quotient(left_pairs);
    a.right = right; a.right_stride = right_stride; a.right_type = type; a.right_shared = Quotient(right_pairs);
    a.rows = rows; a.cols = dim; a.out = out; a.out_type = out_type;
    return dpaps_outer_sums(ps, a, (hipStream_t)stream);
}
