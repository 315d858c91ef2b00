// A shared projection with a low-rank adapter per row, and its gradients.
//
//   y_p = W x_p + s B_a (A_a x_p)               a: the adapter that row p names; W x_p alone where it names none
//   dx_p = W' dy_p + s A_a' (B_a' dy_p)
//   dA_a = s sum over a's rows of (B_a' dy_p) x_p',     dB_a' = s sum of (A_a x_p) dy_p'
// W, the rows of A_a and the rows of B_a' (both `rank` keys of an adapter) lie in the server.  The low-rank numbers s A_a x_p and s B_a' dy_p are worked out first, in the
// order of the groups, and kept in 32 bits; the second launch goes on, after the sum over W's side, with those of the adapters of its rows.
#include "experts.h"

#include <algorithm>

namespace {

template <class CT, class XT, bool TURNED, class T>
__global__ __launch_bounds__(T::THREADS) void k_adapter(AdapterArgs a, int32_t col_tiles, int32_t *err) {
    constexpr int KU = unit_of<CT>(), BR = T::ROWS, BC = T::COLS;
    __shared__ Vec<CT, KU> lds[2][(BR + BC) * UNITS];
    __shared__ int at[BR];
    __shared__ int off;
    look_for_all(err, &off);
    const int first = (int)(blockIdx.x / (uint32_t)col_tiles) * BR, count = a.g.n - first < BR ? a.g.n - first : BR;
    const int c0 = (int)(blockIdx.x % (uint32_t)col_tiles) * BC, tid = threadIdx.x;
    for (int r = tid; r < BR; r += T::THREADS) at[r] = r < count ? row_at(a.g, first + r, err) : -1;
    __syncthreads();
    if (off) return;
    floatx16 acc[T::MC][T::MR] = {};
    const int wave = tid >> 6, wc = wave % T::WC * 32 * T::MC, wr = wave / T::WC * 32 * T::MR, cols = a.N - c0;
    const auto loop = [&](int K, auto load_rows, auto &rows, auto load_columns, auto &columns) {
        const int steps = (K + step_of<CT>() - 1) / step_of<CT>();
        load_rows(0);
        load_columns(0);
        rows.put(lds[0]);
        columns.put(lds[0] + BR * UNITS);
        __syncthreads();
        for (int s = 0; s < steps; ++s) {
            if (s + 1 < steps) { load_rows(s + 1); load_columns(s + 1); }
            const int left = K - s * step_of<CT>(), units = (left + KU - 1) / KU;
            step_products<CT, T::MC, T::MR>(lds[s & 1] + BR * UNITS, lds[s & 1], wc, wr, units < UNITS ? units : UNITS, acc);
            if (s + 1 < steps) { rows.put(lds[(s + 1) & 1]); columns.put(lds[(s + 1) & 1] + BR * UNITS); }
            __syncthreads();
        }
    };
    {
        KMajor<XT, CT, BR, T::THREADS> rows;
        rows.init([&](int r) { return at[r] < 0 ? nullptr : reinterpret_cast<const XT *>(a.x) + (int64_t)at[r] * a.x_stride; });
        if constexpr (TURNED) {
            NMajor<float, CT, BC, T::THREADS> columns;
            loop(a.K, [&](int s) { rows.load(s, a.K); }, rows, [&](int s) { columns.load(s, a.K, cols, [&](int k) { return a.w + (int64_t)k * a.L + c0; }); }, columns);
        } else {
            KMajor<float, CT, BC, T::THREADS> columns;
            columns.init([&](int c) { return c < cols ? a.w + (int64_t)(c0 + c) * a.L : nullptr; });
            loop(a.K, [&](int s) { rows.load(s, a.K); }, rows, [&](int s) { columns.load(s, a.K); }, columns);
        }
    }
    // the adapters of the tile's rows, one after the other: the rows of others are zero
    for (int e = row_tile(a.g, first, 1).group; e < a.g.groups; ++e) {
        const int lo = a.g.start(e) - first, hi = a.g.start(e + 1) - first;
        if (lo >= count) break;
        if (hi <= lo || hi <= 0) continue;
        KMajor<float, CT, BR, T::THREADS> rows;
        rows.init([&](int r) { return r >= lo && r < hi ? a.low + (int64_t)(first + r) * a.low_stride : nullptr; });
        NMajor<float, CT, BC, T::THREADS> columns;
        const float *b = a.b + (int64_t)e * a.rank * a.L + c0;
        loop(a.rank, [&](int s) { rows.load(s, a.rank); }, rows, [&](int s) { columns.load(s, a.rank, cols, [&](int k) { return b + (int64_t)k * a.L; }); }, columns);
    }
    const int l32 = tid & 31, h = (tid & 63) >> 5;
#pragma unroll
    for (int j = 0; j < T::MR; ++j) {
        const int r = wr + 32 * j + l32;
        if (at[r] < 0) continue;
        const int64_t to = (int64_t)at[r] * a.out_stride;
#pragma unroll
        for (int i = 0; i < T::MC; ++i)
#pragma unroll
            for (int q = 0; q < 4; ++q) {
                const int c = wc + 32 * i + 8 * q + 4 * h;
                const Vec<float, 4> v = {acc[i][j][4 * q], acc[i][j][4 * q + 1], acc[i][j][4 * q + 2], acc[i][j][4 * q + 3]};
                if (c < cols) put_typed(a.out, a.out_type, to + c0 + c, v, cols - c);
            }
    }
}

// Few rows, of any adapters: the low-rank part is added to a row's sums number by number.
template <class CT, class XT, bool TURNED, int MT>
__global__ __launch_bounds__((FewRows<CT, XT, TURNED, MT>::THREADS)) void k_adapter_few(AdapterArgs a, int32_t col_tiles, int32_t *err) {
    typedef FewRows<CT, XT, TURNED, MT> F;
    __shared__ float sums[F::SUMS];
    __shared__ int at[16 * MT], group[16 * MT];
    __shared__ int off;
    look_for_all(err, &off);
    const int first = (int)(blockIdx.x / (uint32_t)col_tiles) * 16 * MT, count = a.g.n - first < 16 * MT ? a.g.n - first : 16 * MT;
    const int c0 = (int)(blockIdx.x % (uint32_t)col_tiles) * F::COLS, tid = threadIdx.x;
    if (tid < 16 * MT) {
        at[tid] = tid < count ? row_at(a.g, first + tid, err) : -1;
        group[tid] = tid < count ? a.group_of[first + tid] : a.g.groups;
    }
    __syncthreads();
    if (off) return;
    F f;
    f.run(a.w, a.L, a.K, c0, a.N, [&](int r) { return reinterpret_cast<const XT *>(a.x) + (int64_t)(at[r] < 0 ? 0 : at[r]) * a.x_stride; });
    f.put(sums);
    __syncthreads();
    for (int p = tid; p < F::PIECES; p += F::THREADS) {
        const int r = F::row_of(p), c = F::col_of(p), left = a.N - c0 - c;
        if (at[r] < 0 || left <= 0) continue;
        Vec<float, 4> v = F::sum(sums, p);
        if ((uint32_t)group[r] < (uint32_t)a.g.groups) {              // (whatever the offsets are)
            const float *low = a.low + (int64_t)(first + r) * a.low_stride, *b = a.b + (int64_t)group[r] * a.rank * a.L + c0 + c;
            Vec<float, 4> w = {};
#pragma unroll 8
            for (int i = 0; i < a.rank; ++i) w = w + low[i] * load_some<float, 4>(b + (int64_t)i * a.L, left);
            v = v + w;
        }
        put_typed(a.out, a.out_type, (int64_t)at[r] * a.out_stride + c0 + c, v, left);
    }
}

template <class CT, class XT, bool TURNED, class T> int tiles_of(dpaps_ps *ps, const AdapterArgs &a, hipStream_t st) {
    const int32_t col_tiles = (a.N + T::COLS - 1) / T::COLS;
    const int64_t grid = ceil_div64(a.g.n, T::ROWS) * col_tiles;
    if (grid >= ((int64_t)1 << 24)) { ps->last_error = "adapters: too large for one launch"; return PS_ELIMIT; }
    k_adapter<CT, XT, TURNED, T><<<(unsigned)grid, T::THREADS, 0, st>>>(a, col_tiles, ps->err);
    PS_HIP(ps, hipGetLastError());
    return PS_OK;
}
template <class CT, class XT, bool TURNED, int MT> int few_of(dpaps_ps *ps, const AdapterArgs &a, hipStream_t st) {
    typedef FewRows<CT, XT, TURNED, MT> F;
    const int32_t col_tiles = (a.N + F::COLS - 1) / F::COLS;
    k_adapter_few<CT, XT, TURNED, MT><<<(unsigned)(ceil_div64(a.g.n, 16 * MT) * col_tiles), F::THREADS, 0, st>>>(a, col_tiles, ps->err);
    PS_HIP(ps, hipGetLastError());
    return PS_OK;
}
template <class CT, class XT, bool TURNED> int product_of(dpaps_ps *ps, const AdapterArgs &a, hipStream_t st) {
    if (a.g.n <= 16) return few_of<CT, XT, TURNED, 1>(ps, a, st);
    if (a.g.n <= 128) return few_of<CT, XT, TURNED, 2>(ps, a, st);
    if (ceil_div64(a.g.n, 128) * ceil_div64(a.N, 128) < 2 * ps->num_cu) return tiles_of<CT, XT, TURNED, Tile64>(ps, a, st);
    return tiles_of<CT, XT, TURNED, Tile128>(ps, a, st);
}
template <class CT, class XT> int product_either(dpaps_ps *ps, const AdapterArgs &a, hipStream_t st) {
    return a.turned ? product_of<CT, XT, true>(ps, a, st) : product_of<CT, XT, false>(ps, a, st);
}
int product(dpaps_ps *ps, const AdapterArgs &a, hipStream_t st) {
    const bool precise = a.x_type == PS_F32 || a.out_type == PS_F32;
    if (a.x_type == PS_F32) return product_either<float, float>(ps, a, st);
    if (a.x_type == PS_BF16) return precise ? product_either<float, bf16_t>(ps, a, st) : product_either<bf16_t, bf16_t>(ps, a, st);
    return precise ? product_either<float, f16_t>(ps, a, st) : product_either<f16_t, f16_t>(ps, a, st);
}

// low_p = s M_a x_p in 32 bits, of the rows at the places of the order
int low_numbers(dpaps_ps *ps, const RowGroups &g, const void *x, int32_t type, int64_t stride, int32_t K, const float *m, int32_t rank, float scale, bool precise, float *low,
                int64_t low_stride, int32_t *group_of, hipStream_t st) {
    ExpertArgs a{};
    a.g = g; a.x = x; a.x_stride = stride; a.x_type = type; a.w = m; a.L = ps->L; a.each = rank; a.K = K; a.N = rank; a.scale = scale;
    a.out = low; a.out_stride = low_stride; a.out_type = PS_F32; a.by_place = 1; a.precise = precise; a.group_of = group_of;
    return dpaps_expert_product(ps, a, st);
}

// What both calls check.
int adapter_call(dpaps_ps *ps, int32_t worker, int64_t first_key, int32_t rows, int32_t dim, int64_t first_a, int64_t first_b, int32_t num_adapters, int32_t rank,
                 const int32_t *order, const int32_t *offsets, int64_t n, RowGroups *g) {
    if (!ps || rows <= 0 || rows > ps->L || dim <= 0 || dim > ps->L || rank <= 0 || num_adapters <= 0) return PS_EINVAL;
    if (worker < -1 || worker >= ps->W) return PS_EWORKER;
    const int64_t each = (int64_t)num_adapters * rank;
    if (first_key < 0 || rows > ps->K || first_key > ps->K - rows || each > ps->K || first_a < 0 || first_a > ps->K - each || first_b < 0 || first_b > ps->K - each) return PS_EINVAL;
    return dpaps_row_groups(ps, order, offsets, num_adapters, n, g);
}
int64_t low_stride(int32_t rank) { return (rank + 3) / 4 * 4; }

}  // namespace

extern "C" int adapter_matmul(ps_handle ps, int32_t worker, int64_t first_key, int32_t rows, int32_t dim, int64_t first_a, int64_t first_b, int32_t num_adapters, int32_t rank,
                              float scale, const int32_t *order, const int32_t *offsets, int64_t n, const void *x, int32_t x_type, int64_t x_stride, void *out,
                              int32_t out_type, int64_t out_stride, void *stream) {
    RowGroups g;
    int rc = adapter_call(ps, worker, first_key, rows, dim, first_a, first_b, num_adapters, rank, order, offsets, n, &g);
    if (rc) return rc;
    if (!is_element_type(x_type) || !is_element_type(out_type)) return PS_EINVAL;
    if (n == 0) return PS_OK;
    if (!x || !out || x_stride < 0 || out_stride < rows) return PS_EINVAL;
    hipStream_t st = (hipStream_t)stream;
    const int64_t ld = low_stride(rank);
    rc = dpaps_ws_reserve(ps, (size_t)n * (ld + 1) * sizeof(float));
    if (rc) return rc;
    float *low = (float *)ps->ws;
    int32_t *group_of = (int32_t *)(low + n * ld);
    rc = low_numbers(ps, g, x, x_type, x_stride, dim, ps->val + first_a * ps->L, rank, scale, x_type == PS_F32 || out_type == PS_F32, low, ld, group_of, st);
    if (rc) return rc;
    AdapterArgs a{};
    a.g = g; a.x = x; a.x_stride = x_stride; a.x_type = x_type; a.w = ps->val + first_key * ps->L; a.L = ps->L; a.K = dim; a.N = rows;
    a.low = low; a.low_stride = ld; a.rank = rank; a.b = ps->val + first_b * ps->L; a.group_of = group_of; a.out = out; a.out_stride = out_stride; a.out_type = out_type;
    rc = product(ps, a, st);
    if (rc) return rc;
    GroupKeys k;
    k.first = first_key; k.shared = rows; k.first_a = first_a; k.first_b = first_b; k.each = rank;
    return dpaps_route_groups(ps, worker, g, k, st);
}

extern "C" int adapter_grad(ps_handle ps, int32_t worker, int64_t first_key, int32_t rows, int32_t dim, int64_t first_a, int64_t first_b, int32_t num_adapters, int32_t rank,
                            float scale, const int32_t *order, const int32_t *offsets, int64_t n, const void *x, int64_t x_stride, const void *dout, int64_t dout_stride,
                            int32_t type, void *dx, int32_t dx_type, int64_t dx_stride, float *da, float *db, void *stream) {
    RowGroups g;
    int rc = adapter_call(ps, worker, first_key, rows, dim, first_a, first_b, num_adapters, rank, order, offsets, n, &g);
    if (rc) return rc;
    if (!is_element_type(type) || !is_element_type(dx_type) || !da || !db) return PS_EINVAL;
    if (n > 0 && (!x || !dout || x_stride < 0 || dout_stride < 0 || (dx && dx_stride < dim))) return PS_EINVAL;
    hipStream_t st = (hipStream_t)stream;
    const int64_t ld = low_stride(rank);
    OuterArgs o{};
    o.g = g; o.left_stride = ld; o.left_type = PS_F32; o.left_by_place = 1; o.rows = rank; o.out_type = PS_F32; o.right_type = type;
    size_t part_bytes = 0;
    for (const int32_t c : {dim, rows}) {
        o.cols = c;
        part_bytes = std::max(part_bytes, dpaps_outer_bytes(ps, o));
    }
    const size_t numbers = (size_t)n * (2 * ld + 1), off_part = (numbers + 63) / 64 * 64;
    rc = dpaps_ws_reserve(ps, off_part * sizeof(float) + part_bytes);
    if (rc) return rc;
    float *h = (float *)ps->ws, *t = h + n * ld, *part = h + off_part;
    int32_t *group_of = (int32_t *)(t + n * ld);
    const float *pa = ps->val + first_a * ps->L, *pb = ps->val + first_b * ps->L;
    if (n > 0) {
        rc = low_numbers(ps, g, x, type, x_stride, dim, pa, rank, scale, true, h, ld, group_of, st);
        if (!rc) rc = low_numbers(ps, g, dout, type, dout_stride, rows, pb, rank, scale, true, t, ld, nullptr, st);
        if (rc) return rc;
        if (dx) {
            AdapterArgs a{};
            a.g = g; a.x = dout; a.x_stride = dout_stride; a.x_type = type; a.w = ps->val + first_key * ps->L; a.L = ps->L; a.K = rows; a.N = dim; a.turned = 1;
            a.low = t; a.low_stride = ld; a.rank = rank; a.group_of = group_of; a.b = pa; a.out = dx; a.out_stride = dx_stride; a.out_type = dx_type;
            rc = product(ps, a, st);
            if (rc) return rc;
        }
    }
    o.left = t; o.right = x; o.right_stride = x_stride; o.cols = dim; o.out = da;
    rc = dpaps_outer_sums(ps, o, part, st);
    if (rc) return rc;
    o.left = h; o.right = dout; o.right_stride = dout_stride; o.cols = rows; o.out = db;
    rc = dpaps_outer_sums(ps, o, part, st);
    if (rc) return rc;
    if (n == 0) return PS_OK;
    GroupKeys k;
    k.first = first_key; k.shared = rows; k.first_a = first_a; k.first_b = first_b; k.each = rank;
    return dpaps_route_groups(ps, worker, g, k, st);
}
