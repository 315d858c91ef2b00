// A shared projection with a low-rank adapter per row, and its gradients.
//
//   y_p = W x_p + s B_a (A_a x_p)               a: the adapter that row p names; W x_p alone where it names none
//   dx_p = W' dy_p + s A_a' (B_a' dy_p)
//   dA_a = s sum over a's rows of (B_a' dy_p) x_p',     dB_a' = s sum of (A_a x_p) dy_p'
// W, the rows of A_a and the rows of B_a' (both `rank` keys of an adapter) lie in the server.  The low-rank numbers s A_a x_p and s B_a' dy_p are worked out first, in the
// order of the groups, and kept in 32 bits; the second launch goes on, after the sum over W's side, with those of the adapters of its rows.  Where products are of 16 bits, they
// are rounded for the product with B_a, as B_a is, in every kernel: either costs a term 2^-8 (bf16) or 2^-11 (fp16) of it at most, or 2^-25 of the other factor
// where it is below fp16's normal numbers.
//
// The floor is W's product; what the adapters add are the low-rank numbers' launch, which reads x once more (16,001 rows x 1024 of 24 adapters, rank 32: 12.9 of 84 us), and `rank` further
// terms.  64 rows of 200 adapters, rank 16, 1024 x 1024: 7.5 and 8.3 us, two launches of few workgroups that wait for memory.
#include "experts.h"

#include <algorithm>

namespace {

// v += the low-rank numbers of the row at a place times W columns of its adapter's second matrix; both as numbers of CT, as where they meet on the matrix cores
// (so that what a row's result is made of depends on its types, not on how many rows a call has and of which adapters), their products and sums in 32 bits
template <class CT, int W> __device__ __forceinline__ void add_low(const AdapterArgs &a, int place, int group, int c, int left, Vec<float, W> &v) {
    const float *low = a.low + (int64_t)place * a.low_stride, *b = a.b + (int64_t)group * a.rank * a.L + c;
    Vec<float, W> w = {};
#pragma unroll 4
    for (int i = 0; i < a.rank; ++i) {
        const Vec<float, W> of_b = as_type<float, CT, W>(as_type<CT, float, W>(load_some<float, W>(b + (int64_t)i * a.L, left)));
        if constexpr (sizeof(CT) == 4) w = w + low[i] * of_b;
        else w = __builtin_elementwise_fma(Vec<float, W>((float)(CT)low[i]), of_b, w);      // (a product of two numbers of 16 bits is exact in 32)
    }
    v = v + w;
}

template <class CT, class XT, bool TURNED, class T>
__global__ __launch_bounds__(T::THREADS, T::BLOCKS) void k_adapter(AdapterArgs a, int32_t tiles, int32_t col_tiles, int32_t by_group, int32_t *err) {
    constexpr int KU = unit_of<CT>(), BR = T::ROWS, BC = T::COLS;
    extern __shared__ __align__(16) char shared[];
    Vec<CT, KU> *const lds = reinterpret_cast<Vec<CT, KU> *>(shared);
    __shared__ int at[BR];
    __shared__ int off;
    look_for_all(err, &off);
    const TilePlace place = tile_place(tiles, col_tiles);
    if (place.row < 0) return;
    const int c0 = place.col * BC, tid = threadIdx.x;
    // rows of one adapter, or as they follow each other in the order
    int first, count, group;
    bool alone = true;
    if (by_group) {
        const RowTile t = row_tile(a.g, place.row, BR);
        first = t.first; count = t.rows; group = t.group;
    } else {
        first = place.row * BR;
        count = a.g.n - first < BR ? a.g.n - first : BR;
        group = a.group_of[first];
        alone = group == a.group_of[first + count - 1];
    }
    if (count <= 0) return;
    for (int r = tid; r < BR; r += T::THREADS) at[r] = r < count ? row_at(a.g, first + r, err) : -1;
    __syncthreads();
    if (off) return;
    floatx16 acc[T::MC][T::MR] = {};
    const int wave = tid >> 6, wc = wave % T::WC * 32 * T::MC, wr = wave / T::WC * 32 * T::MR, cols = a.N - c0;
    {
        KMajor<XT, CT, BR, T::THREADS> rows[T::SETS];
        for (auto &r : rows) r.init([&](int r) { return reinterpret_cast<const XT *>(a.x) + (int64_t)(at[r] < 0 ? 0 : at[r]) * a.x_stride; });
        std::conditional_t<TURNED, KeyRows<CT, BC, T::THREADS>, KeyColumns<CT, BC, T::THREADS>> columns[T::SETS];
        for (auto &c : columns) {
            if constexpr (TURNED) c.init(a.w + c0, a.L);
            else c.init(a.w + c0 * a.L, a.L, cols);
        }
        tile_sum<CT, T>(a.K, lds, wc, wr,
            [&](auto set, int s, auto tail) {
                rows[set].template load<decltype(tail)::value>(s, a.K);
                columns[set].template load<decltype(tail)::value>(s, a.K);
            },
            [&](auto set, Vec<CT, KU> *to) {
                rows[set].put(to);
                columns[set].put(to + BR * UNITS);
            }, acc);
    }
    // Rows of one adapter: its product goes on where W's has ended.  Rows of several: a row's part is worked out number by number as the sums leave, so that
    // nothing of one adapter comes near the rows of another (a zero times its infinity would be no number).
    if (alone && (uint32_t)group < (uint32_t)a.g.groups) {
        KMajor<float, CT, BR, T::THREADS> rows;
        rows.init([&](int r) { return a.low + (int64_t)(first + (r < count ? r : 0)) * a.low_stride; });
        KeyRows<CT, BC, T::THREADS> columns;
        columns.init(a.b + (int64_t)group * a.rank * a.L + c0, a.L);
        tile_sum_short<CT, T>(a.rank, lds, wc, wr,
            [&](auto, int s, auto tail) {
                rows.template load<decltype(tail)::value>(s, a.rank);
                columns.template load<decltype(tail)::value>(s, a.rank);
            },
            [&](auto, Vec<CT, KU> *to) {
                rows.put(to);
                columns.put(to + BR * UNITS);
            }, acc);
    }
    put_tile_typed<T>(acc, lds, a.out, a.out_type, c0, a.N, 1.0f, [&](int r) { return at[r] < 0 ? (int64_t)-1 : (int64_t)at[r] * a.out_stride; },
                      [&](int r, int c, int left, Vec<float, 8> &v) {
                          if (alone) return;
                          const uint32_t e = (uint32_t)a.group_of[first + r];
                          if (e < (uint32_t)a.g.groups) add_low<CT, 8>(a, first + r, (int)e, c0 + c, left, v);
                      });
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
        if ((uint32_t)group[r] < (uint32_t)a.g.groups) add_low<CT, 4>(a, first + r, group[r], c0 + c, left, v);       // (whatever the offsets are)
        put_typed<4>(a.out, a.out_type, (int64_t)at[r] * a.out_stride + c0 + c, v, left);
    }
}

template <class CT, class XT, bool TURNED, class T> int tiles_of(dpaps_ps *ps, const AdapterArgs &a, hipStream_t st) {
    const int32_t col_tiles = (a.N + T::COLS - 1) / T::COLS;
    // Tiles of one adapter leave the last tile of each half empty; mixed ones add up to `rank` terms number by number, in 16 bits after rounding them.  K 1024, rows of a
    // few requests an adapter, 16 bits, by adapter and mixed: x 1024 columns, rank 32, 2,000 rows of 100 45 us and 63, 2,400 of 100 52 and 62, 4,000 of 200 76 and 64, 1,500 of 64 31 and
    // 27;   rank 64, 2,000 of 200 71 and 102;   rank 16, 2,000 of 64 42 and 42, 4,000 of 100 53 and 44;   rank 8, 4,100 of 64 46 and 34, 3,800 of 40 30 and 34.   32 bits, where
    // products take longer: 5,000 of 20 132 and 135, of 64 161 and 143, 16,000 of 64 383 and 353; rank 8 139 and 124, 159 and 128, 370 and 341
    const bool by_group = sizeof(CT) == 4 ? a.g.n >= 4 * (int64_t)T::ROWS * a.g.groups : (int64_t)a.g.n * a.rank >= 640 * (int64_t)a.g.groups;
    const int64_t tiles = by_group ? row_tiles(a.g.n, a.g.groups, T::ROWS) : ceil_div64(a.g.n, T::ROWS), grid = tiles * col_tiles;
    if (grid >= ((int64_t)1 << 24)) return dpaps_too_large(ps, "adapters");
    static LdsAllowed allowed;
    const int rc = dpaps_allow_lds(ps, allowed, reinterpret_cast<const void *>(&k_adapter<CT, XT, TURNED, T>), T::LDS);
    if (rc) return rc;
    k_adapter<CT, XT, TURNED, T><<<die_grid(grid), T::THREADS, T::LDS, st>>>(a, (int32_t)tiles, col_tiles, by_group, ps->err);
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
    const int64_t few = ceil_div64(a.g.n, 16) * ceil_div64(a.N, TURNED ? 64 : 16);
    if (4 * few <= (sizeof(CT) == 4 ? 16 : TURNED ? 8 : 5) * ps->num_cu) return few_of<CT, XT, TURNED, 1>(ps, a, st);      // (as products with few experts)
    if (sizeof(CT) == 4 || 2 * ceil_div64(a.g.n, 128) * ceil_div64(a.N, 128) < ps->num_cu) return tiles_of<CT, XT, TURNED, Tile64>(ps, a, st);
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

// low_p = s M_a x_p of the rows at the places of the order, in 32 bits, or, where the second product takes laid matrices, in the rows' type
struct LowNumbers { float *numbers; int64_t stride; void *rounded; int64_t rounded_stride; int32_t *group_of; };
ExpertArgs low_numbers(const dpaps_ps *ps, const RowGroups &g, const void *x, int32_t type, int64_t stride, int32_t K, const float *m, int32_t rank, float scale, bool precise,
                       const LowNumbers &low, int32_t columns) {
    ExpertArgs a{};
    a.g = g; a.x = x; a.x_stride = stride; a.x_type = type; a.w = m; a.L = ps->L; a.each = rank; a.K = K; a.N = columns; a.scale = scale; a.by_place = 1; a.precise = precise;
    a.group_of = low.group_of;
    a.zero_from = columns > rank ? rank : 0;
    if (low.numbers) {
        a.out = low.numbers; a.out_stride = low.stride; a.out_type = PS_F32;
        a.also = low.rounded; a.also_stride = low.rounded_stride; a.also_type = type;
    } else { a.out = low.rounded; a.out_stride = low.rounded_stride; a.out_type = type; }
    return a;
}

// Scratch of a call, and the product with it.  Many rows of 16 bits, tiles of 128 x 128 for one and a half workgroups a compute unit: the shared matrix and the adapters'
// second ones are laid (laid.hip).  1024 x 1024, rank 32, with the laying: 5,000 rows of 20 adapters 32 us and 31 without, 8,000 of 100 54 and 59, 16,384 of 200 99 and
// 123, 16,001 of 64 (24 of them asked for) 71 and 84;   rank 8, 5,000 of 20 32 and 31, 16,384 of 200 100 and 110;   512 x 512, rank 16, 8,000 of 16 20 and 19, 16,384 24 and 29.
struct Scratch {
    bool laid = false;
    int64_t stride = 0, rounded_stride = 0, w_size = 0, b_size = 0;
    size_t numbers[2] = {}, rounded = 0, group_of = 0, w = 0, b = 0, end = 0;
};
// both: the numbers in 32 bits of two products, which gradients need; product: whether there is one with the shared matrix
Scratch scratch_of(const dpaps_ps *ps, const RowGroups &g, const void *x, int64_t x_stride, int32_t K, int32_t N, int32_t rank, bool precise, bool both, bool product) {
    Scratch s;
    const int64_t n = g.n;
    s.w_size = dpaps_laid_size(K, N);
    s.b_size = dpaps_laid_size(rank, N);
    s.laid = product && !precise && ceil_div64(n, 128) * ceil_div64(N, 128) >= 3 * ps->num_cu / 2 && n >= 64 * (int64_t)g.groups && g.groups < 32768 &&
             dpaps_laid_fits(x, x_stride, K) && s.w_size + s.b_size * g.groups <= LAID_MOST;
    s.rounded_stride = (rank + 7) / 8 * 8;
    s.stride = s.rounded_stride;
    const auto take = [&](int64_t bytes) { const size_t at = s.end; s.end += ((size_t)bytes + 255) / 256 * 256; return at; };
    if (!s.laid || both) s.numbers[0] = take(n * s.stride * 4);
    if (both) s.numbers[1] = take(n * s.stride * 4);
    s.group_of = take(n * 4);
    if (s.laid) {
        s.rounded = take(n * s.rounded_stride * 2);
        s.w = take(s.w_size * 2);
        s.b = take(s.b_size * 2 * g.groups);
    }
    return s;
}
LowNumbers low_of(char *ws, const Scratch &s, bool numbers, bool rounded, int which) {
    LowNumbers l{};
    l.stride = s.stride; l.rounded_stride = s.rounded_stride;
    if (numbers || !s.laid) l.numbers = (float *)(ws + s.numbers[which]);
    if (s.laid && rounded) l.rounded = ws + s.rounded;
    l.group_of = (int32_t *)(ws + s.group_of);
    return l;
}
int product_with(dpaps_ps *ps, const Scratch &s, const LowNumbers &low, AdapterArgs a, hipStream_t st) {
    if (!s.laid) {
        a.low = low.numbers; a.low_stride = low.stride; a.group_of = low.group_of;
        return product(ps, a, st);
    }
    char *ws = (char *)ps->ws;
    LayArgs shared{}, second{};
    shared.w = a.w; shared.L = a.L; shared.K = a.K; shared.N = a.N; shared.turned = a.turned; shared.to = ws + s.w;
    second.w = a.b; second.L = a.L; second.each = a.rank; second.K = a.rank; second.N = a.N; second.turned = 1; second.to = ws + s.b; second.size = s.b_size;
    const int rc = dpaps_lay(ps, a.g, a.x_type, second, &shared, st);
    if (rc) return rc;
    LaidArgs p{};
    p.g = a.g; p.x = a.x; p.x_stride = a.x_stride; p.K = a.K; p.N = a.N; p.w = ws + s.w; p.w_size = s.w_size; p.low = low.rounded; p.low_stride = (int32_t)low.rounded_stride;
    p.b = ws + s.b; p.b_size = s.b_size; p.rank = a.rank; p.out = a.out; p.out_stride = a.out_stride; p.out_type = a.out_type;
    return dpaps_laid_product(ps, a.x_type, p, st);
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
    if (!dpaps_strides_fit(ps, x_stride, out_stride)) return PS_ELIMIT;
    hipStream_t st = (hipStream_t)stream;
    const bool precise = x_type == PS_F32 || out_type == PS_F32;
    const Scratch s = scratch_of(ps, g, x, x_stride, dim, rows, rank, precise, false, true);
    rc = dpaps_ws_reserve(ps, s.end);
    if (rc) return rc;
    const LowNumbers low = low_of((char *)ps->ws, s, false, true, 0);
    const ExpertArgs down = low_numbers(ps, g, x, x_type, x_stride, dim, ps->val + first_a * ps->L, rank, scale, precise, low, (int32_t)(s.laid ? s.rounded_stride : rank));
    rc = dpaps_expert_product(ps, &down, 1, st);
    if (rc) return rc;
    AdapterArgs a{};
    a.g = g; a.x = x; a.x_stride = x_stride; a.x_type = x_type; a.w = ps->val + first_key * ps->L; a.L = ps->L; a.K = dim; a.N = rows;
    a.rank = rank; a.b = ps->val + first_b * ps->L; a.out = out; a.out_stride = out_stride; a.out_type = out_type;
    rc = product_with(ps, s, low, a, st);
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
    if (n > 0 && (!dpaps_strides_fit(ps, x_stride, dout_stride) || !dpaps_strides_fit(ps, dx ? dx_stride : 0, 0))) return PS_ELIMIT;
    hipStream_t st = (hipStream_t)stream;
    const Scratch s = scratch_of(ps, g, dout, dout_stride, rows, dim, rank, type == PS_F32 || dx_type == PS_F32, true, dx != nullptr);
    OuterArgs o[2]{};
    for (int i = 0; i < 2; ++i) {
        o[i].g = g; o[i].left_stride = s.stride; o[i].left_type = PS_F32; o[i].left_by_place = 1; o[i].rows = rank; o[i].out_type = PS_F32; o[i].right_type = type;
    }
    o[0].right = x; o[0].right_stride = x_stride; o[0].cols = dim; o[0].out = da;
    o[1].right = dout; o[1].right_stride = dout_stride; o[1].cols = rows; o[1].out = db;
    rc = dpaps_ws_reserve(ps, s.end + dpaps_outer_bytes(ps, o, 2));
    if (rc) return rc;
    char *ws = (char *)ps->ws;
    const LowNumbers h = low_of(ws, s, true, false, 0), t = low_of(ws, s, true, true, 1);
    const float *pa = ps->val + first_a * ps->L, *pb = ps->val + first_b * ps->L;
    if (n > 0) {
        const int32_t columns = (int32_t)(s.laid ? s.rounded_stride : rank);
        const ExpertArgs both[2] = {low_numbers(ps, g, x, type, x_stride, dim, pa, rank, scale, true, h, columns),
                                    low_numbers(ps, g, dout, type, dout_stride, rows, pb, rank, scale, true, t, columns)};
        rc = dpaps_expert_product(ps, both, 2, st);
        if (rc) return rc;
        if (dx) {
            AdapterArgs a{};
            a.g = g; a.x = dout; a.x_stride = dout_stride; a.x_type = type; a.w = ps->val + first_key * ps->L; a.L = ps->L; a.K = rows; a.N = dim; a.turned = 1;
            a.rank = rank; a.b = pa; a.out = dx; a.out_stride = dx_stride; a.out_type = dx_type;
            rc = product_with(ps, s, t, a, st);
            if (rc) return rc;
        }
    }
    o[0].left = t.numbers;
    o[1].left = h.numbers;
    rc = dpaps_outer_sums(ps, o, 2, (float *)(ws + s.end), st);
    if (rc) return rc;
    if (n == 0) return PS_OK;
    GroupKeys k;
    k.first = first_key; k.shared = rows; k.first_a = first_a; k.first_b = first_b; k.each = rank;
    return dpaps_route_groups(ps, worker, g, k, st);
}
