// Products of grouped rows with matrices that lie in the server, and the matrices' gradients.
//
//   product    y_q = W_g(q) x_q,   or W'_g(q) x_q,        W_e: the rows of expert e, keys of the server
//   gradient   dW_e = sum over e's rows of dy_q x_q'
// Rows are taken in the groups' order, in tiles of rows of one group; where they lie stays as it is: they are read, and results are written, through that order.
// Products are of numbers of the rows' 16-bit type, with sums in 32 bits, where rows and results both have 16 bits: the server's numbers of 32 bits are rounded to it, which
// puts as much error on a result as its own rounding does (bf16 2^-8, fp16 2^-11 of each term at most, or 2^-25 of the row's number where the server's is below fp16's normal ones; on
// average over the terms less).  Else of numbers of 32 bits.
#include "experts.h"

#include <algorithm>

namespace {

struct ExpertCall { ExpertArgs a[2]; };

// Tiles of 128 x 128, 64 x 64 or 128 rows x 32 columns by way of LDS, two steps in it and one or two on their way to registers: the server's numbers have to be rounded,
// or turned, on the way, so they cannot come straight into LDS.  64 tokens x 2 of 16 experts, 1024 x 512, fp16: 9.9 us for 17 MB read, of which the trips to memory before
// the first product (the group's place, the row's number, the row) are about half.  Two of 16 experts for 16,384 tokens, 2048 x 1024, bf16, took 281 us so, without laying.
template <class CT, class XT, bool TURNED, class T>
__global__ __launch_bounds__(T::THREADS, T::BLOCKS) void k_expert(ExpertCall call, int32_t tiles, int32_t col_tiles, int32_t *err) {
    const ExpertArgs &a = call.a[blockIdx.y];
    constexpr int KU = unit_of<CT>(), BR = T::ROWS, BC = T::COLS;
    extern __shared__ __align__(16) char shared[];
    Vec<CT, KU> *const lds = reinterpret_cast<Vec<CT, KU> *>(shared);
    __shared__ int at[BR];                                           // the rows' numbers; -1: none
    __shared__ int off;
    look_for_all(err, &off);
    const TilePlace place = tile_place(tiles, col_tiles);
    if (place.row < 0) return;
    const RowTile t = row_tile(a.g, place.row, BR);
    const int c0 = place.col * BC, tid = threadIdx.x;
    if (t.rows == 0) return;
    for (int r = tid; r < BR; r += T::THREADS) {
        at[r] = r < t.rows ? row_at(a.g, t.first + r, err) : -1;
        if (a.group_of && c0 == 0 && r < t.rows) a.group_of[t.first + r] = t.group;
    }
    __syncthreads();
    if (off) return;
    floatx16 acc[T::MC][T::MR] = {};
    const int wave = tid >> 6, wc = wave % T::WC * 32 * T::MC, wr = wave / T::WC * 32 * T::MR, cols = a.columns() - c0;
    if (t.group < a.g.groups) {
        const float *w = a.w + (int64_t)t.group * a.each * a.L;
        KMajor<XT, CT, BR, T::THREADS> rows[T::SETS];
        for (auto &r : rows) r.init([&](int r) { return reinterpret_cast<const XT *>(a.x) + a.x_shared(at[r] < 0 ? 0 : at[r]) * a.x_stride; });
        std::conditional_t<TURNED, KeyRows<CT, BC, T::THREADS>, KeyColumns<CT, BC, T::THREADS>> columns[T::SETS];
        for (auto &c : columns) {
            if constexpr (TURNED) c.init(w + c0, a.L);
            else c.init(w + c0 * a.L, a.L, cols);
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
    if (a.zero_from) {
        const int h = (tid & 63) >> 5;
#pragma unroll
        for (int i = 0; i < T::MC; ++i)
#pragma unroll
            for (int e = 0; e < 16; ++e)
                if (c0 + wc + 32 * i + 8 * (e / 4) + 4 * h + e % 4 >= a.zero_from)
#pragma unroll
                    for (int j = 0; j < T::MR; ++j) acc[i][j][e] = 0.0f;
    }
    put_tile_typed<T>(acc, lds, a.out, a.out_type, c0, a.N, a.scale,
                      [&](int r) { return at[r] < 0 ? (int64_t)-1 : (int64_t)(a.by_place ? t.first + r : at[r]) * a.out_stride; });
    if (a.also)
        put_tile_typed<T>(acc, lds, a.also, a.also_type, c0, a.N, a.scale,
                          [&](int r) { return at[r] < 0 ? (int64_t)-1 : (int64_t)(a.by_place ? t.first + r : at[r]) * a.also_stride; });
}

// Groups of few rows: 16 rows a workgroup, whose wavefronts share the sum, so that a chain is short and all of a matrix is asked for at once.  One token of two experts of
// 512 x 512: 5.5 us; 333 rows of 5, 400 x 100 turned, 32 bits: 7.5.
template <class CT, class XT, bool TURNED, int MT>
__global__ __launch_bounds__((FewRows<CT, XT, TURNED, MT>::THREADS)) void k_expert_few(ExpertCall call, int32_t col_tiles, int32_t *err) {
    const ExpertArgs &a = call.a[blockIdx.y];
    typedef FewRows<CT, XT, TURNED, MT> F;
    __shared__ float sums[F::SUMS];
    __shared__ int at[16 * MT];
    __shared__ int off;
    look_for_all(err, &off);
    const RowTile t = row_tile(a.g, (int)(blockIdx.x / (uint32_t)col_tiles), 16 * MT);
    const int c0 = (int)(blockIdx.x % (uint32_t)col_tiles) * F::COLS, tid = threadIdx.x;
    __syncthreads();
    if (off || t.rows == 0) return;
    if (tid < 16 * MT) {
        at[tid] = tid < t.rows ? row_at(a.g, t.first + tid, err) : -1;
        if (a.group_of && c0 == 0 && tid < t.rows) a.group_of[t.first + tid] = t.group;
    }
    __syncthreads();
    if (t.group < a.g.groups) {
        F f;
        f.run(a.w + (int64_t)t.group * a.each * a.L, a.L, a.K, c0, a.columns(),
              [&](int r) { return reinterpret_cast<const XT *>(a.x) + a.x_shared(at[r] < 0 ? 0 : at[r]) * a.x_stride; });
        f.put(sums);
    }
    __syncthreads();
    for (int p = tid; p < F::PIECES; p += F::THREADS) {
        const int r = F::row_of(p), c = F::col_of(p), left = a.N - c0 - c;
        if (at[r] < 0 || left <= 0) continue;
        Vec<float, 4> v = t.group < a.g.groups ? a.scale * F::sum(sums, p) : Vec<float, 4>{};
        if (a.zero_from) v = cut<float, 4>(v, a.zero_from - c0 - c);
        const int64_t row = a.by_place ? t.first + r : at[r];
        put_typed<4>(a.out, a.out_type, row * a.out_stride + c0 + c, v, left);
        if (a.also) put_typed<4>(a.also, a.also_type, row * a.also_stride + c0 + c, v, left);
    }
}

// out_t = the sum of the rows t b .. t b + b - 1 of `in`, in that order.  (The products leave in 32 bits and are read again, 16,384 rows x 512 in 7.9 us; added in place, by
// atomics, their order would change from run to run.)
__global__ __launch_bounds__(256) void k_pair_sums(const float *in, int64_t n, int32_t b, int32_t N, void *out, int32_t out_type, int64_t out_stride, uint32_t P, double inv_P,
                                                   const int32_t *err) {
    if (*(volatile const int32_t *)err) return;
    for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < n * P; i += (int64_t)gridDim.x * 256) {
        const int64_t t = quotient(i, P, inv_P);
        const int c = (int)(i - t * P) * 4, left = N - c;
        const float *p = in + t * b * N + c;
        Vec<float, 4> v = load_some<float, 4>(p, left);
        for (int j = 1; j < b; ++j) v = v + load_some<float, 4>(p + (int64_t)j * N, left);
        put_typed<4>(out, out_type, t * out_stride + c, v, left);
    }
}
constexpr int64_t PAIR_SUMS_GRID = (int64_t)1 << 20;

}  // namespace

namespace {
constexpr int64_t MOST_GRID = (int64_t)1 << 24;                      // workgroups of a launch, fewer

template <class CT, class XT, bool TURNED, class T> int tiles_of(dpaps_ps *ps, const ExpertCall &c, int count, hipStream_t st) {
    const ExpertArgs &a = c.a[0];
    const int32_t col_tiles = (a.N + T::COLS - 1) / T::COLS;
    const int64_t tiles = row_tiles(a.g.n, a.g.groups, T::ROWS), grid = tiles * col_tiles;
    if (grid >= MOST_GRID) return dpaps_too_large(ps, "product");
    static LdsAllowed allowed;
    const int rc = dpaps_allow_lds(ps, allowed, reinterpret_cast<const void *>(&k_expert<CT, XT, TURNED, T>), T::LDS);
    if (rc) return rc;
    k_expert<CT, XT, TURNED, T><<<dim3(die_grid(grid), (unsigned)count), T::THREADS, T::LDS, st>>>(c, (int32_t)tiles, col_tiles, ps->err);
    PS_HIP(ps, hipGetLastError());
    return PS_OK;
}
template <class CT, class XT, bool TURNED, int MT> int64_t few_grid(const ExpertArgs &a) {
    return row_tiles(a.g.n, a.g.groups, 16 * MT) * ceil_div64(a.N, FewRows<CT, XT, TURNED, MT>::COLS);
}
template <class CT, class XT, bool TURNED, int MT> int few_of(dpaps_ps *ps, const ExpertCall &c, int count, hipStream_t st) {
    const ExpertArgs &a = c.a[0];
    typedef FewRows<CT, XT, TURNED, MT> F;
    const int32_t col_tiles = (a.N + F::COLS - 1) / F::COLS;
    const int64_t grid = few_grid<CT, XT, TURNED, MT>(a);
    if (grid >= MOST_GRID) return dpaps_too_large(ps, "product");
    k_expert_few<CT, XT, TURNED, MT><<<dim3((unsigned)grid, (unsigned)count), F::THREADS, 0, st>>>(c, col_tiles, ps->err);
    PS_HIP(ps, hipGetLastError());
    return PS_OK;
}
template <class CT, class XT, bool TURNED> int product_of(dpaps_ps *ps, const ExpertCall &c, int count, hipStream_t st) {
    const ExpertArgs &a = c.a[0];
    const int64_t n = a.g.n, groups = a.g.groups, cus = ps->num_cu;
    // Few rows, as long as tiles of 16 rows (a group's last one is half full) make no more workgroups than so many a compute unit.  At the borders, K 1024 but for the last:
    //   16 bits, 128 rows of 16 groups x 256 columns 8.0 us and by tiles of 64 8.0, x 512 9.7 and 8.0;   turned, 500 rows of 8 groups x 512 8.4 and 9.2, x 1024 12.3 and 9.5;
    //   32 bits, 333 rows of 5 groups x 400, K 100, 6.6 and 8.0, 1,000 rows 10.5 and 8.1
    const int64_t few = ceil_div64(n + 8 * (groups < n ? groups : n), 16) * ceil_div64(a.N, TURNED ? 64 : 16) * count;
    // Turned in 32 bits, the longer the sum the more of them, as it is a tile's chain and shared by wavefronts here: 400 x 127, K 400, 3,998 rows of 64 experts 31.3 us and
    // 16.5 by tiles of 64, 1,000 rows 12.8 and 15.5;   1024 x 512, K 1024, 1,000 rows of 64 41 and 64
    const int64_t limit = sizeof(CT) == 4 ? (TURNED ? std::min(std::max(a.K / 64, 4), 16) : 16) : TURNED ? 8 : 5;
    // (which launches workgroups for all groups: where those are too many, a quarter as many by tiles of 64)
    if (4 * few <= limit * cus && few_grid<CT, XT, TURNED, 1>(a) < MOST_GRID) return few_of<CT, XT, TURNED, 1>(ps, c, count, st);
    // 32 columns: tiles of 128 rows (16,384 rows of 8 groups, 16 bits, 13.0 us, and 21.2 by the kernel for few rows; 100,000 of 16 groups, 32 bits, 131 and 213), but where the
    // rows' numbers are made longer on their way (two of 16,384 rows of 16 groups, K 512, 26 and 16.5)
    if (a.N <= 32) return sizeof(CT) != sizeof(XT) ? few_of<CT, XT, TURNED, 2>(ps, c, count, st) : tiles_of<CT, XT, TURNED, Narrow>(ps, c, count, st);
    // 32 bits: tiles of 64, whose workgroups cover for each other's meetings (16,384 rows x 1024, K 1024, 345 us, by tiles of 128 371).  16 bits, rows of 8 groups x 1024,
    // K 1024: 1,000 rows 17.0 us by tiles of 64 and 20.4 by tiles of 128, 2,000 rows 28 and 22, 3,000 rows 38 and 24
    if (sizeof(CT) == 4 || 2 * ceil_div64(n, 128) * ceil_div64(a.N, 128) < cus) return tiles_of<CT, XT, TURNED, Tile64>(ps, c, count, st);
    return tiles_of<CT, XT, TURNED, Tile128>(ps, c, count, st);
}
template <class CT, class XT> int product_either(dpaps_ps *ps, const ExpertCall &c, int count, hipStream_t st) {
    return c.a[0].turned ? product_of<CT, XT, true>(ps, c, count, st) : product_of<CT, XT, false>(ps, c, count, st);
}
}  // namespace

int dpaps_expert_product(dpaps_ps *ps, const ExpertArgs *a, int count, hipStream_t st) {
    ExpertCall c{};
    for (int i = 0; i < count; ++i) c.a[i] = a[i];
    if (a->x_type == PS_F32) return product_either<float, float>(ps, c, count, st);
    if (a->x_type == PS_BF16) return a->precise ? product_either<float, bf16_t>(ps, c, count, st) : product_either<bf16_t, bf16_t>(ps, c, count, st);
    return a->precise ? product_either<float, f16_t>(ps, c, count, st) : product_either<f16_t, f16_t>(ps, c, count, st);
}

// From so many rows a group on, and tiles of 128 x 128 for two workgroups a compute unit, matrices are laid before the product (laid.hip).  K 1024, bf16, with the laying and by tiles:
// 16,384 rows of 8 groups x 2048 120 us and 136, x 1024 64 and 73;  of 16 groups, 1,024 rows each, x 2048 139 and 149, x 1024 72 and 77, groups as uneven as rank^-0.7 145 and 139, turned,
// K 2048, 163 and 145;  32,768 rows of 32 309 and 311.  With 512 rows a group it goes either way: 8,192 of 16 x 1024 52 and 60, x 2048 94 and 79;  16,384 of 32 x 2048 196 and 172.
constexpr int64_t LAID_ROWS = 1024;

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
    if (!dpaps_strides_fit(ps, x_stride, out_stride)) return PS_ELIMIT;
    hipStream_t st = (hipStream_t)stream;
    ExpertArgs a{};
    a.g = g; a.x = x; a.x_stride = x_stride; a.x_type = x_type; a.x_shared = Quotient(x_pairs);
    a.w = ps->val + first_key * ps->L; a.L = ps->L; a.each = rows; a.K = K; a.N = N; a.turned = transposed != 0;
    a.scale = 1.0f; a.precise = x_type == PS_F32 || out_type == PS_F32;
    a.out = out; a.out_stride = out_stride; a.out_type = out_type;
    const size_t sums = out_pairs > 1 ? ((size_t)n * N * sizeof(float) + 255) / 256 * 256 : 0;
    const int64_t laid = dpaps_laid_size(K, N);
    const bool lay = !a.precise && n >= LAID_ROWS * num_experts && ceil_div64(n, 128) * ceil_div64(N, 128) >= 2 * ps->num_cu && dpaps_laid_fits(x, x_stride, K) &&
                     num_experts < 32768 && N < (1 << 19) && laid * num_experts <= LAID_MOST;
    rc = dpaps_ws_reserve(ps, sums + (lay ? (size_t)laid * num_experts * 2 : 0));
    if (rc) return rc;
    if (out_pairs > 1) { a.out = ps->ws; a.out_stride = N; a.out_type = PS_F32; }
    if (lay) {
        LayArgs l{};
        l.w = a.w; l.L = a.L; l.each = a.each; l.K = K; l.N = N; l.turned = a.turned; l.to = (char *)ps->ws + sums; l.size = laid;
        rc = dpaps_lay(ps, g, x_type, l, nullptr, st);
        if (rc) return rc;
        LaidArgs p{};
        p.g = g; p.x = x; p.x_stride = x_stride; p.x_shared = a.x_shared; p.K = K; p.N = N; p.w = l.to; p.w_size = laid;
        p.out = a.out; p.out_stride = a.out_stride; p.out_type = a.out_type;
        rc = dpaps_laid_product(ps, x_type, p, st);
    } else rc = dpaps_expert_product(ps, &a, 1, st);
    if (rc) return rc;
    if (out_pairs > 1) {
        const uint32_t P = (uint32_t)((N + 3) / 4);
        const int64_t blocks = ceil_div64(n / out_pairs * P, 256);
        k_pair_sums<<<(unsigned)std::min(blocks, PAIR_SUMS_GRID), 256, 0, st>>>((const float *)ps->ws, n / out_pairs, out_pairs, N, out, out_type, out_stride, P, 1.0 / P, ps->err);
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
    int rc = dpaps_row_groups(ps, order, offsets, num_experts, n, &g);
    if (rc) return rc;
    if (left_pairs < 1 || right_pairs < 1 || n % left_pairs || n % right_pairs || (n > 0 && (!left || !right || left_stride < 0 || right_stride < 0))) return PS_EINVAL;
    if (rows > PS_EMB_MAX_DIM || dim > PS_EMB_MAX_DIM) { ps->last_error = "expert_grad: sides of at most 65536"; return PS_ELIMIT; }
    if (n > 0 && !dpaps_strides_fit(ps, left_stride, right_stride)) return PS_ELIMIT;
    OuterArgs a{};
    a.g = g; a.left = left; a.left_stride = left_stride; a.left_type = type; a.left_shared = Quotient(left_pairs);
    a.right = right; a.right_stride = right_stride; a.right_type = type; a.right_shared = Quotient(right_pairs);
    a.rows = rows; a.cols = dim; a.out = out; a.out_type = out_type;
    rc = dpaps_ws_reserve(ps, dpaps_outer_bytes(ps, &a, 1));
    return rc ? rc : dpaps_outer_sums(ps, &a, 1, (float *)ps->ws, (hipStream_t)stream);
}
