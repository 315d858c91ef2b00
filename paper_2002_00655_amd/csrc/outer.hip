// Sums of products of rows by group: the gradients of matrices that rows were multiplied by.
//
//   out_e[i][j] = sum over the rows q of group e of left_q[i] right_q[j]
// Both operands lie the wrong way round for the matrix instruction, which takes numbers that follow each other in the sum, here the rows.  Rows of 16 bits
// go into LDS as they lie and are turned on their way out of it by the instruction that reads four rows of 16 columns and gives each lane one column; other
// rows are turned in registers on their way in.
// A group's rows are cut into chunks, so that a group of many rows is the work of several workgroups a tile; their sums are added in the chunks' order.
// 16,384 rows of 8 groups, 1024 x 512, bf16: 42 us (410 TFLOP/s; 79 MB read and 31 written) and 8.6 for the sums of the chunks; turned in registers 57.  What bounds it are the chunks:
// about two workgroups a compute unit, whose starts (a row's number, the row) and ways out do not overlap with products.  The same in 32 bits 216 us (80 TFLOP/s of 153).
#include "experts.h"

#include <algorithm>

namespace {

// The first chunk of a group writes to the result, or, where that is not of 32 bits and the group has several, to a slot of part; the others to slots that
// are told apart by their first place, in whole chunks: floor(first / chunk) differs between all chunks but the first ones of groups of several, as it does
// between those.
struct OuterTiles { int32_t rows, cols, chunk; float *part; int32_t slots; };
struct OuterCall { OuterArgs a[2]; OuterTiles o[2]; };
__device__ __forceinline__ float *outer_slot(const OuterArgs &a, const OuterTiles &o, int group, int start, int first) {
    const int64_t size = (int64_t)a.rows * a.cols;
    if (first > start) return o.part + first / o.chunk * size;
    return a.out_type == PS_F32 ? reinterpret_cast<float *>(a.out) + group * size : o.part + (o.slots + first / o.chunk) * size;
}
// Which tile, of which chunk.  False: nothing to do (for the whole workgroup).
constexpr int AT_MOST = 2048;                                        // rows' numbers in LDS
struct OuterPlace { RowTile t; int r0, c0; };
template <int BR, int BC>
__device__ __forceinline__ bool outer_place(const OuterArgs &a, const OuterTiles &o, int32_t *err, OuterPlace &p) {
    __shared__ int off;
    look_for_all(err, &off);
    const int tiles = o.rows * o.cols, tile = (int)(blockIdx.x % (uint32_t)tiles), share = (int)(blockIdx.x / (uint32_t)tiles);
    p.r0 = tile / o.cols * BR;
    p.c0 = tile % o.cols * BC;
    p.t = row_tile(a.g, share, o.chunk);
    if (p.t.group >= a.g.groups) return false;
    // (a group without rows has one chunk, of none: its matrix is cleared)
    if (p.t.rows == 0 && !(p.t.start >= p.t.end && share == p.t.start / o.chunk + p.t.group)) return false;
    __syncthreads();
    return off == 0;
}
// The numbers of the chunk's next rows from its row `from` on, brought into LDS; how many.
__device__ __forceinline__ int outer_rows(const OuterArgs &a, const OuterPlace &p, int from, int *at, int32_t *err) {
    const int rows = p.t.rows - from < AT_MOST ? p.t.rows - from : AT_MOST;
    for (int i0 = threadIdx.x; i0 < rows; i0 += 8 * blockDim.x) {
        int q[8];
#pragma unroll
        for (int u = 0; u < 8; ++u) q[u] = a.g.order[p.t.first + from + (i0 + u * (int)blockDim.x < rows ? i0 + u * (int)blockDim.x : i0)];
#pragma unroll
        for (int u = 0; u < 8; ++u) {
            const int i = i0 + u * (int)blockDim.x;
            if (q[u] < 0 || q[u] >= a.g.n) {                         // (row 0 is read in its place; the error is set)
                atomicExch(err, PS_EKEY);
                q[u] = 0;
            }
            if (i < rows) at[i] = q[u];
        }
    }
    __syncthreads();
    return rows;
}
template <class T> __device__ __forceinline__ void outer_put(const OuterArgs &a, const OuterTiles &o, const OuterPlace &p, const floatx16 (&acc)[T::MC][T::MR], void *lds) {
    const bool whole = p.t.end - p.t.start <= o.chunk;
    void *out = whole ? a.out : outer_slot(a, o, p.t.group, p.t.start, p.t.first);
    const int64_t base = whole ? (int64_t)p.t.group * a.rows * a.cols : 0;
    put_tile_typed<T>(acc, lds, out, whole ? a.out_type : PS_F32, p.c0, a.cols, 1.0f,
                      [&](int r) { return p.r0 + r < a.rows ? base + (int64_t)(p.r0 + r) * a.cols : (int64_t)-1; });
}

// (one multiplication: strides are below 2^31, and rows' numbers are not negative)
template <class T> __device__ __forceinline__ const T *row_of(const T *base, int row, int64_t stride) { return base + (uint64_t)(uint32_t)row * (uint32_t)stride; }

// Turned in registers.  Sums of at most 64 rows, as those of adapters are, by tiles of 32 x 128: two of 16 ranks x 512, 16,384 rows of 16 groups, 32-bit numbers by
// bf16 ones, 21.5 us, and 48 by tiles of 64, of which most rows are nobody's.
// LONG: chunks of more rows than `at` holds.  (In one kernel for both, what the loop keeps in registers left room for two workgroups of the smaller tiles on a compute unit
// instead of three: 29.5 us.)
template <class CT, class LT, class RT, class T, bool LONG>
__global__ __launch_bounds__(T::THREADS, T::BLOCKS) void k_outer(OuterCall call, int32_t *err) {
    constexpr int KU = unit_of<CT>(), BR = T::ROWS, BC = T::COLS;
    extern __shared__ __align__(16) char shared[];
    Vec<CT, KU> *const lds = reinterpret_cast<Vec<CT, KU> *>(shared);
    int *const at = reinterpret_cast<int *>(lds + 2 * (BR + BC) * UNITS);      // the rows' numbers of the chunk
    const OuterArgs a = call.a[blockIdx.y];
    const OuterTiles o = call.o[blockIdx.y];
    OuterPlace p;
    if (!outer_place<BR, BC>(a, o, err, p)) return;
    floatx16 acc[T::MC][T::MR] = {};
    const int wave = threadIdx.x >> 6, wc = wave % T::WC * 32 * T::MC, wr = wave / T::WC * 32 * T::MR;
    ChosenRows<LT, CT, BR, T::THREADS> left[T::SETS];
    ChosenRows<RT, CT, BC, T::THREADS> right[T::SETS];
    for (int from = 0; from < p.t.rows; from += AT_MOST) {
        const int rows = outer_rows(a, p, from, at, err);
        tile_sum<CT, T>(rows, lds, wc, wr,
            [&](auto set, int s, auto tail) {
                left[set].template load<decltype(tail)::value>(s, rows, a.rows - p.r0, [&](int i) {
                    return row_of(reinterpret_cast<const LT *>(a.left) + p.r0, a.left_by_place ? p.t.first + from + i : a.left_shared(at[i]), a.left_stride);
                });
                right[set].template load<decltype(tail)::value>(s, rows, a.cols - p.c0, [&](int i) {
                    return row_of(reinterpret_cast<const RT *>(a.right) + p.c0, a.right_shared(at[i]), a.right_stride);
                });
            },
            [&](auto set, Vec<CT, KU> *to) {
                left[set].put(to);
                right[set].put(to + BR * UNITS);
            }, acc);
        if (!LONG) break;
    }
    outer_put<T>(a, o, p, acc, lds);
}

// Turned out of LDS: rows of 16 bits whose numbers lie on 16 bytes.  A step is 64 rows of the sum, two steps are in LDS and two on their way to registers.  A row's
// columns lie in LDS as in memory, 32 bytes at a time changed over by the row's number, so that the four rows of a read meet all banks.
// (Straight from memory into LDS, the compiler has every turned read wait for all loads on their way: 78 us instead of 60 turned in registers, for
// 16,384 rows of 8 groups, 1024 x 512.)
constexpr int KS = 64;
template <class T> struct Turned {
    static constexpr int STEP = KS * (T::ROWS + T::COLS) * 2, LDS = 2 * STEP, N = KS / 16;    // a thread's rows of a step
    static_assert(T::THREADS == 256 && T::ROWS == 128 && T::COLS == 128);                    // 16 threads a row, on either side
};
typedef short Four __attribute__((ext_vector_type(4)));
typedef short Eight __attribute__((ext_vector_type(8)));
__device__ __forceinline__ Four turned_four(const unsigned char *from) {
    return __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) Four *)from);
}
template <class CT, class T, bool LONG>
__global__ __launch_bounds__(256, T::BLOCKS) void k_outer_turned(OuterCall call, int32_t *err) {
    typedef Turned<T> F;
    constexpr int BR = T::ROWS, BC = T::COLS;
    extern __shared__ __align__(16) unsigned char lds[];
    int *const at = reinterpret_cast<int *>(lds + F::LDS);
    const OuterArgs a = call.a[blockIdx.y];
    const OuterTiles o = call.o[blockIdx.y];
    OuterPlace p;
    if (!outer_place<BR, BC>(a, o, err, p)) return;
    floatx16 acc[T::MC][T::MR] = {};
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const int wc = wave % T::WC * 32 * T::MC, wr = wave / T::WC * 32 * T::MR;
    for (int from = 0; from < p.t.rows; from += AT_MOST) {
        const int rows = outer_rows(a, p, from, at, err), steps = (rows + KS - 1) / KS;
        struct Numbers { Eight left[F::N], right[F::N]; } x, y;
        const int k0 = tid >> 4, c = (tid & 15) * 8;
        const bool in_left = p.r0 + c < a.rows, in_right = p.c0 + c < a.cols;
        const CT *left = reinterpret_cast<const CT *>(a.left) + (in_left ? p.r0 + c : 0), *right = reinterpret_cast<const CT *>(a.right) + (in_right ? p.c0 + c : 0);
        const auto fetch = [&](Numbers &to, int s) {
#pragma unroll
            for (int i = 0; i < F::N; ++i) {
                const int k = s * KS + i * 16 + k0, q = at[k < rows ? k : 0];
                to.left[i] = *reinterpret_cast<const Eight *>(row_of(left, a.left_shared(q), a.left_stride));
                to.right[i] = *reinterpret_cast<const Eight *>(row_of(right, a.right_shared(q), a.right_stride));
            }
        };
        // (rows that do not exist become zero on both sides: a number in their place could be an infinity; columns that do not are nobody's)
        const auto put = [&](const Numbers &from, int s, auto half) {
            unsigned char *to = lds + decltype(half)::value * F::STEP + k0 * 256 + (((c >> 4) ^ (2 * (k0 & 3))) * 32) + (c & 8) * 2;
            if ((s + 1) * KS <= rows) {
#pragma unroll
                for (int i = 0; i < F::N; ++i) {
                    *reinterpret_cast<Eight *>(to + i * 4096) = from.left[i];
                    *reinterpret_cast<Eight *>(to + i * 4096 + KS * 256) = from.right[i];
                }
            } else {
#pragma unroll
                for (int i = 0; i < F::N; ++i) {
                    const bool row = s * KS + i * 16 + k0 < rows;
                    *reinterpret_cast<Eight *>(to + i * 4096) = row ? from.left[i] : Eight{};
                    *reinterpret_cast<Eight *>(to + i * 4096 + KS * 256) = row ? from.right[i] : Eight{};
                }
            }
        };
        typedef Vec<CT, 8> Unit;
        struct Pair { Unit a[T::MC], b[T::MR]; } u, v;
        const int row = lane >> 2 & 3, piece = lane & 3, odd = lane >> 4 & 1, k8 = 8 * (lane >> 5);
        // where this lane reads for a column block of 32: the rest of an address is known before
        const unsigned char *left_at[T::MR], *right_at[T::MC];
#pragma unroll
        for (int j = 0; j < T::MR; ++j) left_at[j] = lds + (k8 + row) * 256 + (((wr + 32 * j) / 16 + odd) ^ (2 * row)) * 32 + piece * 8;
#pragma unroll
        for (int i = 0; i < T::MC; ++i) right_at[i] = lds + KS * 256 + (k8 + row) * 256 + (((wc + 32 * i) / 16 + odd) ^ (2 * row)) * 32 + piece * 8;
        const auto read = [&](Pair &to, auto half, auto pair) {
            constexpr int at = decltype(half)::value * F::STEP + decltype(pair)::value * 16 * 256;
            const auto unit = [&](const unsigned char *from) {
                return __builtin_bit_cast(Unit, __builtin_shufflevector(turned_four(from + at), turned_four(from + at + 4 * 256), 0, 1, 2, 3, 4, 5, 6, 7));
            };
#pragma unroll
            for (int i = 0; i < T::MC; ++i) to.a[i] = unit(right_at[i]);
#pragma unroll
            for (int j = 0; j < T::MR; ++j) to.b[j] = unit(left_at[j]);
        };
        const auto multiply = [&](const Pair &from) {
#pragma unroll
            for (int i = 0; i < T::MC; ++i)
#pragma unroll
                for (int j = 0; j < T::MR; ++j) acc[i][j] = mfma_unit<CT>(from.a[i], from.b[j], acc[i][j]);
        };
        typedef std::integral_constant<int, 0> Zero;
        typedef std::integral_constant<int, 1> One;
        typedef std::integral_constant<int, 2> Two;
        typedef std::integral_constant<int, 3> Three;
        // step s, in that half of LDS, whose first pair has been read; `next` holds the numbers of step s + 1
        const auto step = [&](int s, Numbers &next, auto half, auto other) {
            read(v, half, One{});
            __builtin_amdgcn_sched_barrier(0);
            multiply(u);
            read(u, half, Two{});
            __builtin_amdgcn_sched_barrier(0);
            multiply(v);
            read(v, half, Three{});
            __builtin_amdgcn_sched_barrier(0);
            multiply(u);
            if (s + 1 < steps) {
                put(next, s + 1, other);
                if (s + 3 < steps) fetch(next, s + 3);
                __syncthreads();
                read(u, other, Zero{});
                __builtin_amdgcn_sched_barrier(0);
            }
            multiply(v);
        };
        fetch(x, 0);
        if (steps > 1) fetch(y, 1);
        put(x, 0, Zero{});
        if (steps > 2) fetch(x, 2);
        __syncthreads();
        read(u, Zero{}, Zero{});
        for (int s = 0; s < steps; s += 2) {
            step(s, y, Zero{}, One{});
            if (s + 1 < steps) step(s + 1, x, One{}, Zero{});
        }
        __syncthreads();
        if (!LONG) break;
    }
    outer_put<T>(a, o, p, acc, lds);
}

// The chunks of groups of several, added up in their order.  blockIdx.y: the group
__global__ __launch_bounds__(256) void k_outer_join(OuterCall call, const int32_t *err) {
    if (*(volatile const int32_t *)err) return;
    const OuterArgs &a = call.a[blockIdx.z];
    const OuterTiles &o = call.o[blockIdx.z];
    const int64_t size = (int64_t)a.rows * a.cols;
    for (int group = blockIdx.y; group < a.g.groups; group += gridDim.y) {
        const int start = a.g.start(group), end = a.g.start(group + 1);
        if (end - start <= o.chunk) continue;
        for (int64_t i = ((int64_t)blockIdx.x * 256 + threadIdx.x) * 4; i < size; i += (int64_t)gridDim.x * 1024) {
            const int left = size - i < 4 ? (int)(size - i) : 4;
            Vec<float, 4> v = {};
#pragma unroll 4
            for (int first = start; first < end; first += o.chunk) v = v + load_some<float, 4>(outer_slot(a, o, group, start, first) + i, left);
            put_typed<4>(a.out, a.out_type, group * size + i, v, left);
        }
    }
}

// What a call's sums are worked out by.  Tiles of 64 where tiles of 128 of all groups are fewer than the compute units: 333 rows of 5 groups, 400 x 100, 32 bits, 10.0 us and 17.5 by
// tiles of 128; 16,384 rows of 8, 1024 x 512, 255 and 216.
enum { OUTER_LOW, OUTER_64, OUTER_128, OUTER_TURNED };
int outer_kind(const dpaps_ps *ps, const OuterArgs *a, int count) {
    if (a->rows <= 64) return OUTER_LOW;
    const auto fits = [&](const void *p, int64_t stride, int32_t cols) { return (uintptr_t)p % 16 == 0 && stride % 8 == 0 && cols % 8 == 0; };
    if (count == 1 && a->left_type != PS_F32 && a->right_type != PS_F32 && !a->left_by_place && fits(a->left, a->left_stride, a->rows) && fits(a->right, a->right_stride, a->cols))
        return OUTER_TURNED;
    return ceil_div64(a->rows, 128) * ceil_div64(a->cols, 128) * a->g.groups < ps->num_cu ? OUTER_64 : OUTER_128;
}
// The tiles of a sum, and how many of a group's rows a workgroup takes.
constexpr int CHUNK_MOST = 2048;
constexpr int64_t PART_MOST = (int64_t)1 << 28;                     // bytes of the chunks' sums (twice as many, if the result has 16 bits)
template <class T> OuterTiles outer_tiles(const dpaps_ps *ps, const OuterArgs &a, int64_t want) {
    OuterTiles o{};
    o.rows = (a.rows + T::ROWS - 1) / T::ROWS;
    o.cols = (a.cols + T::COLS - 1) / T::COLS;
    // chunks that make, with the rests of the groups (half a chunk each, if all have rows), one round of `want` workgroups a compute unit: the longest one is
    // what a call takes
    const int64_t round = want * ps->num_cu / ((int64_t)o.rows * o.cols), shares = std::max(round - a.g.groups / 2, round / 2);
    const int64_t rows = shares > 0 ? ceil_div64(ceil_div64(a.g.n, shares), 64) * 64 : CHUNK_MOST, least = a.g.n <= 512 ? 512 : 192;
    int64_t chunk = rows < least ? least : rows > CHUNK_MOST ? CHUNK_MOST : rows;
    // longer ones, where their sums would not fit into the scratch
    while (chunk < a.g.n && (a.g.n / chunk + 1) * a.rows * a.cols * (int64_t)sizeof(float) > PART_MOST) chunk *= 2;
    o.chunk = (int32_t)chunk;
    o.slots = a.g.n / o.chunk + 1;
    return o;
}
OuterTiles outer_plan(const dpaps_ps *ps, const OuterArgs &a, int kind, int count) {
    return kind == OUTER_LOW ? outer_tiles<Low>(ps, a, count == 2 ? 2 : 3) : kind == OUTER_64 ? outer_tiles<Tile64>(ps, a, 2) : outer_tiles<Tile128>(ps, a, 2);
}
size_t outer_part(const OuterArgs &a, const OuterTiles &o) {
    if (a.g.n <= o.chunk) return 0;
    return ((size_t)o.slots * (a.out_type == PS_F32 ? 1 : 2) * (size_t)a.rows * (size_t)a.cols * sizeof(float) + 255) / 256 * 256;
}
int64_t outer_grid(const OuterCall &c, int count) {
    int64_t most = 0;
    for (int i = 0; i < count; ++i) most = std::max(most, row_tiles(c.a[i].g.n, c.a[i].g.groups, c.o[i].chunk) * c.o[i].rows * c.o[i].cols);
    return most;
}
template <class K> int outer_start(dpaps_ps *ps, LdsAllowed &allowed, K kernel, const OuterCall &c, int64_t grid, int count, int threads, int lds, hipStream_t st) {
    if (grid >= ((int64_t)1 << 24)) return dpaps_too_large(ps, "expert_grad");
    const int rc = dpaps_allow_lds(ps, allowed, reinterpret_cast<const void *>(kernel), lds + AT_MOST * sizeof(int));
    if (rc) return rc;
    const int rows = std::min(std::max(c.o[0].chunk, c.o[1].chunk), AT_MOST);
    kernel<<<dim3((unsigned)grid, (unsigned)count), threads, lds + rows * sizeof(int), st>>>(c, ps->err);
    PS_HIP(ps, hipGetLastError());
    return PS_OK;
}
template <class CT, class LT, class RT, class T, bool LONG> int outer_of(dpaps_ps *ps, const OuterCall &c, int count, hipStream_t st) {
    static LdsAllowed allowed;
    return outer_start(ps, allowed, &k_outer<CT, LT, RT, T, LONG>, c, outer_grid(c, count), count, T::THREADS, T::LDS, st);
}
template <class CT, bool LONG> int outer_turned(dpaps_ps *ps, const OuterCall &c, hipStream_t st) {
    static LdsAllowed allowed;
    return outer_start(ps, allowed, &k_outer_turned<CT, Tile128, LONG>, c, outer_grid(c, 1), 1, 256, Turned<Tile128>::LDS, st);
}
bool outer_long(const OuterCall &c) { return std::max(c.o[0].chunk, c.o[1].chunk) > AT_MOST; }
template <class CT, class LT, class RT, class T> int outer_either(dpaps_ps *ps, const OuterCall &c, int count, hipStream_t st) {
    return outer_long(c) ? outer_of<CT, LT, RT, T, true>(ps, c, count, st) : outer_of<CT, LT, RT, T, false>(ps, c, count, st);
}
template <class CT> int outer_turned_either(dpaps_ps *ps, const OuterCall &c, hipStream_t st) {
    return outer_long(c) ? outer_turned<CT, true>(ps, c, st) : outer_turned<CT, false>(ps, c, st);
}
template <class CT, class LT, class RT> int outer_any(dpaps_ps *ps, const OuterCall &c, int count, int kind, hipStream_t st) {
    if (kind == OUTER_LOW) return outer_either<CT, LT, RT, Low>(ps, c, count, st);
    return kind == OUTER_64 ? outer_either<CT, LT, RT, Tile64>(ps, c, count, st) : outer_either<CT, LT, RT, Tile128>(ps, c, count, st);
}

}  // namespace

int dpaps_too_large(dpaps_ps *ps, const char *what) {
    ps->last_error = std::string(what) + ": too large for one launch";
    return PS_ELIMIT;
}

size_t dpaps_outer_bytes(const dpaps_ps *ps, const OuterArgs *a, int count) {
    const int kind = outer_kind(ps, a, count);
    size_t bytes = 0;
    for (int i = 0; i < count; ++i) bytes += outer_part(a[i], outer_plan(ps, a[i], kind, count));
    return bytes;
}
int dpaps_outer_sums(dpaps_ps *ps, const OuterArgs *a, int count, float *part, hipStream_t st) {
    const int kind = outer_kind(ps, a, count);
    char *at = (char *)part;
    OuterCall c{};
    bool join = false;
    int64_t most = 0;
    for (int i = 0; i < count; ++i) {
        c.a[i] = a[i];
        c.o[i] = outer_plan(ps, a[i], kind, count);
        c.o[i].part = (float *)at;
        at += outer_part(a[i], c.o[i]);
        join |= a[i].g.n > c.o[i].chunk;
        most = std::max(most, ceil_div64((int64_t)a[i].rows * a[i].cols, 1024));
    }
    int rc;
    if (kind == OUTER_TURNED) rc = a->left_type == PS_BF16 ? outer_turned_either<bf16_t>(ps, c, st) : outer_turned_either<f16_t>(ps, c, st);
    else if (a->left_type == PS_F32) {
        if (a->right_type == PS_F32) rc = outer_any<float, float, float>(ps, c, count, kind, st);
        else rc = a->right_type == PS_BF16 ? outer_any<float, float, bf16_t>(ps, c, count, kind, st) : outer_any<float, float, f16_t>(ps, c, count, kind, st);
    } else rc = a->left_type == PS_BF16 ? outer_any<bf16_t, bf16_t, bf16_t>(ps, c, count, kind, st) : outer_any<f16_t, f16_t, f16_t>(ps, c, count, kind, st);
    if (rc || !join) return rc;
    k_outer_join<<<dim3((unsigned)std::min<int64_t>(most, 256), (unsigned)std::min(a->g.groups, 1024), (unsigned)count), 256, 0, st>>>(c, ps->err);
    PS_HIP(ps, hipGetLastError());
    return PS_OK;
}
