// Tiles of products of rows with matrices of the server, on the matrix cores.
//
// A tile is sum_k R[k][r] C[k][c]: R, the tile's rows (of a call's tensors), C its columns (of the server's matrices, or of tensors).  Both come into LDS as
// units of 16 bytes, numbers that follow each other in k, of the type CT that the matrix instruction takes: 8 units of a row or column are a step, and lie in one
// line of 128 bytes.  What lies in memory in that order is read so (KMajor, KeyColumns); what lies the other way - neighbouring columns together - is read as blocks of
// a unit's numbers in k by four columns and turned in registers (KeyRows, ChosenRows).  The server's numbers of 32 bits are rounded to CT on the way.
#pragma once
#include "elements.h"

template <class T, int W> struct LooseOf { typedef T type __attribute__((ext_vector_type(W), aligned(sizeof(T)))); };
template <class T, int W> using Loose = typename LooseOf<T, W>::type;          // W neighbouring elements that start on any one

typedef float floatx16 __attribute__((ext_vector_type(16)));

template <class CT> constexpr int unit_of() { return 16 / (int)sizeof(CT); }   // numbers of a unit
constexpr int UNITS = 8;                                                       // units of a step
template <class CT> constexpr int step_of() { return UNITS * unit_of<CT>(); }  // numbers of a step

// Where unit u of row r lies in a tile in LDS.  Turned within the line by the row, so that neither eight neighbouring rows' same units (the
// matrix instruction's reads) nor those of every fourth row (what Blocks writes) share banks.
__device__ __forceinline__ int unit_place(int r, int u) { return r * UNITS + (u ^ ((r ^ (r >> 3)) & 7)); }

template <class CT, class ST, int W> __device__ __forceinline__ Vec<CT, W> as_type(Vec<ST, W> v) {
    if constexpr (std::is_same<CT, ST>::value) return v;
    else return __builtin_convertvector(v, Vec<CT, W>);
}

// Of a unit that starts at k, the numbers from K on become zero.
template <class ST, int W> __device__ __forceinline__ Vec<ST, W> cut(Vec<ST, W> v, int left) {
#pragma unroll
    for (int i = 0; i < W; ++i) v[i] = i < left ? v[i] : (ST)0.0f;
    return v;
}

// The W elements at p of which `left` exist (one at least), the others zero.  (Without a branch for each: their loads are on their way together.)
template <class ST, int W> __device__ __forceinline__ Vec<ST, W> load_some(const ST *p, int left) {
    if (left >= W) return *reinterpret_cast<const Loose<ST, W> *>(p);
    Vec<ST, W> v;
#pragma unroll
    for (int i = 0; i < W; ++i) v[i] = p[i < left ? i : 0];
    return cut<ST, W>(v, left);
}

// ROWS rows of a call's tensor, whose numbers follow each other in k; `row`s are where they start.  Rows that are not wanted may be any: they
// change nothing but their own results.
template <class ST, class CT, int ROWS, int THREADS> struct KMajor {
    static constexpr int KU = unit_of<CT>(), N = ROWS * UNITS / THREADS;
    static_assert(N * THREADS == ROWS * UNITS && THREADS % UNITS == 0);
    const ST *row[N];
    Vec<ST, KU> raw[N];
    template <class F> __device__ __forceinline__ void init(F row_of) {
#pragma unroll
        for (int i = 0; i < N; ++i) row[i] = row_of((i * THREADS + (int)threadIdx.x) / UNITS) + (int)threadIdx.x % UNITS * KU;
    }
    // TAIL: the step goes past K
    template <bool TAIL> __device__ __forceinline__ void load(int step, int K) {
        const int k0 = step * step_of<CT>(), left = K - k0 - (int)threadIdx.x % UNITS * KU;
#pragma unroll
        for (int i = 0; i < N; ++i) {
            if constexpr (!TAIL) raw[i] = *reinterpret_cast<const Loose<ST, KU> *>(row[i] + k0);
            else {
                raw[i] = Vec<ST, KU>{};
                if (left > 0) raw[i] = load_some<ST, KU>(row[i] + k0, left);
            }
        }
    }
    __device__ __forceinline__ void put(Vec<CT, KU> *lds) const {
#pragma unroll
        for (int i = 0; i < N; ++i) lds[unit_place((i * THREADS + (int)threadIdx.x) / UNITS, (int)threadIdx.x % UNITS)] = as_type<CT, ST, KU>(raw[i]);
    }
};

// COLS columns of a matrix in the server that are its keys, so that their numbers follow each other in k, from a key on; `cols` of them exist.  Reads past
// the last number of a key end in the next one, or in the slack behind the store.
// (Four numbers a lane, neighbours in neighbouring lanes: with a whole unit of 16-bit numbers a lane, 32 bytes, both of its accesses touched every line, and the
// die's cache was asked for all of them twice.)
template <class CT, int COLS, int THREADS> struct KeyColumns {
    static constexpr int PIECES = step_of<CT>() / 4, N = COLS * PIECES / THREADS;      // of four numbers
    static_assert(N * THREADS == COLS * PIECES && THREADS % PIECES == 0);
    const float *base;
    uint32_t at[N];
    Vec<float, 4> raw[N];
    __device__ static __forceinline__ int piece() { return (int)threadIdx.x % PIECES; }
    __device__ static __forceinline__ int col(int i) { return (i * THREADS + (int)threadIdx.x) / PIECES; }
    __device__ __forceinline__ void init(const float *w, int64_t L, int cols) {
        base = w;
#pragma unroll
        for (int i = 0; i < N; ++i) at[i] = (uint32_t)(col(i) < cols ? col(i) : cols - 1) * (uint32_t)L + (uint32_t)(piece() * 4);
    }
    template <bool TAIL> __device__ __forceinline__ void load(int step, int K) {
        const int k0 = step * step_of<CT>(), left = K - k0 - piece() * 4;
        const float *from = base + k0;
#pragma unroll
        for (int i = 0; i < N; ++i) {
            raw[i] = *reinterpret_cast<const Loose<float, 4> *>(from + (!TAIL || left > 0 ? at[i] : at[i] - (uint32_t)(piece() * 4)));
            if constexpr (TAIL) raw[i] = cut<float, 4>(raw[i], left);
        }
    }
    __device__ __forceinline__ void put(Vec<CT, unit_of<CT>()> *lds) const {
        constexpr int OF_UNIT = unit_of<CT>() / 4;
#pragma unroll
        for (int i = 0; i < N; ++i)
            reinterpret_cast<Vec<CT, 4> *>(lds + unit_place(col(i), piece() / OF_UNIT))[piece() % OF_UNIT] = as_type<CT, float, 4>(raw[i]);
    }
};

// Blocks of a unit's numbers in k by four columns, turned on their way into LDS.
template <class ST, class CT, int COLS, int THREADS> struct Blocks {
    static constexpr int KU = unit_of<CT>(), BLOCKS = COLS / 4 * UNITS, N = BLOCKS < THREADS ? 1 : BLOCKS / THREADS;
    static constexpr bool ALL = N * THREADS == BLOCKS;                         // else only the first threads have one
    static_assert(ALL || BLOCKS < THREADS);
    Vec<ST, 4> raw[N][KU];
    __device__ static __forceinline__ int block(int b) { return b * THREADS + (int)threadIdx.x; }
    __device__ static __forceinline__ int col(int b) { return block(b) % (COLS / 4) * 4; }
    __device__ static __forceinline__ int unit(int b) { return block(b) / (COLS / 4); }
    __device__ __forceinline__ void put(Vec<CT, KU> *lds) const {
#pragma unroll
        for (int b = 0; b < N; ++b) {
            if (!ALL && block(b) >= BLOCKS) return;
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                Vec<ST, KU> v;
#pragma unroll
                for (int i = 0; i < KU; ++i) v[i] = raw[b][i][j];
                lds[unit_place(col(b) + j, unit(b))] = as_type<CT, ST, KU>(v);
            }
        }
    }
};

// COLS columns of a matrix in the server whose keys follow each other in k; reads past a key's last column end in the next key or in the slack
// behind the store, which has room for 256.
template <class CT, int COLS, int THREADS> struct KeyRows : Blocks<float, CT, COLS, THREADS> {
    typedef Blocks<float, CT, COLS, THREADS> B;
    static_assert(COLS <= 256);
    const float *base;
    int64_t L;
    __device__ __forceinline__ void init(const float *w, int64_t L_) { base = w; L = L_; }
    template <bool TAIL> __device__ __forceinline__ void load(int step, int K) {
        const int k0 = step * step_of<CT>();
#pragma unroll
        for (int b = 0; b < B::N; ++b) {
            const int u = B::ALL || B::block(b) < B::BLOCKS ? B::unit(b) * B::KU : 0;
            const uint32_t at = (uint32_t)u * (uint32_t)L + (uint32_t)B::col(b);
#pragma unroll
            for (int i = 0; i < B::KU; ++i) {
                if constexpr (!TAIL) this->raw[b][i] = *reinterpret_cast<const Loose<float, 4> *>(base + (int64_t)(k0 + i) * L + at);
                else {
                    const int k = k0 + u + i;
                    this->raw[b][i] = *reinterpret_cast<const Loose<float, 4> *>(base + (int64_t)(k < K ? k : K - 1) * L + B::col(b));
                    this->raw[b][i] = cut<float, 4>(this->raw[b][i], k < K ? 4 : 0);
                }
            }
        }
    }
};

// COLS columns, `cols` of which exist, of rows of a call's tensor that are chosen one by one: row_of(k), where they start.
template <class ST, class CT, int COLS, int THREADS> struct ChosenRows : Blocks<ST, CT, COLS, THREADS> {
    typedef Blocks<ST, CT, COLS, THREADS> B;
    template <bool TAIL, class F> __device__ __forceinline__ void load(int step, int K, int cols, F row_of) {
        const int k0 = step * step_of<CT>();
#pragma unroll
        for (int b = 0; b < B::N; ++b) {
            const bool here = B::ALL || B::block(b) < B::BLOCKS;
            const int c = B::col(b), u = here ? B::unit(b) * B::KU : 0, left = here ? cols - c : 0;
            const ST *p[B::KU];
#pragma unroll
            for (int i = 0; i < B::KU; ++i) p[i] = row_of(!TAIL || k0 + u + i < K ? k0 + u + i : K - 1) + c;
            if (left >= 4) {
#pragma unroll
                for (int i = 0; i < B::KU; ++i) this->raw[b][i] = *reinterpret_cast<const Loose<ST, 4> *>(p[i]);
            } else {
#pragma unroll
                for (int i = 0; i < B::KU; ++i) {
                    this->raw[b][i] = Vec<ST, 4>{};
                    if (left > 0) this->raw[b][i] = load_some<ST, 4>(p[i], left);
                }
            }
            if constexpr (TAIL) {
#pragma unroll
                for (int i = 0; i < B::KU; ++i) this->raw[b][i] = cut<ST, 4>(this->raw[b][i], k0 + u + i < K ? 4 : 0);
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

// The instruction for 16 columns by 16 rows, as many units as there are lanes.
typedef float floatx4 __attribute__((ext_vector_type(4)));
template <class CT, int KU> __device__ __forceinline__ floatx4 mfma_small(Vec<CT, KU> a, Vec<CT, KU> b, floatx4 c) {
    if constexpr (sizeof(CT) == 4) {
#pragma unroll
        for (int j = 0; j < KU; ++j) c = __builtin_amdgcn_mfma_f32_16x16x4f32(a[j], b[j], c, 0, 0, 0);
        return c;
    } else if constexpr (std::is_same<CT, bf16_t>::value) return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0);
    else return __builtin_amdgcn_mfma_f32_16x16x32_f16(a, b, c, 0, 0, 0);
}

// What a wavefront multiplies at once: a pair of units of its columns and rows.
template <class CT, class T> struct Operands {
    Vec<CT, unit_of<CT>()> a[T::MC], b[T::MR];
    __device__ __forceinline__ void read(const Vec<CT, unit_of<CT>()> *tile, int c0, int r0, int pair) {
        const int l32 = threadIdx.x & 31, h = (threadIdx.x & 63) >> 5;
#pragma unroll
        for (int i = 0; i < T::MC; ++i) a[i] = tile[T::ROWS * UNITS + unit_place(c0 + 32 * i + l32, 2 * pair + h)];
#pragma unroll
        for (int j = 0; j < T::MR; ++j) b[j] = tile[unit_place(r0 + 32 * j + l32, 2 * pair + h)];
    }
    __device__ __forceinline__ void multiply(floatx16 (&acc)[T::MC][T::MR]) const {
#pragma unroll
        for (int i = 0; i < T::MC; ++i)
#pragma unroll
            for (int j = 0; j < T::MR; ++j) acc[i][j] = mfma_unit<CT>(a[i], b[j], acc[i][j]);
    }
};

// A tile's sum over K.  load(set, step, tail): asks for a step's numbers, put(set, where): brings them into LDS, rows and then columns; a set is what a thread holds of a
// step.  Lane l of the wavefront whose part starts at column c0 and row r0 holds in acc[i][j][4 q + e] the column c0 + 32 i + 8 q + 4 (l / 32) + e of row
// r0 + 32 j + l % 32.
// Two steps are in LDS, and T::SETS more are on their way to registers.  Every pair of units is read from LDS while the one before is multiplied, the first
// pair of a step while the last of the step before is.
template <class CT, class T, class Load, class Put>
__device__ __forceinline__ void tile_sum(int K, Vec<CT, unit_of<CT>()> *lds, int c0, int r0, Load load, Put put, floatx16 (&acc)[T::MC][T::MR]) {
    constexpr int SIZE = (T::ROWS + T::COLS) * UNITS;
    static_assert(UNITS == 8 && (T::SETS == 1 || T::SETS == 2));
    typedef std::integral_constant<int, 0> First;
    typedef std::integral_constant<int, T::SETS - 1> Second;
    const int full = K / step_of<CT>(), steps = (K + step_of<CT>() - 1) / step_of<CT>();
    const auto fetch = [&](auto set, int s) {
        if (s < full) load(set, s, std::false_type{});
        else load(set, s, std::true_type{});
    };
    if (steps <= 0) return;
    Operands<CT, T> x, y;
    fetch(First{}, 0);
    if (T::SETS == 2 && steps > 1) fetch(Second{}, 1);
    put(First{}, lds);
    if (steps > T::SETS) fetch(First{}, T::SETS);
    __syncthreads();
    x.read(lds, c0, r0, 0);
    // step s, which is in that half of LDS; `set` holds the next one
    const auto step = [&](int s, auto set, auto half) {
        const Vec<CT, unit_of<CT>()> *here = lds + decltype(half)::value * SIZE;
        Vec<CT, unit_of<CT>()> *next = lds + (1 - decltype(half)::value) * SIZE;
        y.read(here, c0, r0, 1);
        __builtin_amdgcn_sched_barrier(0);
        x.multiply(acc);
        x.read(here, c0, r0, 2);
        __builtin_amdgcn_sched_barrier(0);
        y.multiply(acc);
        y.read(here, c0, r0, 3);
        __builtin_amdgcn_sched_barrier(0);
        x.multiply(acc);
        if (s + 1 < steps) {
            put(set, next);
            if (s + 1 + T::SETS < steps) fetch(set, s + 1 + T::SETS);
            __syncthreads();
            x.read(next, c0, r0, 0);
            __builtin_amdgcn_sched_barrier(0);
        }
        y.multiply(acc);
    };
    for (int s = 0; s < steps; s += 2) {
        step(s, Second{}, std::integral_constant<int, 0>{});
        if (s + 1 < steps) step(s + 1, First{}, std::integral_constant<int, 1>{});
    }
    __syncthreads();                                                 // (LDS is used again)
}
// The same, of few numbers: up to one step, of the pairs of units that there are.
template <class CT, class T, class Load, class Put>
__device__ __forceinline__ void tile_sum_short(int K, Vec<CT, unit_of<CT>()> *lds, int c0, int r0, Load load, Put put, floatx16 (&acc)[T::MC][T::MR]) {
    for (int s = 0; s * step_of<CT>() < K; ++s) {
        const int left = K - s * step_of<CT>();
        if (left >= step_of<CT>()) load(std::integral_constant<int, 0>{}, s, std::false_type{});
        else load(std::integral_constant<int, 0>{}, s, std::true_type{});
        put(std::integral_constant<int, 0>{}, lds);
        __syncthreads();
        for (int p = 0; 2 * p * unit_of<CT>() < left && p < UNITS / 2; ++p) {
            Operands<CT, T> x;
            x.read(lds, c0, r0, p);
            x.multiply(acc);
        }
        __syncthreads();
    }
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

// A tile's form: WC x WR wavefronts of 32 MC columns by 32 MR rows each.
template <int MC_, int MR_, int WC_, int WR_> struct Form {
    static constexpr int MC = MC_, MR = MR_, WC = WC_, WR = WR_, COLS = 32 * MC * WC, ROWS = 32 * MR * WR, THREADS = 64 * WC * WR;
    static constexpr int LDS = 2 * (ROWS + COLS) * UNITS * 16;              // two steps
    static constexpr int BLOCKS = MC * MR > 4 ? 1 : 2;                  // workgroups a compute unit has to have room for
    static constexpr int SETS = MC * MR == 1 ? 2 : 1;                   // steps on their way to registers
};
typedef Form<1, 1, 2, 2> Tile64;
typedef Form<2, 2, 2, 2> Tile128;
typedef Form<2, 4, 4, 2> Tile256;
typedef Form<1, 1, 1, 4> Narrow;                                     // 32 columns, 128 rows
typedef Form<1, 1, 4, 1> Low;                                        // 128 columns, 32 rows

// Which tile a workgroup has.  Workgroups go to the compute dies in turn: each die gets runs of neighbouring tiles, row by row of tiles in bands of BAND columns of
// them, so that what its cache holds is read by several.  The runs are dealt out in turn, eight or more to a die where there are enough tiles: some
// numbers of tiles of grouped rows have no rows, and lie together.  (All of a die's tiles in one run: 62 us instead of 51 for 16,001 rows of 64 groups, 17 with rows.)
constexpr uint32_t DIES = 8;
constexpr int BAND = 8;
struct TilePlace { int row, col; };                                  // row < 0: none
__host__ __device__ inline uint32_t die_run(uint32_t tiles) {
    uint32_t run = 32;
    while (run > 1 && tiles < 8 * DIES * run) run /= 2;
    return run;
}
inline unsigned die_grid(int64_t tiles) { const int64_t all = DIES * die_run((uint32_t)tiles); return (unsigned)((tiles + all - 1) / all * all); }
__device__ __forceinline__ TilePlace tile_place(int row_tiles, int col_tiles) {
    const uint32_t tiles = (uint32_t)row_tiles * col_tiles, run = die_run(tiles), turn = blockIdx.x / DIES;
    const uint32_t at = (turn / run * DIES + blockIdx.x % DIES) * run + turn % run;
    if (at >= tiles) return TilePlace{-1, 0};
    const uint32_t of_band = (uint32_t)row_tiles * BAND, band = at / of_band, r = at - band * of_band;
    const uint32_t cols = (uint32_t)col_tiles - band * BAND < BAND ? (uint32_t)col_tiles - band * BAND : BAND;
    return TilePlace{(int)(r / cols), (int)(band * BAND + r % cols)};
}

// Neighbouring numbers of a result, of which `left` exist.
template <class T> using Global = __attribute__((address_space(1))) T;
template <class T, int W> __device__ __forceinline__ void put_some(T *to, Vec<float, W> v, int left) {
    Global<T> *p = (Global<T> *)to;
    const Vec<T, W> x = as_type<T, float, W>(v);
    if (left >= W) *(Global<Loose<T, W>> *)p = x;
    else
#pragma unroll
        for (int i = 0; i < W; ++i)
            if (i < left) p[i] = x[i];
}
template <int W> __device__ __forceinline__ void put_typed(void *to, int32_t type, int64_t at, Vec<float, W> v, int left) {
    if (type == PS_F32) put_some<float, W>(reinterpret_cast<float *>(to) + at, v, left);
    else if (type == PS_BF16) put_some<bf16_t, W>(reinterpret_cast<bf16_t *>(to) + at, v, left);
    else put_some<f16_t, W>(reinterpret_cast<f16_t *>(to) + at, v, left);
}

// A tile's sums leave by way of LDS, 32 rows of a wavefront at a time, so that rows are written in whole lines: eight numbers a lane.  to_of(r): where
// row r of the tile starts, counted in elements, or -1: nowhere; c0: the tile's first column of the N.
constexpr int SUMS_PAD = 4;
template <class T, class CT> constexpr bool sums_fit() { return T::WC * T::WR * 32 * (32 * T::MC + SUMS_PAD) * 4 <= T::LDS; }
// add(r, c, left, v): what is added to the eight numbers from column c of the tile on, before they are rounded.
struct Nothing { __device__ __forceinline__ void operator()(int, int, int, Vec<float, 8> &) const {} };
template <class OT, class T, class F, class Add>
__device__ __forceinline__ void put_tile(const floatx16 (&acc)[T::MC][T::MR], float *lds, OT *out, int c0, int N, float scale, F to_of, Add add) {
    constexpr int LD = 32 * T::MC + SUMS_PAD, LANES = 4 * T::MC, AT_ONCE = 64 / LANES;         // lanes of a row, rows at a time
    static_assert(sums_fit<T, float>());
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, l32 = lane & 31, h = lane >> 5;
    const int wc = wave % T::WC * 32 * T::MC, wr = wave / T::WC * 32 * T::MR;
    float *mine = lds + wave * 32 * LD;
#pragma unroll
    for (int j = 0; j < T::MR; ++j) {
#pragma unroll
        for (int i = 0; i < T::MC; ++i)
#pragma unroll
            for (int q = 0; q < 4; ++q)
                *reinterpret_cast<Vec<float, 4> *>(mine + l32 * LD + 32 * i + 8 * q + 4 * h) =
                    Vec<float, 4>{acc[i][j][4 * q], acc[i][j][4 * q + 1], acc[i][j][4 * q + 2], acc[i][j][4 * q + 3]};
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
        const int c = lane % LANES * 8, left = N - c0 - wc - c;
#pragma unroll 4
        for (int r = lane / LANES; r < 32; r += AT_ONCE) {
            const int64_t to = to_of(wr + 32 * j + r);
            const Vec<float, 4> lo = *reinterpret_cast<const Vec<float, 4> *>(mine + r * LD + c), hi = *reinterpret_cast<const Vec<float, 4> *>(mine + r * LD + c + 4);
            if (to < 0 || left <= 0) continue;
            Vec<float, 8> v = scale * __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7);
            add(wr + 32 * j + r, wc + c, left, v);
            put_some<OT, 8>(out + to + c0 + wc + c, v, left);
        }
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    }
}
template <class T, class F, class Add = Nothing>
__device__ __forceinline__ void put_tile_typed(const floatx16 (&acc)[T::MC][T::MR], void *lds, void *out, int32_t type, int c0, int N, float scale, F to_of, Add add = Add{}) {
    float *sums = reinterpret_cast<float *>(lds);
    if (type == PS_F32) put_tile<float, T>(acc, sums, reinterpret_cast<float *>(out), c0, N, scale, to_of, add);
    else if (type == PS_BF16) put_tile<bf16_t, T>(acc, sums, reinterpret_cast<bf16_t *>(out), c0, N, scale, to_of, add);
    else put_tile<f16_t, T>(acc, sums, reinterpret_cast<f16_t *>(out), c0, N, scale, to_of, add);
}

// until at most N of this wavefront's loads are on their way and all it has asked of LDS is there, then until all wavefronts are so far
template <int N> __device__ __forceinline__ void wait_and_meet() {
    asm volatile("" ::: "memory");
    __builtin_amdgcn_s_waitcnt(0x0070 | (N & 15) | ((N >> 4) << 14));
    __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");
}
// The order of a turn's instructions: reads of LDS and loads spread over the products.
template <int PRODUCTS, int READS, int LOADS, int I = 0> __device__ __forceinline__ void spread() {
    constexpr int R = (I + 1) * READS / PRODUCTS - I * READS / PRODUCTS, L = (I + 1) * LOADS / PRODUCTS - I * LOADS / PRODUCTS;
    __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);
    if constexpr (R > 0) __builtin_amdgcn_sched_group_barrier(0x100, R, 0);
    if constexpr (L > 0) __builtin_amdgcn_sched_group_barrier(0x020, L, 0);
    if constexpr (I + 1 < PRODUCTS) spread<PRODUCTS, READS, LOADS, I + 1>();
}

// What stands in LDS where rows or numbers end comes from here.
namespace { __device__ __attribute__((aligned(64))) unsigned char zero_bytes[64]; }
