// Products of many rows of 16 bits with matrices of the server: the matrices are laid first, in 16 bits and in the order in which the product loads them, so that the
// product's operands both go straight from memory into LDS, several stages ahead.
//
// A matrix is laid in blocks of 16 columns and 32 numbers of each, 1,024 bytes: a line of 64 bytes for each column, its four units of eight numbers at the
// places u ^ (column / 4) % 4, where the wavefronts' reads of one unit of 32 columns meet all banks.  Rows come from where they are, 64 bytes each, into
// LDS in the same order: a lane asks for the unit that belongs to its place.
//
// k_lay is bound by memory (16 matrices of 2048 x 1024, 131 MB, of which the counter sees 67 read, and 67 written, in 38 us: 5.2 TB/s), k_laid by how well its loads and reads of LDS
// hide under the products, the matrix units busy for 0.4 to 0.5 of it: 32,768 rows of those 16, with the laying, 202 us (830 TFLOP/s without it) where some hundred calls have followed one
// another, and 209 to 270 in the first thirty after a pause.  That is taken to be the clock, as the card lets it under load: four draws of the groups, of 950 to 6,170 rows, agree within 2 us, and rows of
// zeros take 182.  16,001 rows x 1024 of 24 adapters of 32 ranks, 63 us, 550 TFLOP/s.
#include "experts.h"

namespace {

constexpr int KB = 32;                                       // numbers of a block
constexpr int64_t BLOCK = 16 * KB;                           // elements
inline int64_t col_blocks(int32_t N) { return ceil_div64(N, 256) * 16; }      // (whole tiles)
inline int64_t k_blocks(int32_t K) { return ceil_div64(K, KB); }

// A workgroup lays 16 columns of 256 numbers as they lie, or 64 columns of 64 numbers that it turns in LDS; each[0]: of group blockIdx.z's matrix, each[1]: of the
// one behind them.
struct LayCall {
    LayArgs a[2];
    int32_t cb[2], kb[2], tiles[2];                          // columns and numbers in blocks, workgroups of a matrix
};
template <class T, bool TURNED> __device__ __forceinline__ void lay(const LayArgs &a, int e, int tile, int cb_all, int kb_all) {
    const int tid = threadIdx.x;
    const float *w = a.w + (int64_t)e * a.each * a.L;
    T *to = reinterpret_cast<T *>(a.to) + e * a.size;
    const auto place = [&](int c, int k) { return ((int64_t)(c >> 4) * kb_all + (k >> 5)) * BLOCK + (c & 15) * KB + (((k >> 3 & 3) ^ (c >> 2 & 3)) * 8); };
    if constexpr (!TURNED) {
        const int across = (kb_all * KB + 255) / 256, c = tile / across * 16 + (tid >> 4), k0 = tile % across * 256 + (tid & 15) * 8;
#pragma unroll
        for (int u = 0; u < 2; ++u) {
            const int k = k0 + u * 128;
            if (k >= kb_all * KB) return;
            Vec<float, 8> v = {};
            if (c < a.N && k < a.K) v = cut<float, 8>(*reinterpret_cast<const Loose<float, 8> *>(w + (int64_t)c * a.L + k), a.K - k);
            *reinterpret_cast<Vec<T, 8> *>(to + place(c, k)) = as_type<T, float, 8>(v);
        }
    } else {
        __shared__ float turn[64][65];
        const int across = (kb_all * KB + 63) / 64, c0 = tile / across * 64, k0 = tile % across * 64;
#pragma unroll
        for (int u = 0; u < 4; ++u) {
            const int k = u * 16 + (tid >> 4), c = (tid & 15) * 4;
            Vec<float, 4> v = {};
            if (k0 + k < a.K && c0 + c < a.N) v = load_some<float, 4>(w + (int64_t)(k0 + k) * a.L + c0 + c, a.N - c0 - c);
#pragma unroll
            for (int i = 0; i < 4; ++i) turn[k][c + i] = v[i];
        }
        __syncthreads();
#pragma unroll
        for (int u = 0; u < 2; ++u) {
            const int c = tid & 63, k = (tid >> 6) * 16 + u * 8;
            if (k0 + k >= kb_all * KB || c0 + c >= cb_all * 16) continue;
            Vec<float, 8> v;
#pragma unroll
            for (int i = 0; i < 8; ++i) v[i] = turn[k + i][c];
            *reinterpret_cast<Vec<T, 8> *>(to + place(c0 + c, k0 + k)) = as_type<T, float, 8>(v);
        }
    }
}
template <class T> __global__ __launch_bounds__(256) void k_lay(LayCall call, RowGroups g, const int32_t *err) {
    if (*(volatile const int32_t *)err) return;
    const int e = blockIdx.z, which = e == g.groups ? 1 : 0, tile = blockIdx.x;
    if (tile >= call.tiles[which]) return;
    if (which == 0 && g.start(e) >= g.start(e + 1)) return;
    const LayArgs &a = call.a[which];
    if (a.turned) lay<T, true>(a, which ? 0 : e, tile, call.cb[which], call.kb[which]);
    else lay<T, false>(a, which ? 0 : e, tile, call.cb[which], call.kb[which]);
}

template <class CT, class T> struct LaidForm {
    // (four stages of 32 KB, or three of 16, of which three workgroups share a compute unit)
    static constexpr int STAGES = T::ROWS == 256 ? 4 : 3, STAGE = (T::ROWS + T::COLS) * KB * 2, LDS = STAGES * STAGE, WAVES = T::WC * T::WR, ROW_LOADS = T::ROWS / 16 / WAVES, COL_LOADS = T::COLS / 16 / WAVES, LOADS = ROW_LOADS + COL_LOADS;
};

// The sum of a tile.  A stage is 32 numbers of all rows and columns; while a pair of units is multiplied the next one is read from LDS and half of a later stage's loads are asked
// for, and a wavefront waits for the stage that is needed next only, whatever has been asked for behind it.  LOW: one matrix for all rows, and behind its
// numbers the low-rank ones of the tile's adapter, as further stages.
template <class CT, class T, bool LOW>
__global__ __launch_bounds__(T::THREADS, T::BLOCKS) void k_laid(LaidArgs a, int32_t row_tiles, int32_t col_tiles, int32_t kb_all, int32_t b_kb, int32_t *err) {
    typedef LaidForm<CT, T> F;
    constexpr int BR = T::ROWS, BC = T::COLS, STAGES = F::STAGES;
    extern __shared__ __align__(16) unsigned char lds[];
    __shared__ int at[BR];
    __shared__ int off;
    look_for_all(err, &off);
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const TilePlace place = tile_place(row_tiles, col_tiles);
    if (place.row < 0) return;
    const int tile = place.row, c0 = place.col * BC;
    const RowTile t = row_tile(a.g, tile, BR);
    if (t.rows == 0) return;
    for (int r = tid; r < BR; r += T::THREADS) at[r] = r < t.rows ? row_at(a.g, t.first + r, err) : -1;
    __syncthreads();
    if (off) return;
    floatx16 acc[T::MC][T::MR] = {};
    const int wc = wave % T::WC * 32 * T::MC, wr = wave / T::WC * 32 * T::MR;
    if (LOW || t.group < a.g.groups) {
        // The loads of a stage: this wavefront's blocks of 16 rows, and of 16 columns.  What they come from changes where an adapter's numbers follow
        // the shared matrix's.
        const int unit = (lane & 3) ^ (lane >> 4 & 3);
        const bool low = LOW && t.group < a.g.groups;
        const CT *row[F::ROW_LOADS];
        const CT *col = reinterpret_cast<const CT *>(a.w) + (LOW ? 0 : t.group * a.w_size) + (int64_t)(c0 / 16 + wave * F::COL_LOADS) * kb_all * BLOCK + lane * 8;
        const int stages = kb_all + (low ? b_kb : 0);
        int col_step = kb_all, left = kb_all, K = a.K;
#pragma unroll
        for (int i = 0; i < F::ROW_LOADS; ++i) {
            const int q = at[(wave * F::ROW_LOADS + i) * 16 + (lane >> 2)];
            row[i] = reinterpret_cast<const CT *>(a.x) + a.x_shared(q < 0 ? 0 : q) * a.x_stride + unit * 8;
        }
        const auto to_adapter = [&]() {
#pragma unroll
            for (int i = 0; i < F::ROW_LOADS; ++i) {
                const int r = (wave * F::ROW_LOADS + i) * 16 + (lane >> 2);
                row[i] = reinterpret_cast<const CT *>(a.low) + (int64_t)(t.first + (r < t.rows ? r : 0)) * a.low_stride + unit * 8;
            }
            col = reinterpret_cast<const CT *>(a.b) + t.group * a.b_size + (int64_t)(c0 / 16 + wave * F::COL_LOADS) * b_kb * BLOCK + lane * 8;
            col_step = left = b_kb;
            K = a.rank;
        };
        // half of a stage's loads, the rows' or the columns'; k: where in the sum the stage is
        const auto fetch = [&](int slot, bool rows, int k) {
            unsigned char *to = lds + slot * F::STAGE + (rows ? wave * F::ROW_LOADS : BR / 16 + wave * F::COL_LOADS) * 1024;
            if (rows) {
                const bool here = k + unit * 8 < K;
#pragma unroll
                for (int i = 0; i < F::ROW_LOADS; ++i)
                    __builtin_amdgcn_global_load_lds((const __attribute__((address_space(1))) void *)(here ? row[i] + k : reinterpret_cast<const CT *>(zero_bytes)),
                                                     (__attribute__((address_space(3))) void *)(to + i * 1024), 16, 0, 0);
            } else {
#pragma unroll
                for (int i = 0; i < F::COL_LOADS; ++i)
                    __builtin_amdgcn_global_load_lds((const __attribute__((address_space(1))) void *)(col + ((int64_t)i * col_step + (k >> 5)) * BLOCK),
                                                     (__attribute__((address_space(3))) void *)(to + i * 1024), 16, 0, 0);
            }
        };
        int k_next = 0, fetched = 0;
        // to the stage behind the one that was fetched last; behind the last one that one once more, into a slot that nobody reads, so that all turns are alike
        const auto advance = [&]() {
            if (++fetched >= stages) return;
            if (--left == 0) {
                if constexpr (LOW) to_adapter();
                k_next = 0;
            } else k_next += KB;
        };
        const int l32 = lane & 31, h = lane >> 5;
        typedef Vec<CT, 8> Unit;
        Unit xa[T::MC], xb[T::MR], ya[T::MC], yb[T::MR];
        const auto read = [&](Unit (&ra)[T::MC], Unit (&rb)[T::MR], int slot, int pair) {
            const unsigned char *from = lds + slot * F::STAGE;
            const auto unit_at = [&](int r) { return *reinterpret_cast<const Unit *>(from + r * 64 + (((2 * pair + h) ^ (r >> 2 & 3)) * 16)); };
#pragma unroll
            for (int i = 0; i < T::MC; ++i) ra[i] = unit_at(BR + wc + 32 * i + l32);
#pragma unroll
            for (int j = 0; j < T::MR; ++j) rb[j] = unit_at(wr + 32 * j + l32);
        };
        const auto multiply = [&](const Unit (&ra)[T::MC], const Unit (&rb)[T::MR]) {
#pragma unroll
            for (int i = 0; i < T::MC; ++i)
#pragma unroll
                for (int j = 0; j < T::MR; ++j) acc[i][j] = mfma_unit<CT>(ra[i], rb[j], acc[i][j]);
        };
#pragma unroll
        for (int s = 0; s < STAGES - 1; ++s) {
            fetch(s, true, k_next);
            fetch(s, false, k_next);
            advance();
        }
        wait_and_meet<(STAGES - 2) * F::LOADS>();
        read(xa, xb, 0, 0);
        int slot = 0, into = STAGES - 1;
        for (int s = 0; s < stages; ++s) {
            read(ya, yb, slot, 1);
            fetch(into, true, k_next);
            multiply(xa, xb);
            spread<T::MC * T::MR, T::MC + T::MR, F::ROW_LOADS>();
            // this stage has been read, and the next one is there
            wait_and_meet<(STAGES - 3) * F::LOADS + F::ROW_LOADS>();
            const int next = slot + 1 == STAGES ? 0 : slot + 1;
            read(xa, xb, next, 0);
            fetch(into, false, k_next);
            multiply(ya, yb);
            spread<T::MC * T::MR, T::MC + T::MR, F::COL_LOADS>();
            advance();
            into = slot;
            slot = next;
        }
        wait_and_meet<0>();                                  // nothing is on its way to LDS
    }
    put_tile_typed<T>(acc, lds, a.out, a.out_type, c0, a.N, 1.0f, [&](int r) { return at[r] < 0 ? (int64_t)-1 : (int64_t)at[r] * a.out_stride; });
}

template <class CT, class T, bool LOW> int start(dpaps_ps *ps, const LaidArgs &a, hipStream_t st) {
    typedef LaidForm<CT, T> F;
    const int32_t col_tiles = (a.N + T::COLS - 1) / T::COLS;
    const int64_t tiles = row_tiles(a.g.n, a.g.groups, T::ROWS), grid = tiles * col_tiles;
    if (grid >= ((int64_t)1 << 24)) return dpaps_too_large(ps, "product");
    static LdsAllowed allowed;
    const int rc = dpaps_allow_lds(ps, allowed, reinterpret_cast<const void *>(&k_laid<CT, T, LOW>), F::LDS);
    if (rc) return rc;
    k_laid<CT, T, LOW><<<die_grid(grid), T::THREADS, F::LDS, st>>>(a, (int32_t)tiles, col_tiles, (int32_t)k_blocks(a.K), (int32_t)k_blocks(a.rank), ps->err);
    PS_HIP(ps, hipGetLastError());
    return PS_OK;
}
template <class CT> int start_any(dpaps_ps *ps, const LaidArgs &a, hipStream_t st) {
    // tiles of 256 where nearly all of them are full, and there is one for every compute unit: 16,384 rows of one group, 1024 x 1024, 44 us and 53 by tiles of 128; of
    // four groups 69 and 57, because the rests of the groups leave the last round of the compute units half empty
    const bool large = a.g.n >= 16384 * (int64_t)a.g.groups && ceil_div64(a.g.n, 256) * ceil_div64(a.N, 256) >= ps->num_cu;
    if (a.low) return large ? start<CT, Tile256, true>(ps, a, st) : start<CT, Tile128, true>(ps, a, st);
    return large ? start<CT, Tile256, false>(ps, a, st) : start<CT, Tile128, false>(ps, a, st);
}

}  // namespace

int64_t dpaps_laid_size(int32_t K, int32_t N) { return col_blocks(N) * k_blocks(K) * BLOCK; }
bool dpaps_laid_fits(const void *x, int64_t x_stride, int32_t K) { return K % 8 == 0 && (uintptr_t)x % 16 == 0 && x_stride % 8 == 0; }

int dpaps_lay(dpaps_ps *ps, const RowGroups &g, int32_t type, const LayArgs &each, const LayArgs *one, hipStream_t st) {
    LayCall c{};
    int32_t most = 0;
    for (int i = 0; i < (one ? 2 : 1); ++i) {
        c.a[i] = i ? *one : each;
        const LayArgs &a = c.a[i];
        c.cb[i] = (int32_t)col_blocks(a.N);
        c.kb[i] = (int32_t)k_blocks(a.K);
        c.tiles[i] = (int32_t)(a.turned ? c.cb[i] / 4 * ceil_div64(c.kb[i] * KB, 64) : c.cb[i] * ceil_div64(c.kb[i] * KB, 256));
        most = c.tiles[i] > most ? c.tiles[i] : most;
    }
    const dim3 grid((unsigned)most, 1, (unsigned)(g.groups + (one ? 1 : 0)));
    if (type == PS_BF16) k_lay<bf16_t><<<grid, 256, 0, st>>>(c, g, ps->err);
    else k_lay<f16_t><<<grid, 256, 0, st>>>(c, g, ps->err);
    PS_HIP(ps, hipGetLastError());
    return PS_OK;
}

int dpaps_laid_product(dpaps_ps *ps, int32_t type, const LaidArgs &a, hipStream_t st) {
    return type == PS_BF16 ? start_any<bf16_t>(ps, a, st) : start_any<f16_t>(ps, a, st);
}
