// Tokens: the lookup of their embeddings in the server, the gradient of that lookup, and a step of AdaGrad with it.
//
// Token t is key first_key + t, its embedding the first `dim` values of the key.
//   lookup     out_p = s E[t_p]                                     (zero where t_p is padding)
//   gradient   g_v = s sum over the p with t_p = v of dout_p
//   AdaGrad    G_v += g_v^2,  E_v -= lr g_v / sqrt(G_v + eps)       (G_v: the key's next `dim` values)
// The sums go over sorted tokens: the pairs (token, position) are brought into that order (key_sort.hip) and cut into
// ranges, and the terms of a token inside one range are added one after the other in increasing position, in 32 bits,
// from zero; the sums of a token's ranges are then added in range order.  No floating-point atomics: the result
// depends on the arguments only.
#include "elements.h"
#include "token_ids.h"

#include <type_traits>

namespace {

inline unsigned grid_for(int64_t n, int block) { return (unsigned)((n + block - 1) / block); }
inline size_t up256(size_t x) { return (x + 255) / 256 * 256; }

__device__ __forceinline__ uint64_t readlane_u64(uint64_t x, int l) {
    const uint32_t lo = (uint32_t)__builtin_amdgcn_readlane((int)(uint32_t)x, l);
    const uint32_t hi = (uint32_t)__builtin_amdgcn_readlane((int)(uint32_t)(x >> 32), l);
    return ((uint64_t)hi << 32) | lo;
}

__global__ __launch_bounds__(256) void k_emb_check(TokenIds t, int32_t *err) {
    const int64_t p = (int64_t)blockIdx.x * blockDim.x + threadIdx.x;
    if (p < t.n && t.bad(t.at(p))) atomicExch(err, PS_EKEY);
}

__global__ __launch_bounds__(256) void k_route_tokens(RouteArgs a, TokenIds t, const int32_t *err) {
    __shared__ RouteLds l;
    route_tokens_block(a, t, l, blockIdx.x, flag_ahead(err));
}

// the replies of an access have set the requester's location cache (k_cache_replies, for tokens)
__global__ __launch_bounds__(256) void k_token_replies(TokenIds t, int32_t worker, const int32_t *owner, int16_t *loc_row, const int32_t *err) {
    if (*(volatile const int32_t *)err) return;
    const int64_t p = (int64_t)blockIdx.x * blockDim.x + threadIdx.x;
    if (p >= t.n) return;
    const int64_t id = t.at(p);
    if (t.padding(id)) return;
    const int32_t o = owner[t.first + id];
    if (o != worker) loc_row[t.first + id] = (int16_t)o;
}

// ---- lookup ---------------------------------------------------------------------------------------------------------
// The result in pieces of W values, P a row, a workgroup 256 * AHEAD consecutive pieces, a thread every 256th: its tokens,
// then its pieces of the rows, are asked for together.  The first route.blocks workgroups count the statistics.
// Memory bounds it: 65,537 tokens of 50,000, by rank, 512 numbers to bf16: 96 MB (the rows mentioned once, the result) in 20 us, 4.8 TB/s; with pieces of 4
// instead of 8, whose stores are of 8 bytes, 25 us.  More than a few tokens are checked in a launch before it (4 us), so that a bad one leaves
// the result as it was.
template <class Out, int W, int AHEAD>
__global__ __launch_bounds__(256) void k_emb_lookup(RouteArgs route, TokenIds t, uint32_t P, double inv_P, int64_t L, float scale, const float *val, Out *out,
                                                    int64_t stride, int32_t *err) {
    const bool few = t.n <= FEW_KEYS;
    const int32_t stop = few ? 0 : flag_ahead(err);
    __shared__ RouteLds l;
    if ((int)blockIdx.x < route.blocks) {
        if (few && few_tokens_off(t, err)) return;
        route_tokens_block(route, t, l, blockIdx.x, stop);
        return;
    }
    const int64_t block = blockIdx.x - route.blocks;
    // (the quotients of numbers up to 1023 + 2048: see k_pull)
    const int64_t first = block * (256 * AHEAD), total = t.n * P;
    const int64_t p0 = quotient(first, P, inv_P);
    const uint32_t c0 = (uint32_t)(first - p0 * P);
    const float inv_Pf = (float)inv_P;
    int64_t id[AHEAD];
    uint32_t c[AHEAD], row[AHEAD];
#pragma unroll
    for (int u = 0; u < AHEAD; ++u) {
        const uint32_t at = c0 + u * 256u + threadIdx.x;
        row[u] = (uint32_t)(((float)at + 0.5f) * inv_Pf);
        c[u] = at - row[u] * P;
        id[u] = first + u * 256 + threadIdx.x < total ? t.at(p0 + row[u]) : 0;
    }
    if (few ? few_tokens_off(t, err) : stop != 0) return;
    Vec<float, W> x[AHEAD];
#pragma unroll
    for (int u = 0; u < AHEAD; ++u) {
        x[u] = Vec<float, W>{};
        if (first + u * 256 + threadIdx.x < total && !t.padding(id[u])) x[u] = load_vec<float, W>(val + (t.first + id[u]) * L + (int64_t)c[u] * W) * scale;
    }
#pragma unroll
    for (int u = 0; u < AHEAD; ++u)
        if (first + u * 256 + threadIdx.x < total) store_vec<Out, W>(out + (p0 + row[u]) * stride + (int64_t)c[u] * W, x[u]);
}

// ---- sums over sorted tokens ----------------------------------------------------------------------------------------
struct EmbSums {
    const uint64_t *skeys; const uint32_t *spos; int64_t n;      // the sorted pairs
    int64_t count, first;                                        // tokens, the key of token 0
    int32_t range;                                               // sorted positions of a range, at most 64
    int32_t D;
    const void *dout; int64_t stride;
    float scale;
    float *part;                                                 // two rows of D per range
    float *to; int64_t L;                                        // where a token's row is: the gradient (L = D) or the store
    float lr, eps;
};

// What becomes of a token's sum: a row of the gradient, added to what is there, or a step of AdaGrad.
enum EmbMode { EMB_GRAD, EMB_GRAD_ADD, EMB_ADAGRAD };
template <int MODE, int W> struct Old { Vec<float, W> v[MODE == EMB_GRAD ? 1 : MODE]; };
template <int MODE, int W>
__device__ __forceinline__ void emb_read(Old<MODE, W> &o, const EmbSums &a, int64_t token, int c) {
    const float *p = a.to + (a.first + token) * a.L + (int64_t)c * W;
    if constexpr (MODE >= EMB_GRAD_ADD) o.v[0] = load_vec<float, W>(p);
    if constexpr (MODE == EMB_ADAGRAD) o.v[1] = load_vec<float, W>(p + a.D);
}
template <int MODE, int W>
__device__ __forceinline__ void emb_finish(const Old<MODE, W> &o, const EmbSums &a, int64_t token, int c, Vec<float, W> sum) {
    float *p = a.to + (a.first + token) * a.L + (int64_t)c * W;
    const Vec<float, W> g = sum * a.scale;
    if constexpr (MODE == EMB_GRAD) store_vec<float, W>(p, g);
    if constexpr (MODE == EMB_GRAD_ADD) store_vec<float, W>(p, o.v[0] + g);
    if constexpr (MODE == EMB_ADAGRAD) {
        const Vec<float, W> G = o.v[1] + g * g;
        Vec<float, W> e = o.v[0];
        if constexpr (W == 1) e = e - a.lr * g / sqrtf(G + a.eps);
        else
            for (int i = 0; i < W; ++i) e[i] = e[i] - a.lr * g[i] / sqrtf(G[i] + a.eps);
        store_vec<float, W>(p, e);
        store_vec<float, W>(p + a.D, G);
    }
}

// D zeros, by a wavefront (16 bytes a lane at most: neighbouring lanes' stores make whole lines)
template <int W> __device__ __forceinline__ void clear_row(float *p, int D) {
    constexpr int V = W < 4 ? W : 4;
    for (int c = (threadIdx.x & 63) * V; c < D; c += 64 * V) store_vec<float, V>(p + c, Vec<float, V>{});
}

constexpr int CLEAR_ROWS = 16;                         // rows of tokens not mentioned that a wavefront clears at a time
constexpr int64_t CLEARERS = (int64_t)1 << 20;         // workgroups at most that clear rows
constexpr uint64_t NOKEY = ~0ull;                      // no token looks like this

// Which of the rows v0 .. v0 + CLEAR_ROWS - 1 are mentioned, a bit each, the same in all lanes: their first place among the sorted tokens, 64 places
// looked at in one trip to memory, and the 64 tokens from there on.  Where those do not reach the last row - tokens mentioned often -, four lanes look
// for each row in what is behind, a fifth left after every trip.  (38,438 tokens of 231: the join 10 us; row after row with all lanes 25.)
__device__ __forceinline__ uint32_t emb_mentioned(const EmbSums &a, int64_t v0) {
    const int lane = threadIdx.x & 63;
    uint32_t rows = 0;
    int64_t lo = 0, hi = a.n;                                          // the first place of a token v0 or above is one of these, or hi
    while (hi - lo > 64) {
        const int64_t by = (hi - lo + 63) / 64, at = lo + lane * by;
        const int below = __popcll(__ballot(at < hi && (int64_t)a.skeys[at < hi ? at : lo] < v0));
        const int64_t base = lo;
        if (below > 0) lo = base + (below - 1) * by + 1;
        if (base + below * by < hi) hi = base + below * by;
        if (below == 0) break;
    }
    const int64_t k = lo + lane < a.n ? (int64_t)a.skeys[lo + lane] : INT64_MAX;
#pragma unroll
    for (int i = 0; i < CLEAR_ROWS; ++i)
        if (__ballot(k == v0 + i) != 0) rows |= 1u << i;
    if ((int64_t)readlane_u64((uint64_t)k, 63) >= v0 + CLEAR_ROWS - 1) return rows;
    static_assert(CLEAR_ROWS * 4 == 64);
    const int64_t v = v0 + (lane >> 2);
    lo += 64;
    hi = a.n;
    while (__ballot(lo < hi) != 0) {
        const int64_t by = (hi - lo + 4) / 5, at = lo + ((lane & 3) + 1) * by - 1;
        const int below = __popcll(__ballot(at < hi && (int64_t)a.skeys[at < hi ? at : 0] < v) >> (lane & ~3) & 15);
        if (lo < hi && below < 4 && lo + (below + 1) * by - 1 < hi) hi = lo + (below + 1) * by - 1;
        lo += below * by;
    }
    const u64 there = __ballot(lo < a.n && (int64_t)a.skeys[lo < a.n ? lo : 0] == v);
#pragma unroll
    for (int i = 0; i < CLEAR_ROWS; ++i) rows |= (uint32_t)(there >> (4 * i) & 1) << i;
    return rows;
}

// A wavefront per range and 64 pieces of W values; UN rows are on their way together.  The first workgroups count the statistics.
// Memory bounds it where there are many terms: 262,144 of 512 bf16 numbers onto a gradient of 128,000, by rank: 268 MB of terms in any order, 200 MB of the
// gradient, 119 us, 3.9 TB/s; AdaGrad of 65,536 49 us.  With 16,384 of 1024 (15 us) it is the chain of trips: tokens, rows, sums.
template <class T, int W, int MODE>
__global__ __launch_bounds__(256) void k_emb_sums(RouteArgs route, TokenIds t, EmbSums a, const int32_t *err) {
    constexpr int UN = MODE == EMB_ADAGRAD ? 8 : W >= 4 ? 8 : 16;
    const int32_t stop = flag_ahead(err);
    const int lane = threadIdx.x & 63;
    int64_t block = blockIdx.x;
    if constexpr (MODE == EMB_ADAGRAD) {
        __shared__ RouteLds l;
        if (block < route.blocks) {
            if (blockIdx.y == 0) route_tokens_block(route, t, l, (int)block, stop);
            return;
        }
        block -= route.blocks;
    }
    const int64_t r = block * 4 + __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6), q0 = r * a.range;
    if (q0 >= a.n) return;
    const int here = (int)(a.n - q0 < a.range ? a.n - q0 : a.range);
    const uint64_t mk = lane < here ? a.skeys[q0 + lane] : NOKEY;       // lane i: sorted position q0 + i
    const uint64_t before = lane < here && q0 + lane > 0 ? a.skeys[q0 + lane - 1] : NOKEY;
    const uint64_t next = q0 + here < a.n ? a.skeys[q0 + here] : NOKEY;
    const int mp = lane < here ? (int)a.spos[q0 + lane] : 0;
    if (stop) return;
    const int cnt = __popcll(__ballot(lane < here && (int64_t)mk < a.count));          // padding comes last
    if (cnt == 0) return;
    u64 heads = __ballot(lane < cnt && before != mk);                   // positions where a token's terms start
    const bool first_open = (heads & 1) == 0;                           // the first token's terms continue from the range before,
    const bool last_open = next == readlane_u64(mk, cnt - 1);           // the last one's go on in the range behind
    const u64 ends = (heads >> 1) | (1ull << (cnt - 1));                // positions where they end
    const int c = blockIdx.y * 64 + lane;
    const bool in = c * W < a.D;
    const T *dout = reinterpret_cast<const T *>(a.dout) + (int64_t)c * W;
    Vec<float, W> v = {};
    Old<MODE, W> kept;                                                  // of the token whose terms are being added
    bool from_zero = first_open;                                        // its terms started in a range before
    for (int i0 = 0; i0 < cnt; i0 += UN) {
        Vec<float, W> d[UN];
        Old<MODE, W> old[UN];
#pragma unroll
        for (int i = 0; i < UN; ++i) {
            d[i] = Vec<float, W>{};
            if (in && i0 + i < cnt) {
                d[i] = load_vec<T, W>(dout + (int64_t)(uint32_t)__builtin_amdgcn_readlane(mp, i0 + i) * a.stride);
                if constexpr (MODE != EMB_GRAD)
                    if ((heads >> (i0 + i)) & 1) emb_read<MODE, W>(old[i], a, (int64_t)readlane_u64(mk, i0 + i), c);
            }
        }
#pragma unroll
        for (int i = 0; i < UN; ++i) {
            const int u = i0 + i;
            if (u < cnt) {
                if ((heads >> u) & 1) {
                    v = Vec<float, W>{};
                    from_zero = false;
                    if constexpr (MODE != EMB_GRAD) kept = old[i];
                }
                v = v + d[i];
                if ((ends >> u) & 1) {
                    const bool open = u == cnt - 1 && last_open;
                    if (in) {
                        if (from_zero || open) store_vec<float, W>(a.part + (2 * r + (from_zero ? 0 : 1)) * (int64_t)a.D + (int64_t)c * W, v);
                        else emb_finish<MODE, W>(kept, a, (int64_t)readlane_u64(mk, u), c, v);
                    }
                }
            }
        }
    }
}

// Tokens whose terms fill more than one range: the workgroup of the range in which they start adds the sums of the ranges behind it, each
// wavefront a quarter of them in order, and then the four.  blockIdx.y: which 64 pieces.  The other workgroups, of a gradient that is not added to,
// clear the rows of tokens that are not mentioned meanwhile: the few trips to memory, one behind the other, of a join hide behind that.
// 50,000 rows of 1024, 44,800 of them not mentioned: 184 MB in 29 us, 6.3 TB/s; without rows to clear, 4,096 ranges of 64 x 512, 17 us, most of it a frequent
// token's thousands of ranges (8 or 16 wavefronts a range instead of 4: 25 and 55 us).  Clearing all of the gradient on a second stream beside
// the sort costs more than it hides: 82 us instead of 60.
constexpr int JOIN_AHEAD = 16;
template <int W, int MODE>
__global__ __launch_bounds__(256) void k_emb_join(EmbSums a, int64_t joins, const int32_t *err) {
    const int32_t stop = flag_ahead(err);
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6);
    if (MODE == EMB_GRAD && blockIdx.x >= joins) {
        if (blockIdx.y != 0 || stop) return;
        for (int64_t v0 = ((blockIdx.x - joins) * 4 + wave) * CLEAR_ROWS; v0 < a.count; v0 += (gridDim.x - joins) * 4 * CLEAR_ROWS) {
            const uint32_t mentioned = emb_mentioned(a, v0);
            for (int i = 0; i < CLEAR_ROWS && v0 + i < a.count; ++i)
                if (!(mentioned >> i & 1))
                    clear_row<W>(a.to + (v0 + i) * a.L, a.D);
        }
        return;
    }
    __shared__ Vec<float, W> sums[4][64];
    const int64_t r = blockIdx.x, R = a.range, q1 = (r + 1) * R;
    if (q1 >= a.n) return;
    const uint64_t key = a.skeys[q1 - 1], next = a.skeys[q1];
    const uint64_t start = r > 0 ? a.skeys[q1 - R] : NOKEY, before = r > 0 ? a.skeys[q1 - R - 1] : NOKEY;
    if (stop != 0 || next != key || (int64_t)key >= a.count) return;
    if (start == key && before == key) return;                                         // they started earlier
    // the ranges behind that begin with the token follow one another: 64 are looked at, spread over what is left
    const int64_t nranges = (a.n + R - 1) / R;
    int64_t lo = r + 1, hi = nranges, by = 1;
    while (lo < hi) {
        const int64_t at = lo + lane * by;
        const u64 b = __ballot(at < hi && a.skeys[(at < hi ? at : lo) * R] == key);
        const int run = b == ~0ull ? 64 : __ffsll((long long)~b) - 1;
        if (run < 64 && lo + run * by < hi) hi = lo + run * by;
        if (run > 0) lo += (run - 1) * by + 1;
        by = (hi - lo + 63) / 64;
    }
    // sum 0 is of range r, sum j of range r + j, j <= m
    const int64_t m = lo - (r + 1), j0 = (m + 1) * wave / 4, j1 = (m + 1) * (wave + 1) / 4;
    const int c = blockIdx.y * 64 + lane;
    const bool in = c * W < a.D;
    const float *part = a.part + (in ? (int64_t)c * W : 0);
    Old<MODE, W> old;
    if (wave == 0 && in) emb_read<MODE, W>(old, a, (int64_t)key, c);
    Vec<float, W> v = {};
    for (int64_t j = j0; j < j1; j += JOIN_AHEAD) {
        Vec<float, W> d[JOIN_AHEAD];
#pragma unroll
        for (int i = 0; i < JOIN_AHEAD; ++i) d[i] = j + i < j1 ? load_vec<float, W>(part + (2 * (r + j + i) + (j + i == 0 ? 1 : 0)) * (int64_t)a.D) : Vec<float, W>{};
#pragma unroll
        for (int i = 0; i < JOIN_AHEAD; ++i)
            if (j + i < j1) v = v + d[i];
    }
    sums[wave][lane] = v;
    __syncthreads();
    if (wave == 0 && in) emb_finish<MODE, W>(old, a, (int64_t)key, c, sums[0][lane] + sums[1][lane] + sums[2][lane] + sums[3][lane]);
}

// ---- few tokens: one launch, without a sort -----------------------------------------------------------------------------
// Every workgroup checks all tokens and has them in LDS.  A wavefront takes a position: if no position before it has the same token, the
// positions that have it are the token's terms, in order.  They are added one after the other; more than FEW_OWN by the whole workgroup,
// a sixteenth each, and then the sixteen.  Further workgroups clear the rows of tokens not mentioned, FEW_CLEAR each; the first ones count the
// statistics.
// The launch and a few trips to memory bound it: 64 tokens of 128 numbers 6.5 us, 1,024 8 to 10 (of 5,000, bf16, evenly spread to as their rank),
// where a sort and the sums take 11.4 and 14.  By 2,048 tokens the two meet: 11.9 us and 13.9 evenly spread, 14.4 and 13.9 by rank, a single
// token, all of whose terms one workgroup adds, 38 and 18.  FEW_OWN 16: by rank 512 tokens 7.8 us and 1,024 10.0, with 64 13.7 and 13.7, with 8 7.9 and 10.0.
constexpr int FEW_THREADS = 1024, FEW_WAVES = FEW_THREADS / 64, FEW_OWN = 16, FEW_CLEAR = 64;
template <class T, int W, int MODE>
__global__ __launch_bounds__(FEW_THREADS) void k_emb_few(RouteArgs route, TokenIds t, EmbSums a, int32_t *err) {
    constexpr size_t SUMS = (size_t)FEW_KEYS * 8, ALL = SUMS + (size_t)FEW_WAVES * 64 * W * 4;
    __shared__ __attribute__((aligned(32))) unsigned char mem[ALL > sizeof(RouteLds) ? ALL : sizeof(RouteLds)];
    __shared__ uint32_t many;                                          // which wavefronts' tokens the whole workgroup works on,
    __shared__ u64 many_mask[FEW_WAVES][FEW_KEYS / 64], many_key[FEW_WAVES];   // and what they found of them
    __shared__ int many_count[FEW_WAVES];
    __shared__ bool named[FEW_CLEAR];
    uint64_t *lk = reinterpret_cast<uint64_t *>(mem);
    Vec<float, W> *sums = reinterpret_cast<Vec<float, W> *>(mem + SUMS);
    const int n = (int)t.n;
    if (threadIdx.x == 0) many = 0;
    if (few_tokens_off<2>(t, err, [&](int64_t p, int64_t id) { lk[p] = t.padding(id) ? NOKEY : (uint64_t)id; })) return;
    int block = blockIdx.x;
    if constexpr (MODE == EMB_ADAGRAD) {
        if (block < route.blocks) {
            __syncthreads();                                           // (the tokens in LDS are not needed here)
            if (blockIdx.y == 0) route_tokens_block(route, t, *reinterpret_cast<RouteLds *>(mem), block, 0);
            return;
        }
        block -= route.blocks;
    }
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6), chunks = (n + 63) / 64;
    const int groups = (n + FEW_WAVES - 1) / FEW_WAVES;
    if constexpr (MODE == EMB_GRAD) {
        if (block >= groups) {
            if (blockIdx.y != 0) return;
            for (int64_t v0 = (int64_t)(block - groups) * FEW_CLEAR; v0 < a.count; v0 += (int64_t)((int)gridDim.x - groups) * FEW_CLEAR) {
                if (threadIdx.x < FEW_CLEAR) named[threadIdx.x] = false;
                __syncthreads();
                for (int p = threadIdx.x; p < n; p += FEW_THREADS)
                    if (lk[p] - (uint64_t)v0 < FEW_CLEAR) named[lk[p] - (uint64_t)v0] = true;
                __syncthreads();
                for (int r = wave; r < FEW_CLEAR && v0 + r < a.count; r += FEW_WAVES)
                    if (!named[r])
                        clear_row<W>(a.to + (v0 + r) * a.L, a.D);
                __syncthreads();
            }
            return;
        }
    }
    // (the positions dealt out to the workgroups in turn, shifted from turn to turn: frequent tokens are first named by the first
    // positions, or at equal distances, and a workgroup takes its own one after the other)
    const int mine = wave * groups + (block + 5 * wave) % groups;
    const int c = blockIdx.y * 64 + lane;
    const bool in = c * W < a.D;
    const T *dout = reinterpret_cast<const T *>(a.dout) + (in ? (int64_t)c * W : 0);
    u64 mask = 0;                                                      // lane i: which of the positions 64 i .. have the token
    int count = 0;
    uint64_t key = NOKEY;
    const auto look = [&](int p) {
        if (p >= n) return false;
        key = lk[p];
        key = readlane_u64(key, 0);
        if (key == NOKEY) return false;
        for (int i = 0; i < chunks; ++i) {
            const u64 same = __ballot(64 * i + lane < n && lk[64 * i + lane] == key);
            if (64 * i <= p && (64 * i + 63 < p ? same : same & ((1ull << (p & 63)) - 1ull)) != 0) return false;
            count += __popcll(same);
            mask = lane == i ? same : mask;
        }
        return true;
    };
    // the sum of the token's terms [lo, hi), one after the other
    const auto sum = [&](int lo, int hi) {
        constexpr int UN = W >= 4 ? 8 : 16;
        Vec<float, W> v = {};
        if (lo >= hi) return v;
        int at = 0, seen = 0;                                          // the positions from 64 at on, `seen` terms are before those
        u64 m = readlane_u64(mask, 0);
        while (seen + __popcll(m) <= lo) { seen += __popcll(m); m = readlane_u64(mask, ++at); }
        for (; seen < lo; ++seen) m &= m - 1ull;
        while (lo < hi) {
            Vec<float, W> d[UN];
            int got = 0;
#pragma unroll
            for (int u = 0; u < UN; ++u) {
                d[u] = Vec<float, W>{};
                if (lo + u < hi) {
                    while (m == 0) m = readlane_u64(mask, ++at);
                    const int p = 64 * at + __ffsll((long long)m) - 1;
                    m &= m - 1ull;
                    if (in) d[u] = load_vec<T, W>(dout + (int64_t)p * a.stride);
                    ++got;
                }
            }
#pragma unroll
            for (int u = 0; u < UN; ++u)
                if (u < got) v = v + d[u];
            lo += got;
        }
        return v;
    };
    if (look(mine)) {
        if (count <= FEW_OWN) {
            Old<MODE, W> old;
            if (in) emb_read<MODE, W>(old, a, (int64_t)key, c);
            const Vec<float, W> v = sum(0, count);
            if (in) emb_finish<MODE, W>(old, a, (int64_t)key, c, v);
        } else {
            if (lane < (int)FEW_KEYS / 64) many_mask[wave][lane] = mask;
            if (lane == 0) { many_key[wave] = key; many_count[wave] = count; atomicOr(&many, 1u << wave); }
        }
    }
    __syncthreads();
    uint32_t left = (uint32_t)__builtin_amdgcn_readfirstlane((int)many);
    while (left != 0) {
        const int w = __ffs((int)left) - 1;
        left &= left - 1u;
        mask = lane < (int)FEW_KEYS / 64 ? many_mask[w][lane] : 0;
        key = readlane_u64(many_key[w], 0);
        count = __builtin_amdgcn_readfirstlane(many_count[w]);
        sums[wave * 64 + lane] = sum(count * wave / FEW_WAVES, count * (wave + 1) / FEW_WAVES);
        __syncthreads();
        if (wave == 0 && in) {
            Old<MODE, W> old;
            emb_read<MODE, W>(old, a, (int64_t)key, c);
            Vec<float, W> v = sums[lane];
            for (int k = 1; k < FEW_WAVES; ++k) v = v + sums[k * 64 + lane];
            emb_finish<MODE, W>(old, a, (int64_t)key, c, v);
        }
        __syncthreads();                                               // the sums' place is used again
    }
}

// ---- host ---------------------------------------------------------------------------------------------------------
// What all calls check of their tokens.
int token_ids(dpaps_ps *ps, int64_t first_key, int64_t num_tokens, bool in_store, const void *tokens, int32_t token_type, int64_t n, int64_t pad, TokenIds *t) {
    if (n < 0 || (n > 0 && !tokens) || num_tokens <= 0 || first_key < 0 || (token_type != PS_I32 && token_type != PS_I64)) return PS_EINVAL;
    if (in_store && (num_tokens > ps->K || first_key > ps->K - num_tokens)) return PS_EINVAL;
    if (n > PS_EMB_MAX_TOKENS || num_tokens >= ((int64_t)1 << 31)) {
        ps->last_error = "tokens: at most 2^29 in a call, of a vocabulary of less than 2^31";
        return PS_ELIMIT;
    }
    t->ids = tokens; t->wide = token_type == PS_I64; t->n = n; t->first = first_key; t->count = num_tokens; t->pad = pad; t->padded = pad != PS_NO_PAD;
    return PS_OK;
}

template <class Out>
int lookup(dpaps_ps *ps, const RouteArgs &a, const TokenIds &t, int32_t dim, float scale, Out *out, int32_t type, int64_t stride, hipStream_t st) {
    const auto fits = [&](int w) { return rows_allow(ps->val, PS_F32, dim, ps->L, w) && rows_allow(out, type, dim, stride, w); };
#define LOOKUP(W, AHEAD)                                                                                                                          \
    do {                                                                                                                                          \
        const uint32_t P = (uint32_t)(dim / W);                                                                                                   \
        const int64_t blocks = a.blocks + ceil_div64(t.n * P, 256 * AHEAD);                                                                       \
        if (blocks >= ((int64_t)1 << 24)) { ps->last_error = "emb_lookup: the result is too large for one launch"; return PS_ELIMIT; }            \
        const unsigned grid = (unsigned)blocks;                                                                                                   \
        if (t.n > FEW_KEYS) {                                                                                                                     \
            k_emb_check<<<grid_for(t.n, 256), 256, 0, st>>>(t, ps->err);                                                                          \
            PS_HIP(ps, hipGetLastError());                                                                                                        \
        }                                                                                                                                         \
        k_emb_lookup<Out, W, AHEAD><<<grid, 256, 0, st>>>(a, t, P, 1.0 / P, ps->L, scale, ps->val, out, stride, ps->err);                  \
    } while (0)
    if (sizeof(Out) == 2 && fits(8)) LOOKUP(8, 2);
    else if (fits(4)) LOOKUP(4, 4);
    else if (fits(2)) LOOKUP(2, 4);
    else LOOKUP(1, 8);
#undef LOOKUP
    PS_HIP(ps, hipGetLastError());
    return PS_OK;
}

// The sorted pairs and what the sums need, in the handle's scratch.
int sums_of(dpaps_ps *ps, const RouteArgs &route, const TokenIds &t, EmbSums a, int32_t dout_type, int mode, hipStream_t st) {
    const int bits = dpaps_key_bits(t.count + 1);
    // Values of a lane, and so the wavefronts that a row takes.  16-bit rows 16 bytes at a time, unless rows of 32 bits are read and written as often: a
    // wavefront's accesses to those then have gaps.  16,384 rows of 1024 into a gradient that is cleared: the sums 15 us with 8, 20 with 4;
    // 262,144 of 512 added to one: 126 with 8, 118 with 4.
    const auto fits = [&](int w) { return rows_allow(a.dout, dout_type, a.D, a.stride, w) && rows_allow(a.to, PS_F32, a.D, a.L, w); };
    const int W = dout_type != PS_F32 && mode == EMB_GRAD && a.D > 256 && fits(8) ? 8 : a.D > 64 && fits(4) ? 4 : 1;
    const int64_t slices = (a.D / W + 63) / 64;
    a.n = t.n; a.count = t.count; a.first = t.first;
    const bool few = t.n <= FEW_KEYS;
    // workgroups that clear `rows` rows at a time (a launch has less than 2^32 threads)
    const auto clearers = [&](int64_t rows) { const int64_t all = ceil_div64(t.count, rows); return all < CLEARERS ? all : CLEARERS; };
    dim3 grid, join;
    int64_t joins = 0;
    if (few) {
        grid = dim3((unsigned)((mode == EMB_GRAD ? clearers(FEW_CLEAR) : 0) + route.blocks + ceil_div64(t.n, FEW_WAVES)), (unsigned)slices);
    } else {
        // ranges of 64 positions, shorter ones where those would be fewer wavefronts (of 256 values) than the compute units hold; by the
        // number of tokens and the length of a row alone, so that a gradient that is added to gets the same sums (4,096 terms of 256: the whole call 15 us, with
        // ranges of 64 33; 16,384 of 1024 39 and 51; 65,536 of 512 51 and 59)
        a.range = 64;
        while (a.range > 8 && ceil_div64(t.n, a.range) * ceil_div64(a.D, 256) < 16 * (int64_t)ps->num_cu) a.range /= 2;
        const int64_t nranges = ceil_div64(t.n, a.range);
        const size_t off_spos = up256((size_t)t.n * 8), off_part = off_spos + up256((size_t)t.n * 4),
                     off_sort = off_part + up256((size_t)nranges * 2 * (size_t)a.D * sizeof(float));
        int rc = dpaps_ws_reserve(ps, off_sort + dpaps_sort_scratch_bytes(t.n, bits));
        if (rc) return rc;
        char *ws = (char *)ps->ws;
        a.skeys = (const uint64_t *)ws;
        a.spos = (const uint32_t *)(ws + off_spos);
        rc = dpaps_sort_tokens(ps, t, (uint64_t *)ws, (uint32_t *)(ws + off_spos), ws + off_sort, st);
        if (rc) return rc;
        a.part = (float *)(ws + off_part);
        joins = nranges - 1;
        grid = dim3((unsigned)(route.blocks + ceil_div64(nranges, 4)), (unsigned)slices);
        join = dim3((unsigned)(joins + (mode == EMB_GRAD ? clearers(4 * CLEAR_ROWS) : 0)), (unsigned)slices);
    }
    if (grid.x == 0) return PS_OK;
#define SUMS(T, WW, MODE)                                                                     \
    do {                                                                                      \
        if (few) { k_emb_few<T, WW, MODE><<<grid, FEW_THREADS, 0, st>>>(route, t, a, ps->err); break; } \
        k_emb_sums<T, WW, MODE><<<grid, 256, 0, st>>>(route, t, a, ps->err);                  \
        PS_HIP(ps, hipGetLastError());                                                        \
        k_emb_join<WW, MODE><<<join, 256, 0, st>>>(a, joins, ps->err);                        \
    } while (0)
#define MODES(T, WW)                                                                          \
    do {                                                                                      \
        if (mode == EMB_GRAD) SUMS(T, WW, EMB_GRAD);                                          \
        else if constexpr (WW < 8) {                                                          \
            if (mode == EMB_GRAD_ADD) SUMS(T, WW, EMB_GRAD_ADD);                              \
            else SUMS(T, WW, EMB_ADAGRAD);                                                    \
        }                                                                                     \
    } while (0)
#define WIDTHS(T)                                                                             \
    do {                                                                                      \
        if (W == 1) MODES(T, 1);                                                              \
        else if (W == 4) MODES(T, 4);                                                         \
        else if constexpr (sizeof(T) == 2) MODES(T, 8);                                       \
    } while (0)
    if (dout_type == PS_F32) WIDTHS(float);
    else if (dout_type == PS_BF16) WIDTHS(bf16_t);
    else WIDTHS(f16_t);
#undef WIDTHS
#undef MODES
#undef SUMS
    PS_HIP(ps, hipGetLastError());
    return PS_OK;
}

}  // namespace

int dpaps_route_tokens(dpaps_ps *ps, int32_t worker, const TokenIds &t, bool pull, bool push, hipStream_t st) {
    if (worker < 0 || t.n == 0) return PS_OK;
    if (ps->loc && pull && push) {       // with location caches the second access is routed after the first one's replies
        const int rc = dpaps_route_tokens(ps, worker, t, true, false, st);
        return rc ? rc : dpaps_route_tokens(ps, worker, t, false, true, st);
    }
    const RouteArgs a = dpaps_route_args(ps, worker, t.n, pull ? PS_STAT_PULL_LOCAL : PS_STAT_PUSH_LOCAL, pull ? PS_STAT_PULL_REMOTE : PS_STAT_PUSH_REMOTE,
                                         pull && push ? PS_STAT_PUSH_LOCAL : -1, pull && push ? PS_STAT_PUSH_REMOTE : -1, st);
    k_route_tokens<<<a.blocks, 256, 0, st>>>(a, t, ps->err);
    PS_HIP(ps, hipGetLastError());
    if (ps->loc) {
        k_token_replies<<<grid_for(t.n, 256), 256, 0, st>>>(t, worker, ps->owner, ps->loc + (int64_t)worker * ps->K, ps->err);
        PS_HIP(ps, hipGetLastError());
    }
    return PS_OK;
}

extern "C" int emb_lookup(ps_handle ps, int32_t worker, int64_t first_key, int64_t num_tokens, int32_t dim, const void *tokens, int32_t token_type, int64_t n,
                          int64_t pad_token, float scale, void *out, int32_t out_type, int64_t out_stride, void *stream) {
    if (!ps || !is_element_type(out_type) || dim <= 0 || dim > ps->L || (n > 0 && (!out || out_stride < dim))) return PS_EINVAL;
    if (worker < -1 || worker >= ps->W) return PS_EWORKER;
    TokenIds t;
    int rc = token_ids(ps, first_key, num_tokens, true, tokens, token_type, n, pad_token, &t);
    if (rc || n == 0) return rc;
    hipStream_t st = (hipStream_t)stream;
    RouteArgs a{};
    if (!ps->loc) a = dpaps_route_args(ps, worker, n, PS_STAT_PULL_LOCAL, PS_STAT_PULL_REMOTE, -1, -1, st);
    if (out_type == PS_F32) rc = lookup(ps, a, t, dim, scale, (float *)out, out_type, out_stride, st);
    else if (out_type == PS_BF16) rc = lookup(ps, a, t, dim, scale, (bf16_t *)out, out_type, out_stride, st);
    else rc = lookup(ps, a, t, dim, scale, (f16_t *)out, out_type, out_stride, st);
    if (rc || !ps->loc) return rc;
    return dpaps_route_tokens(ps, worker, t, true, false, st);         // (behind the check, which few tokens have in the lookup)
}

extern "C" int emb_grad(ps_handle ps, int64_t num_tokens, int32_t dim, const void *tokens, int32_t token_type, int64_t n, int64_t pad_token, float scale,
                        const void *dout, int32_t dout_type, int64_t dout_stride, float *grad, int32_t accumulate, void *stream) {
    if (!ps || !is_element_type(dout_type) || dim <= 0 || dim > PS_EMB_MAX_DIM || !grad || (n > 0 && (!dout || dout_stride < 0))) return PS_EINVAL;
    TokenIds t;
    const int rc = token_ids(ps, 0, num_tokens, false, tokens, token_type, n, pad_token, &t);
    if (rc) return rc;
    EmbSums a{};
    a.D = dim; a.dout = dout; a.stride = dout_stride; a.scale = scale; a.to = grad; a.L = dim;
    return sums_of(ps, RouteArgs{}, t, a, dout_type, accumulate ? EMB_GRAD_ADD : EMB_GRAD, (hipStream_t)stream);
}

extern "C" int emb_adagrad_step(ps_handle ps, int32_t worker, int64_t first_key, int64_t num_tokens, int32_t dim, const void *tokens, int32_t token_type,
                                int64_t n, int64_t pad_token, float scale, const void *dout, int32_t dout_type, int64_t dout_stride, float lr, float eps,
                                void *stream) {
    if (!ps || !is_element_type(dout_type) || dim <= 0 || dim > ps->L / 2 || !(eps > 0.0f) || (n > 0 && (!dout || dout_stride < 0))) return PS_EINVAL;
    if (worker < -1 || worker >= ps->W) return PS_EWORKER;
    TokenIds t;
    int rc = token_ids(ps, first_key, num_tokens, true, tokens, token_type, n, pad_token, &t);
    if (rc || n == 0) return rc;
    hipStream_t st = (hipStream_t)stream;
    EmbSums a{};
    a.D = dim; a.dout = dout; a.stride = dout_stride; a.scale = scale; a.to = ps->val; a.L = ps->L; a.lr = lr; a.eps = eps;
    RouteArgs route{};
    if (!ps->loc) route = dpaps_route_args(ps, worker, n, PS_STAT_PULL_LOCAL, PS_STAT_PULL_REMOTE, PS_STAT_PUSH_LOCAL, PS_STAT_PUSH_REMOTE, st);
    rc = sums_of(ps, route, t, a, dout_type, EMB_ADAGRAD, st);
    return rc || !ps->loc ? rc : dpaps_route_tokens(ps, worker, t, true, true, st);
}
