// Rows ordered by the group that they name (an expert, an adapter): a stable counting sort, and where the groups start.
//
// place of row p = #{q: g_q < g_p} + #{q < p: g_q = g_p};  rows of no group (padding) stand behind all others, as group `groups`.
// A wavefront takes 64 neighbouring rows at a time: the lanes that name one group are found by a vote per bit of the group's number, so that a
// row's place within the 64 is a count of bits, and a wavefront's counts of a group are its own word in LDS.  No atomics on places: the order is stable.
//
// Few bytes move (131,072 int32 ids in, their order out: 1 MB); what a call takes are launches and the chain of trips to memory and of votes in each.
#include "groups.h"

#include <algorithm>

namespace {

constexpr int THREADS = 1024, WAVES = THREADS / 64;
constexpr int MOST_GROUPS = 2046;                  // beside the rows of no group: 128 KB of counts in LDS
constexpr int MOST_BLOCKS = 128;                   // each looks at the counts of all
constexpr int MOST_CHUNK = 16384;                  // rows of a workgroup
constexpr int64_t ONE_CHUNK = 4096;                // ... of the only one

struct GroupArgs {
    TokenIds t;
    int32_t groups, chunk, blocks, bits;
    uint32_t *count;                               // blocks x (groups + 1)
    int32_t *order, *offsets;
};

// The lanes that hold the same key; `in`: this lane has one.
__device__ __forceinline__ uint64_t same_key(bool in, uint32_t key, int bits) {
    uint64_t m = __ballot(in);
    for (int b = 0; b < bits; ++b) {
        const bool one = key >> b & 1u;
        const uint64_t v = __ballot(one);
        m &= one ? v : ~v;
    }
    return m;
}
// A wavefront's rows, HELD times 64 of them at once (so that their ids are asked for together): f(row, is there one, key, lanes with that key).  Up to that many, what has
// been read for the count is kept for the places.  Returns whether a row names no group that there is.
constexpr int HELD = 4;
struct Held { uint32_t key[HELD]; uint64_t same[HELD]; };
template <bool AGAIN, class F> __device__ __forceinline__ bool each_64(const GroupArgs &a, int64_t first, Held &held, F f) {
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int64_t end = first + a.chunk < a.t.n ? first + a.chunk : a.t.n, share = (a.chunk + 64 * WAVES - 1) / (64 * WAVES) * 64;
    int64_t stop = first + (wave + 1) * share;
    if (stop > end) stop = end;
    const bool keep = share <= 64 * HELD;
    bool bad = false;
    for (int64_t p0 = first + wave * share; p0 < stop; p0 += 64 * HELD) {
        if (!(AGAIN && keep)) {
            int64_t id[HELD];
#pragma unroll
            for (int i = 0; i < HELD; ++i) id[i] = p0 + 64 * i + lane < stop ? a.t.at(p0 + 64 * i + lane) : 0;
#pragma unroll
            for (int i = 0; i < HELD; ++i) {
                if (p0 + 64 * i >= stop) break;
                const bool in = p0 + 64 * i + lane < stop;
                bad |= in && a.t.bad(id[i]);
                held.key[i] = a.t.padding(id[i]) || a.t.bad(id[i]) ? (uint32_t)a.groups : (uint32_t)id[i];
                held.same[i] = same_key(in, held.key[i], a.bits);
            }
        }
#pragma unroll
        for (int i = 0; i < HELD; ++i) {
            if (p0 + 64 * i >= stop) break;
            f(p0 + 64 * i + lane, p0 + 64 * i + lane < stop, held.key[i], held.same[i]);
            __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");       // what one lane has counted, another reads next
        }
    }
    return bad;
}
// count[key * WAVES + wave]: a wavefront's rows of a key.  Returns whether a row of the workgroup is bad, in all threads.
__device__ __forceinline__ bool count_keys(const GroupArgs &a, int64_t first, uint32_t *count, Held &held) {
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    for (int i = threadIdx.x; i < (a.groups + 1) * WAVES; i += THREADS) count[i] = 0;
    __syncthreads();
    const bool bad = each_64<false>(a, first, held, [&](int64_t, bool in, uint32_t key, uint64_t same) {
        if (in && __ffsll((unsigned long long)same) - 1 == lane) count[key * WAVES + wave] += (uint32_t)__popcll(same);
    });
    return __syncthreads_or(bad ? 1 : 0) != 0;
}
// x[0 .. n) becomes the sums of what stands before; all threads call it
__device__ __forceinline__ void sums_before(uint32_t *x, int n) {
    __shared__ uint32_t waves[WAVES];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, each = (n + THREADS - 1) / THREADS, at = threadIdx.x * each;
    uint32_t own = 0;
    for (int i = 0; i < each; ++i)
        if (at + i < n) own += x[at + i];
    uint32_t sum = own;
    for (int d = 1; d < 64; d <<= 1) {
        const uint32_t y = __shfl_up(sum, d);
        if (lane >= d) sum += y;
    }
    if (lane == 63) waves[wave] = sum;
    __syncthreads();
    uint32_t before = sum - own;
    for (int w = 0; w < wave; ++w) before += waves[w];
    for (int i = 0; i < each; ++i)
        if (at + i < n) { const uint32_t y = x[at + i]; x[at + i] = before; before += y; }
    __syncthreads();
}
__device__ __forceinline__ void put_rows(const GroupArgs &a, int64_t first, uint32_t *next, Held &held) {
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    each_64<true>(a, first, held, [&](int64_t p, bool in, uint32_t key, uint64_t same) {
        if (in) a.order[next[key * WAVES + wave] + (uint32_t)__popcll(same & ((1ull << lane) - 1))] = (int32_t)p;
        if (in && __ffsll((unsigned long long)same) - 1 == lane) next[key * WAVES + wave] += (uint32_t)__popcll(same);
    });
}

// Few rows, by one workgroup: 128 rows 3.4 us, 3,998 rows 7.0.
__global__ __launch_bounds__(THREADS) void k_group_one(GroupArgs a, int32_t *err) {
    extern __shared__ uint32_t count[];
    __shared__ int off;
    look_for_all(err, &off);
    Held held;
    const bool bad = count_keys(a, 0, count, held);
    if (off) return;
    if (bad) {
        if (threadIdx.x == 0) atomicExch(err, PS_EKEY);
        return;
    }
    sums_before(count, (a.groups + 1) * WAVES);
    for (int e = threadIdx.x; e <= a.groups; e += THREADS) a.offsets[e] = (int32_t)count[e * WAVES];
    __syncthreads();
    put_rows(a, 0, count, held);
}

// More of them: what every workgroup counts, and then the places - each workgroup reads its own ids and votes on them once more, for its wavefronts' counts, which
// the first launch leaves as one sum a group, and adds up the counts of those before it, which are at most 128.  131,072 rows of 64 groups: 4.2 and 7.8 us.  (In one launch, which would
// save the second reading, workgroups would have to wait for each other.)
__global__ __launch_bounds__(THREADS) void k_group_count(GroupArgs a, int32_t *err) {
    extern __shared__ uint32_t count[];
    Held held;
    const bool bad = count_keys(a, (int64_t)blockIdx.x * a.chunk, count, held);
    if (bad && threadIdx.x == 0) atomicExch(err, PS_EKEY);
    for (int e = threadIdx.x; e <= a.groups; e += THREADS) {
        uint32_t s = 0;
        for (int w = 0; w < WAVES; ++w) s += count[e * WAVES + w];
        a.count[(int64_t)blockIdx.x * (a.groups + 1) + e] = s;
    }
}
__global__ __launch_bounds__(THREADS) void k_group_place(GroupArgs a, const int32_t *err) {
    extern __shared__ uint32_t count[];
    __shared__ int off;
    const int keys = a.groups + 1;
    uint32_t *total = count + keys * WAVES, *before = total + keys;
    look_for_all(err, &off);
    Held held;
    count_keys(a, (int64_t)blockIdx.x * a.chunk, count, held);
    if (off) return;
    for (int i = threadIdx.x; i < 2 * keys; i += THREADS) total[i] = 0;
    __syncthreads();
    const int parts = keys < THREADS ? THREADS / keys : 1;
    for (int i = threadIdx.x; i < parts * keys; i += THREADS) {
        const int key = i % keys, part = i / keys, lo = a.blocks * part / parts, hi = a.blocks * (part + 1) / parts;
        uint32_t all = 0, first = 0;
#pragma unroll 8
        for (int b = lo; b < hi; ++b) {
            const uint32_t c = a.count[(int64_t)b * keys + key];
            all += c;
            first += b < (int)blockIdx.x ? c : 0u;
        }
        atomicAdd(&total[key], all);
        atomicAdd(&before[key], first);
    }
    __syncthreads();
    sums_before(total, keys);
    if (blockIdx.x == 0)
        for (int e = threadIdx.x; e < keys; e += THREADS) a.offsets[e] = (int32_t)total[e];
    for (int e = threadIdx.x; e < keys; e += THREADS) {
        uint32_t at = total[e] + before[e];
        for (int w = 0; w < WAVES; ++w) { const uint32_t c = count[e * WAVES + w]; count[e * WAVES + w] = at; at += c; }
    }
    __syncthreads();
    put_rows(a, (int64_t)blockIdx.x * a.chunk, count, held);
}

// From rows sorted as keys: more groups than counts have room for in LDS, or more rows than 128 workgroups of 16,384.
__global__ __launch_bounds__(256) void k_group_sorted(const uint64_t *skeys, const uint32_t *spos, int64_t n, int32_t groups, int32_t *order, int32_t *offsets,
                                                      const int32_t *err) {
    if (*(volatile const int32_t *)err) return;
    const int64_t p = (int64_t)blockIdx.x * blockDim.x + threadIdx.x;
    if (p > n) return;
    // the groups that start here: those after the key before, up to this one
    const int64_t was = p > 0 ? (int64_t)skeys[p - 1] : -1, is = p < n ? (int64_t)skeys[p] : groups;
    for (int64_t e = was + 1; e <= is && e <= groups; ++e) offsets[e] = (int32_t)p;
    if (p < n) order[p] = (int32_t)spos[p];
}

__global__ __launch_bounds__(256) void k_route_groups(RouteArgs a, RowGroups g, GroupKeys k, const int32_t *err) {
    __shared__ RouteLds l;
    route_access_block(a, l, blockIdx.x, flag_ahead(err), [&](int64_t p, int64_t &key) {
        key = 0;
        if (p < k.shared) { key = k.first + p; return true; }
        p -= k.shared;
        const int64_t all = (int64_t)g.groups * k.each;
        const bool second = p >= all;
        if (second) p -= all;
        const int e = (int)(p / k.each);
        if (g.start(e) >= g.start(e + 1)) return false;
        key = (second ? k.first_b : k.first_a) + p;
        return true;
    });
}
__global__ __launch_bounds__(256) void k_group_replies(int64_t n, RowGroups g, GroupKeys k, int32_t worker, const int32_t *owner, int16_t *loc_row, const int32_t *err) {
    if (*(volatile const int32_t *)err) return;
    int64_t p = (int64_t)blockIdx.x * blockDim.x + threadIdx.x;
    if (p >= n) return;
    int64_t key = k.first + p;
    if (p >= k.shared) {
        p -= k.shared;
        const int64_t all = (int64_t)g.groups * k.each;
        const bool second = p >= all;
        if (second) p -= all;
        const int e = (int)(p / k.each);
        if (g.start(e) >= g.start(e + 1)) return;
        key = (second ? k.first_b : k.first_a) + p;
    }
    const int32_t o = owner[key];
    if (o != worker) loc_row[key] = (int16_t)o;
}

size_t up256(size_t x) { return (x + 255) / 256 * 256; }

template <class K> int start_groups(dpaps_ps *ps, LdsAllowed &allowed, K kernel, const GroupArgs &a, int blocks, size_t words, hipStream_t st) {
    const size_t bytes = words * 4;
    if (bytes > 65536) {
        const int rc = dpaps_allow_lds(ps, allowed, reinterpret_cast<const void *>(kernel), bytes);
        if (rc) return rc;
    }
    kernel<<<(unsigned)blocks, THREADS, bytes, st>>>(a, ps->err);
    PS_HIP(ps, hipGetLastError());
    return PS_OK;
}

}  // namespace

int dpaps_row_groups(dpaps_ps *ps, const int32_t *order, const int32_t *offsets, int32_t groups, int64_t n, RowGroups *g) {
    if (n < 0 || groups <= 0 || !offsets || (n > 0 && !order)) return PS_EINVAL;
    if (n > PS_EMB_MAX_TOKENS || groups > PS_MAX_GROUPS) {
        ps->last_error = "groups: at most 65536, of at most 2^29 rows";
        return PS_ELIMIT;
    }
    g->order = order; g->offsets = offsets; g->groups = groups; g->n = (int32_t)n;
    return PS_OK;
}

bool dpaps_strides_fit(dpaps_ps *ps, int64_t a, int64_t b) {
    if (a < ((int64_t)1 << 31) && b < ((int64_t)1 << 31)) return true;
    ps->last_error = "rows at most 2^31 - 1 elements apart";
    return false;
}

int dpaps_route_groups(dpaps_ps *ps, int32_t worker, const RowGroups &g, const GroupKeys &k, hipStream_t st) {
    if (worker < 0) return PS_OK;
    const int64_t n = k.shared + (int64_t)g.groups * k.each * (k.first_b >= 0 ? 2 : 1);
    const RouteArgs a = dpaps_route_args(ps, worker, n, PS_STAT_PULL_LOCAL, PS_STAT_PULL_REMOTE, -1, -1, st);
    if (a.blocks == 0) return PS_OK;
    k_route_groups<<<a.blocks, 256, 0, st>>>(a, g, k, ps->err);
    PS_HIP(ps, hipGetLastError());
    if (ps->loc) {
        k_group_replies<<<(unsigned)ceil_div64(n, 256), 256, 0, st>>>(n, g, k, worker, ps->owner, ps->loc + (int64_t)worker * ps->K, ps->err);
        PS_HIP(ps, hipGetLastError());
    }
    return PS_OK;
}

extern "C" int group_rows(ps_handle ps, int32_t num_groups, const void *ids, int32_t id_type, int64_t n, int64_t pad_id, int32_t *order, int32_t *offsets,
                          void *stream) {
    if (!ps || n < 0 || num_groups <= 0 || (id_type != PS_I32 && id_type != PS_I64) || !offsets || (n > 0 && (!ids || !order))) return PS_EINVAL;
    if (n > PS_EMB_MAX_TOKENS || num_groups > PS_MAX_GROUPS) {
        ps->last_error = "groups: at most 65536, of at most 2^29 rows";
        return PS_ELIMIT;
    }
    hipStream_t st = (hipStream_t)stream;
    GroupArgs a{};
    a.t.ids = ids; a.t.wide = id_type == PS_I64; a.t.n = n; a.t.count = num_groups; a.t.pad = pad_id; a.t.padded = pad_id != PS_NO_PAD;
    a.groups = num_groups; a.order = order; a.offsets = offsets;
    a.bits = dpaps_key_bits((int64_t)num_groups + 1);
    const int64_t keys = (int64_t)num_groups + 1;
    if (num_groups <= MOST_GROUPS && n <= ONE_CHUNK) {
        static LdsAllowed allowed;
        a.chunk = (int32_t)(n > 0 ? n : 1);
        return start_groups(ps, allowed, &k_group_one, a, 1, keys * WAVES, st);
    }
    if (num_groups <= MOST_GROUPS && n <= (int64_t)MOST_CHUNK * MOST_BLOCKS) {
        static LdsAllowed allowed_count, allowed_place;
        a.chunk = THREADS;
        while (ceil_div64(n, a.chunk) > MOST_BLOCKS) a.chunk *= 2;
        a.blocks = (int32_t)ceil_div64(n, a.chunk);
        int rc = dpaps_ws_reserve(ps, (size_t)a.blocks * keys * 4);
        if (rc) return rc;
        a.count = (uint32_t *)ps->ws;
        rc = start_groups(ps, allowed_count, &k_group_count, a, a.blocks, keys * WAVES, st);
        return rc ? rc : start_groups(ps, allowed_place, &k_group_place, a, a.blocks, keys * (WAVES + 2), st);
    }
    const size_t off_spos = up256((size_t)n * 8), off_sort = off_spos + up256((size_t)n * 4);
    int rc = dpaps_ws_reserve(ps, off_sort + dpaps_sort_scratch_bytes(n, a.bits));
    if (rc) return rc;
    char *ws = (char *)ps->ws;
    if (n > 0) rc = dpaps_sort_tokens(ps, a.t, (uint64_t *)ws, (uint32_t *)(ws + off_spos), ws + off_sort, st);
    if (rc) return rc;
    k_group_sorted<<<(unsigned)ceil_div64(n + 1, 256), 256, 0, st>>>((const uint64_t *)ws, (const uint32_t *)(ws + off_spos), n, num_groups, order, offsets, ps->err);
    PS_HIP(ps, hipGetLastError());
    return PS_OK;
}
