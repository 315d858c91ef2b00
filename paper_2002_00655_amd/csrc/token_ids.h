// The keys that a call names by tokens: token t is key first + t.
#pragma once
#include "route.h"
#include "together.h"

struct TokenIds {
    const void *ids = nullptr;   // int32 or int64 (wide), on the device; NULL: token p is p
    int64_t n = 0, first = 0, count = 0, pad = 0;
    int32_t wide = 0, padded = 0;   // padded: there is padding, the token `pad` (PS_NO_PAD is a token that a batch can hold, by mistake)
    __device__ __forceinline__ int64_t at(int64_t p) const {
        return !ids ? p : wide ? reinterpret_cast<const int64_t *>(ids)[p] : (int64_t)reinterpret_cast<const int32_t *>(ids)[p];
    }
    __device__ __forceinline__ bool padding(int64_t t) const { return padded && t == pad; }
    __device__ __forceinline__ bool bad(int64_t t) const { return (t < 0 || t >= count) && !padding(t); }
};

// Whether a call of few tokens is to do nothing: few_keys_off, for tokens.  keep(p, id): called for every token as it is read.
template <int AHEAD, class Keep>
__device__ __forceinline__ bool few_tokens_off(const TokenIds &t, int32_t *err, Keep keep) {
    const bool was_off = *(volatile const int32_t *)err != 0;
    bool off = was_off;
#pragma unroll AHEAD
    for (int64_t p = threadIdx.x; p < t.n; p += blockDim.x) {
        const int64_t id = t.at(p);
        keep(p, id);
        off |= t.bad(id);
    }
    const bool any = __syncthreads_or(off ? 1 : 0) != 0;
    if (any && threadIdx.x == 0 && !was_off) atomicExch(err, PS_EKEY);
    return any;
}
__device__ __forceinline__ bool few_tokens_off(const TokenIds &t, int32_t *err) {
    return few_tokens_off<4>(t, err, [](int64_t, int64_t) {});
}

// The statistics of an access to the tokens' keys; padding is no access.
__device__ __forceinline__ void route_tokens_block(const RouteArgs &a, const TokenIds &t, RouteLds &l, int block, int32_t stop) {
    route_access_block(a, l, block, stop, [&](int64_t p, int64_t &k) {
        const int64_t id = t.at(p);
        const bool padding = t.padding(id);
        k = padding ? 0 : t.first + id;
        return !padding;
    });
}

// emb.hip: the statistics of a pull of the tokens' keys, and of a push of them right after it if `push`, in launches of their own, and with location
// caches the replies
int dpaps_route_tokens(dpaps_ps *ps, int32_t worker, const TokenIds &t, bool pull, bool push, hipStream_t st);
// key_sort.hip: the pairs (token, position) ordered by token (see there)
int dpaps_sort_tokens(dpaps_ps *ps, const TokenIds &t, uint64_t *skeys, uint32_t *spos, void *scratch, hipStream_t st);
