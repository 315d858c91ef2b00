// For tests on the CPU: what device code of csrc/ needs to be compiled as plain C++ (by clang), one thread at a time, so that its arithmetic and its reads
// can be looked at.  Threads have no LDS in common and no barrier; what the lanes of a wavefront tell each other (votes, a lane's number) goes by wave(), below.
#pragma once
#include <hip/hip_runtime.h>
#include <cstdint>
#include <cstdio>
#include <cstdlib>
#include <cstring>
#include <functional>
#include <setjmp.h>
#include <sys/mman.h>
#include <vector>

struct Dim { unsigned x, y, z; };
static Dim threadIdx, blockIdx, blockDim, gridDim;

#undef __shared__
#define __shared__ static
template <class T> static T atomicAdd(T *p, T v) { const T o = *p; *p += v; return o; }
template <class T> static T atomicOr(T *p, T v) { const T o = *p; *p |= v; return o; }
template <class T, class U> static T atomicExch(T *p, U v) { const T o = *p; *p = (T)v; return o; }
#define __HIP_MEMORY_SCOPE_AGENT 0
#define __hip_atomic_load(p, order, scope) (*(p))
#define __hip_atomic_store(p, v, order, scope) ((void)(*(p) = (v)))
static inline void __syncthreads() {}
static inline int __syncthreads_or(int p) { return p; }
static inline int __popc(uint32_t x) { return __builtin_popcount(x); }
static inline int __popcll(unsigned long long x) { return __builtin_popcountll(x); }

// A wavefront's 64 lanes run one after the other, again and again: a lane that comes to a vote whose outcome is not known yet says what it votes and ends; when
// all have, the outcome is known to the next run.
static std::vector<std::vector<uint64_t>> told;       // per vote, what each lane has said
static size_t known, asked;                           // votes whose outcome is known; votes of this lane so far
static jmp_buf lane_ends;
static std::vector<uint64_t> said(64);
static inline const std::vector<uint64_t> &of_all(uint64_t mine) {
    if (asked < known) return told[asked++];
    said[threadIdx.x & 63] = mine;
    longjmp(lane_ends, 1);
}
static inline unsigned long long __ballot(bool p) {
    const std::vector<uint64_t> &v = of_all(p);
    unsigned long long m = 0;
    for (int l = 0; l < 64; ++l) m |= (unsigned long long)(v[l] != 0) << l;
    return m;
}
static inline int read_lane(int x, int lane) {
    const std::vector<uint64_t> &v = of_all((uint32_t)x);
    if (lane < 0 || lane > 63) abort();
    return (int)(uint32_t)v[lane];
}
#define __builtin_amdgcn_readlane(x, lane) read_lane(x, lane)
#define __builtin_amdgcn_readfirstlane(x) read_lane(x, 0)
static inline void wave(const std::function<void(int)> &lane) {
    told.clear();
    for (known = 0;;) {
        static int through;
        through = 0;
        for (int l = 0; l < 64; ++l) {
            threadIdx.x = (unsigned)l;
            asked = 0;
            if (!setjmp(lane_ends)) { lane(l); ++through; }
        }
        if (through == 64) return;
        if (through != 0) { fprintf(stderr, "lanes part\n"); abort(); }
        told.push_back(said);
        ++known;
    }
}

// what is multiplied does not matter to these tests
#define __builtin_amdgcn_mfma_f32_32x32x2f32(a, b, c, x, y, z) (c)
#define __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, b, c, x, y, z) (c)
#define __builtin_amdgcn_mfma_f32_32x32x16_f16(a, b, c, x, y, z) (c)
#define __builtin_amdgcn_mfma_f32_16x16x4f32(a, b, c, x, y, z) (c)
#define __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, x, y, z) (c)
#define __builtin_amdgcn_mfma_f32_16x16x32_f16(a, b, c, x, y, z) (c)
#define __builtin_amdgcn_fence(order, scope) ((void)0)
#define __builtin_amdgcn_sched_barrier(m) ((void)0)
#define __builtin_amdgcn_sched_group_barrier(m, n, g) ((void)0)
#define __builtin_amdgcn_s_waitcnt(n) ((void)0)
#define __builtin_amdgcn_s_barrier() ((void)0)

// Memory whose last byte is followed by a page, and whose first one is preceded by one, that cannot be read.
template <class T> static T *fenced(size_t count) {
    const size_t page = 4096, bytes = count * sizeof(T), pages = (bytes + page - 1) / page;
    char *p = (char *)mmap(nullptr, (pages + 2) * page, PROT_READ | PROT_WRITE, MAP_PRIVATE | MAP_ANONYMOUS, -1, 0);
    if (p == MAP_FAILED || mprotect(p, page, PROT_NONE) || mprotect(p + (pages + 1) * page, page, PROT_NONE)) abort();
    return (T *)(p + page + pages * page - bytes);
}
static inline void unfence(void *p, size_t bytes) {
    const size_t page = 4096, pages = (bytes + page - 1) / page;
    munmap((char *)p - (pages * page - bytes) - page, (pages + 2) * page);
}
