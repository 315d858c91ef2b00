// A stand-in for the HIP runtime, for tests of what the library's host code launches, on a machine without a GPU: nothing runs, device memory is
// addresses only, and launches are kept with their names, grids and, of products of grouped rows, the numbers of the server that they may read.
// Loaded with global symbols before the library.
#include "experts.h"

#include <cstring>
#include <map>

namespace {
struct Launch { std::string name; dim3 grid; int64_t first, end; };
std::vector<Launch> launches;
std::map<const void *, std::string> kernels;
struct Block { char *at; size_t bytes; };
std::vector<Block> blocks;
size_t next_address = (size_t)1 << 40, refuse_from = SIZE_MAX;
dim3 cfg_grid, cfg_block;
size_t cfg_lds;
hipStream_t cfg_stream;

struct ExpertCall { ExpertArgs a[2]; };               // (as in expert.hip)
// numbers of the store, counted from its start
void reads(Launch &l, const float *w, int64_t key, int64_t keys, int64_t L) {
    const Block *b = nullptr;
    for (const Block &x : blocks) if ((const char *)w >= x.at && (const char *)w < x.at + x.bytes) b = &x;
    const int64_t at = b ? w - (const float *)b->at : INT64_MAX / 2, first = at + key * L, end = at + (key + keys) * L;
    if (l.end == 0 || first < l.first) l.first = first;
    if (end > l.end) l.end = end;
}
}  // namespace

extern "C" {
int launch_count() { return (int)launches.size(); }
const char *launch_name(int i) { return launches[i].name.c_str(); }
int64_t launch_groups(int i) { const dim3 &g = launches[i].grid; return (int64_t)g.x * g.y * g.z; }
int64_t launch_reads_from(int i) { return launches[i].first; }
int64_t launch_reads_to(int i) { return launches[i].end; }
void launch_clear() { launches.clear(); }
void refuse_allocations_from(int64_t bytes) { refuse_from = (size_t)bytes; }

void **__hipRegisterFatBinary(const void *) { static void *h; return &h; }
void __hipUnregisterFatBinary(void **) {}
void __hipRegisterFunction(void **, const void *host, char *, const char *name, unsigned, void *, void *, void *, void *, int *) { kernels[host] = name; }
void __hipRegisterVar(void **, void *, char *, char *, int, size_t, int, int) {}
hipError_t __hipPushCallConfiguration(dim3 g, dim3 b, size_t s, hipStream_t st) { cfg_grid = g; cfg_block = b; cfg_lds = s; cfg_stream = st; return hipSuccess; }
hipError_t __hipPopCallConfiguration(dim3 *g, dim3 *b, size_t *s, hipStream_t *st) { *g = cfg_grid; *b = cfg_block; *s = cfg_lds; *st = cfg_stream; return hipSuccess; }
hipError_t hipLaunchKernel(const void *f, dim3 g, dim3, void **args, size_t, hipStream_t) {
    Launch l{kernels[f], g, 0, 0};
    const bool few = l.name.find("12k_expert_few") != std::string::npos, tiles = l.name.find("8k_expertI") != std::string::npos;
    if (few || tiles) {
        const ExpertCall &c = *(const ExpertCall *)args[0];
        for (unsigned i = 0; i < g.y; ++i) {
            const ExpertArgs &a = c.a[i];
            reads(l, a.w, 0, (int64_t)(a.g.groups - 1) * a.each + (a.turned ? a.K : a.columns()), a.L);
        }
    }
    if (l.name.find("k_adapter") != std::string::npos) {
        const AdapterArgs &a = *(const AdapterArgs *)args[0];
        reads(l, a.w, 0, a.turned ? a.K : a.N, a.L);
        reads(l, a.b, 0, (int64_t)a.g.groups * a.rank, a.L);
    }
    launches.push_back(l);
    return hipSuccess;
}
hipError_t hipMalloc(void **p, size_t bytes) {
    if (bytes >= refuse_from) { *p = nullptr; return hipErrorOutOfMemory; }
    *p = (void *)next_address;
    blocks.push_back({(char *)*p, bytes});
    next_address += (bytes + 8191) / 4096 * 4096;
    return hipSuccess;
}
hipError_t hipFree(void *p) {
    for (size_t i = 0; i < blocks.size(); ++i) if (blocks[i].at == p) { blocks.erase(blocks.begin() + i); break; }
    return hipSuccess;
}
hipError_t hipMemset(void *, int, size_t) { return hipSuccess; }
hipError_t hipMemsetAsync(void *, int, size_t, hipStream_t) { return hipSuccess; }
hipError_t hipMemcpyAsync(void *, const void *, size_t, hipMemcpyKind, hipStream_t) { return hipSuccess; }
hipError_t hipGetLastError() { return hipSuccess; }
const char *hipGetErrorString(hipError_t) { return "stand-in"; }
hipError_t hipGetDevice(int *d) { *d = 0; return hipSuccess; }
hipError_t hipDeviceGetAttribute(int *v, hipDeviceAttribute_t a, int) { *v = a == hipDeviceAttributeMultiprocessorCount ? 256 : 163840; return hipSuccess; }
hipError_t hipGetSymbolAddress(void **p, const void *) { static char x[16]; *p = x; return hipSuccess; }
hipError_t hipDeviceSynchronize() { return hipSuccess; }
hipError_t hipStreamSynchronize(hipStream_t) { return hipSuccess; }
hipError_t hipFuncSetAttribute(const void *, hipFuncAttribute, int) { return hipSuccess; }
}
