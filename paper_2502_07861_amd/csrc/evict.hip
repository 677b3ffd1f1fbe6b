// Eviction by accumulated attention weight: of every sequence's cache the first n_sink and the last n_recent tokens and the
// heaviest of the others stay, `keep` in all, in their order; the rows move to a dense cache.
//
// Order of two tokens: protected ones first, then the larger mass, then the lower place; places without a token never stay.  A
// token's rank is a 32-bit number (mass_rank) that orders like this but for the place, so the keep-th largest rank and how many
// of its equals stay say everything: found by four passes over 8 bits each with a histogram in LDS.
#include "bkv_device.h"
#include "bkv_host.h"

namespace bkv {

constexpr int kSelectThreads = 1024;
constexpr int kGatherThreads = 256;

// 0: no token; 0xffffffff: protected; in between the mass in its own order (-0 equals 0, NaN counts as -inf)
__device__ __forceinline__ unsigned int mass_rank(float mass, float w, bool window) {
    if (!(w > 0.f)) return 0u;
    if (window) return 0xffffffffu;
    const unsigned int u = __float_as_uint(mass == mass ? mass + 0.f : -INFINITY);
    return (u & 0x80000000u) ? ~u : u | 0x80000000u;
}

__global__ __launch_bounds__(kSelectThreads) void evict_select_kernel(const EvictArgs a) {
    __shared__ unsigned int hist[256];
    __shared__ unsigned int prefix_s, need_s;
    __shared__ int above[kSelectThreads / 64], equal[kSelectThreads / 64];
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const int64_t seq = blockIdx.x;
    const float* w = a.w + (size_t)seq * a.stride;
    const float* mass = a.mass + (size_t)seq * a.stride;
    auto rank = [&](int p) { return mass_rank(mass[p], w[p], p < a.n_sink || p >= a.count - a.n_recent); };

    unsigned int prefix = 0, need = (unsigned int)a.keep;           // the keep-th largest rank starts with `prefix`; it is the need-th of those
    for (int shift = 24; shift >= 0; shift -= 8) {
        for (int i = tid; i < 256; i += kSelectThreads) hist[i] = 0;
        __syncthreads();
        for (int p = tid; p < a.count; p += kSelectThreads) {
            const unsigned int x = rank(p);
            if (shift == 24 || (x >> (shift + 8)) == (prefix >> (shift + 8))) atomicAdd(&hist[(x >> shift) & 255u], 1u);
        }
        __syncthreads();
        if (tid == 0) {
            unsigned int left = need, b = 256;
            while (b-- > 0) {
                if (hist[b] >= left) break;
                left -= hist[b];
            }
            prefix_s = prefix | (b << shift);
            need_s = left;
        }
        __syncthreads();
        prefix = prefix_s; need = need_s;
    }
    // ranks above `prefix` stay, of those equal to it the first `need` (none where it says: no token)
    if (prefix == 0u) need = 0;
    int32_t* pick = a.pick + (size_t)seq * a.keep;
    int base_above = 0, base_equal = 0;
    for (int c = 0; c < a.count; c += kSelectThreads) {
        const int p = c + tid;
        const unsigned int x = p < a.count ? rank(p) : 0u;
        const unsigned long long up = __ballot(x > prefix), eq = __ballot(x == prefix && x != 0u);
        if (lane == 0) { above[wave] = __popcll(up); equal[wave] = __popcll(eq); }
        __syncthreads();
        int before_above = base_above, before_equal = base_equal;
        for (int k = 0; k < kSelectThreads / 64; ++k) {
            if (k < wave) { before_above += above[k]; before_equal += equal[k]; }
            base_above += above[k]; base_equal += equal[k];
        }
        const unsigned long long below = (1ull << lane) - 1ull;
        before_above += __popcll(up & below);
        before_equal += __popcll(eq & below);
        const bool mine_eq = x == prefix && x != 0u && (unsigned int)before_equal < need;
        if (x > prefix || mine_eq) pick[before_above + min(before_equal, (int)need)] = p;
        __syncthreads();
    }
    const int total = base_above + min(base_equal, (int)need);
    for (int i = total + tid; i < a.keep; i += kSelectThreads) pick[i] = -1;
    if (tid == 0 && a.count_out) a.count_out[seq] = total;
}

__global__ __launch_bounds__(kGatherThreads) void evict_gather_kernel(const EvictArgs a) {
    const int slots = a.row_bytes / 16;
    const int64_t seq = blockIdx.y;
    const int32_t* pick = a.pick + (size_t)seq * a.keep;
    const size_t in = (size_t)seq * a.stride, out = (size_t)seq * a.keep;
    const int64_t pieces = (int64_t)a.keep * slots;
    for (int64_t i = (int64_t)blockIdx.x * kGatherThreads + threadIdx.x; i < pieces; i += (int64_t)gridDim.x * kGatherThreads) {
        const int r = (int)(i / slots), s = (int)(i - (int64_t)r * slots);
        const int p = pick[r];
        const size_t from = (in + (size_t)max(p, 0)) * a.row_bytes + s * 16, to = (out + r) * a.row_bytes + s * 16;
        uintx4 k = {0u, 0u, 0u, 0u}, v = k;
        if (p >= 0) { k = *reinterpret_cast<const uintx4*>(a.K + from); v = *reinterpret_cast<const uintx4*>(a.V + from); }
        *reinterpret_cast<uintx4*>(a.K_out + to) = k;
        *reinterpret_cast<uintx4*>(a.V_out + to) = v;
        if (s == 0) {
            if (a.w_out) a.w_out[out + r] = p >= 0 ? a.w[in + p] : 0.f;
            if (a.mass_out) a.mass_out[out + r] = p >= 0 ? a.mass[in + p] : 0.f;
            if (a.idx_out) a.idx_out[out + r] = p < 0 ? -1 : a.idx ? a.idx[in + p] : p;
        }
    }
}

size_t evict_workspace_bytes(int64_t n_seq, int64_t count) { return (size_t)n_seq * count * sizeof(int32_t); }

hipError_t launch_evict(EvictArgs& a, void* workspace, hipStream_t st) {
    a.pick = (int32_t*)workspace;
    hipLaunchKernelGGL(evict_select_kernel, dim3((uint32_t)a.n_seq), dim3(kSelectThreads), 0, st, a);
    hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
    const int64_t pieces = (int64_t)a.keep * (a.row_bytes / 16);
    const int64_t gx = (pieces + kGatherThreads - 1) / kGatherThreads;
    hipLaunchKernelGGL(evict_gather_kernel, dim3((uint32_t)(gx > 4096 ? 4096 : gx), (uint32_t)a.n_seq), dim3(kGatherThreads), 0, st, a);
    return hipGetLastError();
}

}  // namespace bkv
