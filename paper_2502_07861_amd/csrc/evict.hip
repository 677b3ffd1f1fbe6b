// Eviction by accumulated attention weight: of every sequence's cache the first n_sink and the last n_recent tokens and the
// heaviest of the others stay, `keep` in all, in their order; the rows move to a dense cache.
//
// Order of two tokens: protected ones first, then the larger mass, then the lower place; places without a token never stay.  A
// token's rank is a 32-bit number (mass_rank) that orders like this but for the place, so the keep-th largest rank and how many
// of its equals stay say everything.
// The search is the latency of its steps (8 x 16384 places 11.2 us, 256 x 32768 27), the copy memory's rate (256 x 8192 rows of 256 bytes, keys and
// values: 371 us, 5.8 TB/s read and written).
#include "bkv_device.h"
#include "bkv_host.h"

namespace bkv {

constexpr int kSelectThreads = 1024;
constexpr int kGatherThreads = 256;

typedef float floatx4_any __attribute__((ext_vector_type(4), aligned(4)));     // four consecutive floats, any alignment

// 0: no token; 0xffffffff: protected; in between the mass in its own order (-0 equals 0, NaN counts as -inf)
__device__ __forceinline__ unsigned int mass_rank(float mass, float w, bool window) {
    if (!(w > 0.f)) return 0u;
    if (window) return 0xffffffffu;
    const unsigned int u = __float_as_uint(mass == mass ? mass + 0.f : -INFINITY);
    return (u & 0x80000000u) ? ~u : u | 0x80000000u;
}

// Ranks of places p .. p + 3 of one sequence (0 behind the last one).
__device__ __forceinline__ void load_ranks(const EvictArgs& a, int64_t seq, int p, unsigned int* x) {
    const float* w = a.w + (size_t)seq * a.stride;
    const float* mass = a.mass + (size_t)seq * a.stride;
    const int recent_from = a.count - a.n_recent;
    float wv[4] = {0.f, 0.f, 0.f, 0.f}, mv[4] = {0.f, 0.f, 0.f, 0.f};
    if (p + 4 <= a.count) {
        const floatx4_any w4 = *reinterpret_cast<const floatx4_any*>(w + p), m4 = *reinterpret_cast<const floatx4_any*>(mass + p);
#pragma unroll
        for (int e = 0; e < 4; ++e) { wv[e] = w4[e]; mv[e] = m4[e]; }
    } else {
#pragma unroll
        for (int e = 0; e < 4; ++e) if (p + e < a.count) { wv[e] = w[p + e]; mv[e] = mass[p + e]; }
    }
#pragma unroll
    for (int e = 0; e < 4; ++e) x[e] = mass_rank(mv[e], wv[e], p + e < a.n_sink || p + e >= recent_from);
}

// What stays: ranks from `from` on, and the first `need` of those equal to `equal` (0: of none).
struct EvictCut { unsigned int from, equal; int need; };
// t: the keep-th largest rank, or, where all of the `in` ranks that it can be stay (in == left), a bound that they reach and the
// smaller ones do not.  Rank 0, no token, never stays.
__device__ __forceinline__ EvictCut evict_cut(unsigned int t, unsigned int in, unsigned int left) {
    if (in == left) return {max(t, 1u), 0u, 0};
    return {t + 1u, t, t ? (int)left : 0};        // (t == 0xffffffff: no more tokens are protected than stay, so they all do)
}

// A wavefront has 64 KPT consecutive places, group j of a lane (ranks 4 j .. 4 j + 3) the places first + 4 (64 j + lane) ...: every
// load of a wavefront is one stretch, and where its list starts takes one sum over the wavefronts in front.
__device__ __forceinline__ int place_of(int kpt, int j) {
    return (int)(threadIdx.x >> 6) * 64 * kpt + 4 * (64 * j + (int)(threadIdx.x & 63u));
}

// inclusive sum over the wavefront's lanes
__device__ __forceinline__ unsigned int lane_sums(unsigned int x) {
    x += (unsigned int)__builtin_amdgcn_update_dpp(0, (int)x, 0x111, 0xf, 0xf, false);     // row_shr:1
    x += (unsigned int)__builtin_amdgcn_update_dpp(0, (int)x, 0x112, 0xf, 0xf, false);
    x += (unsigned int)__builtin_amdgcn_update_dpp(0, (int)x, 0x114, 0xf, 0xf, false);
    x += (unsigned int)__builtin_amdgcn_update_dpp(0, (int)x, 0x118, 0xf, 0xf, false);
    x += (unsigned int)__builtin_amdgcn_update_dpp(0, (int)x, 0x142, 0xa, 0xf, false);     // row_bcast:15 to rows 1 and 3
    x += (unsigned int)__builtin_amdgcn_update_dpp(0, (int)x, 0x143, 0xc, 0xf, false);     // row_bcast:31 to rows 2 and 3
    return x;
}

// Which of the workgroup's places stay, (above, equal) of them after `base`: what lies in front of this wavefront, and the sum of all.
template <int KPT>
__device__ __forceinline__ void sum_ranks(const unsigned int (&x)[KPT], const EvictCut& cut, int2 base, int2* waves /*[16]*/, int2& before, int2& total) {
    constexpr int W = kSelectThreads / 64;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    int up = 0, eq = 0;
#pragma unroll
    for (int i = 0; i < KPT; ++i) up += (int)__popcll(__ballot(x[i] >= cut.from));
    if (cut.equal) {
#pragma unroll
        for (int i = 0; i < KPT; ++i) eq += (int)__popcll(__ballot(x[i] == cut.equal));
    }
    if (lane == 0) waves[wave] = make_int2(up, eq);
    __syncthreads();
    const int2 v = lane < W ? waves[lane] : make_int2(0, 0);
    const int su = (int)lane_sums((unsigned int)v.x), se = (int)lane_sums((unsigned int)v.y);
    before = make_int2(base.x + __builtin_amdgcn_readlane(su, wave) - up, base.y + __builtin_amdgcn_readlane(se, wave) - eq);
    total = make_int2(base.x + __builtin_amdgcn_readlane(su, W - 1), base.y + __builtin_amdgcn_readlane(se, W - 1));
}

__device__ __forceinline__ int lanes_below(unsigned long long m) {
    return (int)__builtin_amdgcn_mbcnt_hi((unsigned int)(m >> 32), __builtin_amdgcn_mbcnt_lo((unsigned int)m, 0u));
}

// The places that stay, each to its own place of the list; `before` of them lie in front of this wavefront.
template <int KPT>
__device__ __forceinline__ void list_ranks(const unsigned int (&x)[KPT], EvictCut cut, int first, int32_t* pick, int2 before) {
    // The compiler is not to know that it had these comparisons (sum_ranks) and places (load_ranks) before: kept, they take two scalar
    // registers and most of a vector register a rank, and 64 ranks a thread went to memory for it.
    first += place_of(KPT, 0);
    cut.from = __builtin_amdgcn_readfirstlane(cut.from);
    cut.equal = __builtin_amdgcn_readfirstlane(cut.equal);
    asm("" : "+s"(cut.from), "+s"(cut.equal), "+v"(first));
#pragma unroll
    for (int j = 0; j < KPT / 4; ++j) {
        int up = before.x, eq = before.y;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const unsigned long long m = __ballot(x[4 * j + e] >= cut.from);
            up += lanes_below(m);
            before.x += (int)__popcll(m);
        }
        if (cut.equal) {
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const unsigned long long m = __ballot(x[4 * j + e] == cut.equal);
                eq += lanes_below(m);
                before.y += (int)__popcll(m);
            }
        }
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const bool is_up = x[4 * j + e] >= cut.from, is_eq = cut.equal != 0u && x[4 * j + e] == cut.equal;
            if (is_up || (is_eq && eq < cut.need)) pick[up + min(eq, cut.need)] = first + 256 * j + e;
            up += is_up; eq += is_eq;
        }
    }
}

// Behind the last kept token: no place.
__device__ __forceinline__ void end_list(const EvictArgs& a, int64_t seq, int2 total, const EvictCut& cut) {
    const int n = total.x + min(total.y, cut.need);
    for (int i = n + (int)threadIdx.x; i < a.keep; i += kSelectThreads) a.pick[(size_t)seq * a.keep + i] = -1;
    if (threadIdx.x == 0 && a.count_out) a.count_out[seq] = n;
}

// Rows to their places: 16 bytes of keys and of values a lane and step, kGatherSteps of them on their way; piece `first` and every
// `step`-th after it.
constexpr int kGatherSteps = 4;
template <int SLOTS, int THREADS>
__device__ __forceinline__ void gather_rows(const EvictArgs& a, int64_t seq, int first, int step) {
    constexpr int RPS = THREADS / SLOTS;                             // rows of a step
    const int32_t* pick = a.pick + (size_t)seq * a.keep;
    const size_t in = (size_t)seq * a.stride, out = (size_t)seq * a.keep;
    const int slot = threadIdx.x % SLOTS, r0 = threadIdx.x / SLOTS;
    for (int64_t base = (int64_t)first * (RPS * kGatherSteps); base < a.keep; base += (int64_t)step * (RPS * kGatherSteps)) {
        int p[kGatherSteps];
        uintx4 k[kGatherSteps], v[kGatherSteps];
#pragma unroll
        for (int i = 0; i < kGatherSteps; ++i) {
            const int r = (int)base + RPS * i + r0;
            p[i] = pick[min(r, a.keep - 1)];
        }
#pragma unroll
        for (int i = 0; i < kGatherSteps; ++i) {
            const size_t from = (in + (size_t)max(p[i], 0)) * (SLOTS * 16) + slot * 16;
            k[i] = __builtin_nontemporal_load(reinterpret_cast<const uintx4*>(a.K + from));
            v[i] = __builtin_nontemporal_load(reinterpret_cast<const uintx4*>(a.V + from));
        }
#pragma unroll
        for (int i = 0; i < kGatherSteps; ++i) {
            const int r = (int)base + RPS * i + r0;
            if (r >= a.keep) break;
            const size_t to = (out + r) * (SLOTS * 16) + slot * 16;
            if (p[i] < 0) { k[i] = uintx4{0u, 0u, 0u, 0u}; v[i] = k[i]; }
            __builtin_nontemporal_store(k[i], reinterpret_cast<uintx4*>(a.K_out + to));
            __builtin_nontemporal_store(v[i], reinterpret_cast<uintx4*>(a.V_out + to));
        }
        const int r = (int)base + (int)threadIdx.x;
        if (threadIdx.x < RPS * kGatherSteps && r < a.keep) {
            const int at = pick[r];
            if (a.w_out) a.w_out[out + r] = at >= 0 ? a.w[in + at] : 0.f;
            if (a.mass_out) a.mass_out[out + r] = at >= 0 ? a.mass[in + at] : 0.f;
            if (a.idx_out) a.idx_out[out + r] = at < 0 ? -1 : a.idx ? a.idx[in + at] : at;
        }
    }
}

template <int SLOTS>
__global__ __launch_bounds__(kGatherThreads) void evict_gather_kernel(const EvictArgs a) {
    gather_rows<SLOTS, kGatherThreads>(a, blockIdx.y, blockIdx.x, gridDim.x);
}

// A workgroup a sequence, KPT ranks a thread in registers.  The keep-th largest rank is found seven bits at a time from counts of
// 128 bins, every lane with counters of its own (masses share their upper bits: bins that lanes share are all hit at once, 81 us for
// 8 x 16384 places in all; bit by bit by ballots of all ranks 19), until few ranks are left that it can be, mostly after two steps;
// those one wavefront searches bit by bit.
// SLOTS: it moves the rows, of so many 16-byte slots, as well; 0: a launch behind this one does.
constexpr int kFew = 512, kDigit = 7, kBins = 1 << kDigit;
template <int KPT, int SLOTS = 0>
__global__ __launch_bounds__(kSelectThreads) void evict_select_kernel(const EvictArgs a) {
    __shared__ __align__(16) unsigned int bins[2][kBins * 64];
    __shared__ __align__(16) unsigned int sums[kBins];
    __shared__ unsigned int few[kFew];
    __shared__ int2 waves[kSelectThreads / 64];
    __shared__ unsigned int few_n, found[3];
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int64_t seq = blockIdx.x;
    unsigned int x[KPT];
#pragma unroll
    for (int j = 0; j < KPT / 4; ++j) load_ranks(a, seq, place_of(KPT, j), x + 4 * j);
    auto clear = [&](int buf) {
#pragma unroll
        for (int i = 0; i < kBins * 64 / (4 * kSelectThreads); ++i) *reinterpret_cast<uintx4*>(&bins[buf][4 * (kSelectThreads * i + tid)]) = uintx4{0u, 0u, 0u, 0u};
    };
    clear(0);
    clear(1);
    if (tid == 0) few_n = 0u;
    __syncthreads();

    // t: the rank's upper bits; of the `in` ranks that start with them it is the left-th largest
    unsigned int t = 0u, left = (unsigned int)a.keep, in = (unsigned int)(KPT * kSelectThreads);
    int shift = 32;
    for (int pass = 0; shift > 0 && in > kFew && in != left; ++pass) {
        const unsigned int mask = pass == 0 ? 0u : 0xffffffffu << shift;
        const int bits = min(shift, kDigit);
        shift -= bits;
        unsigned int* mine = &bins[pass & 1][lane];
        const unsigned int low = (1u << bits) - 1u;
#pragma unroll
        for (int i = 0; i < KPT; ++i)
            if (((x[i] ^ t) & mask) == 0u) atomicAdd(mine + ((x[i] >> shift) & low) * 64, 1u);
        __syncthreads();
        {   // eight threads a bin
            const uintx4 c0 = *reinterpret_cast<const uintx4*>(&bins[pass & 1][8 * tid]), c1 = *reinterpret_cast<const uintx4*>(&bins[pass & 1][8 * tid + 4]);
            const unsigned int c = c0[0] + c0[1] + c0[2] + c0[3] + c1[0] + c1[1] + c1[2] + c1[3];
            const float sum = group_sum<8>((float)c);                   // (at most 65536: exact)
            if ((tid & 7) == 0) sums[tid >> 3] = (unsigned int)sum;
        }
        __syncthreads();
        // two bins a lane, the upper ones first
        const unsigned int hi = sums[kBins - 1 - 2 * lane], lo = sums[kBins - 2 - 2 * lane];
        const unsigned int upto = lane_sums(hi + lo), before = upto - hi - lo;
        const int at = (int)__builtin_ctzll(__ballot(upto >= left));     // (left <= in, the sum of all)
        const unsigned int b = (unsigned int)__builtin_amdgcn_readlane((int)before, at), h = (unsigned int)__builtin_amdgcn_readlane((int)hi, at);
        const bool upper = b + h >= left;
        t |= (unsigned int)(kBins - 1 - 2 * at - (upper ? 0 : 1)) << shift;
        in = upper ? h : (unsigned int)__builtin_amdgcn_readlane((int)lo, at);
        left -= upper ? b : b + h;
        clear(pass & 1);                                                 // (for the step after the next one)
    }
    if (shift > 0 && in != left) {
        const unsigned int mask = 0xffffffffu << shift;
#pragma unroll
        for (int i = 0; i < KPT; ++i)
            if (((x[i] ^ t) & mask) == 0u) few[atomicAdd(&few_n, 1u)] = x[i];
        __syncthreads();
        if (wave == 0) {
            unsigned int y[kFew / 64];
#pragma unroll
            for (int i = 0; i < kFew / 64; ++i) y[i] = 64u * i + lane < in ? few[64 * i + lane] : ~t;      // (~t: never starts with t)
            for (int bit = shift - 1; bit >= 0 && in != left; --bit) {
                const unsigned int cand = t | (1u << bit);
                unsigned int c = 0;                                      // of those that t can be, the ones with this bit
#pragma unroll
                for (int i = 0; i < kFew / 64; ++i) c += (unsigned int)__popcll(__ballot(((y[i] ^ cand) >> bit) == 0u));
                if (c >= left) { t = cand; in = c; }
                else { left -= c; in -= c; }
            }
            if (lane == 0) { found[0] = t; found[1] = in; found[2] = left; }
        }
        __syncthreads();
        t = found[0]; in = found[1]; left = found[2];
    }
    const EvictCut cut = evict_cut(t, in, left);
    int2 before, total;
    sum_ranks<KPT>(x, cut, make_int2(0, 0), waves, before, total);
    list_ranks<KPT>(x, cut, 0, a.pick + (size_t)seq * a.keep, before);
    end_list(a, seq, total, cut);
    if constexpr (SLOTS > 0) {
        __syncthreads();
        gather_rows<SLOTS, kSelectThreads>(a, seq, 0, 1);
    }
}

// Longer sequences: a workgroup per 8192 places (few enough that places of one bin do not hold each other up for long), the same
// search in steps of 11, 11 and 10 bits over counts in memory that every workgroup of a sequence adds to and the next launch reads.
constexpr int kLongKpt = 8, kLongPlaces = kLongKpt * kSelectThreads, kLongBins = 2048;
__device__ __forceinline__ int long_shift(int pass) { return pass == 0 ? 21 : pass == 1 ? 10 : 0; }

// the bits that `passes` finished counts of this sequence have settled
__device__ __forceinline__ void long_prefix(const EvictArgs& a, int64_t seq, int passes, unsigned int& t, unsigned int& in, unsigned int& left) {
    __shared__ unsigned int wave_sum[kSelectThreads / 64], found[3];
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    t = 0u; left = (unsigned int)a.keep; in = 0xffffffffu;
    for (int pass = 0; pass < passes; ++pass) {
        // two bins a thread, the upper ones first
        const unsigned int* h = a.hist + ((size_t)seq * 3 + pass) * kLongBins;
        const int hi = kLongBins - 1 - 2 * tid;
        const unsigned int c1 = h[hi], c0 = h[hi - 1];
        unsigned int sum = c1 + c0;
#pragma unroll
        for (int o = 1; o < 64; o <<= 1) { const unsigned int up = __shfl_up(sum, o); if (lane >= o) sum += up; }
        if (lane == 63) wave_sum[wave] = sum;
        __syncthreads();
        unsigned int before = sum - c1 - c0;
        for (int k = 0; k < wave; ++k) before += wave_sum[k];
        const unsigned int sh = (unsigned int)long_shift(pass);
        if (before < left && left <= before + c1) { found[0] = (unsigned int)hi << sh; found[1] = c1; found[2] = left - before; }
        else if (before + c1 < left && left <= before + c1 + c0) { found[0] = (unsigned int)(hi - 1) << sh; found[1] = c0; found[2] = left - before - c1; }
        __syncthreads();
        t |= found[0]; in = found[1]; left = found[2];
        __syncthreads();
    }
}

__device__ __forceinline__ void load_long(const EvictArgs& a, int64_t seq, int first, unsigned int (&x)[kLongKpt]) {
#pragma unroll
    for (int j = 0; j < kLongKpt / 4; ++j) {
        load_ranks(a, seq, first + place_of(kLongKpt, j), x + 4 * j);
    }
}

__global__ __launch_bounds__(kSelectThreads) void evict_count_kernel(const EvictArgs a, int pass) {
    __shared__ unsigned int bins[kLongBins];
    const int64_t seq = blockIdx.y;
    const int first = (int)blockIdx.x * kLongPlaces;
    unsigned int x[kLongKpt], t, in, left;
    load_long(a, seq, first, x);
    for (int i = threadIdx.x; i < kLongBins; i += kSelectThreads) bins[i] = 0u;
    long_prefix(a, seq, pass, t, in, left);
    __syncthreads();
    const int shift = long_shift(pass);
    const unsigned int mask = pass == 0 ? 0u : 0xffffffffu << long_shift(pass - 1);
#pragma unroll
    for (int i = 0; i < kLongKpt; ++i) {
        if (first + place_of(kLongKpt, i / 4) + i % 4 < a.count && ((x[i] ^ t) & mask) == 0u) atomicAdd(&bins[(x[i] >> shift) & (kLongBins - 1)], 1u);
    }
    __syncthreads();
    unsigned int* h = a.hist + ((size_t)seq * 3 + pass) * kLongBins;
    for (int i = threadIdx.x; i < kLongBins; i += kSelectThreads)
        if (bins[i]) atomicAdd(h + i, bins[i]);
}

// list == 0: how many of a workgroup's places stay; 1: the list, its places after those of the workgroups in front
__global__ __launch_bounds__(kSelectThreads) void evict_list_kernel(const EvictArgs a, int list) {
    __shared__ int2 waves[kSelectThreads / 64];
    __shared__ int base_s[2];
    const int64_t seq = blockIdx.y;
    const int first = (int)blockIdx.x * kLongPlaces;
    unsigned int x[kLongKpt], t, in, left;
    load_long(a, seq, first, x);
    long_prefix(a, seq, 3, t, in, left);
    const EvictCut cut = evict_cut(t, in, left);
    int2* chunk = a.chunk + (size_t)seq * gridDim.x;
    int2 base = make_int2(0, 0);
    if (list) {
        if (threadIdx.x < 2) base_s[threadIdx.x] = 0;
        __syncthreads();
        int up = 0, eq = 0;
        for (unsigned int i = threadIdx.x; i < blockIdx.x; i += kSelectThreads) { const int2 c = chunk[i]; up += c.x; eq += c.y; }
#pragma unroll
        for (int o = 1; o < 64; o <<= 1) { up += __shfl_xor(up, o); eq += __shfl_xor(eq, o); }
        if ((threadIdx.x & 63) == 0 && (up | eq)) { atomicAdd(&base_s[0], up); atomicAdd(&base_s[1], eq); }
        __syncthreads();
        base = make_int2(base_s[0], base_s[1]);
    }
    int2 before, total;
    sum_ranks<kLongKpt>(x, cut, base, waves, before, total);
    if (!list) {
        if (threadIdx.x == 0) chunk[blockIdx.x] = total;
        return;
    }
    list_ranks<kLongKpt>(x, cut, first, a.pick + (size_t)seq * a.keep, before);
    if (blockIdx.x + 1 == gridDim.x) end_list(a, seq, total, cut);
}

// Places whose ranks fit the registers of one workgroup, 64 a thread; more of them take the search by many.  By one / by many, a quarter of the rows
// kept, d = 128, bf16, us a call: 8 x 33000 41.5 / 46.7, 8 x 65536 54 / 59, 64 x 65536 217 / 240, 256 x 33000 405 / 484, 256 x 65536 793 / 929; by many alone:
// 8 x 131072 82 (3.4 TB/s read and written), 512 x 131072 3900 (4.6).
constexpr int kOnePlaces = 64 * kSelectThreads;

static size_t list_bytes(int64_t n_seq, int64_t count) { return ((size_t)n_seq * count * sizeof(int32_t) + 255) / 256 * 256; }
static size_t hist_bytes(int64_t n_seq) { return (size_t)n_seq * 3 * kLongBins * sizeof(unsigned int); }
size_t evict_workspace_bytes(int64_t n_seq, int64_t count) {
    size_t n = list_bytes(n_seq, count);
    if (count > kOnePlaces) n += hist_bytes(n_seq) + (size_t)n_seq * ((count + kLongPlaces - 1) / kLongPlaces) * sizeof(int2);
    return n;
}

template <int SLOTS>
static hipError_t launch_gather(const EvictArgs& a, hipStream_t st) {
    const int per = kGatherThreads / SLOTS * kGatherSteps;
    const int gx = (a.keep + per - 1) / per;
    return launch_timed(kProfEvictCopy, a.n_seq * a.keep, evict_gather_kernel<SLOTS>, dim3((uint32_t)(gx > 65535 ? 65535 : gx), (uint32_t)a.n_seq), dim3(kGatherThreads), 0, st, a);
}

static hipError_t launch_long(const EvictArgs& a, hipStream_t st) {
    const dim3 grid((uint32_t)((a.count + kLongPlaces - 1) / kLongPlaces), (uint32_t)a.n_seq), block(kSelectThreads);
    const int64_t units = a.n_seq * a.count;
    hipError_t e = launch_fill_u32(a.hist, 0u, a.n_seq * 3 * kLongBins, st);
    for (int pass = 0; pass < 3 && e == hipSuccess; ++pass) e = launch_timed(kProfEvict, units, evict_count_kernel, grid, block, 0, st, a, pass);
    for (int list = 0; list < 2 && e == hipSuccess; ++list) e = launch_timed(kProfEvict, units, evict_list_kernel, grid, block, 0, st, a, list);
    return e;
}

template <int KPT, int SLOTS = 0>
static hipError_t launch_select(const EvictArgs& a, hipStream_t st) {
    return launch_timed(kProfEvict, a.n_seq * a.count, evict_select_kernel<KPT, SLOTS>, dim3((uint32_t)a.n_seq), dim3(kSelectThreads), 0, st, a);
}

template <int SLOTS>
static hipError_t launch_whole(const EvictArgs& a, hipStream_t st) {
    return a.count <= 4 * kSelectThreads ? launch_select<4, SLOTS>(a, st) : launch_select<16, SLOTS>(a, st);
}

hipError_t launch_evict(EvictArgs& a, void* workspace, hipStream_t st) {
    a.pick = (int32_t*)workspace;
    a.hist = (unsigned int*)((char*)workspace + list_bytes(a.n_seq, a.count));
    a.chunk = (int2*)((char*)a.hist + hist_bytes(a.n_seq));
    hipError_t e;
    // Few rows: the workgroup that chose them moves them, one launch.  One compute unit copies slower than the launch of many takes from
    // here on.  Both sides, us a call, 8 sequences / the same in a captured graph / 256 sequences: 50 KB kept 8.5 for 11.9 / 8.5 for 8.7 / 12.1 for 14.3,
    // 128 KB (of 4000 places) 9.6 for 12.6 / 9.6 for 9.7 / 19.2 for 22.3, 256 KB 12.0 for 12.7 / 12.1 for 9.7 / 31.6 for 34.2, 500 KB 16.8 for 13.0.
    if (a.count <= 16 * kSelectThreads && (int64_t)2 * a.keep * a.row_bytes <= 192 * 1024) {
        if (a.row_bytes == 128) return launch_whole<8>(a, st);
        if (a.row_bytes == 256) return launch_whole<16>(a, st);
        return launch_whole<32>(a, st);
    }
    if (a.count > kOnePlaces) e = launch_long(a, st);
    else if (a.count <= 4 * kSelectThreads) e = launch_select<4>(a, st);
    else if (a.count <= 8 * kSelectThreads) e = launch_select<8>(a, st);
    else if (a.count <= 16 * kSelectThreads) e = launch_select<16>(a, st);
    else if (a.count <= 32 * kSelectThreads) e = launch_select<32>(a, st);
    else e = launch_select<64>(a, st);
    if (e != hipSuccess) return e;
    if (a.row_bytes == 128) return launch_gather<8>(a, st);
    if (a.row_bytes == 256) return launch_gather<16>(a, st);
    return launch_gather<32>(a, st);
}

}  // namespace bkv
