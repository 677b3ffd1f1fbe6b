// Attention weight that every cached token gets, summed over the queries of its cache:
//   mass_out_j = decay mass_j + sum_q P_qj,   P_qj = w_j e^{<k_j,q>/sqrt d} / sum_i w_i e^{<k_i,q>/sqrt d}
// The denominators are known once the attention pass in front of this one is over, so the logits are formed a second time, by
// keys: a workgroup of four wavefronts keeps 128 keys in registers, 32 each, and its queries go by through LDS, 64 at a time in
// two buffers.  No weight leaves its lane: lane (n, h) adds up query n's share of its 16 keys, and the 32 lanes meet at the end.
#include "bkv_device.h"
#include "bkv_host.h"
#include "tile_device.h"

namespace bkv {

constexpr int kMassThreads = 256;
constexpr int kMassKeys = 128;               // keys of a workgroup
constexpr int kMassRows = 64;                // queries of a tile

template <typename T, int D>
__global__ __launch_bounds__(kMassThreads) void mass_kernel(const MassArgs a) {
    using R = TileRows<T, D>;
    constexpr int ROWB = R::kRowB, SLOTS = R::kSlots, NP = kMassRows * SLOTS / kMassThreads;
    __shared__ __align__(16) char lds[2][kMassRows * ROWB];
    __shared__ __align__(16) floatx2 st[2][kMassRows];

    const int tid = threadIdx.x, lane = tid & 63, n = lane & 31, h = lane >> 5;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const unsigned int block = blockIdx.y * gridDim.x + blockIdx.x;
    const unsigned int per_seq = (unsigned int)a.n_kb * (unsigned int)a.splits;
    const int64_t seq = block / per_seq;
    if (seq >= a.n_seq) return;
    const int in_seq = (int)(block % per_seq);
    const int kb = in_seq % a.n_kb, split = in_seq / a.n_kb;
    const int k0 = kb * kMassKeys + 32 * wave;

    // queries of this workgroup: of a causal set the first ones see none of its keys
    int r0 = split * a.rows_per_split, r1 = min(a.rows, r0 + a.rows_per_split);
    if (a.causal) {
        const int64_t from = (kb * kMassKeys + 1 - a.visible) * a.inner;                // first row that sees the first key
        if (from > r0) r0 = (int)min(from, (int64_t)r1);
    }

    const char* Kb = a.K + (size_t)seq * a.stride * ROWB;
    const float* wb = a.w + (size_t)seq * a.stride;
    uintx4 kf[R::kPieces];
    floatx16 bias;
    {
        const int key = min(k0 + n, a.count - 1);
        const bool live = k0 + n < a.count && wb[key] > 0.f;
#pragma unroll
        for (int c = 0; c < R::kPieces; ++c) {
            kf[c] = *reinterpret_cast<const uintx4*>(Kb + (size_t)key * ROWB + 32 * c + 16 * h);
            if (!live) kf[c] = uintx4{0u, 0u, 0u, 0u};
        }
#pragma unroll
        for (int r = 0; r < 16; ++r) {
            const int k = k0 + tile_row(r, h);
            const float w = wb[min(k, a.count - 1)];
            bias[r] = k < a.count && w > 0.f ? __builtin_amdgcn_logf(w) * a.inv_scale : kTileDead;
        }
    }
    uintx4 qreg[NP];
    floatx2 streg = {0.f, 0.f};
    auto q_row = [&](int r) {
        const int outer = r / a.inner;
        return seq * a.q_stream + (int64_t)outer * a.q_outer + (int64_t)(r - outer * a.inner) * a.q_inner;
    };
    auto load = [&](int r) {
#pragma unroll
        for (int i = 0; i < NP; ++i) {
            const int piece = tid + kMassThreads * i;
            qreg[i] = *reinterpret_cast<const uintx4*>(a.Q + (size_t)q_row(min(r + piece / SLOTS, r1 - 1)) * ROWB + (piece % SLOTS) * 16);
        }
        if (tid < kMassRows)
            streg = r + tid < r1 ? *reinterpret_cast<const floatx2*>(a.stats + 2 * q_row(r + tid)) : floatx2{-kTileDead, 0.f};
    };
    auto store = [&](int buf) {
#pragma unroll
        for (int i = 0; i < NP; ++i) {
            const int piece = tid + kMassThreads * i, r = piece / SLOTS, s = piece % SLOTS;
            *reinterpret_cast<uintx4*>(lds[buf] + r * ROWB + R::key_slot(r, s) * 16) = qreg[i];
        }
        if (tid < kMassRows) st[buf][tid] = streg;
    };
    float acc[16];
#pragma unroll
    for (int r = 0; r < 16; ++r) acc[r] = 0.f;

    if (r0 < r1) {
        load(r0);
        store(0);
        __syncthreads();
        int buf = 0;
        for (int r = r0;; r += kMassRows) {
            const bool more = r + kMassRows < r1;
            if (more) load(r + kMassRows);
#pragma unroll
            for (int sub = 0; sub < kMassRows / 32; ++sub) {
                if (r + 32 * sub >= r1) break;
                const int qr = 32 * sub + n;
                floatx16 s = bias;
                if constexpr (R::kB16) {
#pragma unroll
                    for (int c = 0; c < R::kPieces; ++c)
                        s = tile_mma<T>(kf[c], *reinterpret_cast<const uintx4*>(lds[buf] + qr * ROWB + R::key_slot(qr, 2 * c + h) * 16), s);
                } else {
                    floatx16 s1;
#pragma unroll
                    for (int x = 0; x < 16; ++x) s1[x] = 0.f;
                    floatx16 s0 = s1;
#pragma unroll
                    for (int c = 0; c < R::kPieces; c += 2) {
                        s0 = tile_mma<T>(kf[c], *reinterpret_cast<const uintx4*>(lds[buf] + qr * ROWB + R::key_slot(qr, 2 * c + h) * 16), s0);
                        s1 = tile_mma<T>(kf[c + 1], *reinterpret_cast<const uintx4*>(lds[buf] + qr * ROWB + R::key_slot(qr, 2 * c + 2 + h) * 16), s1);
                    }
                    s = s + (s0 + s1);
                }
                if (a.causal) {
                    const int64_t sees = a.visible + min(r + qr, r1 - 1) / a.inner;
                    if (__builtin_amdgcn_ballot_w64(sees < k0 + 32) != 0ull) {
#pragma unroll
                        for (int x = 0; x < 16; ++x) s[x] = k0 + tile_row(x, h) < sees ? s[x] : kTileDead;
                    }
                }
                const floatx2 ml = st[buf][qr];
#pragma unroll
                for (int x = 0; x < 16; ++x) acc[x] = fmaf(fast_exp2(fmaf(s[x], a.scale_log2, -ml[0])), ml[1], acc[x]);
            }
            if (!more) break;
            store(buf ^ 1);
            __syncthreads();
            buf ^= 1;
        }
    }
    const int s = lane & 15;
    const float total = xor_sum<16>(row16_transpose_sum(acc, s));
    const int key = k0 + tile_row(s, h);
    if ((lane & 16) != 0 || key >= a.count) return;
    if (a.splits > 1) {
        a.part[((size_t)split * a.n_seq + seq) * a.count + key] = total;
    } else {
        const size_t at = (size_t)seq * a.stride + key;
        a.mass_out[at] = a.mass ? fmaf(a.decay, a.mass[at], total) : total;
    }
}

__global__ __launch_bounds__(kMassThreads) void mass_merge_kernel(const MassArgs a) {
    const int64_t seq = blockIdx.y;
    for (int64_t key = (int64_t)blockIdx.x * kMassThreads + threadIdx.x; key < a.count; key += (int64_t)gridDim.x * kMassThreads) {
        float total = 0.f;
        for (int s = 0; s < a.splits; ++s) total += a.part[((size_t)s * a.n_seq + seq) * a.count + key];
        const size_t at = (size_t)seq * a.stride + key;
        a.mass_out[at] = a.mass ? fmaf(a.decay, a.mass[at], total) : total;
    }
}

// The queries are split until there are two workgroups per compute unit, so the partial sums are at most so many times its keys.
constexpr int kMassTarget = 512;
size_t mass_part_bytes() { return (size_t)kMassTarget * kMassKeys * sizeof(float); }

static int mass_splits(int64_t n_seq, int64_t count, int64_t rows) {
    const int64_t wgs = n_seq * ((count + kMassKeys - 1) / kMassKeys);
    int64_t splits = kMassTarget / wgs;
    const int64_t tiles = (rows + kMassRows - 1) / kMassRows;
    if (splits > tiles) splits = tiles;
    return splits < 1 ? 1 : (int)splits;
}

template <typename T, int D>
static hipError_t launch_mass_t(MassArgs& a, hipStream_t st) {
    a.n_kb = (a.count + kMassKeys - 1) / kMassKeys;
    const int splits = mass_splits(a.n_seq, a.count, a.rows);
    const int tiles = (a.rows + kMassRows - 1) / kMassRows;
    const int per = (tiles + splits - 1) / splits;
    a.rows_per_split = per * kMassRows;
    a.splits = (tiles + per - 1) / per;
    const uint64_t blocks = (uint64_t)a.n_seq * a.n_kb * a.splits;
    if (blocks >= (uint64_t)1 << 31) return hipErrorInvalidValue;
    const uint32_t gx = blocks > 65536 ? 65536u : (uint32_t)blocks;
    hipError_t e = launch_timed(kProfAttend, a.n_seq * a.count, mass_kernel<T, D>, dim3(gx, (uint32_t)((blocks + gx - 1) / gx)), dim3(kMassThreads), 0, st, a);
    if (e != hipSuccess || a.splits == 1) return e;
    const uint32_t mx = (uint32_t)((a.count + kMassThreads - 1) / kMassThreads);
    return launch_timed(kProfAttendMerge, a.n_seq * a.count, mass_merge_kernel, dim3(mx > 4096 ? 4096 : mx, (uint32_t)a.n_seq), dim3(kMassThreads), 0, st, a);
}

hipError_t launch_mass(int dtype, int d, MassArgs& a, hipStream_t st) {
    if (dtype == BKV_BF16 && d == 128) return launch_mass_t<__bf16, 128>(a, st);
    if (dtype == BKV_BF16 && d == 64) return launch_mass_t<__bf16, 64>(a, st);
    if (dtype == BKV_F32 && d == 128) return launch_mass_t<float, 128>(a, st);
    if (dtype == BKV_F32 && d == 64) return launch_mass_t<float, 64>(a, st);
    return hipErrorInvalidValue;
}

}  // namespace bkv
