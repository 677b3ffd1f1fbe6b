// Attention weight that every cached token gets, summed over the queries of its cache:
//   mass_out_j = decay mass_j + sum_q P_qj,   P_qj = w_j e^{<k_j,q>/sqrt d} / sum_i w_i e^{<k_i,q>/sqrt d}
// The denominators are known once the attention pass in front of this one is over, so the logits are formed a second time, by
// keys: a workgroup of four wavefronts keeps 128 keys in registers, 32 each, and its queries go by through LDS, 64 at a time in
// two buffers, in the order in which they lie in memory.  No weight leaves its lane: lane (n, h) adds up query n's share of its 16
// keys, and the 32 lanes meet at the end.
// Bound by the vector unit first (exponentials: 51 % of the cycles, products 31 %; bf16, d = 128, 8 x 4096 tokens x 4 x 4096 queries, causal: 98 us,
// 700 TFLOP/s), with few queries by the trips of a few tiles (8 x 8704 tokens x 256: 14 us).
#include <type_traits>

#include "bkv_device.h"
#include "bkv_host.h"
#include "tile_device.h"

namespace bkv {

constexpr int kMassThreads = 256;
constexpr int kMassKeys = 128;               // keys of a workgroup
constexpr int kMassRows = 64;                // queries of a tile

template <typename T, int D>
__global__ __launch_bounds__(kMassThreads, sizeof(T) == 2 ? 3 : 1) void mass_kernel(const MassArgs a) {
    using R = TileRows<T, D>;
    using F = TileFetch<T, D>;
    constexpr int ROWB = R::kRowB, TILEB = kMassRows * ROWB;
    __shared__ __align__(16) char lds[2][TILEB];

    const int tid = threadIdx.x, lane = tid & 63, n = lane & 31, h = lane >> 5;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    // workgroup -> (sequence, keys, split): the workgroups of a sequence read the same queries and go to one XCD; the first keys of a
    // causal set, which the most queries see, come first
    const unsigned int block = blockIdx.y * gridDim.x + blockIdx.x;
    const unsigned int per_seq = (unsigned int)a.n_kb * (unsigned int)a.splits;
    const unsigned int in_xcd = a.by_xcd ? block >> 3 : block;
    const int64_t seq = a.by_xcd ? (int64_t)(in_xcd / per_seq) * 8 + (block & 7u) : in_xcd / per_seq;
    if (seq >= a.n_seq) return;
    const int in_seq = (int)(in_xcd % per_seq);
    const int kb = in_seq / a.splits, split = in_seq % a.splits;
    const int kb0 = kb * kMassKeys, k0 = kb0 + 32 * wave;

    const char* Kb = a.K + (size_t)seq * a.stride * ROWB;
    const char* Qb = a.Q + (size_t)seq * a.rows * ROWB;
    const floatx2* Sb = reinterpret_cast<const floatx2*>(a.stats) + (size_t)seq * a.rows;
    const float* wb = a.w + (size_t)seq * a.stride;

    // keys of this wavefront, on their way first
    uintx4 kf[R::kPieces];
    const int key = min(k0 + n, a.count - 1);
#pragma unroll
    for (int c = 0; c < R::kPieces; ++c) kf[c] = *reinterpret_cast<const uintx4*>(Kb + (size_t)key * ROWB + 32 * c + 16 * h);
    const float w_raw = wb[key], w = k0 + n < a.count ? w_raw : 0.f;

    // tiles split, split + splits, ... of the sequence's queries (row = head nq + position); of a causal set those of which no query
    // sees a key are passed over.  p0: position of the tile's first row
    const int tiles = (a.rows + kMassRows - 1) / kMassRows;
    int p0 = a.causal ? split * kMassRows % a.nq : 0;
    const int p_step = a.causal ? a.splits * kMassRows % a.nq : 0;
    auto in_one_head = [&](int t) { return p0 + min(kMassRows, a.rows - t * kMassRows) <= a.nq; };
    auto next_tile = [&](int t) {
        if (a.causal)
            for (; t < tiles; t += a.splits) {
                if (a.visible + (in_one_head(t) ? p0 + min(kMassRows, a.rows - t * kMassRows) - 1 : a.nq - 1) > kb0) break;
                p0 += p_step;
                if (p0 >= a.nq) p0 -= a.nq;
            }
        return t;
    };
    unsigned int qo[F::kSteps];
#pragma unroll
    for (int i = 0; i < F::kSteps; ++i) {
        const int r = 16 * wave + F::row(i, lane);
        qo[i] = r * ROWB + R::key_slot(r, lane % R::kSlots) * 16;
    }
    const unsigned int lds0 = lds_address(&lds[0][0]) + 16 * wave * ROWB;
    auto fetch = [&](int t, int buf) {
        const char* from = Qb + (size_t)t * TILEB;
        const int left = a.rows - 1 - t * kMassRows;
#pragma unroll
        for (int i = 0; i < F::kSteps; ++i)                          // (rows past the end repeat it, their statistics say 0)
            to_lds(from, qo[i] - (left < kMassRows - 1 ? max(16 * wave + F::row(i, lane) - left, 0) * ROWB : 0), lds0 + buf * TILEB + 1024 * i);
    };
    floatx2 st0[2], st1[2];
    auto load_stats = [&](floatx2 (&st)[2], int t) {
#pragma unroll
        for (int u = 0; u < 2; ++u) {
            const int r = t * kMassRows + 32 * u + n;
            st[u] = Sb[min(r, a.rows - 1)];
            if (r >= a.rows) st[u] = floatx2{-kTileDead, 0.f};
        }
    };
    int t = next_tile(split);
    if (t < tiles) { fetch(t, 0); load_stats(st0, t); }

    floatx16 bias;                               // log2 w of the keys, in units of 1 / scale
    {
        const bool live = w > 0.f;
        if (__ballot(!live) != 0ull) {
#pragma unroll
            for (int c = 0; c < R::kPieces; ++c)
                if (!live) kf[c] = uintx4{0u, 0u, 0u, 0u};           // (whatever the row holds)
        }
        const float mine = live ? log2_weight(w) * a.inv_scale : kTileDead;
#pragma unroll
        for (int r = 0; r < 16; ++r) bias[r] = __shfl(mine, tile_row(r, h));
    }
    unsigned int ro[R::kPieces];
#pragma unroll
    for (int c = 0; c < R::kPieces; ++c) ro[c] = n * ROWB + R::key_slot(n, 2 * c + h) * 16;
    float acc[16];
#pragma unroll
    for (int r = 0; r < 16; ++r) acc[r] = 0.f;

    auto compute = [&](auto buf_c, int tile) {
        constexpr int BUF = decltype(buf_c)::value;
        const bool masked = a.causal && a.visible + (in_one_head(tile) ? p0 : 0) < k0 + 32;        // a query does not see all keys
#pragma unroll
        for (int u = 0; u < 2; ++u) {
            floatx16 s = bias;
            if constexpr (R::kB16) {
#pragma unroll
                for (int c = 0; c < R::kPieces; ++c) s = tile_mma<T>(kf[c], *reinterpret_cast<const uintx4*>(lds[BUF] + ro[c] + 32 * u * ROWB), s);
            } else {
                floatx16 s0, s1;
#pragma unroll
                for (int x = 0; x < 16; ++x) s0[x] = 0.f;
                s1 = s0;
#pragma unroll
                for (int c = 0; c < R::kPieces; c += 2) {
                    s0 = tile_mma<T>(kf[c], *reinterpret_cast<const uintx4*>(lds[BUF] + ro[c] + 32 * u * ROWB), s0);
                    s1 = tile_mma<T>(kf[c + 1], *reinterpret_cast<const uintx4*>(lds[BUF] + ro[c + 1] + 32 * u * ROWB), s1);
                }
                s = s + (s0 + s1);
            }
            if (masked) {
                const int r = min(tile * kMassRows + 32 * u + n, a.rows - 1) - tile * kMassRows;
                const int64_t sees = a.visible + (p0 + r) % a.nq;
#pragma unroll
                for (int x = 0; x < 16; ++x) s[x] = k0 + tile_row(x, h) < sees ? s[x] : kTileDead;
            }
#pragma unroll
            for (int x = 0; x < 16; ++x) acc[x] = fmaf(fast_exp2(fmaf(s[x], a.scale_log2, -st0[u][0])), st0[u][1], acc[x]);
        }
    };
    if (t < tiles) {
        all_arrived_so_far();
        tile_barrier();
        auto step = [&](auto buf_c) {            // true: this was the last tile
            constexpr int BUF = decltype(buf_c)::value;
            const int p_now = p0;
            p0 += p_step;
            if (p0 >= a.nq) p0 -= a.nq;
            const int tn = next_tile(t + a.splits), p_next = p0;
            const bool more = tn < tiles;
            if (more) { load_stats(st1, tn); fetch(tn, BUF ^ 1); }
            p0 = p_now;
            compute(buf_c, t);
            if (!more) return true;
            p0 = p_next;
            tile_arrived();
            tile_barrier();
            t = tn;
#pragma unroll
            for (int u = 0; u < 2; ++u) st0[u] = st1[u];
            return false;
        };
        while (!step(std::integral_constant<int, 0>{}) && !step(std::integral_constant<int, 1>{})) {}
    }
    const int s = lane & 15;
    const bool live = __shfl(w, tile_row(s, h)) > 0.f;               // (a NaN query reaches no place without a token)
    const float sum = xor_sum<16>(row16_transpose_sum(acc, s)), total = live ? sum : 0.f;
    const int to = k0 + tile_row(s, h);
    if ((lane & 16) != 0 || to >= a.count) return;
    if (a.splits > 1) {
        a.part[((size_t)split * a.n_seq + seq) * a.count + to] = total;
    } else {
        const size_t at = (size_t)seq * a.stride + to;
        a.mass_out[at] = a.mass ? fmaf(a.decay, a.mass[at], total) : total;
    }
}

__global__ __launch_bounds__(kMassThreads) void mass_merge_kernel(const MassArgs a) {
    const int64_t seq = blockIdx.y;
    for (int64_t key = (int64_t)blockIdx.x * kMassThreads + threadIdx.x; key < a.count; key += (int64_t)gridDim.x * kMassThreads) {
        constexpr int U = 8;                                         // partial sums on their way at a time
        float total = 0.f;
        for (int s0 = 0; s0 < a.splits; s0 += U) {
            float x[U];
#pragma unroll
            for (int u = 0; u < U; ++u) x[u] = a.part[((size_t)min(s0 + u, a.splits - 1) * a.n_seq + seq) * a.count + key];
#pragma unroll
            for (int u = 0; u < U; ++u) total += s0 + u < a.splits ? x[u] : 0.f;
        }
        const size_t at = (size_t)seq * a.stride + key;
        a.mass_out[at] = a.mass ? fmaf(a.decay, a.mass[at], total) : total;
    }
}

// The queries are split until there are eight workgroups per compute unit (causal sets: of very different length), so the partial sums are at most so many times its keys.
constexpr int kMassTarget = 2048;
size_t mass_part_bytes() { return (size_t)kMassTarget * kMassKeys * sizeof(float); }

static int mass_splits(int64_t n_seq, int64_t count, int64_t rows, int elem) {
    const int64_t wgs = n_seq * ((count + kMassKeys - 1) / kMassKeys);
    // (bf16: a workgroup takes the time of two or three tiles to begin and to end: eight tiles each, where there are workgroups enough.
    // fp32: a tile takes longer than that by itself.  Three tiles or fewer are over before another launch would have added them up.)
    const int64_t tiles = (rows + kMassRows - 1) / kMassRows, fill = (256 + wgs - 1) / wgs;
    int64_t most = elem == 2 ? tiles / 8 > fill ? tiles / 8 : fill : tiles;
    if (most > tiles) most = tiles;
    if (tiles < 4) most = 1;
    int64_t splits = (elem == 2 ? kMassTarget : kMassTarget / 2) / wgs;
    if (splits > most) splits = most;
    return splits < 1 ? 1 : (int)splits;
}

template <typename T, int D>
static hipError_t launch_mass_t(MassArgs& a, hipStream_t st) {
    a.n_kb = (a.count + kMassKeys - 1) / kMassKeys;
    const int splits = mass_splits(a.n_seq, a.count, a.rows, (int)sizeof(T));
    a.splits = splits;
    a.by_xcd = a.n_seq % 8 == 0 || a.n_seq >= 48;              // (equal shares for all XCDs)
    const uint64_t blocks = (uint64_t)(a.by_xcd ? (a.n_seq + 7) / 8 * 8 : a.n_seq) * a.n_kb * a.splits;
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
