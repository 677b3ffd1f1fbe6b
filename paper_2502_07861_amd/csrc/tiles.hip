// Attention of many queries against weighted caches: batches that share a prefix, observation windows, whole prompts.
//   z = sum_i w_i e^{<k_i,q>/sqrt d} v_i / sum_i w_i e^{<k_i,q>/sqrt d}
// over the tokens i of one or two caches, optionally only the first few of them per query (causal).
//
// A workgroup of four wavefronts takes 32, 64 or 128 queries of one cache against a range of its keys, 64 at a time: keys and
// values go from memory to LDS once for all its queries, in two buffers, the next tile's are under way while the current one is
// multiplied.  A wavefront has 32 queries in registers; where the workgroup has fewer than 128, wavefronts share queries and
// split the keys of a tile.  Softmax weights stay in the lane that the next product wants them in (tile_device.h).
//
// What bounds it (bf16, d = 128): memory with few queries to a row (256 prefixes x 8192 tokens x 64 queries, 4096 sequences of 151 own tokens on
// average in 301 places: 277 us, 5.3 TB/s of rows that are fetched); with hundreds the products (45 % of the cycles) and the vector unit (43 %), which a
// wavefront keeps busy in turn, two of them to a SIMD (8 x 16385 tokens x 1280 queries 136 us, 940 TFLOP/s with both numbers of a weight; 8 x 4096
// tokens x 4 x 4096 queries, causal, 224 us, 920); start, two trips to memory and a store with little to do (8 x 4096 x 16: 8.2 us).
#include <type_traits>

#include "bkv_device.h"
#include "bkv_host.h"
#include "tile_device.h"

namespace bkv {

constexpr int kTileKeys = 64;
constexpr int kTileThreads = 256;
constexpr int kTilePad = 4;                  // floats behind the D sums of a partial row: [0] reference exponent, [1] denominator

// Two tiles, so that the next one is on its way while one is multiplied; of rows of 512 bytes (fp32, whose products take four times as
// long as their loads) one, and two workgroups a compute unit that wait in turn.
template <typename T, int D> struct TileLds {
    static constexpr int kBuffers = D * sizeof(T) == 512 ? 1 : 2;
    __align__(16) char rows[kBuffers][2][kTileKeys * D * sizeof(T)];        // [buffer][keys, values]
};

// Short caches of many sequences: a wavefront each, 32 keys at a time, nothing shared; so many wavefronts of a workgroup have room in LDS.
template <typename T, int D> constexpr int kSoloWaves = D * sizeof(T) == 512 ? 2 : 4;

// QW: wavefronts with queries of their own; 4 / QW share the same ones.  0: a wavefront is on its own.
template <typename T, int D, int QW>
__device__ __forceinline__ void tile_body(const TileArgs& a, const TileJob& J, int64_t stream /* SOLO: a workgroup's */, int split, int qt, TileLds<T, D>& lds) {
    using R = TileRows<T, D>;
    using F = TileFetch<T, D>;
    constexpr int ROWB = R::kRowB, EPN = R::kEpn, P = D + kTilePad;
    constexpr bool SOLO = QW == 0;
    constexpr int Q1 = SOLO ? 1 : QW;
    constexpr int KEYS = SOLO ? 32 : kTileKeys, TILEB = KEYS * ROWB, BUFS = SOLO ? 1 : TileLds<T, D>::kBuffers;
    constexpr int SHARE = SOLO ? KEYS : KEYS / 4, STEPS = SHARE / F::kRps;        // rows of a tile that a wavefront brings
    // wavefronts a query has; groups of 32 keys a wavefront takes of a tile at a time, times (fp32: registers)
    constexpr int KW = SOLO ? 1 : 4 / Q1, NS = QW == 4 && R::kB16 ? 2 : 1, TIMES = QW == 4 ? 2 / NS : 1;

    const int tid = threadIdx.x, lane = tid & 63, n = lane & 31, h = lane >> 5;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int qsub = SOLO ? 0 : wave & (Q1 - 1), ksub = SOLO ? 0 : wave / Q1;
    if constexpr (SOLO) {
        stream = stream * kSoloWaves<T, D> + wave;
        if (wave >= kSoloWaves<T, D> || stream >= J.n_streams) return;          // (no barrier below)
    }
    const int row_first = qt * 32 * QW, row0 = row_first + 32 * qsub;
    const bool has_rows = row0 < J.rows && ksub * 32 < KEYS;
    const int row = min(row0 + n, J.rows - 1);
    const int outer = row / J.inner;
    const int64_t q_row = stream * J.q_stream + (int64_t)outer * J.q_outer + (int64_t)(row - outer * J.inner) * J.q_inner;

    // tiles of keys of this workgroup
    const int tiles = (J.count + KEYS - 1) / KEYS;
    const int t0 = split * J.tiles_per_split;
    int t1 = min(tiles, t0 + J.tiles_per_split);
    int sees = J.count, sees_min = J.count, most = J.count;          // places: that this query, any one of the wavefront, one of the workgroup sees
    if (a.causal) {
        auto visible = [&](int i) { return (int)min((int64_t)J.count, max((int64_t)0, a.visible + i)); };
        sees = visible(outer);
        most = visible((min(row_first + 32 * Q1, J.rows) - 1) / J.inner);
        t1 = min(t1, (most + KEYS - 1) / KEYS);
        if (split > 0 && t0 >= t1) return;                           // (none of its queries sees this split: the merge does not look at it)
        sees_min = visible(min(row0, J.rows - 1) / J.inner);
    }

    const char* Kb = J.K + (size_t)stream * J.stride * ROWB;
    const char* Vb = J.V + (size_t)stream * J.stride * ROWB;
    const float* wb = J.w + (size_t)stream * J.stride;

    // ---- a tile on its way: this lane's bytes of each step, the slots exchanged as the rows are stored
    const int share0 = SOLO ? 0 : SHARE * wave;
    unsigned int kgo[STEPS], vgo[STEPS];
#pragma unroll
    for (int i = 0; i < STEPS; ++i) {
        const int r = share0 + F::row(i, lane), s = lane % R::kSlots;
        kgo[i] = r * ROWB + R::key_slot(r, s) * 16;
        vgo[i] = r * ROWB + R::value_slot(r, s) * 16;
    }
    char* mine = &lds.rows[0][0][0] + (SOLO ? wave * 2 * TILEB : 0);           // [buffer][keys, values] of this wavefront or workgroup
    const unsigned int lds0 = lds_address(mine) + share0 * ROWB;
    auto fetch = [&](int t, int buf) {
        const char* kp = Kb + (size_t)t * TILEB;
        const char* vp = Vb + (size_t)t * TILEB;
        const unsigned int to = lds0 + buf * 2 * TILEB;
        const int left = J.count - 1 - t * KEYS;                     // last row there is
        if (left >= KEYS - 1) {
#pragma unroll
            for (int i = 0; i < STEPS; ++i) { to_lds(kp, kgo[i], to + 1024 * i); to_lds(vp, vgo[i], to + TILEB + 1024 * i); }
        } else {                                                     // (rows past the end repeat it, with weight 0)
#pragma unroll
            for (int i = 0; i < STEPS; ++i) {
                const int r = share0 + F::row(i, lane);
                const unsigned int back = max(r - left, 0) * ROWB;
                to_lds(kp, kgo[i] - back, to + 1024 * i);
                to_lds(vp, vgo[i] - back, to + TILEB + 1024 * i);
            }
        }
    };
    auto weight = [&](int t) {                                       // lane (SOLO: and lane + 32): key
        const int key = t * KEYS + (lane & (KEYS - 1));
        const float w = wb[min(key, J.count - 1)];
        return key < most ? w : 0.f;
    };
    // rows of places without a token, whatever they hold: 0 (each wavefront those it brought)
    auto clear_dead = [&](int buf, unsigned long long live) {
        unsigned int dead = (unsigned int)(~live >> share0) & (SOLO ? 0xffffffffu : 0xffffu);
        if (live == 0ull) return;                                    // (not fetched, not looked at)
        while (dead != 0u) {
            const int r = share0 + __builtin_ctz(dead);
            dead &= dead - 1u;
#pragma unroll
            for (int k = 0; k < 2; ++k) {
                char* to = mine + (2 * buf + k) * TILEB + r * ROWB + lane * (ROWB / 64);
                if constexpr (ROWB == 128) *reinterpret_cast<unsigned short*>(to) = 0;
                else if constexpr (ROWB == 256) *reinterpret_cast<unsigned int*>(to) = 0u;
                else *reinterpret_cast<uint2*>(to) = make_uint2(0u, 0u);
            }
        }
    };

    // where a lane reads: key row n (of the wavefront's group), value columns (see tile_device.h)
    unsigned int ko[R::kPieces];
#pragma unroll
    for (int c = 0; c < R::kPieces; ++c) ko[c] = ksub * 32 * ROWB + n * ROWB + R::key_slot(n, 2 * c + h) * 16;
    constexpr int NV = R::kB16 ? EPN : 1;
    unsigned int vo[NV];
    if constexpr (R::kB16) {
        const int i16 = lane & 15, half = (lane >> 4) & 1, r = 4 * h + (i16 >> 2);
#pragma unroll
        for (int e = 0; e < EPN; ++e)
            vo[e] = ksub * 32 * ROWB + r * ROWB + R::value_slot(r, 4 * e + 2 * half + ((i16 & 3) >> 1)) * 16 + (i16 & 1) * 8;
    } else vo[0] = ksub * 32 * ROWB + 4 * h * ROWB + n * (EPN * 4);

    float w0 = 0.f, w1 = 0.f, w2 = 0.f;
    unsigned long long live0 = 0ull, live1 = 0ull;
    if (t0 < t1) {
        fetch(t0, 0);                                                // (before its weights are there, whether they say so or not)
        w0 = weight(t0);
        if (t0 + 1 < t1) w1 = weight(t0 + 1);
    }
    uintx4 qf[R::kPieces];
#pragma unroll
    for (int c = 0; c < R::kPieces; ++c) qf[c] = *reinterpret_cast<const uintx4*>(a.Q + (size_t)q_row * ROWB + 32 * c + 16 * h);

    float m = kTileLow, l = 0.f;
    floatx16 o[EPN];
#pragma unroll
    for (int e = 0; e < EPN; ++e)
#pragma unroll
        for (int r = 0; r < 16; ++r) o[e][r] = 0.f;

    auto compute = [&](auto buf_c, int t, float w, int group) {      // groups group .. group + NS - 1 of the tile's keys (and ksub)
        constexpr int BUF = decltype(buf_c)::value;
        const char* Kt = mine + 2 * BUF * TILEB + group * (32 * ROWB);
        const char* Vt = Kt + TILEB;
        const int k0 = t * KEYS + 32 * (ksub + group);
        // ---- logits, in units of 1 / scale
        __builtin_amdgcn_s_setprio(1);
        floatx16 s[NS];
#pragma unroll
        for (int u = 0; u < NS; ++u) {
#pragma unroll
            for (int r = 0; r < 16; ++r) s[u][r] = 0.f;
            if constexpr (R::kB16) {
#pragma unroll
                for (int c = 0; c < R::kPieces; ++c)
                    s[u] = tile_mma<T>(*reinterpret_cast<const uintx4*>(Kt + ko[c] + 32 * u * ROWB), qf[c], s[u]);
            } else {
                // two chains, so that no sum is rounded more than d / 4 times at its full size
                floatx16 s1 = s[u];
#pragma unroll
                for (int c = 0; c < R::kPieces; c += 2) {
                    s[u] = tile_mma<T>(*reinterpret_cast<const uintx4*>(Kt + ko[c] + 32 * u * ROWB), qf[c], s[u]);
                    s1 = tile_mma<T>(*reinterpret_cast<const uintx4*>(Kt + ko[c + 1] + 32 * u * ROWB), qf[c + 1], s1);
                }
                s[u] = s[u] + s1;
            }
        }
        __builtin_amdgcn_s_setprio(0);
        // ---- token weights: one for the whole tile (the usual tile), or ln2 w of every key as one more product: its three bf16
        // parts (together all its bits) times ones, in the half of the wavefront that holds the group's keys.  An infinite weight makes NaN of
        // the queries that see its token, so it is never the tile's
        const float first = __uint_as_float(__builtin_amdgcn_readfirstlane(__float_as_uint(w)));
        const bool one = first > 0.f && first < INFINITY && __ballot(w == first) == ~0ull;
        const float b = one ? log2_weight(first) : 0.f;
        if (!one) {
            const float x = w > 0.f ? log2_weight(w) * a.inv_scale : kTileDead;
#pragma unroll
            for (int u = 0; u < NS; ++u) {
                const float y = h == ksub + group + u ? x : 0.f;
                if constexpr (R::kB16) {
                    const unsigned int y0 = __float_as_uint(y) & 0xffff0000u;
                    const float rest = y - __uint_as_float(y0);
                    const unsigned int y1 = __float_as_uint(rest) & 0xffff0000u;
                    const uintx4 part = {(y0 >> 16) | y1, __float_as_uint(rest - __uint_as_float(y1)) >> 16, 0u, 0u};
                    const uintx4 ones = {0x3f803f80u, 0x00003f80u, 0u, 0u};
                    s[u] = tile_mma<T>(part, ones, s[u]);
                } else s[u] = __builtin_amdgcn_mfma_f32_32x32x2f32(y, 1.f, s[u], 0, 0, 0);
            }
        }
        if (a.causal && k0 + 32 * NS > sees_min) {
#pragma unroll
            for (int u = 0; u < NS; ++u)
#pragma unroll
                for (int r = 0; r < 16; ++r) s[u][r] = k0 + 32 * u + tile_row(r, h) < sees ? s[u][r] : kTileDead;
        }
        // ---- weights 2^(logit - m); m moves when a logit passes it by more than the slack
        float mx = s[0][0];
#pragma unroll
        for (int u = 0; u < NS; ++u)
#pragma unroll
            for (int r = 0; r < 16; ++r) mx = fmaxf(mx, s[u][r]);
        mx = fmaf(mx, a.scale_log2, b);
        if (__builtin_amdgcn_ballot_w64(mx > m + kTileSlack) != 0ull) {
            const float mnew = fmaxf(m, half_max(mx));
            const float sc = fast_exp2(m - mnew);
            m = mnew;
            l *= sc;
#pragma unroll
            for (int e = 0; e < EPN; ++e) o[e] *= sc;
        }
        const float shift = b - m;
#pragma unroll
        for (int u = 0; u < NS; ++u)
#pragma unroll
            for (int r = 0; r < 16; ++r) { s[u][r] = fast_exp2(fmaf(s[u][r], a.scale_log2, shift)); l += s[u][r]; }
        // ---- values.  bf16: a weight multiplies its value row as two bf16 numbers, its upper bits and what they leave (relative error 2^-17,
        // for any number of queries; the second one of a weight is never 0, so that an infinite value stays infinite)
#pragma unroll
        for (int u = 0; u < NS; ++u) {
            if constexpr (R::kB16) {
#pragma unroll
                for (int j = 0; j < 2; ++j) {
                    uintx4 x, y;
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        const float p0 = s[u][8 * j + 2 * i], p1 = s[u][8 * j + 2 * i + 1];
                        const unsigned int b0 = __float_as_uint(p0), b1 = __float_as_uint(p1);
                        x[i] = __builtin_amdgcn_perm(b1, b0, 0x07060302u);
                        const floatx2 rest = {fmaf(p0, 0x1p-40f, p0 - __uint_as_float(b0 & 0xffff0000u)),
                                              fmaf(p1, 0x1p-40f, p1 - __uint_as_float(b1 & 0xffff0000u))};
                        y[i] = __builtin_bit_cast(unsigned int, __builtin_convertvector(rest, bf16x2_tile));
                    }
#pragma unroll
                    for (int e = 0; e < EPN; ++e) {
                        typedef __attribute__((address_space(3))) shortx4* lds4;
                        const shortx4 v0 = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds4)(Vt + vo[e] + (32 * u + 16 * j) * ROWB));
                        const shortx4 v1 = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds4)(Vt + vo[e] + (32 * u + 16 * j + 8) * ROWB));
                        struct { shortx4 a, b; } both = {v0, v1};
                        const bf16x8_t vf = __builtin_bit_cast(bf16x8_t, both);
                        o[e] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(vf, __builtin_bit_cast(bf16x8_t, x), o[e], 0, 0, 0);
                        o[e] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(vf, __builtin_bit_cast(bf16x8_t, y), o[e], 0, 0, 0);
                    }
                }
            } else {
                typedef float vecf __attribute__((ext_vector_type(EPN)));
#pragma unroll
                for (int r = 0; r < 16; ++r) {
                    const vecf v = *reinterpret_cast<const vecf*>(Vt + vo[0] + (32 * u + tile_row(r, 0)) * ROWB);
#pragma unroll
                    for (int e = 0; e < EPN; ++e) o[e] = __builtin_amdgcn_mfma_f32_32x32x2f32(v[e], s[u][r], o[e], 0, 0, 0);
                }
            }
        }
    };

    auto barrier = [] {
        if constexpr (SOLO) asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
        else tile_barrier();
    };
    if (t0 < t1) {
        all_arrived_so_far();
        live0 = __ballot(w0 > 0.f);
        clear_dead(0, live0);
        barrier();
        // one tile: the next one is requested, this one multiplied, the next one awaited; true: this was the last one
        auto step = [&](auto buf_c, int t) {
            constexpr int BUF = decltype(buf_c)::value;
            const bool more = t + 1 < t1;
            if (t + 2 < t1) w2 = weight(t + 2);
            live1 = more ? __ballot(w1 > 0.f) : 0ull;
            if (BUFS == 2 && live1 != 0ull) fetch(t + 1, BUF ^ 1);
            if (has_rows)
                for (int i = 0; i < TIMES; ++i)
                    if ((live0 >> (32 * (ksub + i)) & (NS == 2 ? ~0ull : 0xffffffffull)) != 0ull) compute(buf_c, t, w0, i);
            if (!more) return true;
            if constexpr (BUFS == 1) {
                barrier();
                if (live1 != 0ull) fetch(t + 1, 0);
            }
            tile_arrived();
            clear_dead(BUFS == 2 ? BUF ^ 1 : 0, live1);
            barrier();
            w0 = w1; w1 = w2; live0 = live1;
            return false;
        };
        if constexpr (BUFS == 2) {
            for (int t = t0;; t += 2) {
                if (step(std::integral_constant<int, 0>{}, t)) break;
                if (step(std::integral_constant<int, 1>{}, t + 1)) break;
            }
        } else {
            for (int t = t0; !step(std::integral_constant<int, 0>{}, t); ++t) {}
        }
    }
    l = half_sum(l);

    // ---- wavefronts that share queries meet in LDS, register by register
    if constexpr (KW > 1) {
        constexpr int PER = 16 * EPN * 64 + 128;
        __syncthreads();
        float* all = reinterpret_cast<float*>(&lds.rows[0][0][0]);
        if (ksub == 1) {
            float* mine = all + qsub * PER;
#pragma unroll
            for (int e = 0; e < EPN; ++e)
#pragma unroll
                for (int r = 0; r < 16; ++r) mine[(16 * e + r) * 64 + lane] = o[e][r];
            mine[16 * EPN * 64 + lane] = m;
            mine[16 * EPN * 64 + 64 + lane] = l;
        }
        __syncthreads();
        if (ksub > 0) return;
        const float* other = all + qsub * PER;
        const float mo = other[16 * EPN * 64 + lane], lo = other[16 * EPN * 64 + 64 + lane];
        const float mn = fmaxf(m, mo), f0 = fast_exp2(m - mn), f1 = fast_exp2(mo - mn);
        m = mn;
        l = fmaf(l, f0, lo * f1);
#pragma unroll
        for (int e = 0; e < EPN; ++e)
#pragma unroll
            for (int r = 0; r < 16; ++r) o[e][r] = fmaf(o[e][r], f0, other[(16 * e + r) * 64 + lane] * f1);
    }
    if (row0 + n >= J.rows) return;

    // ---- store: a lane has four (fp32: EPN) consecutive columns at a time
    if (J.part) {
        float* dst = J.part + ((size_t)split * a.n_rows + q_row) * P;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            if constexpr (R::kB16) {
#pragma unroll
                for (int e = 0; e < EPN; ++e)
                    *reinterpret_cast<floatx4*>(dst + 32 * e + 8 * i + 4 * h) = floatx4{o[e][4 * i], o[e][4 * i + 1], o[e][4 * i + 2], o[e][4 * i + 3]};
            } else {
#pragma unroll
                for (int j = 0; j < 4; ++j)
#pragma unroll
                    for (int e = 0; e < EPN; e += 2)
                        *reinterpret_cast<floatx2*>(dst + EPN * tile_row(4 * i + j, h) + e) = floatx2{o[e][4 * i + j], o[e + 1][4 * i + j]};
            }
        }
        if (h == 0) *reinterpret_cast<floatx2*>(dst + D) = floatx2{m, l};
        return;
    }
    const float f = l != 0.f ? 1.f / l : 0.f;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        if constexpr (R::kB16) {
#pragma unroll
            for (int e = 0; e < EPN; ++e) {
                uint2 x;
                x.x = f32_to_bf16_bits(o[e][4 * i] * f) | (f32_to_bf16_bits(o[e][4 * i + 1] * f) << 16);
                x.y = f32_to_bf16_bits(o[e][4 * i + 2] * f) | (f32_to_bf16_bits(o[e][4 * i + 3] * f) << 16);
                *reinterpret_cast<uint2*>(a.out + ((size_t)q_row * D + 32 * e + 8 * i + 4 * h) * 2) = x;
            }
        } else {
#pragma unroll
            for (int j = 0; j < 4; ++j)
#pragma unroll
                for (int e = 0; e < EPN; e += 2)
                    *reinterpret_cast<floatx2*>(a.out + ((size_t)q_row * D + EPN * tile_row(4 * i + j, h) + e) * 4) =
                        floatx2{o[e][4 * i + j] * f, o[e + 1][4 * i + j] * f};
        }
    }
    if (h == 0) {
        if (a.lse) a.lse[q_row] = l != 0.f ? (m + __builtin_amdgcn_logf(l)) * 0.6931471805599453f : -INFINITY;
        if (a.stats) *reinterpret_cast<floatx2*>(a.stats + 2 * q_row) = l != 0.f ? floatx2{m, f} : floatx2{-kTileDead, 0.f};
    }
}

template <typename T, int D>
__global__ __launch_bounds__(kTileThreads, 2) void tile_kernel(const TileArgs a) {
    __shared__ TileLds<T, D> lds;
    // workgroup -> (job, cache, split, query tile); the query tiles of a split go to one XCD (blocks are dealt out to the eight
    // of them in turn), whose L2 then serves all but the first read of its rows
    unsigned int block = blockIdx.y * gridDim.x + blockIdx.x;
    const int which = block >= a.first ? 1 : 0;
    block -= which ? a.first : 0u;
    const TileJob J = which ? a.job[1] : a.job[0];
    const unsigned int units = (unsigned int)J.units, in_xcd = block >> 3;
    const unsigned int unit = J.by_xcd ? in_xcd / (unsigned int)J.n_qt * 8u + (block & 7u) : block % units;
    const unsigned int turn = J.by_xcd ? in_xcd % (unsigned int)J.n_qt : block / units;
    if (unit >= units || turn >= (unsigned int)J.n_qt) return;
    const int qt = J.n_qt - 1 - (int)turn;                                      // (causal: the longest first)
    const unsigned int splits = (unsigned int)J.splits;
    // (causal: the first splits have the most to do, and where 2, 4 or 8 of them divide the XCDs among themselves, they take turns)
    const int split = (int)((unit + (a.causal && 8u % splits == 0u ? unit >> 3 : 0u)) % splits);
    const int64_t stream = unit / splits;
    if (J.qw == 4) tile_body<T, D, 4>(a, J, stream, split, qt, lds);
    else if (J.qw == 2) tile_body<T, D, 2>(a, J, stream, split, qt, lds);
    else if (J.qw == 1) tile_body<T, D, 1>(a, J, stream, split, qt, lds);
    else tile_body<T, D, 0>(a, J, stream, split, qt, lds);
}

// Partial rows of all splits of a query -> its result.  D / 4 lanes a query, four columns each; SG groups of lanes take its splits in
// turn, so that many splits are not one trip to memory after the other, and meet in LDS (128 queries x 65 splits 8.9 -> 3.7 us).
constexpr int kTileMergeThreads = 256;
template <typename T, int D, int SG>
__device__ __forceinline__ void merge_rows(const TileArgs& a, const float* part, int splits, int64_t block, float* red /*[SG > 1 ? 2048 : 0]*/) {
    constexpr int P = D + kTilePad, LPR = D / 4, ROWS = kTileMergeThreads / LPR / SG, U = 4;
    const int lane = threadIdx.x % LPR, sg = threadIdx.x / LPR % SG;
    const int64_t row = block * ROWS + threadIdx.x / (LPR * SG);
    const bool there = row < a.n_rows;
    const int col = 4 * lane;
    if (a.causal) {                                                  // the splits that this query sees something of (job 0 alone; head by head in memory)
        const TileJob& J = a.job[0];
        const int64_t sees = a.visible + (int)((uint32_t)row % (uint32_t)J.rows % (uint32_t)J.q_inner);
        const int per = J.tiles_per_split * kTileKeys;
        splits = (int)min((int64_t)splits, max((int64_t)1, (min(sees, (int64_t)J.count) + per - 1) / per));
    }
    const float* src = part + (size_t)(there ? row : 0) * P;
    const size_t step = (size_t)a.n_rows * P;
    floatx4 acc = {0.f, 0.f, 0.f, 0.f};
    float m = kTileLow, l = 0.f;
    auto join = [&](float mo, float lo, const floatx4& x) {
        const float mn = fmaxf(m, mo), f0 = fast_exp2(m - mn), f1 = fast_exp2(mo - mn);
        m = mn;
        l = fmaf(l, f0, lo * f1);
#pragma unroll
        for (int e = 0; e < 4; ++e) acc[e] = fmaf(acc[e], f0, x[e] * f1);
    };
    for (int s0 = sg; s0 < splits; s0 += U * SG) {
        floatx2 ml[U];
        floatx4 x[U];
#pragma unroll
        for (int u = 0; u < U; ++u) {                                // (splits behind the last one: that one again)
            const float* p = src + (size_t)min(s0 + u * SG, splits - 1) * step;
            ml[u] = *reinterpret_cast<const floatx2*>(p + D);
            x[u] = *reinterpret_cast<const floatx4*>(p + col);
        }
#pragma unroll
        for (int u = 0; u < U; ++u)
            if (s0 + u * SG < splits) join(ml[u][0], ml[u][1], x[u]);
    }
    if constexpr (SG > 1) {
        float* mine = red + threadIdx.x * 8;
        *reinterpret_cast<floatx4*>(mine) = acc;
        *reinterpret_cast<floatx2*>(mine + 4) = floatx2{m, l};
        __syncthreads();
        if (sg != 0) return;
        for (int k = 1; k < SG; ++k) {
            const float* other = mine + k * LPR * 8;
            join(other[4], other[5], *reinterpret_cast<const floatx4*>(other));
        }
    }
    if (!there) return;
    const float f = l != 0.f ? 1.f / l : 0.f;
    if constexpr (sizeof(T) == 2) {
        uint2 x;
        x.x = f32_to_bf16_bits(acc[0] * f) | (f32_to_bf16_bits(acc[1] * f) << 16);
        x.y = f32_to_bf16_bits(acc[2] * f) | (f32_to_bf16_bits(acc[3] * f) << 16);
        *reinterpret_cast<uint2*>(a.out + ((size_t)row * D + col) * 2) = x;
    } else {
        *reinterpret_cast<floatx4*>(a.out + ((size_t)row * D + col) * 4) = acc * f;
    }
    if (col == 0) {
        if (a.lse) a.lse[row] = l != 0.f ? (m + __builtin_amdgcn_logf(l)) * 0.6931471805599453f : -INFINITY;
        if (a.stats) *reinterpret_cast<floatx2*>(a.stats + 2 * row) = l != 0.f ? floatx2{m, f} : floatx2{-kTileDead, 0.f};
    }
}

template <typename T, int D, int SG>
__global__ __launch_bounds__(kTileMergeThreads) void tile_merge_kernel(const TileArgs a, const float* part, int splits) {
    __shared__ __align__(16) float red[SG > 1 ? kTileMergeThreads * 8 : 8];
    merge_rows<T, D, SG>(a, part, splits, (int64_t)blockIdx.y * gridDim.x + blockIdx.x, red);
}

// ---------------------------------------------------------------------------------------------------------------------
constexpr int kTileTarget = 512;             // workgroups a launch is cut into where there are fewer: two per compute unit
constexpr int kTileFull = 256;               // ... one

static int tile_qw(int64_t rows) { return rows > 64 ? 4 : rows > 32 ? 2 : 1; }
static int64_t tile_units(int64_t n_streams, int64_t rows, int qw) { return n_streams * ((rows + 32 * qw - 1) / (32 * qw)); }

// Splits of a job of this shape at most (any token count; with fewer queries to a workgroup there are more workgroups, and fewer splits).
// Causal jobs in fp32 may be cut twice as fine, as about half of their workgroups have little or nothing to do (d = 128, us a call: 13 x 1959 x 1959
// 396 -> 295, 9 x 730 x 4 x 730 166 -> 134, 3 x 1235 x 4 x 1235 as long).  bf16, where a cut costs more of its work, mostly takes as long either way
// (8 x 687 x 8 x 687 48, 2118 x 8 x 2118, d = 64, 52; 3156 x 4 x 3156 63.5 -> 58).
static int64_t tile_target(int elem, bool causal) { return elem == 4 && causal ? 2 * kTileTarget : kTileTarget; }
int tile_most_splits(int64_t n_streams, int64_t rows, int elem, bool causal) {
    const int64_t wgs = tile_units(n_streams, rows, tile_qw(rows));
    return wgs > 0 ? (int)max((int64_t)1, tile_target(elem, causal) / wgs) : 1;
}

static bool tile_by_xcd(int64_t units) { return units % 8 == 0 || units >= 48; }

// Splits of a job with workgroups of 128 queries (bf16: of 64 too), at most `most`: the least of (rounds of workgroups, by the fullest XCD) x (tiles of a split and
// what a workgroup takes to begin and to end) + what the merge reads, in times of a tile; two workgroups of a compute unit side by side
// take 1.5 times (fp32 1.8, causal bf16, of different lengths, 1.3) what one does.  `seen`: tiles that a query sees on average.  The constants are
// fitted to such times.  As many splits as give two workgroups a compute unit (bf16, 128 queries: of at least eight tiles) / this, us a call, d = 128:
// fp32 13 x 1959 x 1959 324 / 293, bf16 8 x 8704 x 256 52.8 / 49.5, 106 prefixes x 487 tokens x 40 queries 22.2 / 18.2, 6 x 3004 x 96 23.2 / 21.5,
// equal within 2 %: 8 x 420 x 8 x 420, 8 x 4096 x 4 x 4096, 8 prefixes x 16385 x 1280, 106 x 199 x 200, 94 x 1543 x 34, 4 x 2616 x 75.  (Workgroups of 64 in fp32 lose:
// 8 x 200 x 1120 22.5 / 28.5.)
static int best_splits(int64_t n_streams, int n_qt, int tiles, int most, bool b16, bool causal, int seen) {
    const float side = !b16 ? 0.9f : causal ? 0.65f : 0.75f, ends = b16 ? 4.f : 1.f, merge = b16 ? 0.011f : 0.0025f;
    float least = 0.f;
    int best = 1;
    for (int k = 1; k <= most; k += most / 64 + 1) {
        const int per = (tiles + k - 1) / k, s = (tiles + per - 1) / per;
        const int64_t units = n_streams * s;
        const bool mixed = s % 8 != 0 && (8 % s != 0 || units >= 8 * s);          // every XCD has all splits, early ones and late ones
        const float share = causal && mixed ? fminf(1.f, ((float)seen / (float)per + 0.5f) / (float)s) : 1.f;
        const float in_xcd = (float)(tile_by_xcd(units) ? (units + 7) / 8 * n_qt : (units * n_qt + 7) / 8) * share;
        const float rounds = ceilf(in_xcd * (8.f / kTileFull));
        float cost = (rounds <= 1.f ? 1.f : side * rounds) * ((float)per + ends) + merge * (float)(units * n_qt);
        if (causal && s > 1) cost += ends;                                         // (the merge's launch; a prefix has one anyway)
        if (k == 1 || cost < least) { least = cost; best = s; }
    }
    return best;
}

// Queries of a workgroup and cuts of the keys.  Workgroups of 128 queries read the fewest keys; where they do not give every compute
// unit one even with the keys cut, smaller ones are taken.  taken: workgroups of the launch that others have; first: places that the first
// query of a causal job sees.
void tile_plan(TileJob& j, int row_bytes, int elem, bool causal, int64_t taken, int64_t first) {
    const int tiles = (j.count + kTileKeys - 1) / kTileKeys;
    const int seen = (int)(((max(min(first, (int64_t)j.count), (int64_t)0) + j.count) / 2 + kTileKeys - 1) / kTileKeys);     // tiles, on average
    for (j.qw = tile_qw(j.rows);; j.qw /= 2) {
        const int64_t wgs = tile_units(j.n_streams, j.rows, j.qw);
        j.n_qt = (j.rows + 32 * j.qw - 1) / (32 * j.qw);
        // (A few others that the chip has no place for beside these cost a second round, so they are taken off: 8 x 64 tiles beside 32 workgroups
        // may then be cut into 60, which whole tiles make 32 of two.  512 + 32 workgroups, two a compute unit, 11.6 us, 256 + 32 8.2.  Many
        // others are the launch's work themselves.)
        int64_t splits = (tile_target(elem, causal) - (taken <= kTileTarget / 8 ? taken : 0)) / wgs;
        splits = max((int64_t)1, min(splits, (int64_t)tiles));
        if ((j.qw == 4 || (j.qw == 2 && elem == 2)) && tiles > 1) splits = best_splits(j.n_streams, j.n_qt, tiles, (int)splits, elem == 2, causal, seen);
        j.tiles_per_split = (int)((tiles + splits - 1) / splits);
        j.splits = j.tiles_per_split > 0 ? (tiles + j.tiles_per_split - 1) / j.tiles_per_split : 1;
        if (j.qw == 1 || wgs * j.splits >= kTileFull * 3 / 4) break;
    }
    // XCDs take the query tiles of a split each where that gives them equal shares, else whatever comes next
    j.units = j.n_streams * j.splits;
    // More short sequences of at most 32 queries than a round of workgroups has places: a wavefront each, which waits for nobody (call
    // times, a workgroup each beside: 7232 x 3 keys on 113 prefixes x 195 bf16 81 -> 35 us; 4096 x 60 keys bf16 56 -> 34, fp32 111 -> 87,
    // x 250 fp32 348 -> 296, bf16 123 -> 115; but 320 x 250 16.4 -> 20.9, the chip half empty and the keys one after the other).
    if (j.rows <= 32 && j.n_streams > kTileTarget / 2 && j.count <= (j.n_streams >= 2 * kTileTarget ? 256 : 128)) {
        const int per = row_bytes == 512 ? 2 : 4;
        j.qw = 0; j.n_qt = 1; j.splits = 1; j.tiles_per_split = 8;             // (tiles of 32 keys)
        j.units = (j.n_streams + per - 1) / per;
    }
    j.by_xcd = tile_by_xcd(j.units);
}

size_t tile_part_bytes(int d, int64_t n_rows, int splits) { return (size_t)n_rows * splits * (d + kTilePad) * sizeof(float); }

template <typename T, int D>
static hipError_t launch_tiles_t(TileArgs& a, int n_jobs, float* part, hipStream_t st) {
    int splits = 0;
    uint64_t blocks = 0, units = 0;
    for (int k = 0; k < n_jobs; ++k) {
        TileJob& j = a.job[k];
        if (k == 1) a.first = (uint32_t)blocks;
        const uint64_t own = (uint64_t)j.units;
        blocks += j.by_xcd ? (own + 7) / 8 * 8 * j.n_qt : (own * j.n_qt + 7) / 8 * 8;
        units += (uint64_t)j.n_streams * j.count;
        splits += j.splits;
    }
    if (n_jobs == 1) a.first = 0xffffffffu;
    if (blocks >= (uint64_t)1 << 31) return hipErrorInvalidValue;
    int at = 0;
    for (int k = 0; k < n_jobs; ++k) {
        a.job[k].part = splits > 1 ? part + (size_t)at * a.n_rows * (D + kTilePad) : nullptr;
        at += a.job[k].splits;
    }
    // (two dimensions: a grid may not exceed 2^32 threads in one of them)
    const uint32_t gx = blocks > 65536 ? 65536u : (uint32_t)blocks;
    hipError_t e = launch_timed(kProfAttend, (int64_t)units, tile_kernel<T, D>, dim3(gx, (uint32_t)((blocks + gx - 1) / gx)), dim3(kTileThreads), 0, st, a);
    if (e != hipSuccess) return e;
    if (splits == 1) return e;
    auto merge = [&](auto sg_c) {
        constexpr int SG = decltype(sg_c)::value, per = kTileMergeThreads / (D / 4) / SG;
        const uint64_t mb = ((uint64_t)a.n_rows + per - 1) / per;
        const uint32_t mx = mb > 65536 ? 65536u : (uint32_t)mb;
        return launch_timed(kProfAttendMerge, a.n_rows, tile_merge_kernel<T, D, SG>, dim3(mx, (uint32_t)((mb + mx - 1) / mx)), dim3(kTileMergeThreads), 0, st, a,
                            (const float*)part, splits);
    };
    // (eight groups a query only where the queries alone do not fill the chip: 10240 of them and 7 splits 7.3 us, in groups 11.4)
    return splits > 4 && a.n_rows <= 2048 ? merge(std::integral_constant<int, 8>{}) : merge(std::integral_constant<int, 1>{});
}

hipError_t launch_tiles(int dtype, int d, TileArgs& a, int n_jobs, float* part, hipStream_t st) {
    if (dtype == BKV_BF16 && d == 128) return launch_tiles_t<__bf16, 128>(a, n_jobs, part, st);
    if (dtype == BKV_BF16 && d == 64) return launch_tiles_t<__bf16, 64>(a, n_jobs, part, st);
    if (dtype == BKV_F32 && d == 128) return launch_tiles_t<float, 128>(a, n_jobs, part, st);
    if (dtype == BKV_F32 && d == 64) return launch_tiles_t<float, 64>(a, n_jobs, part, st);
    return hipErrorInvalidValue;
}

}  // namespace bkv
