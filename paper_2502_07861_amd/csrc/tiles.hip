// Attention of many queries against weighted caches: batches that share a prefix, observation windows, whole prompts.
//   z = sum_i w_i e^{<k_i,q>/sqrt d} v_i / sum_i w_i e^{<k_i,q>/sqrt d}
// over the tokens i of one or two caches, optionally only the first few of them per query (causal).
//
// A workgroup of four wavefronts takes 32, 64 or 128 queries of one cache against a range of its keys, 64 at a time: keys and
// values go through LDS once for all its queries, in two buffers, the next tile's loads are under way while the current one is
// multiplied.  A wavefront has 32 queries in registers; where the workgroup has fewer than 128, wavefronts share queries and
// split the keys of a tile.  Softmax weights stay in the lane that the next product wants them in (tile_device.h).
#include "bkv_device.h"
#include "bkv_host.h"
#include "tile_device.h"

namespace bkv {

constexpr int kTileKeys = 64;
constexpr int kTileThreads = 256;
constexpr int kTilePad = 4;                  // floats behind the D sums of a partial row: [0] reference exponent, [1] denominator

template <typename T, int D>
__global__ __launch_bounds__(kTileThreads, sizeof(T) == 2 ? 2 : 1) void tile_kernel(const TileArgs a) {
    using R = TileRows<T, D>;
    constexpr int ROWB = R::kRowB, SLOTS = R::kSlots, NP = kTileKeys * SLOTS / kTileThreads, EPN = R::kEpn, P = D + kTilePad;
    __shared__ __align__(16) char lds[2][2][kTileKeys * ROWB];         // [buffer][keys, values]
    __shared__ __align__(16) float bias[2][kTileKeys];

    const int tid = threadIdx.x, lane = tid & 63, n = lane & 31, h = lane >> 5;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);

    // workgroup -> (job, cache, split, query tile); the query tiles of a split go to one XCD (blocks are dealt out to the eight
    // of them in turn), whose L2 then serves all but the first read of its rows
    unsigned int block = blockIdx.y * gridDim.x + blockIdx.x;
    const int which = block >= a.first ? 1 : 0;
    block -= which ? a.first : 0u;
    const TileJob J = which ? a.job[1] : a.job[0];
    const unsigned int in_xcd = block >> 3;
    const unsigned int unit = in_xcd / (unsigned int)J.n_qt * 8u + (block & 7u);
    const int qt = J.n_qt - 1 - (int)(in_xcd % (unsigned int)J.n_qt);           // (causal: the longest first)
    if (unit >= (unsigned int)J.n_streams * (unsigned int)J.splits) return;
    const int split = (int)(unit % (unsigned int)J.splits);
    const int64_t stream = unit / (unsigned int)J.splits;

    const int qw = J.qw, kw = 4 / qw;
    const int qsub = wave & (qw - 1), ksub = wave / qw;
    const int row_first = qt * 32 * qw, row0 = row_first + 32 * qsub;
    const bool has_rows = row0 < J.rows;
    const int row = min(row0 + n, J.rows - 1);
    const int outer = row / J.inner;
    const int64_t q_row = stream * J.q_stream + (int64_t)outer * J.q_outer + (int64_t)(row - outer * J.inner) * J.q_inner;

    // keys of this workgroup
    const int tiles = (J.count + kTileKeys - 1) / kTileKeys;
    const int t0 = split * J.tiles_per_split;
    int t1 = min(tiles, t0 + J.tiles_per_split);
    int sees = J.count, sees_min = J.count;
    if (a.causal) {
        const int64_t v = a.visible + outer;
        sees = (int)min((int64_t)J.count, max((int64_t)0, v));
        const int row_last = min(row_first + 32 * qw, J.rows) - 1;
        const int most = (int)min((int64_t)J.count, max((int64_t)0, a.visible + row_last / J.inner));
        t1 = min(t1, (most + kTileKeys - 1) / kTileKeys);
        sees_min = (int)min((int64_t)J.count, max((int64_t)0, a.visible + min(row0, J.rows - 1) / J.inner));
    }

    const char* Kb = J.K + (size_t)stream * J.stride * ROWB;
    const char* Vb = J.V + (size_t)stream * J.stride * ROWB;
    const float* wb = J.w + (size_t)stream * J.stride;

    // a tile on its way: pieces tid + 256 i of its 64 rows
    uintx4 kreg[NP], vreg[NP];
    float wreg[NP], wkey = 0.f;
    auto load = [&](int t) {
#pragma unroll
        for (int i = 0; i < NP; ++i) {
            const int piece = tid + kTileThreads * i, r = piece / SLOTS, s = piece % SLOTS;
            const int key = t * kTileKeys + r, at = min(key, J.count - 1);
            const size_t off = (size_t)at * ROWB + s * 16;
            kreg[i] = *reinterpret_cast<const uintx4*>(Kb + off);
            vreg[i] = *reinterpret_cast<const uintx4*>(Vb + off);
            const float w = wb[at];
            wreg[i] = key < J.count ? w : 0.f;
        }
        if (tid < kTileKeys) {
            const int key = t * kTileKeys + tid;
            const float w = wb[min(key, J.count - 1)];
            wkey = key < J.count ? w : 0.f;
        }
    };
    auto store = [&](int buf) {
        bool dead = false;
#pragma unroll
        for (int i = 0; i < NP; ++i) dead |= !(wreg[i] > 0.f);
        if (__builtin_amdgcn_ballot_w64(dead) != 0ull) {              // (whatever an absent token's row holds)
#pragma unroll
            for (int i = 0; i < NP; ++i) {
                const unsigned int keep = wreg[i] > 0.f ? 0xffffffffu : 0u;
#pragma unroll
                for (int j = 0; j < 4; ++j) { kreg[i][j] &= keep; vreg[i][j] &= keep; }
            }
        }
#pragma unroll
        for (int i = 0; i < NP; ++i) {
            const int piece = tid + kTileThreads * i, r = piece / SLOTS, s = piece % SLOTS;
            *reinterpret_cast<uintx4*>(lds[buf][0] + r * ROWB + R::key_slot(r, s) * 16) = kreg[i];
            *reinterpret_cast<uintx4*>(lds[buf][1] + r * ROWB + R::value_slot(r, s) * 16) = vreg[i];
        }
        if (tid < kTileKeys) bias[buf][tid] = wkey > 0.f ? __builtin_amdgcn_logf(wkey) * a.inv_scale : kTileDead;
    };

    if (t0 < t1) load(t0);
    uintx4 qf[R::kPieces];
#pragma unroll
    for (int c = 0; c < R::kPieces; ++c) qf[c] = *reinterpret_cast<const uintx4*>(a.Q + (size_t)q_row * ROWB + 32 * c + 16 * h);

    float m = kTileLow, l = 0.f;
    floatx16 o[EPN];
#pragma unroll
    for (int e = 0; e < EPN; ++e)
#pragma unroll
        for (int r = 0; r < 16; ++r) o[e][r] = 0.f;

    auto compute = [&](int buf, int t) {
        const char* Kt = lds[buf][0];
        const char* Vt = lds[buf][1];
        for (int sub = ksub; sub < kTileKeys / 32; sub += kw) {
            const int k0 = t * kTileKeys + 32 * sub;
            // ---- logits, in units of 1 / scale
            floatx16 s;
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const floatx4 b = *reinterpret_cast<const floatx4*>(&bias[buf][32 * sub + 8 * i + 4 * h]);
#pragma unroll
                for (int j = 0; j < 4; ++j) s[4 * i + j] = b[j];
            }
            const int kr = 32 * sub + n;
            if constexpr (R::kB16) {
#pragma unroll
                for (int c = 0; c < R::kPieces; ++c) {
                    const uintx4 kf = *reinterpret_cast<const uintx4*>(Kt + kr * ROWB + R::key_slot(kr, 2 * c + h) * 16);
                    s = tile_mma<T>(kf, qf[c], s);
                }
            } else {
                // two chains, so that no sum is rounded more than d / 4 times at its full size
                floatx16 s1;
#pragma unroll
                for (int r = 0; r < 16; ++r) s1[r] = 0.f;
                floatx16 s0 = s1;
#pragma unroll
                for (int c = 0; c < R::kPieces; c += 2) {
                    const uintx4 ka = *reinterpret_cast<const uintx4*>(Kt + kr * ROWB + R::key_slot(kr, 2 * c + h) * 16);
                    const uintx4 kb = *reinterpret_cast<const uintx4*>(Kt + kr * ROWB + R::key_slot(kr, 2 * c + 2 + h) * 16);
                    s0 = tile_mma<T>(ka, qf[c], s0);
                    s1 = tile_mma<T>(kb, qf[c + 1], s1);
                }
                s = s + (s0 + s1);
            }
            if (a.causal && k0 + 32 > sees_min) {
#pragma unroll
                for (int r = 0; r < 16; ++r) s[r] = k0 + tile_row(r, h) < sees ? s[r] : kTileDead;
            }
            // ---- weights 2^(logit - m); m moves when a logit passes it by more than the slack
            float mx = s[0];
#pragma unroll
            for (int r = 1; r < 16; ++r) mx = fmaxf(mx, s[r]);
            mx *= a.scale_log2;
            if (__builtin_amdgcn_ballot_w64(mx > m + kTileSlack) != 0ull) {
                const float mnew = fmaxf(m, half_max(mx));
                const float sc = fast_exp2(m - mnew);
                m = mnew;
                l *= sc;
#pragma unroll
                for (int e = 0; e < EPN; ++e) o[e] *= sc;
            }
#pragma unroll
            for (int r = 0; r < 16; ++r) { s[r] = fast_exp2(fmaf(s[r], a.scale_log2, -m)); l += s[r]; }
            // ---- values
            if constexpr (R::kB16) {
                // two bf16 numbers for a weight, its upper bits and what they leave
                bf16x8_t hi[2], lo[2];
#pragma unroll
                for (int j = 0; j < 2; ++j) {
                    uintx4 x, y;
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        const float p0 = s[8 * j + 2 * i], p1 = s[8 * j + 2 * i + 1];
                        const unsigned int b0 = __float_as_uint(p0), b1 = __float_as_uint(p1);
                        x[i] = __builtin_amdgcn_perm(b1, b0, 0x07060302u);
                        const floatx2 rest = {p0 - __uint_as_float(b0 & 0xffff0000u), p1 - __uint_as_float(b1 & 0xffff0000u)};
                        y[i] = __builtin_bit_cast(unsigned int, __builtin_convertvector(rest, bf16x2_tile));
                    }
                    hi[j] = __builtin_bit_cast(bf16x8_t, x); lo[j] = __builtin_bit_cast(bf16x8_t, y);
                }
                const int i16 = lane & 15, half = (lane >> 4) & 1;
#pragma unroll
                for (int j = 0; j < 2; ++j)
#pragma unroll
                    for (int e = 0; e < EPN; ++e) {
                        const int r0 = 32 * sub + 16 * j + 4 * h + (i16 >> 2), r1 = r0 + 8, slot = 4 * e + 2 * half + ((i16 & 3) >> 1);
                        typedef __attribute__((address_space(3))) shortx4* lds4;
                        const shortx4 v0 = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds4)(Vt + r0 * ROWB + R::value_slot(r0, slot) * 16 + (i16 & 1) * 8));
                        const shortx4 v1 = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds4)(Vt + r1 * ROWB + R::value_slot(r1, slot) * 16 + (i16 & 1) * 8));
                        struct { shortx4 a, b; } both = {v0, v1};
                        const bf16x8_t vf = __builtin_bit_cast(bf16x8_t, both);
                        o[e] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(vf, hi[j], o[e], 0, 0, 0);
                        o[e] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(vf, lo[j], o[e], 0, 0, 0);
                    }
            } else {
                typedef float vecf __attribute__((ext_vector_type(EPN)));
#pragma unroll
                for (int r = 0; r < 16; ++r) {
                    const int vr = 32 * sub + tile_row(r, h);
                    const vecf v = *reinterpret_cast<const vecf*>(Vt + vr * ROWB + n * (EPN * 4));
#pragma unroll
                    for (int e = 0; e < EPN; ++e) o[e] = __builtin_amdgcn_mfma_f32_32x32x2f32(v[e], s[r], o[e], 0, 0, 0);
                }
            }
        }
    };

    if (t0 < t1) {
        store(0);
        __syncthreads();
        int buf = 0;
        for (int t = t0;; ++t) {
            const bool more = t + 1 < t1;
            if (more) load(t + 1);
            if (has_rows) compute(buf, t);
            if (!more) break;
            store(buf ^ 1);
            __syncthreads();
            buf ^= 1;
        }
    }
    l = half_sum(l);

    // ---- wavefronts that share queries meet in LDS, register by register
    if (kw > 1) {
        __syncthreads();
        float* mine = reinterpret_cast<float*>(&lds[0][0][0]) + (wave - qw) * (16 * EPN * 64 + 128);
        if (ksub > 0) {
#pragma unroll
            for (int e = 0; e < EPN; ++e)
#pragma unroll
                for (int r = 0; r < 16; ++r) mine[(16 * e + r) * 64 + lane] = o[e][r];
            mine[16 * EPN * 64 + lane] = m;
            mine[16 * EPN * 64 + 64 + lane] = l;
        }
        __syncthreads();
        if (ksub > 0) return;
        for (int k = 1; k < min(kw, kTileKeys / 32); ++k) {
            const float* other = reinterpret_cast<const float*>(&lds[0][0][0]) + (wave + (k - 1) * qw) * (16 * EPN * 64 + 128);
            const float mo = other[16 * EPN * 64 + lane], lo = other[16 * EPN * 64 + 64 + lane];
            const float mn = fmaxf(m, mo), f0 = fast_exp2(m - mn), f1 = fast_exp2(mo - mn);
            m = mn;
            l = fmaf(l, f0, lo * f1);
#pragma unroll
            for (int e = 0; e < EPN; ++e)
#pragma unroll
                for (int r = 0; r < 16; ++r) o[e][r] = fmaf(o[e][r], f0, other[(16 * e + r) * 64 + lane] * f1);
        }
    }
    if (!has_rows || row0 + n >= J.rows) return;

    // ---- store: a lane has four consecutive columns at a time
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

// Partial rows of all splits of a query -> its result.  D / 4 lanes a query, four columns each.
constexpr int kTileMergeThreads = 256;
template <typename T, int D>
__global__ __launch_bounds__(kTileMergeThreads) void tile_merge_kernel(const TileArgs a, const float* part, int splits) {
    constexpr int P = D + kTilePad, LPR = D / 4;
    const int64_t row = ((int64_t)blockIdx.y * gridDim.x + blockIdx.x) * (kTileMergeThreads / LPR) + threadIdx.x / LPR;
    if (row >= a.n_rows) return;
    const int col = 4 * (threadIdx.x % LPR);
    const float* src = part + (size_t)row * P;
    const size_t step = (size_t)a.n_rows * P;
    floatx4 acc = {0.f, 0.f, 0.f, 0.f};
    float m = kTileLow, l = 0.f;
#pragma unroll 4
    for (int s = 0; s < splits; ++s) {
        const floatx2 ml = *reinterpret_cast<const floatx2*>(src + s * step + D);
        const floatx4 x = *reinterpret_cast<const floatx4*>(src + s * step + col);
        const float mn = fmaxf(m, ml[0]), f0 = fast_exp2(m - mn), f1 = fast_exp2(ml[0] - mn);
        m = mn;
        l = fmaf(l, f0, ml[1] * f1);
#pragma unroll
        for (int e = 0; e < 4; ++e) acc[e] = fmaf(acc[e], f0, x[e] * f1);
    }
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

// ---------------------------------------------------------------------------------------------------------------------
constexpr int kTileTarget = 512;             // workgroups a launch is cut into where there are fewer: two per compute unit

static int tile_qw(int64_t rows) { return rows > 64 ? 4 : rows > 32 ? 2 : 1; }

// Splits of a job of this shape at most (any token count).
int tile_most_splits(int64_t n_streams, int64_t rows) {
    const int64_t wgs = n_streams * ((rows + 32 * tile_qw(rows) - 1) / (32 * tile_qw(rows)));
    return wgs > 0 ? (int)max((int64_t)1, kTileTarget / wgs) : 1;
}

void tile_plan(TileJob& j) {
    j.qw = tile_qw(j.rows);
    j.n_qt = (j.rows + 32 * j.qw - 1) / (32 * j.qw);
    const int tiles = (j.count + kTileKeys - 1) / kTileKeys;
    int splits = tile_most_splits(j.n_streams, j.rows);
    if (splits > tiles) splits = tiles;
    if (splits < 1) splits = 1;
    j.tiles_per_split = (tiles + splits - 1) / splits;
    j.splits = j.tiles_per_split > 0 ? (tiles + j.tiles_per_split - 1) / j.tiles_per_split : 1;
}

size_t tile_part_bytes(int d, int64_t n_rows, int splits) { return (size_t)n_rows * splits * (d + kTilePad) * sizeof(float); }

template <typename T, int D>
static hipError_t launch_tiles_t(TileArgs& a, int n_jobs, float* part, hipStream_t st) {
    int splits = 0;
    uint64_t blocks = 0, units = 0;
    for (int k = 0; k < n_jobs; ++k) {
        TileJob& j = a.job[k];
        if (k == 1) a.first = (uint32_t)blocks;
        blocks += ((uint64_t)j.n_streams * j.splits + 7) / 8 * 8 * j.n_qt;
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
    if (e != hipSuccess || splits == 1) return e;
    constexpr int per = kTileMergeThreads / (D / 4);
    const uint64_t mb = ((uint64_t)a.n_rows + per - 1) / per;
    const uint32_t mx = mb > 65536 ? 65536u : (uint32_t)mb;
    return launch_timed(kProfAttendMerge, a.n_rows, tile_merge_kernel<T, D>, dim3(mx, (uint32_t)((mb + mx - 1) / mx)), dim3(kTileMergeThreads), 0, st, a,
                        (const float*)part, splits);
}

hipError_t launch_tiles(int dtype, int d, TileArgs& a, int n_jobs, float* part, hipStream_t st) {
    if (dtype == BKV_BF16 && d == 128) return launch_tiles_t<__bf16, 128>(a, n_jobs, part, st);
    if (dtype == BKV_BF16 && d == 64) return launch_tiles_t<__bf16, 64>(a, n_jobs, part, st);
    if (dtype == BKV_F32 && d == 128) return launch_tiles_t<float, 128>(a, n_jobs, part, st);
    if (dtype == BKV_F32 && d == 64) return launch_tiles_t<float, 64>(a, n_jobs, part, st);
    return hipErrorInvalidValue;
}

}  // namespace bkv
