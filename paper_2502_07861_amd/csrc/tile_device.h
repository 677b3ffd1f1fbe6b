// Building blocks of the kernels that take many queries against a cache (tiles.hip, mass.hip): rows of keys, values or queries in
// LDS, and the 32x32 matrix-core products between them.
//
// Layout of a product: lane = 32 h + n.  S^T = K Q^T (rows = keys, columns = queries): lane (n, h) brings bytes 32 c + 16 h .. of
// key row n and of query row n for piece c of a row, the same bytes on both sides, so the contraction meets every column once.
// The result's register r is key 8 (r / 4) + 4 h + r % 4 of query n.  O^T += V^T P takes P from where it is: product j of a step
// contracts the keys that registers 8 j .. 8 j + 7 (bf16; register j, fp32) of both halves hold, if lane (n, h) brings column n of
// exactly those value rows.  bf16: ds_read_b64_tr_b16 hands a lane one column of four consecutive rows; fp32: a lane reads EPN
// consecutive columns of a row, column EPN n + e is row n of product tile e.
#pragma once
#include "bkv_device.h"

namespace bkv {

constexpr float kTileDead = -1.0e30f;        // logit of a place without a token, or one that the query does not see
constexpr float kTileLow = -1.0e28f;         // running reference before the first live token: above every dead logit (scale >= 0.1)
constexpr float kTileSlack = 6.f;            // weights may exceed the running reference by 2^6 before it moves

typedef short shortx4 __attribute__((ext_vector_type(4)));
typedef __bf16 bf16x2_tile __attribute__((ext_vector_type(2)));

template <typename T, int D> struct TileRows {
    static constexpr bool kB16 = sizeof(T) == 2;
    static constexpr int kRowB = D * (int)sizeof(T);
    static constexpr int kSlots = kRowB / 16;             // 16-byte slots of a row
    static constexpr int kPieces = kRowB / 32;            // contraction pieces of a row
    static constexpr int kEpn = D / 32;                   // product tiles along the head dimension
    // Rows are whole multiples of half the LDS banks, so slot s of row r is stored at another place: 8 (or 16) rows read at one
    // slot, and 8 rows read at two neighbouring slots by the transposing read, then meet different banks.
    static __device__ __forceinline__ int key_slot(int r, int s) {
        if constexpr (kRowB == 128) return s ^ ((r >> 1) & 7);
        else return s ^ (r & 15);
    }
    static __device__ __forceinline__ int value_slot(int r, int s) {
        if constexpr (!kB16) return s;
        else if constexpr (kRowB == 128) return s ^ (((r >> 1) & 3) << 1);
        else return s ^ ((r & 7) << 1);
    }
};

// acc + one piece of rows a (rows of the result) and b (columns)
template <typename T>
__device__ __forceinline__ floatx16 tile_mma(const uintx4& a, const uintx4& b, floatx16 acc) {
    if constexpr (sizeof(T) == 2) {
        return __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8_t, a), __builtin_bit_cast(bf16x8_t, b), acc, 0, 0, 0);
    } else {
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const unsigned int ae = a[e], be = b[e];
            acc = __builtin_amdgcn_mfma_f32_32x32x2f32(__uint_as_float(ae), __uint_as_float(be), acc, 0, 0, 0);
        }
        return acc;
    }
}

__device__ __forceinline__ int tile_row(int r, int h) { return 8 * (r >> 2) + 4 * h + (r & 3); }

// (x of this half, x of the other half), the same pair in both
__device__ __forceinline__ float half_max(float x) { return xor_max<32>(x); }
__device__ __forceinline__ float half_sum(float x) { return xor_sum<32>(x); }

}  // namespace bkv
