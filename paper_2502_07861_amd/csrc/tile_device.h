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
    // Rows are whole multiples of half the LDS banks, so slot s of row r is stored at another place: 16 rows read at one slot (keys), and
    // four rows read at four neighbouring slots by 32 lanes of the transposing read (values), then meet different banks.
    static __device__ __forceinline__ int key_slot(int r, int s) {
        if constexpr (kRowB == 128) return s ^ ((r >> 1) & 7);
        else return s ^ (r & 15);
    }
    static __device__ __forceinline__ int value_slot(int r, int s) {
        if constexpr (!kB16) return s;
        else if constexpr (kRowB == 128) return s ^ (((r >> 1) & 1) << 2);
        else return s ^ ((r & 3) << 2);
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

__device__ __forceinline__ float half_max(float x) { return xor_max<32>(x); }
__device__ __forceinline__ float half_sum(float x) { return xor_sum<32>(x); }

// ---- memory to LDS without registers: lane l's 16 bytes at base + off go to LDS address `to` + 16 l.  In assembly because the
// compiler waits for all of them before any LDS read that follows; tile_arrived() waits for this wavefront's own.
__device__ __forceinline__ unsigned int lds_address(const void* p) {
    return (unsigned int)(uintptr_t)(__attribute__((address_space(3))) const char*)p;
}
// m0 is written: declared, so that nothing behind takes it for what it was (the compiler sets it for each use of its own, and warns that
// it does not keep it across the statement, which nothing asks for).
#pragma clang diagnostic push
#pragma clang diagnostic ignored "-Winline-asm"
__device__ __forceinline__ void to_lds(const char* base, unsigned int off, unsigned int to) {
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, %2" ::"s"(to), "v"(off), "s"(base) : "memory", "m0");
}
#pragma clang diagnostic pop
__device__ __forceinline__ void tile_arrived() { asm volatile("s_waitcnt vmcnt(0)" ::: "memory"); }
// The same in the compiler's books too (which hold the loads it made itself): nothing behind it waits for those again.
__device__ __forceinline__ void all_arrived_so_far() {
    __builtin_amdgcn_s_waitcnt(0x0f70);          // vmcnt(0)
    tile_arrived();
}
// All wavefronts' LDS writes are done and seen: loads under way stay so (a __syncthreads would wait for them).
__device__ __forceinline__ void tile_barrier() {
    asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory");
}

// This lane's share of a tile of 64 rows: wavefront w of four brings rows 16 w .. 16 w + 15, step i of them RPS rows.
template <typename T, int D> struct TileFetch {
    using R = TileRows<T, D>;
    static constexpr int kRps = 64 / R::kSlots;                  // rows of a step
    static constexpr int kSteps = 16 / kRps;
    // row of step i within the wavefront's sixteen, and the slot of it that is stored where this lane writes
    static __device__ __forceinline__ int row(int i, int lane) { return kRps * i + lane / R::kSlots; }
};

}  // namespace bkv
