// What the kernels on the MFMA units of gfx950 share: fragments, K and V tiles in LDS and their permutation, direct loads.
#pragma once

#include "st3_common.h"

#if defined(__HIPCC__)

namespace st3 {

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef float f32x2 __attribute__((ext_vector_type(2)));
typedef float f32x4_a4 __attribute__((ext_vector_type(4), aligned(4)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
typedef short i16x4 __attribute__((ext_vector_type(4)));

constexpr int kTileKeys = 64;        // keys per LDS tile where nothing else is asked for

// An LDS tile is BN rows of D elements, no padding.  The 64 banks are 256 bytes wide together, so
// RPB rows share one pass over the banks.  K rows are read 16 bytes per lane by lanes holding
// consecutive rows: unit u ^ ((r / RPB) % UPR) spreads 16 consecutive rows over all banks.  V rows
// are read by the transpose read, 32 lanes covering 8 consecutive rows x 32 bytes (2 units): the
// permutation 2 * ((r / RPB) % (UPR / 2)) puts the eight rows on disjoint eighths of the banks.
template <int D, int BN = kTileKeys> struct TileLayout {
    static constexpr int UPR = D / 8;                   // 16-byte units per row
    static constexpr int RPB = 256 / (2 * D);           // rows per 256 bytes: 1 or 2
    static constexpr int RPI = 1024 / (2 * D);          // rows per wave-wide direct load (1 KB): 4 or 8
    static constexpr int NI = BN / (RPI * 4);           // direct loads of K, and of V, per wave and tile
    static constexpr int TILE = BN * D;                // elements of one K (or V) tile
    __device__ static __forceinline__ int k_swz(int row) { return (row / RPB) & (UPR - 1); }
    __device__ static __forceinline__ int v_swz(int row) { return 2 * ((row / RPB) & (UPR / 2 - 1)); }
};

union Frag {
    bf16x8 v;
    u32x4 u4;
    uint32_t w[4];
    i16x4 h[2];
};

// One wave-wide direct load: every lane fetches the 16 bytes at base + lane_byte_off (global memory;
// the base is the same for all lanes and sits in scalar registers, the offset is 32 bits wide) and
// the wave's 64 x 16 bytes land at LDS byte address lds_byte_addr .. + 1023 in lane order (gfx950:
// global_load_lds_dwordx4, LDS base in M0).  Issued through inline assembly: the compiler treats the
// builtin form as an access that is outstanding on the LDS counter as well, and then makes every
// later wait for an LDS read a wait for ALL LDS reads in flight, which serialises the fragment
// reads of the whole tile.  What it does not know about is handled here: wait_direct_loads() before
// the barrier that publishes a buffer; M0 is declared clobbered; "memory" keeps LDS reads in place.
__device__ __forceinline__ void direct_load16(const uint16_t* base, uint32_t lane_byte_off, uint32_t lds_byte_addr) {
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, %2"
                 :
                 : "s"(lds_byte_addr), "v"(lane_byte_off), "s"(base)
                 : "memory", "m0");
}

// The same for data that is read once and should not displace what the caches hold.
__device__ __forceinline__ void direct_load16_stream(const uint8_t* base, uint32_t lane_byte_off, uint32_t lds_byte_addr) {
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, %2 nt"
                 :
                 : "s"(lds_byte_addr), "v"(lane_byte_off), "s"(base)
                 : "memory", "m0");
}

// A value that is the same in every lane, moved to scalar registers.
__device__ __forceinline__ const uint16_t* uniform_ptr(const uint16_t* p) {
    const uint64_t v = reinterpret_cast<uint64_t>(p);
    const uint32_t lo = __builtin_amdgcn_readfirstlane((uint32_t)v), hi = __builtin_amdgcn_readfirstlane((uint32_t)(v >> 32));
    return reinterpret_cast<const uint16_t*>(((uint64_t)hi << 32) | lo);
}

// LDS byte address of a __shared__ object.
__device__ __forceinline__ uint32_t lds_addr(const void* p) {
    return (uint32_t)reinterpret_cast<uintptr_t>((__attribute__((address_space(3))) const void*)p);
}

// Starts the direct loads of the K/V tile at key k0 into the buffer at LDS byte address `lds_buf` (K
// tile, then V tile).  Rows past n-1 are clamped: such keys lie above every valid query's diagonal
// and are masked there.  Every address read is a row of the caller's tensors; every LDS address
// written lies inside the buffer.
// Kp / Vp: row 0 of the strip (uniform).  k_lane / v_lane: byte offset of this lane's 16 bytes within
// the first 1 KB group of a tile at key 0 (row min(row0, n-1) and permuted unit folded in).
// Offsets from the strip's row 0 fit 32 bits (checked by the launcher).  wave_s: the wave's index, scalar.
template <int D, int BN = kTileKeys>
__device__ __forceinline__ void issue_tile(uint32_t lds_buf, const uint16_t* Kp, const uint16_t* Vp, uint32_t k_lane,
                                           uint32_t v_lane, int64_t k_st, int64_t v_st, int k0, int n, int lane, int wave,
                                           int wave_s) {
    using L = TileLayout<D, BN>;
    const int row0 = wave * L::RPI + lane / L::UPR;     // this lane's row in the wave's first group
    if (k0 + BN <= n) {                                // all rows of the tile exist: plain strides
#pragma unroll
        for (int i = 0; i < L::NI; ++i) {
            const uint32_t dst = lds_buf + (4 * i + wave_s) * 1024;    // which 1 KB of the tile this wave-wide load fills
            const int key = k0 + 4 * i * L::RPI;
            direct_load16(uniform_ptr(Kp + key * k_st), k_lane, dst);
            direct_load16(uniform_ptr(Vp + key * v_st), v_lane, dst + 2 * L::TILE);
        }
    } else {
        const uint16_t* Ku = uniform_ptr(Kp);
        const uint16_t* Vu = uniform_ptr(Vp);
#pragma unroll
        for (int i = 0; i < L::NI; ++i) {
            const uint32_t dst = lds_buf + (4 * i + wave_s) * 1024;
            const int key = max(0, min(k0 + 4 * i * L::RPI, n - 1 - row0));     // this lane's row, key + row0, stays <= n - 1
            direct_load16(Ku, k_lane + (uint32_t)key * (uint32_t)(2 * k_st), dst);
            direct_load16(Vu, v_lane + (uint32_t)key * (uint32_t)(2 * v_st), dst + 2 * L::TILE);
        }
    }
}

// All direct loads this wave has issued have landed in LDS (vmcnt(0); other counters untouched).
__device__ __forceinline__ void wait_direct_loads() { __builtin_amdgcn_s_waitcnt(0x0F70); }

// The same but for this wave's last N direct loads.
template <int N>
__device__ __forceinline__ void wait_direct_loads_but() {
    static_assert(N < 16, "the counter's low bits");
    __builtin_amdgcn_s_waitcnt(0x0F70 | N);
}

// LDS reads at a byte address: 16 bytes, and the transpose read (4 consecutive rows of one column; see the header comment for the lane map).
__device__ __forceinline__ u32x4 lds_read16(uint32_t at) { return *reinterpret_cast<__attribute__((address_space(3))) const u32x4*>(at); }
__device__ __forceinline__ i16x4 lds_read_tr(uint32_t at) {
    return __builtin_amdgcn_ds_read_tr16_b64_v4i16(reinterpret_cast<__attribute__((address_space(3))) i16x4*>(at));
}

// Where a lane finds its operands in a tile (byte offsets, fixed for the whole kernel).  K fragment s of row c: unit (4s + g) ^ k_swz(c),
// which is the first one's address ^ 64 s; transpose read of the 16 columns dt: row 4g + c/4, unit (2dt + (c%4)/2) ^ v_swz(row),
// half c%2: the first one's ^ 32 dt.  (g < 4 and (c%4)/2 < 2, so the + is an ^ too; tiles start at multiples of a row's bytes, so the ^ may
// come last: two registers, not twelve.)
template <int D>
struct LaneMap {
    uint32_t k, v;
    __device__ __forceinline__ void init(int c, int g) {
        using L = TileLayout<D>;
        k = (uint32_t)(2 * (c * D + (g ^ L::k_swz(c)) * 8));
        const int row = 4 * g + (c >> 2);
        v = (uint32_t)(2 * (row * D + (((c & 3) >> 1) ^ L::v_swz(row)) * 8 + 4 * (c & 1)));
    }
};

}  // namespace st3

#endif  // __HIPCC__
