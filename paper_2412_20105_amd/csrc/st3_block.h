// Shared by the calls for grouped heads: argument checks, the cache of 8-bit blocks as kernels see it, its quantiser.
#pragma once

#include "st3_mfma.h"

namespace st3 {

constexpr int kBlk = ST3_BLOCK_TOKENS;      // rows of a block
constexpr int kMostRows = 0x3fffffff;       // rows of a sequence: what is added to them on the way stays below 2^31

// The limits of a grid: y, and x in threads.
inline bool grid_fits(int64_t x, int threads, int64_t y) { return x * threads < (int64_t)1 << 32 && y <= 65535; }

inline st3_status check_gqa_shape(const st3_gqa_shape* s) {
    if (!s) return ST3_ERR_INVALID_ARG;
    if (s->batch <= 0 || s->heads <= 0 || s->kv_heads <= 0) return ST3_ERR_INVALID_ARG;
    if (s->dtype != ST3_F32 && s->dtype != ST3_BF16) return ST3_ERR_UNSUPPORTED;
    if (s->head_dim != 64 && s->head_dim != 128) return ST3_ERR_UNSUPPORTED;
    if (s->heads > 1024 || s->batch > 65535) return ST3_ERR_UNSUPPORTED;
    if (s->heads % s->kv_heads != 0) return ST3_ERR_INVALID_ARG;
    if (!(s->softmax_scale >= 0.0f)) return ST3_ERR_INVALID_ARG;
    return ST3_OK;
}

inline float gqa_scale_log2(const st3_gqa_shape* s) {
    const float sc = s->softmax_scale > 0.0f ? s->softmax_scale : 1.0f / sqrtf((float)s->head_dim);
    return sc * kLog2e;
}

// Rows of eb-byte elements: 16-byte aligned, no stride below a row (heads may lie outside rows: [H, T, d] seen as [T, H, d]).
inline st3_status check_rows(const st3_rows* r, int D, int eb) {
    if (!r || !r->data) return ST3_ERR_INVALID_ARG;
    if (r->stride_t < D || r->stride_h < D) return ST3_ERR_INVALID_ARG;
    if (!aligned16(r->data) || r->stride_t * eb % 16 != 0 || r->stride_h * eb % 16 != 0) return ST3_ERR_INVALID_ARG;
    return ST3_OK;
}

// Rows that are written, T of them: none lies on another.
inline st3_status check_output(const st3_rows* r, int heads, int64_t T, int D, int eb) {
    const st3_status s = check_rows(r, D, eb);
    if (s != ST3_OK) return s;
    if (T <= 1 || r->stride_t >= (heads - 1) * r->stride_h + D || r->stride_h >= (T - 1) * r->stride_t + D) return ST3_OK;
    for (int64_t h = 1; h < heads; ++h) {           // head h of a row and head 0 of one of the two nearest to it
        const int64_t at = h * r->stride_h, near = at / r->stride_t;
        if (near < T && at - near * r->stride_t < D) return ST3_ERR_INVALID_ARG;
        if (near + 1 < T && (near + 1) * r->stride_t - at < D) return ST3_ERR_INVALID_ARG;
    }
    return ST3_OK;
}

// Whether a row of x (D elements) meets a row of y (Dy of them, or as many).  Of tensors with equal strides it is told exactly (slices of one buffer may
// alternate); of others, all that lies between the first byte and the last counts.  Where there are several rows, strides of rows are a row long at least.
inline bool packed_rows_meet(const st3_rows* x, int hx, const st3_rows* y, int hy, int64_t T, int D, int eb, int Dy = -1) {
    const int64_t row = (int64_t)D * eb, row_y = Dy < 0 ? row : (int64_t)Dy * eb, d = (int64_t)(reinterpret_cast<intptr_t>(y->data) - reinterpret_cast<intptr_t>(x->data));
    auto extent = [&](const st3_rows* t, int h, int64_t last) { return ((h - 1) * t->stride_h + (T - 1) * t->stride_t) * eb + last; };
    if (d >= extent(x, hx, row) || -d >= extent(y, hy, row_y)) return false;
    // (one row of each, or one head: that stride says nothing, and may be 0)
    if ((T > 1 && x->stride_t != y->stride_t) || ((hx > 1 || hy > 1) && x->stride_h != y->stride_h)) return true;
    const int64_t sh = x->stride_h * eb, st = x->stride_t * eb;
    for (int64_t h = 1 - hx; h < hy; ++h) {
        // rows i of x and j of y begin gap + (j - i) * st apart; the two nearest values of j - i on either side of -gap / st
        const int64_t gap = d + h * sh, near = T > 1 ? -gap / st : 0;
        for (int64_t k = near - 1; k <= near + 1; ++k)
            if (k > -T && k < T && gap + k * st < row && -(gap + k * st) < row_y) return true;
    }
    return false;
}

inline st3_status check_block_cache(const st3_gqa_shape* s, const st3_block_cache* c) {
    if (!c || !c->k_codes || !c->v_codes || !c->k_scale || !c->v_scale || !c->k_tail || !c->v_tail || !c->table || !c->len) return ST3_ERR_INVALID_ARG;
    if (s->dtype != ST3_BF16) return ST3_ERR_UNSUPPORTED;
    if (c->code != ST3_BLOCK_INT8 && c->code != ST3_BLOCK_E4M3) return ST3_ERR_INVALID_ARG;
    if (c->n_pages <= 0 || c->table_blocks <= 0 || c->table_stride < c->table_blocks) return ST3_ERR_INVALID_ARG;
    if (!aligned16(c->k_codes) || !aligned16(c->v_codes) || !aligned16(c->k_tail) || !aligned16(c->v_tail)) return ST3_ERR_INVALID_ARG;
    return ST3_OK;
}

// The cache as kernels take it.
struct BlockPages {
    uint8_t* k_codes; uint8_t* v_codes;
    float* k_scale; float* v_scale;
    uint16_t* k_tail; uint16_t* v_tail;
    const int32_t* table; int64_t table_stride;
    const int32_t* len;
    int32_t table_blocks, n_pages;
};

inline BlockPages block_pages(const st3_block_cache* c) {
    return BlockPages{reinterpret_cast<uint8_t*>(c->k_codes), reinterpret_cast<uint8_t*>(c->v_codes), c->k_scale, c->v_scale,
                      reinterpret_cast<uint16_t*>(c->k_tail), reinterpret_cast<uint16_t*>(c->v_tail), c->table, c->table_stride, c->len,
                      c->table_blocks, c->n_pages};
}

#if defined(__HIPCC__)

// Inclusive sum over the wave's lanes (DPP: row_shr 1, 2, 4, 8, row_bcast 15, 31); the sum, and the largest of values that are not negative, the same
// in every lane.
__device__ __forceinline__ int wave_prefix(int x) {
    x += __builtin_amdgcn_update_dpp(0, x, 0x111, 0xf, 0xf, true);
    x += __builtin_amdgcn_update_dpp(0, x, 0x112, 0xf, 0xf, true);
    x += __builtin_amdgcn_update_dpp(0, x, 0x114, 0xf, 0xf, true);
    x += __builtin_amdgcn_update_dpp(0, x, 0x118, 0xf, 0xf, true);
    x += __builtin_amdgcn_update_dpp(0, x, 0x142, 0xa, 0xf, true);
    x += __builtin_amdgcn_update_dpp(0, x, 0x143, 0xc, 0xf, true);
    return x;
}
__device__ __forceinline__ int wave_total(int x) { return __builtin_amdgcn_readlane(wave_prefix(x), 63); }
__device__ __forceinline__ int wave_most(int x) {
    x = max(x, __builtin_amdgcn_update_dpp(0, x, 0x111, 0xf, 0xf, true));
    x = max(x, __builtin_amdgcn_update_dpp(0, x, 0x112, 0xf, 0xf, true));
    x = max(x, __builtin_amdgcn_update_dpp(0, x, 0x114, 0xf, 0xf, true));
    x = max(x, __builtin_amdgcn_update_dpp(0, x, 0x118, 0xf, 0xf, true));
    x = max(x, __builtin_amdgcn_update_dpp(0, x, 0x142, 0xa, 0xf, true));
    x = max(x, __builtin_amdgcn_update_dpp(0, x, 0x143, 0xc, 0xf, true));
    return __builtin_amdgcn_readlane(x, 63);
}

// Two float32 as two bf16, rounded to nearest even (NaN stays NaN).
__device__ __forceinline__ uint32_t bf16_pair(float lo, float hi) {
    const f32x2 v = {lo, hi};
    return __builtin_bit_cast(uint32_t, __builtin_convertvector(v, bf16x2));
}

// A block's K lies in a wave's own LDS, rows of D bytes, the 16-byte units of a row permuted: unit u of row r is at u ^ swz(r), so that the 16 rows
// that a fragment's lanes read (16 (c / 4) + c % 4 + 4 t) lie in 16 different units of the banks.
template <int D> struct KeyTile {
    static constexpr int UPR = D / 16, RPI = 1024 / D, NI = kBlk / RPI;     // units of a row; rows of a wave-wide load; loads of a block
    __device__ static __forceinline__ int swz(int row) { return D == 128 ? ((row >> 4 & 3) << 1 | (row >> 1 & 1)) : row >> 4 & 3; }
};

// Page of block j of sequence b; -1: there is none.
__device__ __forceinline__ int page_of(const BlockPages& c, int b, int j) {
    if (j >= c.table_blocks) return -1;
    const int p = c.table[b * c.table_stride + j];
    return p >= 0 && p < c.n_pages ? p : -1;
}

// x / scale, correctly rounded, for many x and one scale: two corrections of x * (1 / scale) by the remainder, which a fused multiply-add gives
// exactly (Markstein). That holds while nothing on the way leaves the normal range.  Else, and where a block holds what is not finite, x is divided
// with care first (`care`: the caller puts careful(x) in x's place): an infinity counts as the largest finite magnitude, and the quotients are then
// "divided" by one.
struct Divider {
    float by, inv, scale, top;
    bool care;
    __device__ __forceinline__ Divider(float s, float largest, bool all_finite) : scale(s), top(largest) {
        care = !(all_finite && s > 0x1p-60f && s < 0x1p60f);
        by = care ? 1.0f : s;
        inv = __fdiv_rn(1.0f, by);
    }
    // most: the largest code.  A scale of a few of the smallest float32 is rounded by so much that a quotient can pass it.
    __device__ __forceinline__ float careful(float x, float if_nan, float most) const {
        return !(x == x) ? if_nan : scale > 0.f ? fminf(fmaxf(__fdiv_rn(fminf(fmaxf(x, -top), top), scale), -most), most) : copysignf(0.f, x);
    }
    __device__ __forceinline__ float operator()(float x) const {
        float q = x * inv;                                  // (with the remainder's sign this way round zeros keep theirs)
        q = fmaf(-fmaf(q, by, -x), inv, q);
        return fmaf(-fmaf(q, by, -x), inv, q);
    }
};

// Magnitudes compare as integers: what is not finite is above all that is.
constexpr uint32_t kInfinity = 0x7f800000u;
__device__ __forceinline__ uint32_t magnitude(float x) { return __float_as_uint(x) & 0x7fffffffu; }

// The largest magnitude of a workgroup's values (`mine` of a thread's), as its bits; all threads call it and get it.  sm: a word for each wave.
template <int WAVES>
__device__ __forceinline__ uint32_t largest_of(uint32_t mine, uint32_t* sm, int tid) {
    mine = (uint32_t)wave_most((int)mine);
    if ((tid & 63) == 0) sm[tid >> 6] = mine;
    __syncthreads();
    uint32_t all = sm[0];
#pragma unroll
    for (int w = 1; w < WAVES; ++w) all = max(all, sm[w]);
    return all;
}

// The two formats.  code4: four quotients (of x[0..3], no larger than kMost by more than a rounding that its code takes back) as four
// bytes.
template <int CODE> struct BlockCode;
template <> struct BlockCode<ST3_BLOCK_INT8> {
    static constexpr float kMost = 127.0f, kUnit = 1.0f / kMost;
    __device__ static __forceinline__ float nan_code() { return 0.f; }
    __device__ static __forceinline__ uint32_t code4(const float* x, const Divider& d) {
        uint32_t u[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) u[i] = __float_as_uint(d(x[i]) + 12582912.0f);      // the sum's last bits are the integer nearest, ties to even
        const uint32_t lo = __builtin_amdgcn_perm(u[1], u[0], 0x0c0c0400u), hi = __builtin_amdgcn_perm(u[3], u[2], 0x04000c0cu);
        return lo | hi;
    }
    __device__ static __forceinline__ float value(uint32_t byte) { return (float)(int8_t)byte; }
    __device__ static __forceinline__ f32x4 value4(uint32_t w) {
        return f32x4{(float)(int8_t)w, (float)(int8_t)(w >> 8), (float)(int8_t)(w >> 16), (float)(int8_t)(w >> 24)};
    }
    // four codes as four bf16 (exact: at most seven bits)
    __device__ static __forceinline__ uint2 to_bf16(uint32_t w) {
        asm("" : "+v"(w));              // (opaque: else the bytes are taken apart where the word is loaded, and wait in four registers for one)
        const float f0 = (float)(int8_t)w, f1 = (float)(int8_t)(w >> 8), f2 = (float)(int8_t)(w >> 16), f3 = (float)(int8_t)(w >> 24);
        return make_uint2(__builtin_amdgcn_perm(__float_as_uint(f1), __float_as_uint(f0), 0x07060302u),
                          __builtin_amdgcn_perm(__float_as_uint(f3), __float_as_uint(f2), 0x07060302u));
    }
};
template <> struct BlockCode<ST3_BLOCK_E4M3> {
    static constexpr float kMost = 448.0f, kUnit = 1.0f / kMost;
    __device__ static __forceinline__ float nan_code() { return __uint_as_float(0x7fc00000u); }
    __device__ static __forceinline__ uint32_t code4(const float* x, const Divider& d) {
        uint32_t w = __builtin_amdgcn_cvt_pk_fp8_f32(d(x[0]), d(x[1]), 0, false);
        w = __builtin_amdgcn_cvt_pk_fp8_f32(d(x[2]), d(x[3]), w, true);
        return w;
    }
    __device__ static __forceinline__ float value(uint32_t byte) { return __builtin_amdgcn_cvt_f32_fp8((int)byte, 0); }
    __device__ static __forceinline__ f32x4 value4(uint32_t w) {
        const auto lo = __builtin_amdgcn_cvt_pk_f32_fp8(w, false), hi = __builtin_amdgcn_cvt_pk_f32_fp8(w, true);
        return f32x4{lo[0], lo[1], hi[0], hi[1]};
    }
    __device__ static __forceinline__ uint2 to_bf16(uint32_t w) {
        const bf16x2 lo = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w, 1.0f, false), hi = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w, 1.0f, true);
        return make_uint2(__builtin_bit_cast(uint32_t, lo), __builtin_bit_cast(uint32_t, hi));
    }
};

#endif  // __HIPCC__

}  // namespace st3
