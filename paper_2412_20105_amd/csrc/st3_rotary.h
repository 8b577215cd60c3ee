// The rotation of rows by a table of cosines and sines, as kernels take it.
#pragma once

#include "st3_block.h"

namespace st3 {

struct Rotation {
    const float* table;     // null: none
    int64_t stride;
    int32_t pairs;
};

inline st3_status check_rotary(const st3_rotary* r, int D) {
    if (!r || !r->table || !aligned16(r->table) || r->pairs < 1) return ST3_ERR_INVALID_ARG;
    if (r->layout != ST3_ROTARY_HALVES && r->layout != ST3_ROTARY_ADJACENT) return ST3_ERR_INVALID_ARG;
    if (r->pairs % 8 != 0 || r->pairs > 64) return ST3_ERR_UNSUPPORTED;
    if (2 * r->pairs > D || r->stride_t % 4 != 0 || r->stride_t < 2 * r->pairs) return ST3_ERR_INVALID_ARG;
    return ST3_OK;
}

inline Rotation rotation(const st3_rotary* r) { return r ? Rotation{r->table, r->stride_t, r->pairs} : Rotation{nullptr, 0, 0}; }

// Whether a table of T rows meets what is written to `out`: all that lies between the first byte and the last counts.
inline bool table_meets(const st3_rotary* r, int64_t T, const st3_rows* out, int heads, int D, int eb) {
    const char* t = reinterpret_cast<const char*>(r->table);
    const char* o = reinterpret_cast<const char*>(out->data);
    const int64_t table = ((T - 1) * r->stride_t + 2 * r->pairs) * 4, rows = ((heads - 1) * out->stride_h + (T - 1) * out->stride_t + D) * eb;
    return t < o + rows && o < t + table;
}

#if defined(__HIPCC__)

// (a, b) turned: each product rounded by itself, so that the result does not hang on how a kernel is compiled.
__device__ __forceinline__ void turn(float& a, float& b, float c, float s) {
#pragma clang fp contract(off)
    const float ac = a * c, bs = b * s, bc = b * c, as = a * s;
    a = ac - bs;
    b = bc + as;
}

// A vector of 16 bytes from float32, rounded to nearest even.
template <typename T> __device__ __forceinline__ uint4 packed(const float* f);
template <> __device__ __forceinline__ uint4 packed<float>(const float* f) { return ElemTraits<float>::pack(f); }
template <> __device__ __forceinline__ uint4 packed<bf16_t>(const float* f) {
    return make_uint4(bf16_pair(f[0], f[1]), bf16_pair(f[2], f[3]), bf16_pair(f[4], f[5]), bf16_pair(f[6], f[7]));
}

#endif  // __HIPCC__

}  // namespace st3
