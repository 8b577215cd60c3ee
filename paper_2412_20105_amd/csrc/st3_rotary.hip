// Rotary positions: a table of cosines and sines from positions with several axes, and rows turned by it.
#include "st3_block.h"
#include "st3_rotary.h"

namespace st3 {
namespace {

constexpr int kThreads = 256;

// ---------------------------------------------------------------------------------------------------------------------------------
// The table.  angle = position * inv_freq, exact as the sum of two float64; its distance r from the nearest multiple of pi/2 in
// float64 (pi/2 in two parts), then sin r and cos r from their series about 0, |r| <= pi/4, in float32.  A thread makes two pairs, 16 bytes,
// of one token, or of four from kManyVectors of them on, whose positions are on their way together.  Bound by the writes: 200000 tokens of 64 pairs 25.5 us,
// 4.0 TB/s (one token each 30.3), 50176 10.1 us with the launch (10.4); up to 20000 the host's 6.3 us.
// ---------------------------------------------------------------------------------------------------------------------------------
struct TableArgs {
    const float* inv_freq; const int32_t* positions; int64_t p_stride;
    float* table; int64_t t_stride;
    uint64_t axis[2];               // two bits for each pair
    int32_t total, pairs, per, rows;       // per: threads of a token; rows: tokens of a workgroup
};

__device__ __forceinline__ float2 cos_sin(int position, float freq) {
    constexpr double kHalfPi = 1.5707963267948966, kHalfPiRest = 6.123233995736766e-17, kPerHalfPi = 0.6366197723675814;
    constexpr double kWhole = 6755399441055744.0;           // 1.5 * 2^52: a sum's last bits are the integer nearest
    const double p = (double)position, f = (double)freq;
    const double angle = p * f, rest = __fma_rn(p, f, -angle);
    const double turns = __fma_rn(angle, kPerHalfPi, kWhole), n = turns - kWhole;
    const float r = (float)(__fma_rn(-n, kHalfPiRest, __fma_rn(-n, kHalfPi, angle)) + rest);
    const int quarter = (int)__double_as_longlong(turns) & 3;
    const float x = r * r;
    // r - r^3/3! + ... + r^9/9! and 1 - r^2/2! + ... - r^10/10!: the next terms are 2e-9 and 2e-10 at pi/4
    float s = fmaf(x, 2.7557319e-6f, -1.9841270e-4f);
    s = fmaf(x, s, 8.3333333e-3f);
    s = fmaf(x, s, -1.6666667e-1f);
    s = fmaf(x * r, s, r);
    float c = fmaf(x, -2.7557319e-7f, 2.4801587e-5f);
    c = fmaf(x, c, -1.3888889e-3f);
    c = fmaf(x, c, 4.1666667e-2f);
    c = fmaf(x, c, -0.5f);
    c = fmaf(x, c, 1.0f);
    const float a = quarter & 1 ? s : c, b = quarter & 1 ? c : s;
    return make_float2(quarter == 1 || quarter == 2 ? -a : a, quarter >= 2 ? -b : b);
}

constexpr int kManyVectors = 1 << 19;

template <int U>
__global__ __launch_bounds__(kThreads) void rotary_table_kernel(TableArgs a) {
    const int row = threadIdx.x / a.per, c = 2 * (threadIdx.x - row * a.per);
    const int64_t t0 = (int64_t)blockIdx.x * (U * a.rows) + row;
    if (row >= a.rows) return;
    const float2 f = *reinterpret_cast<const float2*>(a.inv_freq + c);
    const uint32_t axes = (uint32_t)(a.axis[c >> 5] >> (2 * (c & 31)));
    const int32_t* first = a.positions + (axes & 3) * a.p_stride;
    const int32_t* second = a.positions + (axes >> 2 & 3) * a.p_stride;
    int p[U], q[U];
#pragma unroll
    for (int i = 0; i < U; ++i) {
        const int64_t t = min(t0 + i * a.rows, (int64_t)a.total - 1);
        p[i] = first[t];
        q[i] = second[t];
    }
#pragma unroll
    for (int i = 0; i < U; ++i) {
        const int64_t t = t0 + i * a.rows;
        if (t >= a.total) return;
        const float2 x = cos_sin(p[i], f.x), y = cos_sin(q[i], f.y);
        *reinterpret_cast<float4*>(a.table + t * a.t_stride + 2 * c) = make_float4(x.x, x.y, y.x, y.y);
    }
}

// ---------------------------------------------------------------------------------------------------------------------------------
// Rows.  An item is two 16-byte vectors of a row that hold as many pairs (columns c .. and c + pairs .., or two vectors side by side), or two behind
// the columns that turn, which are copied.  A workgroup takes a few tokens, all heads.
// ---------------------------------------------------------------------------------------------------------------------------------
struct RotateArgs {
    const void* x; void* out;
    int64_t x_st, x_sh, o_st, o_sh;
    Rotation r;
    int32_t total, heads, tokens;          // tokens of a workgroup
    uint32_t items, per_token;             // items of a token; 2^32 / items, rounded up
    bool inverse, copies;
};

template <typename T, int D, bool ADJACENT>
__global__ __launch_bounds__(kThreads) void rotate_rows_kernel(RotateArgs a) {
    using E = ElemTraits<T>;
    constexpr int V = E::kPerVec, PER = D / (2 * V), U = 4;         // items of a row; items of a thread on their way at a time
    const int64_t t0 = (int64_t)blockIdx.x * a.tokens;
    const int n = (int)min((int64_t)a.tokens, a.total - t0) * (int)a.items;
    for (int e0 = threadIdx.x; e0 < n; e0 += U * kThreads) {
        uint4 x[U], y[U];
        int64_t to[U];
        const float* table[U];
        int u[U], second[U];
#pragma unroll
        for (int i = 0; i < U; ++i) {
            const int e = min(e0 + i * kThreads, n - 1), t = (int)__umulhi((uint32_t)e, a.per_token), left = e - t * (int)a.items, h = left / PER;
            u[i] = left % PER;
            const bool turns = u[i] < a.r.pairs / V;
            const int col = turns && !ADJACENT ? u[i] * V : u[i] * 2 * V;
            second[i] = turns && !ADJACENT ? a.r.pairs : V;
            const T* row = reinterpret_cast<const T*>(a.x) + (t0 + t) * a.x_st + h * a.x_sh + col;
            x[i] = *reinterpret_cast<const uint4*>(row);
            y[i] = *reinterpret_cast<const uint4*>(row + second[i]);
            to[i] = (t0 + t) * a.o_st + h * a.o_sh + col;
            table[i] = a.r.table + (t0 + t) * a.r.stride + 2 * V * (turns ? u[i] : 0);
        }
#pragma unroll
        for (int i = 0; i < U; ++i) {
            if (e0 + i * kThreads >= n) break;
            if (u[i] < a.r.pairs / V) {
                float p[V], q[V], cs[2 * V];
                E::unpack(x[i], p);
                E::unpack(y[i], q);
#pragma unroll
                for (int j = 0; j < V / 2; ++j) *reinterpret_cast<float4*>(cs + 4 * j) = reinterpret_cast<const float4*>(table[i])[j];
#pragma unroll
                for (int j = 0; j < V; ++j) {
                    const float c = cs[2 * j], s = a.inverse ? -cs[2 * j + 1] : cs[2 * j + 1];
                    if constexpr (ADJACENT) {
                        float* pair = j < V / 2 ? p + 2 * j : q + 2 * j - V;
                        turn(pair[0], pair[1], c, s);
                    } else {
                        turn(p[j], q[j], c, s);
                    }
                }
                x[i] = packed<T>(p);
                y[i] = packed<T>(q);
            } else if (!a.copies) {
                continue;
            }
            T* row = reinterpret_cast<T*>(a.out) + to[i];
            *reinterpret_cast<uint4*>(row) = x[i];
            *reinterpret_cast<uint4*>(row + second[i]) = y[i];
        }
    }
}

}  // namespace
}  // namespace st3

extern "C" st3_status st3_rotary_table(int32_t axes, int32_t pairs, const uint8_t* axis, const float* inv_freq, const int32_t* positions,
                                       int64_t position_stride, int32_t total, float* table, int64_t table_stride, void* stream) {
    using namespace st3;
    if (axes < 1 || pairs < 1 || total < 0) return ST3_ERR_INVALID_ARG;
    if (axes > 4 || pairs > 64 || pairs % 8 != 0) return ST3_ERR_UNSUPPORTED;
    TableArgs a{};
    for (int c = 0; c < pairs && axis; ++c) {
        if (axis[c] >= axes) return ST3_ERR_INVALID_ARG;
        a.axis[c >> 5] |= (uint64_t)axis[c] << (2 * (c & 31));
    }
    if (!inv_freq || (reinterpret_cast<uintptr_t>(inv_freq) & 7) != 0) return ST3_ERR_INVALID_ARG;
    if (total == 0) return ST3_OK;          // (an empty tensor may have no address)
    if (!positions || !table || !aligned16(table) || (axes > 1 && position_stride != 0 && position_stride < total)) return ST3_ERR_INVALID_ARG;
    if (table_stride % 4 != 0 || table_stride < 2 * pairs) return ST3_ERR_INVALID_ARG;
    a.inv_freq = inv_freq; a.positions = positions; a.p_stride = position_stride; a.table = table; a.t_stride = table_stride;
    a.total = total; a.pairs = pairs; a.per = pairs / 2; a.rows = kThreads / a.per;
    auto launch = [&](auto kernel, int tokens) {
        const int64_t groups = ((int64_t)total + tokens - 1) / tokens;
        if (!grid_fits(groups, kThreads, 1)) return ST3_ERR_UNSUPPORTED;
        kernel<<<(unsigned)groups, kThreads, 0, reinterpret_cast<hipStream_t>(stream)>>>(a);
        return check_launch();
    };
    return (int64_t)total * a.per >= kManyVectors ? launch(rotary_table_kernel<4>, 4 * a.rows) : launch(rotary_table_kernel<1>, a.rows);
}

extern "C" st3_status st3_rotate_rows(const st3_rows* x, const st3_rows* out, int32_t heads, int32_t total, int32_t head_dim, int32_t dtype,
                                      const st3_rotary* rotary, int32_t inverse, void* stream) {
    using namespace st3;
    if (heads < 1 || total < 0) return ST3_ERR_INVALID_ARG;
    if (dtype != ST3_F32 && dtype != ST3_BF16) return ST3_ERR_UNSUPPORTED;
    if ((head_dim != 64 && head_dim != 128) || heads > 1024) return ST3_ERR_UNSUPPORTED;
    if (total == 0) return ST3_OK;          // (an empty tensor may have no address)
    const int eb = elem_bytes(dtype);
    st3_status s = check_rows(x, head_dim, eb);
    if (s != ST3_OK || (s = check_output(out, heads, total, head_dim, eb)) != ST3_OK || (s = check_rotary(rotary, head_dim)) != ST3_OK) return s;
    const bool in_place = x->data == out->data && (total == 1 || x->stride_t == out->stride_t) && (heads == 1 || x->stride_h == out->stride_h);
    if (!in_place && packed_rows_meet(x, heads, out, heads, total, head_dim, eb)) return ST3_ERR_INVALID_ARG;
    if (table_meets(rotary, total, out, heads, head_dim, eb)) return ST3_ERR_INVALID_ARG;
    RotateArgs a{};
    a.x = x->data; a.out = out->data;
    a.x_st = x->stride_t; a.x_sh = x->stride_h; a.o_st = out->stride_t; a.o_sh = out->stride_h;
    a.r = rotation(rotary);
    a.total = total; a.heads = heads; a.inverse = inverse != 0; a.copies = !in_place;
    const int per = head_dim * eb / 32;
    a.items = (uint32_t)(heads * per);
    a.per_token = (uint32_t)((((uint64_t)1 << 32) + a.items - 1) / a.items);
    // tokens of a workgroup: about kItems items, where that leaves enough workgroups
    constexpr int kItems = 4 * kThreads, kGroups = 1024;
    int64_t tokens = (kItems + a.items - 1) / a.items;
    if (tokens * kGroups > total) tokens = total / kGroups;
    a.tokens = (int)(tokens < 1 ? 1 : tokens);
    const int64_t groups = ((int64_t)total + a.tokens - 1) / a.tokens;
    if (!grid_fits(groups, kThreads, 1)) return ST3_ERR_UNSUPPORTED;
    hipStream_t st = reinterpret_cast<hipStream_t>(stream);
    auto launch = [&](auto kernel) { kernel<<<(unsigned)groups, kThreads, 0, st>>>(a); };
    const bool adjacent = rotary->layout == ST3_ROTARY_ADJACENT;
    if (dtype == ST3_BF16) {
        if (head_dim == 128) adjacent ? launch(rotate_rows_kernel<bf16_t, 128, true>) : launch(rotate_rows_kernel<bf16_t, 128, false>);
        else adjacent ? launch(rotate_rows_kernel<bf16_t, 64, true>) : launch(rotate_rows_kernel<bf16_t, 64, false>);
    } else {
        if (head_dim == 128) adjacent ? launch(rotate_rows_kernel<float, 128, true>) : launch(rotate_rows_kernel<float, 128, false>);
        else adjacent ? launch(rotate_rows_kernel<float, 64, true>) : launch(rotate_rows_kernel<float, 64, false>);
    }
    return check_launch();
}
