// Attention of single tokens over a cache of 8-bit blocks, with grouped heads, appended rows and accumulated weights.
//
// A workgroup of four waves takes a chunk of the blocks of one (sequence, key head); a wave takes a block of 64 keys at a time, with
// v_mfma_f32_16x16x32_bf16 (A: lane (c, g) holds A[c][8g..8g+7], B: B[8g..8g+7][c], C: C[4g..4g+3][c]); the group's query heads are the columns
// (up to 16; a larger group is several workgroups).  8-bit codes are at most 8 significant bits: exact in bf16, so the products are exact and the block's
// scale multiplies the finished sums.
//   S^T = K Q^T    product t of four: row 4g'+i of A is key 16 g' + 4 t + i, so that lane (c, g) of C ends with keys 16 g .. 16 g + 15 of query c.  A lane
//                  reads 16 codes of its row at once: columns 64 x + 16 g .. + 15, contraction steps 2 x and 2 x + 1.
//   O^T = V^T P^T  the lane's 16 keys are the contraction slots 8g..8g+7 of two steps: P^T is where S^T left it, and V^T, whose rows lie in memory, is
//                  read 16 codes at a time too.
// No value crosses lanes but the maximum.  Bound by memory: 256 bytes a key and key head at d = 128 against some 25 cycles of a SIMD.
#include <algorithm>

#include "st3_block.h"

namespace st3 {
namespace {

constexpr int kMaxChunks = 64;
constexpr int kCols = 16;               // query heads of a workgroup

struct BlockDecodeArgs {
    BlockPages c;
    const uint16_t* q; const uint16_t* k_new; const uint16_t* v_new; uint16_t* out;
    int64_t q_st, q_sh, k_st, k_sh, v_st, v_sh, o_st, o_sh;
    int32_t max_len, H, Hk, G, QG;      // QG: workgroups that share a key head's chunk
    int32_t chunk, nsplit;              // blocks of a chunk; chunks of the longest sequence
    float scale_l2;
    float* score; int64_t s_sb, s_sh;
    float* part_o;                      // [B][H][nsplit][D]
    float* part_ml;                     // [B][H][nsplit][2]
    float* logits;                      // [B][H][logit_stride], in the log2 domain
    int64_t logit_stride;
};


// Blocks that hold rows to attend (the last one may be the tail).
__device__ __forceinline__ int units_of(int n, bool fresh) { return n / kBlk + (n % kBlk + (fresh ? 1 : 0) > 0 ? 1 : 0); }

template <int D, int CODE>
__global__ __launch_bounds__(256, 2) void block_attend_kernel(BlockDecodeArgs a) {
    using F = BlockCode<CODE>;
    constexpr int KS = D / 32, DT = D / 16, KH = D / 64;    // contraction steps of S, row tiles of O, 16-byte pieces of a K row per lane
    __shared__ float sm_o[4][kCols][D + 4];
    __shared__ float sm_m[4][kCols], sm_l[4][kCols];
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), g = lane >> 4, c = lane & 15;
    const int kh = blockIdx.x / a.QG, q0 = (blockIdx.x % a.QG) * kCols, b = blockIdx.z, ch = blockIdx.y;
    const int nq = min(kCols, a.G - q0);                    // query heads of this workgroup
    const bool fresh = a.k_new != nullptr;
    const int n = min(a.c.len[b], a.max_len);
    const int units = n < 0 ? 0 : units_of(n, fresh), blocks = n / kBlk;
    if (ch > 0 && ch * a.chunk >= units) return;
    const int h0 = kh * a.G + q0, u_end = min(units, (ch + 1) * a.chunk);
    const int hq = h0 + min(c, nq - 1);                     // this lane's query head (columns past the last repeat it)
    Frag qf[KS];
    {
        const uint16_t* row = a.q + (int64_t)b * a.q_st + (int64_t)hq * a.q_sh;
#pragma unroll
        for (int s = 0; s < KS; ++s) qf[s].u4 = *reinterpret_cast<const u32x4*>(row + 64 * (s / 2) + 16 * g + 8 * (s & 1));
    }
    f32x4 o[DT];
#pragma unroll
    for (int dt = 0; dt < DT; ++dt) o[dt] = f32x4{0.f, 0.f, 0.f, 0.f};
    float m = -3.402823466e38f, l = 0.f;
    float* logit = a.score != nullptr && c < nq ? a.logits + ((int64_t)b * a.H + hq) * a.logit_stride : nullptr;

    // softmax of 64 keys (s[t][i]: key 16 g + 4 t + i, in the log2 domain) and the weights of V, times vs, as two bf16 terms
    auto weigh = [&](f32x4 (&s)[4], float vs, int u, Frag (&hi)[2], Frag (&lo)[2]) {
        if (logit != nullptr) {
#pragma unroll
            for (int t = 0; t < 4; ++t) *reinterpret_cast<f32x4*>(logit + u * kBlk + 16 * g + 4 * t) = s[t];
        }
        float mx = -INFINITY;
#pragma unroll
        for (int t = 0; t < 4; ++t) mx = fmaxf(mx, fmaxf(fmaxf(s[t][0], s[t][1]), fmaxf(s[t][2], s[t][3])));
        constexpr float kLazy = 8.0f;
        if (__any(mx - m > kLazy)) {
            const float cand = fmaxf(m, wave_max_from<16>(mx));
            const float m_new = cand - m > kLazy ? cand : m;
            const float alpha = exp2_fast(m - m_new);
            m = m_new;
            l *= alpha;
#pragma unroll
            for (int dt = 0; dt < DT; ++dt) o[dt] *= alpha;
        }
#pragma unroll
        for (int t = 0; t < 4; ++t)
#pragma unroll
            for (int j = 0; j < 2; ++j) {
                const float p0 = exp2_fast(s[t][2 * j] - m), p1 = exp2_fast(s[t][2 * j + 1] - m);
                l += p0 + p1;
                const float w0 = p0 * vs, w1 = p1 * vs;
                const uint32_t b0 = __float_as_uint(w0), b1 = __float_as_uint(w1);
                hi[t / 2].w[2 * (t & 1) + j] = __builtin_amdgcn_perm(b1, b0, 0x07060302u);
                const f32x2 rest = {w0 - __uint_as_float(b0 & 0xffff0000u), w1 - __uint_as_float(b1 & 0xffff0000u)};
                lo[t / 2].w[2 * (t & 1) + j] = __builtin_bit_cast(uint32_t, __builtin_convertvector(rest, bf16x2));
            }
    };
    const int krow = 16 * (c >> 2) + (c & 3);               // + 4 t: the key of row c of product t
    for (int u = ch * a.chunk + wave; u < min(u_end, blocks); u += 4) {
        const int page = page_of(a.c, b, u);
        if (page < 0) {                                     // (whatever lies elsewhere is not read)
            if (logit != nullptr) {
#pragma unroll
                for (int t = 0; t < 4; ++t) *reinterpret_cast<f32x4*>(logit + u * kBlk + 16 * g + 4 * t) = f32x4{-INFINITY, -INFINITY, -INFINITY, -INFINITY};
            }
            continue;
        }
        const int64_t at = (int64_t)page * a.Hk + kh;
        const uint8_t* kp = a.c.k_codes + at * kBlk * D;
        const uint8_t* vp = a.c.v_codes + at * kBlk * D;
        const float ks = a.c.k_scale[at] * a.scale_l2, vs = a.c.v_scale[at];
        uint4 kr[4][KH], vr[DT];
#pragma unroll
        for (int t = 0; t < 4; ++t)
#pragma unroll
            for (int x = 0; x < KH; ++x) kr[t][x] = *reinterpret_cast<const uint4*>(kp + (krow + 4 * t) * D + 64 * x + 16 * g);
#pragma unroll
        for (int dt = 0; dt < DT; ++dt) vr[dt] = *reinterpret_cast<const uint4*>(vp + (16 * dt + c) * kBlk + 16 * g);
        f32x4 s[4];
#pragma unroll
        for (int t = 0; t < 4; ++t) {
            s[t] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int x = 0; x < KH; ++x) {
                const uint2 w0 = F::to_bf16(kr[t][x].x), w1 = F::to_bf16(kr[t][x].y), w2 = F::to_bf16(kr[t][x].z), w3 = F::to_bf16(kr[t][x].w);
                Frag f0, f1;
                f0.u4 = u32x4{w0.x, w0.y, w1.x, w1.y};
                f1.u4 = u32x4{w2.x, w2.y, w3.x, w3.y};
                s[t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(f0.v, qf[2 * x].v, s[t], 0, 0, 0);
                s[t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(f1.v, qf[2 * x + 1].v, s[t], 0, 0, 0);
            }
            s[t] *= ks;
        }
        Frag hi[2], lo[2];
        weigh(s, vs, u, hi, lo);
#pragma unroll
        for (int dt = 0; dt < DT; ++dt) {
            const uint2 w0 = F::to_bf16(vr[dt].x), w1 = F::to_bf16(vr[dt].y), w2 = F::to_bf16(vr[dt].z), w3 = F::to_bf16(vr[dt].w);
            Frag f[2];
            f[0].u4 = u32x4{w0.x, w0.y, w1.x, w1.y};
            f[1].u4 = u32x4{w2.x, w2.y, w3.x, w3.y};
#pragma unroll
            for (int x = 0; x < 2; ++x) {
                o[dt] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(f[x].v, hi[x].v, o[dt], 0, 0, 0);
                o[dt] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(f[x].v, lo[x].v, o[dt], 0, 0, 0);
            }
        }
    }
    // ---- the rows in 16 bits, and the new one ------------------------------------------------------------------------------------
    if (units > blocks && blocks >= ch * a.chunk && blocks < u_end && (blocks - ch * a.chunk) % 4 == wave) {
        const int r = n % kBlk;                             // rows in the tail; the new row's place
        const int64_t at = ((int64_t)b * a.Hk + kh) * kBlk * D;
        const uint16_t* kt = a.c.k_tail + at;
        const uint16_t* vt = a.c.v_tail + at;
        const uint16_t* kn = fresh ? a.k_new + (int64_t)b * a.k_st + (int64_t)kh * a.k_sh : nullptr;
        const uint16_t* vn = fresh ? a.v_new + (int64_t)b * a.v_st + (int64_t)kh * a.v_sh : nullptr;
        f32x4 s[4];
#pragma unroll
        for (int t = 0; t < 4; ++t) {
            const int key = krow + 4 * t;
            const uint16_t* row = fresh && key == r ? kn : kt + key * D;
            s[t] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int i = 0; i < KS; ++i) {
                Frag f;
                f.u4 = *reinterpret_cast<const u32x4*>(row + 64 * (i / 2) + 16 * g + 8 * (i & 1));
                s[t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(f.v, qf[i].v, s[t], 0, 0, 0);
            }
            s[t] *= a.scale_l2;
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const int key_c = 16 * g + 4 * t + i;
                if (key_c > r || (key_c == r && !fresh)) s[t][i] = -INFINITY;       // whatever lies there
            }
        }
        Frag hi[2], lo[2];
        weigh(s, 1.0f, blocks, hi, lo);
#pragma unroll
        for (int dt = 0; dt < DT; ++dt) {
            const uint32_t fresh_v = fresh ? vn[16 * dt + c] : 0u;
#pragma unroll
            for (int x = 0; x < 2; ++x) {
                Frag f;
                f.u4 = *reinterpret_cast<const u32x4*>(vt + (16 * dt + c) * kBlk + 16 * g + 8 * x);
#pragma unroll
                for (int i = 0; i < 8; ++i) {               // rows that hold nothing weigh nothing, whatever their bits are
                    const int key = 16 * g + 8 * x + i;
                    const uint32_t keep = i & 1 ? 0x0000ffffu : 0xffff0000u;
                    if (key >= r) f.w[i / 2] = (f.w[i / 2] & keep) | (key == r ? fresh_v << (16 * (i & 1)) : 0u);
                }
                o[dt] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(f.v, hi[x].v, o[dt], 0, 0, 0);
                o[dt] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(f.v, lo[x].v, o[dt], 0, 0, 0);
            }
        }
        if (fresh && q0 == 0) {
            for (int e = lane; e < D; e += kWave) {
                a.c.k_tail[at + r * D + e] = kn[e];
                a.c.v_tail[at + e * kBlk + r] = vn[e];
            }
        }
    }
    // ---- the four waves' parts ----------------------------------------------------------------------------------------------------
    l = wave_sum_from<16>(l);
    if (g == 0) { sm_m[wave][c] = m; sm_l[wave][c] = l; }
#pragma unroll
    for (int dt = 0; dt < DT; ++dt) *reinterpret_cast<f32x4*>(&sm_o[wave][c][16 * dt + 4 * g]) = o[dt];
    __syncthreads();
    for (int e = tid; e < nq * D; e += 256) {
        const int col = e / D, dim = e % D;
        float top = sm_m[0][col];
#pragma unroll
        for (int w = 1; w < 4; ++w) top = fmaxf(top, sm_m[w][col]);
        float sum = 0.f, x = 0.f;
#pragma unroll
        for (int w = 0; w < 4; ++w) {
            const float f = exp2_fast(sm_m[w][col] - top);
            sum = fmaf(sm_l[w][col], f, sum);
            x = fmaf(sm_o[w][col][dim], f, x);
        }
        const int64_t part = ((int64_t)b * a.H + h0 + col) * a.nsplit + ch;
        a.part_o[part * D + dim] = x;
        if (dim == 0) { a.part_ml[2 * part] = top; a.part_ml[2 * part + 1] = sum; }
    }
}

// Maximum and sum of a head over its chunks.
__device__ __forceinline__ float2 head_sum(const BlockDecodeArgs& a, int64_t part, int chunks) {
    float top = a.part_ml[2 * part], sum = 0.f;
    for (int i = 1; i < chunks; ++i) top = fmaxf(top, a.part_ml[2 * (part + i)]);
    for (int i = 0; i < chunks; ++i) sum = fmaf(a.part_ml[2 * (part + i) + 1], exp2_fast(a.part_ml[2 * (part + i)] - top), sum);
    return make_float2(top, sum > 0.f ? 1.0f / sum : 0.f);
}

// Behind the attention: workgroups [0, H) merge a head's chunks, the next Hk code a block that is whole now, the rest add 256 keys' weights.
template <int D, int CODE>
__global__ __launch_bounds__(256) void block_finish_kernel(BlockDecodeArgs a) {
    using F = BlockCode<CODE>;
    const int tid = threadIdx.x, b = blockIdx.y;
    const bool fresh = a.k_new != nullptr;
    const int n = min(a.c.len[b], a.max_len);
    const int units = n < 0 ? 0 : units_of(n, fresh), chunks = max(1, (units + a.chunk - 1) / a.chunk);
    int x = blockIdx.x;
    if (x < a.H) {
        const int64_t part = ((int64_t)b * a.H + x) * a.nsplit;
        const float2 hs = head_sum(a, part, chunks);
        for (int e = tid; e < D; e += 256) {
            float v = 0.f;
            for (int i = 0; i < chunks; ++i) v = fmaf(a.part_o[(part + i) * D + e], exp2_fast(a.part_ml[2 * (part + i)] - hs.x), v);
            a.out[(int64_t)b * a.o_st + (int64_t)x * a.o_sh + e] = (uint16_t)f32_to_bf16_bits(v * hs.y);
        }
        return;
    }
    x -= a.H;
    if (x < a.Hk) {
        if (!fresh || n < 0 || n % kBlk != kBlk - 1) return;
        const int page = page_of(a.c, b, n / kBlk);
        if (page < 0) return;
        __shared__ float sm[4];
        const int64_t at = (int64_t)page * a.Hk + x, tail = ((int64_t)b * a.Hk + x) * kBlk * D;
        for (int which = 0; which < 2; ++which) {
            const uint16_t* src = (which ? a.c.v_tail : a.c.k_tail) + tail;     // (codes lie in the tails' own order)
            uint8_t* dst = (which ? a.c.v_codes : a.c.k_codes) + at * kBlk * D;
            float mx = 0.f;
            for (int e = tid; e < kBlk * D; e += 256) mx = fmaxf(mx, finite_abs(__uint_as_float((uint32_t)src[e] << 16)));
            mx = wave_max_from<1>(mx);
            __syncthreads();
            if ((tid & 63) == 0) sm[tid >> 6] = mx;
            __syncthreads();
            const float scale = fmaxf(fmaxf(sm[0], sm[1]), fmaxf(sm[2], sm[3])) * F::kUnit;
            for (int e = tid; e < kBlk * D; e += 256) dst[e] = (uint8_t)F::code(__uint_as_float((uint32_t)src[e] << 16), scale);
            if (tid == 0) (which ? a.c.v_scale : a.c.k_scale)[at] = scale;
        }
        return;
    }
    x -= a.Hk;
    if (a.score == nullptr || n < 0) return;
    const int kh = x % a.Hk, key = x / a.Hk * 256 + tid, rows = n + (fresh ? 1 : 0);
    if (x / a.Hk * 256 >= rows) return;
    float w = 0.f;
    for (int h = kh * a.G; h < (kh + 1) * a.G; ++h) {
        const float2 hs = head_sum(a, ((int64_t)b * a.H + h) * a.nsplit, chunks);
        if (key < rows) w = fmaf(exp2_fast(a.logits[((int64_t)b * a.H + h) * a.logit_stride + key] - hs.x), hs.y, w);
    }
    if (key < rows) {
        float* s = a.score + b * a.s_sb + kh * a.s_sh + key;
        *s = key < n ? *s + w : w;
    }
}

struct BlockWs { size_t part_o, part_ml, logits, total; int64_t logit_stride; int chunk, nsplit; };

// Chunks: enough workgroups to fill the card, no more than kMaxChunks a sequence.
inline BlockWs block_ws(const st3_gqa_shape* s, int max_len) {
    const int G = s->heads / s->kv_heads, QG = (G + kCols - 1) / kCols;
    const int64_t units = max_len / kBlk + 1, strips = (int64_t)s->batch * s->kv_heads * QG;
    int64_t chunk = std::max<int64_t>(4, (units * strips + 511) / 512);
    chunk = std::max(chunk, (units + kMaxChunks - 1) / kMaxChunks);
    BlockWs w{};
    w.chunk = (int)chunk;
    w.nsplit = (int)((units + chunk - 1) / chunk);
    w.logit_stride = units * kBlk;
    const size_t BH = (size_t)s->batch * s->heads;
    size_t off = 0;
    w.part_o = off;  off = align_up(off + BH * w.nsplit * s->head_dim * sizeof(float), 256);
    w.part_ml = off; off = align_up(off + BH * w.nsplit * 2 * sizeof(float), 256);
    w.logits = off;  off = align_up(off + BH * w.logit_stride * sizeof(float), 256);
    w.total = off;
    return w;
}

template <int D, int CODE>
void launch_decode(const BlockDecodeArgs& a, int B, hipStream_t st) {
    block_attend_kernel<D, CODE><<<dim3(a.Hk * a.QG, a.nsplit, B), 256, 0, st>>>(a);
    const int tiles = a.score ? (a.max_len + 1 + 255) / 256 : 0;
    block_finish_kernel<D, CODE><<<dim3(a.H + a.Hk + a.Hk * tiles, B), 256, 0, st>>>(a);
}

}  // namespace
}  // namespace st3

extern "C" size_t st3_block_workspace_bytes(const st3_gqa_shape* shape, int32_t max_len) {
    if (st3::check_gqa_shape(shape) != ST3_OK || max_len < 0) return 0;
    return st3::block_ws(shape, max_len).total;
}

extern "C" st3_status st3_block_decode(const st3_gqa_shape* shape, const st3_rows* q, const st3_rows* k_new, const st3_rows* v_new,
                                       const st3_block_cache* cache, int32_t max_len, const st3_rows* out, float* score, int64_t score_stride_b,
                                       int64_t score_stride_h, void* workspace, size_t workspace_bytes, void* stream) {
    using namespace st3;
    st3_status s = check_gqa_shape(shape);
    if (s != ST3_OK) return s;
    if ((s = check_block_cache(shape, cache)) != ST3_OK) return s;
    const int B = shape->batch, H = shape->heads, Hk = shape->kv_heads, D = shape->head_dim, G = H / Hk;
    if ((s = check_rows(q, H, D, 2)) != ST3_OK || (s = check_rows(out, H, D, 2)) != ST3_OK) return s;
    if (!k_new != !v_new) return ST3_ERR_INVALID_ARG;
    if (k_new && ((s = check_rows(k_new, Hk, D, 2)) != ST3_OK || (s = check_rows(v_new, Hk, D, 2)) != ST3_OK)) return s;
    if (max_len < 0 || max_len > 0x3fffffff) return ST3_ERR_INVALID_ARG;
    // (a row that fills its block needs that block's page)
    if (cache->table_blocks < (max_len + (k_new ? 1 : 0)) / kBlk) return ST3_ERR_INVALID_ARG;
    if (score && (score_stride_h < (int64_t)max_len + 1 || (B > 1 && score_stride_b < (int64_t)max_len + 1))) return ST3_ERR_INVALID_ARG;
    if (!workspace || !aligned16(workspace)) return ST3_ERR_INVALID_ARG;
    const BlockWs wl = block_ws(shape, max_len);
    if (workspace_bytes < wl.total) return ST3_ERR_WORKSPACE_TOO_SMALL;
    char* ws = reinterpret_cast<char*>(workspace);
    auto bits = [](const st3_rows* r) { return r ? reinterpret_cast<uint16_t*>(r->data) : nullptr; };
    BlockDecodeArgs a{};
    a.c = block_pages(cache);
    a.q = bits(q); a.k_new = bits(k_new); a.v_new = bits(v_new); a.out = bits(out);
    a.q_st = q->stride_t; a.q_sh = q->stride_h; a.o_st = out->stride_t; a.o_sh = out->stride_h;
    if (k_new) { a.k_st = k_new->stride_t; a.k_sh = k_new->stride_h; a.v_st = v_new->stride_t; a.v_sh = v_new->stride_h; }
    a.max_len = max_len; a.H = H; a.Hk = Hk; a.G = G; a.QG = (G + kCols - 1) / kCols;
    a.chunk = wl.chunk; a.nsplit = wl.nsplit;
    a.scale_l2 = gqa_scale_log2(shape);
    a.score = score; a.s_sb = score_stride_b; a.s_sh = score_stride_h;
    a.part_o = reinterpret_cast<float*>(ws + wl.part_o);
    a.part_ml = reinterpret_cast<float*>(ws + wl.part_ml);
    a.logits = reinterpret_cast<float*>(ws + wl.logits);
    a.logit_stride = wl.logit_stride;
    hipStream_t st = reinterpret_cast<hipStream_t>(stream);
    if (cache->code == ST3_BLOCK_INT8) {
        if (D == 128) launch_decode<128, ST3_BLOCK_INT8>(a, B, st);
        else launch_decode<64, ST3_BLOCK_INT8>(a, B, st);
    } else {
        if (D == 128) launch_decode<128, ST3_BLOCK_E4M3>(a, B, st);
        else launch_decode<64, ST3_BLOCK_E4M3>(a, B, st);
    }
    return check_launch();
}
