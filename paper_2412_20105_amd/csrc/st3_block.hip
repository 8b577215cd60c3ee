// The cache of 8-bit blocks: packed prompts into pages, and eviction by accumulated weight into other pages.
//
// Both write blocks the same way (BlockWriter): a workgroup holds the 64 x d values of one block and key head in registers, thread (wave w,
// lane i) row i and the columns w d/4 .. + d/4 - 1, finds the largest magnitude, and codes.  K codes are rows, V codes columns.
#include <algorithm>
#include <utility>

#include "st3_block.h"

namespace st3 {
namespace {

constexpr int kThreads = 256;
constexpr int kRankThreads = 1024;

// Largest magnitude over the workgroup; every thread gets it.
__device__ __forceinline__ float block_max(float x, float* sm, int tid) {
    x = wave_max_from<1>(x);
    __syncthreads();                    // (sm may still be read from the last time)
    if ((tid & 63) == 0) sm[tid >> 6] = x;
    __syncthreads();
    return fmaxf(fmaxf(sm[0], sm[1]), fmaxf(sm[2], sm[3]));
}

// Codes one block of K (columns: false) or V (true) from x[d/4] of each thread into its page.
template <int D, int CODE, bool COLUMNS>
__device__ __forceinline__ void write_block(const float (&x)[D / 4], uint8_t* codes, float* scale_out, float* sm, int tid) {
    using F = BlockCode<CODE>;
    const int lane = tid & 63, col = (tid >> 6) * (D / 4);
    float mx = 0.f;
#pragma unroll
    for (int e = 0; e < D / 4; ++e) mx = fmaxf(mx, finite_abs(x[e]));
    const float scale = block_max(mx, sm, tid) * F::kUnit;
    if (tid == 0) *scale_out = scale;
    if constexpr (COLUMNS) {
#pragma unroll
        for (int e = 0; e < D / 4; ++e) codes[(col + e) * kBlk + lane] = (uint8_t)F::code(x[e], scale);
    } else {
#pragma unroll
        for (int e = 0; e < D / 4; e += 16) {
            uint32_t w[4];
#pragma unroll
            for (int j = 0; j < 4; ++j)
                w[j] = F::code(x[e + 4 * j], scale) | F::code(x[e + 4 * j + 1], scale) << 8 | F::code(x[e + 4 * j + 2], scale) << 16 |
                       F::code(x[e + 4 * j + 3], scale) << 24;
            *reinterpret_cast<uint4*>(codes + lane * D + col + e) = make_uint4(w[0], w[1], w[2], w[3]);
        }
    }
}

__device__ __forceinline__ float bf16_value(uint16_t b) { return __uint_as_float((uint32_t)b << 16); }

// ---------------------------------------------------------------------------------------------------------------------------------
// prompts into pages: workgroup (key head, block, sequence)
// ---------------------------------------------------------------------------------------------------------------------------------
struct StoreArgs {
    BlockPages c;
    const uint16_t* k; const uint16_t* v;
    int64_t k_st, k_sh, v_st, v_sh;
    const int32_t* cu;
    int32_t total, max_len, Hk;
};

template <int D, int CODE>
__global__ __launch_bounds__(kThreads) void block_store_kernel(StoreArgs a) {
    __shared__ float sm[4];
    const int tid = threadIdx.x, lane = tid & 63, col = (tid >> 6) * (D / 4);
    const int kh = blockIdx.x, j = blockIdx.y, b = blockIdx.z;
    const int start = max(0, min(a.cu[b], a.total)), n = min(max(start, min(a.cu[b + 1], a.total)) - start, a.max_len);
    if (j * kBlk >= n) return;
    const int row = j * kBlk + lane;
    const bool whole = (j + 1) * kBlk <= n;
    const int page = whole ? page_of(a.c, b, j) : 0;
    if (page < 0) return;
#pragma unroll
    for (int which = 0; which < 2; ++which) {
        const uint16_t* src = (which ? a.v + kh * a.v_sh : a.k + kh * a.k_sh) + (int64_t)(start + min(row, n - 1)) * (which ? a.v_st : a.k_st) + col;
        uint4 raw[D / 32];
#pragma unroll
        for (int e = 0; e < D / 32; ++e) raw[e] = *reinterpret_cast<const uint4*>(src + 8 * e);
        if (!whole) {
            const int64_t at = ((int64_t)b * a.Hk + kh) * kBlk * D;
            if (row < n) {
                const uint16_t* h = reinterpret_cast<const uint16_t*>(raw);
                if (which) {
#pragma unroll
                    for (int e = 0; e < D / 4; ++e) a.c.v_tail[at + (col + e) * kBlk + lane] = h[e];
                } else {
#pragma unroll
                    for (int e = 0; e < D / 32; ++e) *reinterpret_cast<uint4*>(a.c.k_tail + at + lane * D + col + 8 * e) = raw[e];
                }
            }
            continue;
        }
        float x[D / 4];
#pragma unroll
        for (int e = 0; e < D / 32; ++e) ElemTraits<bf16_t>::unpack(raw[e], x + 8 * e);
        const int64_t at = (int64_t)page * a.Hk + kh;
        if (which) write_block<D, CODE, true>(x, a.c.v_codes + at * kBlk * D, a.c.v_scale + at, sm, tid);
        else write_block<D, CODE, false>(x, a.c.k_codes + at * kBlk * D, a.c.k_scale + at, sm, tid);
    }
}

// ---------------------------------------------------------------------------------------------------------------------------------
// eviction: rank, then rows into their new blocks
// ---------------------------------------------------------------------------------------------------------------------------------
struct EvictBlockArgs {
    BlockPages from, to;
    int32_t max_len, keep, n_sink, n_recent, Hk;
    const float* score; int64_t s_sb, s_sh;
    float* to_score; int64_t t_sb, t_sh;
    int32_t* kept; int64_t i_sb, i_sh;
};

// Greater means better; NaN below everything, -0 as +0.
__device__ __forceinline__ uint32_t rank_key(float x) {
    if (!(x == x)) return 0;
    const uint32_t u = __float_as_uint(x == 0.f ? 0.f : x);
    return u & 0x80000000u ? ~u : u | 0x80000000u;
}

// Workgroup (key head, sequence): the key of the last row kept by a radix search (11 + 11 + 10 bits), then one pass in order that writes the rows kept, their
// scores, and, of the rows with that last key, as many of the first as are wanted.
__global__ __launch_bounds__(kRankThreads) void block_rank_kernel(EvictBlockArgs a) {
    __shared__ uint32_t hist[2048];
    __shared__ uint32_t waves[2][kRankThreads / 64];
    __shared__ uint32_t found[2];
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, kh = blockIdx.x, b = blockIdx.y;
    const int n = min(a.from.len[b], a.max_len);
    if (n < 0) return;
    const float* score = a.score + b * a.s_sb + kh * a.s_sh;
    float* to = a.to_score + b * a.t_sb + kh * a.t_sh;
    int32_t* kept = a.kept + b * a.i_sb + kh * a.i_sh;
    const int lo = a.n_sink, hi = n - a.n_recent;
    uint32_t want = 0, key = 0;             // candidates wanted; key of the last of them
    if (n > a.keep) {
        want = a.keep - a.n_sink - a.n_recent;
        uint32_t mask = 0;
        if (want > 0) {
            for (int pass = 0; pass < 3; ++pass) {
                const int shift = pass == 0 ? 21 : pass == 1 ? 10 : 0, bits = pass == 2 ? 10 : 11;
                for (int i = tid; i < 2048; i += kRankThreads) hist[i] = 0;
                __syncthreads();
                for (int i = lo + tid; i < hi; i += kRankThreads) {
                    const uint32_t u = rank_key(score[i]);
                    if ((u & mask) == key) atomicAdd(&hist[(u >> shift) & ((1u << bits) - 1)], 1u);
                }
                __syncthreads();
                // bins from the top: thread t owns bins 2047 - 2 t and 2046 - 2 t
                const uint32_t h0 = hist[2047 - 2 * tid], h1 = hist[2046 - 2 * tid];
                uint32_t incl = h0 + h1;
#pragma unroll
                for (int off = 1; off < 64; off <<= 1) {
                    const uint32_t up = __shfl_up(incl, off);
                    if (lane >= off) incl += up;
                }
                if (lane == 63) waves[0][wave] = incl;
                __syncthreads();
                uint32_t before = incl - h0 - h1;
                for (int w = 0; w < wave; ++w) before += waves[0][w];
                if (before < want && before + h0 >= want) { found[0] = 2047 - 2 * tid; found[1] = want - before; }
                else if (before + h0 < want && before + h0 + h1 >= want) { found[0] = 2046 - 2 * tid; found[1] = want - before - h0; }
                __syncthreads();
                key |= found[0] << shift;
                mask |= ((1u << bits) - 1) << shift;
                want = found[1];
                __syncthreads();
            }
        } else {
            key = 0xffffffffu;              // (no row has it: no candidate is kept)
        }
    }
    const bool all = n <= a.keep;
    uint32_t out = 0, ties = 0;             // rows written, rows with the last key met
    for (int i0 = 0; i0 < n; i0 += kRankThreads) {
        const int i = i0 + tid;
        const float x = i < n ? score[i] : 0.f;
        const uint32_t u = rank_key(x);
        const bool safe = all || i < lo || i >= hi;
        const bool tie = i < n && !safe && u == key;
        const uint64_t tie_mask = __ballot(tie);
        if (lane == 0) waves[0][wave] = __popcll(tie_mask);
        __syncthreads();
        uint32_t t = ties + __popcll(tie_mask & ((1ull << lane) - 1)), t_all = ties;
        for (int w = 0; w < kRankThreads / 64; ++w) { t += w < wave ? waves[0][w] : 0; t_all += waves[0][w]; }
        const bool keep = i < n && (safe || u > key || (tie && t < want));
        const uint64_t keep_mask = __ballot(keep);
        if (lane == 0) waves[1][wave] = __popcll(keep_mask);
        __syncthreads();                    // (every thread has read its score: to_score may be score)
        uint32_t at = out + __popcll(keep_mask & ((1ull << lane) - 1)), all_kept = out;
        for (int w = 0; w < kRankThreads / 64; ++w) { at += w < wave ? waves[1][w] : 0; all_kept += waves[1][w]; }
        if (keep) { kept[at] = i; to[at] = x; }
        out = all_kept;
        ties = t_all;
    }
    for (int i = min(n, a.keep) + tid; i < a.keep; i += kRankThreads) kept[i] = -1;
}

// Workgroup (key head, new block, sequence).
template <int D, int CODE>
__global__ __launch_bounds__(kThreads) void block_move_kernel(EvictBlockArgs a) {
    using F = BlockCode<CODE>;
    __shared__ float sm[4];
    const int tid = threadIdx.x, lane = tid & 63, col = (tid >> 6) * (D / 4);
    const int kh = blockIdx.x, j = blockIdx.y, b = blockIdx.z;
    const int n = min(a.from.len[b], a.max_len), count = min(n, a.keep);
    if (j * kBlk >= count) return;
    const int32_t* kept = a.kept + b * a.i_sb + kh * a.i_sh;
    const bool whole = (j + 1) * kBlk <= count;
    const int to_page = whole ? page_of(a.to, b, j) : 0;
    if (to_page < 0) return;
    const int i = min(j * kBlk + lane, count - 1), row = kept[i];
    const int whole_rows = n / kBlk * kBlk;
    const bool coded = row < whole_rows;
    const int page = coded ? page_of(a.from, b, row / kBlk) : -1, r = row % kBlk;
    // one whole old block?
    const bool same = whole && coded && page >= 0 && r == lane && __ballot(row - lane == __builtin_amdgcn_readfirstlane(row)) == ~0ull;
    const bool verbatim = __ballot(same) == ~0ull;
    const int64_t to_at = (int64_t)to_page * a.Hk + kh, tail_at = ((int64_t)b * a.Hk + kh) * kBlk * D, from_at = (int64_t)max(page, 0) * a.Hk + kh;
#pragma unroll
    for (int which = 0; which < 2; ++which) {
        const uint8_t* codes = (which ? a.from.v_codes : a.from.k_codes) + from_at * kBlk * D;
        uint8_t* to_codes = (which ? a.to.v_codes : a.to.k_codes) + to_at * kBlk * D;
        const float* scales = which ? a.from.v_scale : a.from.k_scale;
        float* to_scales = which ? a.to.v_scale : a.to.k_scale;
        if (verbatim) {                     // (the same in every wave)
            for (int e = tid; e < kBlk * D / 16; e += kThreads) reinterpret_cast<uint4*>(to_codes)[e] = reinterpret_cast<const uint4*>(codes)[e];
            if (tid == 0) to_scales[to_at] = scales[from_at];
            continue;
        }
        float x[D / 4];
        if (coded) {
            const float scale = page >= 0 ? scales[from_at] : 0.f;
#pragma unroll
            for (int e = 0; e < D / 4; ++e) x[e] = page >= 0 ? F::value(which ? codes[(col + e) * kBlk + r] : codes[r * D + col + e]) * scale : 0.f;
        } else {
            const uint16_t* tail = (which ? a.from.v_tail : a.from.k_tail) + tail_at;
#pragma unroll
            for (int e = 0; e < D / 4; ++e) x[e] = bf16_value(which ? tail[(col + e) * kBlk + r] : tail[r * D + col + e]);
        }
        if (whole) {
            if (which) write_block<D, CODE, true>(x, to_codes, to_scales + to_at, sm, tid);
            else write_block<D, CODE, false>(x, to_codes, to_scales + to_at, sm, tid);
        } else if (j * kBlk + lane < count) {
            uint16_t* tail = (which ? a.to.v_tail : a.to.k_tail) + tail_at;
#pragma unroll
            for (int e = 0; e < D / 4; ++e) tail[which ? (col + e) * kBlk + lane : lane * D + col + e] = (uint16_t)f32_to_bf16_bits(x[e]);
        }
    }
}

}  // namespace
}  // namespace st3

extern "C" st3_status st3_block_store(const st3_gqa_shape* shape, const st3_rows* k, const st3_rows* v, const int32_t* cu_len, int32_t total,
                                      int32_t max_len, const st3_block_cache* cache, void* stream) {
    using namespace st3;
    st3_status s = check_gqa_shape(shape);
    if (s != ST3_OK) return s;
    if ((s = check_block_cache(shape, cache)) != ST3_OK) return s;
    const int Hk = shape->kv_heads, D = shape->head_dim;
    if ((s = check_rows(k, Hk, D, 2)) != ST3_OK || (s = check_rows(v, Hk, D, 2)) != ST3_OK) return s;
    if (!cu_len || total < 0 || max_len < 0 || max_len > total) return ST3_ERR_INVALID_ARG;
    const int blocks = (max_len + kBlk - 1) / kBlk;
    if (blocks == 0) return ST3_OK;
    if (blocks > 65535) return ST3_ERR_UNSUPPORTED;
    if (cache->table_blocks < max_len / kBlk) return ST3_ERR_INVALID_ARG;
    const StoreArgs a{block_pages(cache), reinterpret_cast<const uint16_t*>(k->data), reinterpret_cast<const uint16_t*>(v->data), k->stride_t, k->stride_h,
                      v->stride_t, v->stride_h, cu_len, total, max_len, Hk};
    const dim3 grid(Hk, blocks, shape->batch);
    hipStream_t st = reinterpret_cast<hipStream_t>(stream);
    if (cache->code == ST3_BLOCK_INT8) {
        if (D == 128) block_store_kernel<128, ST3_BLOCK_INT8><<<grid, kThreads, 0, st>>>(a);
        else block_store_kernel<64, ST3_BLOCK_INT8><<<grid, kThreads, 0, st>>>(a);
    } else {
        if (D == 128) block_store_kernel<128, ST3_BLOCK_E4M3><<<grid, kThreads, 0, st>>>(a);
        else block_store_kernel<64, ST3_BLOCK_E4M3><<<grid, kThreads, 0, st>>>(a);
    }
    return check_launch();
}

extern "C" st3_status st3_block_evict(const st3_gqa_shape* shape, const st3_block_cache* from, const st3_block_cache* to, int32_t max_len, int32_t keep,
                                      int32_t n_sink, int32_t n_recent, const float* score, int64_t score_stride_b, int64_t score_stride_h,
                                      float* to_score, int64_t to_score_stride_b, int64_t to_score_stride_h, int32_t* kept, int64_t kept_stride_b,
                                      int64_t kept_stride_h, void* stream) {
    using namespace st3;
    st3_status s = check_gqa_shape(shape);
    if (s != ST3_OK) return s;
    if ((s = check_block_cache(shape, from)) != ST3_OK || (s = check_block_cache(shape, to)) != ST3_OK) return s;
    const int B = shape->batch, Hk = shape->kv_heads, D = shape->head_dim;
    if (from->code != to->code || !score || !to_score || !kept) return ST3_ERR_INVALID_ARG;
    if (max_len < 0 || keep < 1 || n_sink < 0 || n_recent < 0 || (int64_t)n_sink + n_recent > keep) return ST3_ERR_INVALID_ARG;
    const int most = std::min(max_len, keep);
    if (from->table_blocks < max_len / kBlk || to->table_blocks < most / kBlk) return ST3_ERR_INVALID_ARG;
    if (score_stride_h < max_len || to_score_stride_h < most || kept_stride_h < keep) return ST3_ERR_INVALID_ARG;
    if (B > 1 && (score_stride_b < max_len || to_score_stride_b < most || kept_stride_b < keep)) return ST3_ERR_INVALID_ARG;
    const int64_t tail = (int64_t)B * Hk * kBlk * D * 2;
    for (auto [x, y] : {std::pair{from->k_tail, to->k_tail}, {from->v_tail, to->v_tail}, {from->k_tail, to->v_tail}, {from->v_tail, to->k_tail}}) {
        const int64_t d = reinterpret_cast<intptr_t>(x) - reinterpret_cast<intptr_t>(y);
        if (d < tail && -d < tail) return ST3_ERR_INVALID_ARG;
    }
    const int blocks = (most + kBlk - 1) / kBlk;
    if (blocks > 65535) return ST3_ERR_UNSUPPORTED;
    const EvictBlockArgs a{block_pages(from), block_pages(to), max_len, keep, n_sink, n_recent, Hk, score, score_stride_b, score_stride_h, to_score,
                           to_score_stride_b, to_score_stride_h, kept, kept_stride_b, kept_stride_h};
    hipStream_t st = reinterpret_cast<hipStream_t>(stream);
    block_rank_kernel<<<dim3(Hk, B), kRankThreads, 0, st>>>(a);
    if (blocks == 0) return check_launch();
    const dim3 grid(Hk, blocks, B);
    if (from->code == ST3_BLOCK_INT8) {
        if (D == 128) block_move_kernel<128, ST3_BLOCK_INT8><<<grid, kThreads, 0, st>>>(a);
        else block_move_kernel<64, ST3_BLOCK_INT8><<<grid, kThreads, 0, st>>>(a);
    } else {
        if (D == 128) block_move_kernel<128, ST3_BLOCK_E4M3><<<grid, kThreads, 0, st>>>(a);
        else block_move_kernel<64, ST3_BLOCK_E4M3><<<grid, kThreads, 0, st>>>(a);
    }
    return check_launch();
}
