// The cache of 8-bit blocks: packed prompts into pages, and eviction by accumulated weight into other pages.
//
// A workgroup of 256 threads makes one block of one key head, K and V.  Thread (group y = tid / 16, x = tid % 16) holds rows 4 y .. + 3 of it and columns
// w x .. + w - 1, w = d / 16: 16 threads read and write whole rows of K; V's codes, whose rows lie in memory as columns, are packed four rows to a word and
// change places through LDS, so that they too leave as 16 bytes a thread.  Bound by memory: both read and write what they must once, but for the lines
// of a page's V of which an eviction keeps a part.
#include <algorithm>
#include <utility>

#include "st3_block.h"

namespace st3 {
namespace {

constexpr int kThreads = 256;
constexpr int kRankThreads = 1024;

// Largest magnitudes of K's and V's values over the workgroup; every thread gets both.
__device__ __forceinline__ float2 block_max(float k, float v, float2* sm, int tid) {
    k = wave_max_from<1>(k);
    v = wave_max_from<1>(v);
    if ((tid & 63) == 0) sm[tid >> 6] = make_float2(k, v);
    __syncthreads();
    return make_float2(fmaxf(fmaxf(sm[0].x, sm[1].x), fmaxf(sm[2].x, sm[3].x)), fmaxf(fmaxf(sm[0].y, sm[1].y), fmaxf(sm[2].y, sm[3].y)));
}

// LDS words of V's codes: [d][64 / 4], a row of 16 words followed by 4 of padding.
constexpr int kWordRow = kBlk / 4 + 4;

// Codes a block from the threads' values (k, v [row][column] as above) into a page.
template <int D, int CODE>
__device__ __forceinline__ void write_block(const float (&k)[4][D / 16], const float (&v)[4][D / 16], const BlockPages& c, int64_t at, uint32_t* words,
                                            float2* sm, int tid) {
    using F = BlockCode<CODE>;
    constexpr int W = D / 16;
    const int x = tid & 15, y = tid >> 4;
    float mk = 0.f, mv = 0.f;
#pragma unroll
    for (int r = 0; r < 4; ++r)
#pragma unroll
        for (int e = 0; e < W; ++e) { mk = fmaxf(mk, finite_abs(k[r][e])); mv = fmaxf(mv, finite_abs(v[r][e])); }
    const float2 top = block_max(mk, mv, sm, tid);
    const Divider dk(top.x * F::kUnit, top.x), dv(top.y * F::kUnit, top.y);
    if (tid == 0) { c.k_scale[at] = dk.scale; c.v_scale[at] = dv.scale; }
    uint8_t* kc = c.k_codes + at * (kBlk * D);
#pragma unroll
    for (int r = 0; r < 4; ++r) {
        uint32_t w[W / 4];
#pragma unroll
        for (int j = 0; j < W / 4; ++j) w[j] = F::code4(k[r] + 4 * j, dk);
        uint32_t* to = reinterpret_cast<uint32_t*>(kc + (4 * y + r) * D + W * x);
        if constexpr (W == 8) *reinterpret_cast<uint2*>(to) = make_uint2(w[0], w[1]);
        else *to = w[0];
    }
#pragma unroll
    for (int e = 0; e < W; ++e) {
        const float col[4] = {v[0][e], v[1][e], v[2][e], v[3][e]};
        words[(W * x + e) * kWordRow + y] = F::code4(col, dv);
    }
    __syncthreads();
    uint4* vc = reinterpret_cast<uint4*>(c.v_codes + at * (kBlk * D));
#pragma unroll
    for (int i = tid; i < D * 4; i += kThreads) vc[i] = *reinterpret_cast<const uint4*>(words + (i >> 2) * kWordRow + 4 * (i & 3));
}

// The rows [0, rows) of a partial block into the tails, `put(r, e, k, v)` being the bits of row r's column e.
template <int D, typename Bits>
__device__ __forceinline__ void write_tail(const Bits& bits, const BlockPages& c, int64_t strip, int rows, int tid) {
    constexpr int W = D / 16;
    const int x = tid & 15, y = tid >> 4;
    uint16_t* kt = c.k_tail + strip * (kBlk * D);
    uint16_t* vt = c.v_tail + strip * (kBlk * D);
#pragma unroll
    for (int r = 0; r < 4; ++r) {
        if (4 * y + r >= rows) continue;
#pragma unroll
        for (int e = 0; e < W; ++e) {
            kt[(4 * y + r) * D + W * x + e] = bits(0, r, e);
            vt[(W * x + e) * kBlk + 4 * y + r] = bits(1, r, e);
        }
    }
}

// W bf16 at p (16 or 8 bytes).
template <int W>
__device__ __forceinline__ void load_bf16(const uint16_t* p, uint32_t (&raw)[W / 2]) {
    if constexpr (W == 8) {
        const uint4 q = *reinterpret_cast<const uint4*>(p);
        raw[0] = q.x; raw[1] = q.y; raw[2] = q.z; raw[3] = q.w;
    } else {
        const uint2 q = *reinterpret_cast<const uint2*>(p);
        raw[0] = q.x; raw[1] = q.y;
    }
}

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
    constexpr int W = D / 16;
    __shared__ __attribute__((aligned(16))) uint32_t words[D * kWordRow];
    __shared__ float2 sm[4];
    const int tid = threadIdx.x, x = tid & 15, y = tid >> 4;
    const int kh = blockIdx.x, j = blockIdx.y, b = blockIdx.z;
    const int start = max(0, min(a.cu[b], a.total)), n = min(max(start, min(a.cu[b + 1], a.total)) - start, a.max_len);
    if (j * kBlk >= n) return;
    const bool whole = (j + 1) * kBlk <= n;
    uint32_t kr[4][W / 2], vr[4][W / 2];
#pragma unroll
    for (int r = 0; r < 4; ++r) {
        const int64_t row = start + min(j * kBlk + 4 * y + r, n - 1);
        load_bf16<W>(a.k + kh * a.k_sh + row * a.k_st + W * x, kr[r]);
        load_bf16<W>(a.v + kh * a.v_sh + row * a.v_st + W * x, vr[r]);
    }
    if (!whole) {
        write_tail<D>([&](int which, int r, int e) { return (uint16_t)((which ? vr[r][e / 2] : kr[r][e / 2]) >> (16 * (e & 1))); }, a.c,
                      (int64_t)b * a.Hk + kh, n - j * kBlk, tid);
        return;
    }
    const int page = page_of(a.c, b, j);
    if (page < 0) return;
    float k[4][W], v[4][W];
#pragma unroll
    for (int r = 0; r < 4; ++r)
#pragma unroll
        for (int e = 0; e < W; e += 2) {
            k[r][e] = bf16_lo(kr[r][e / 2]); k[r][e + 1] = bf16_hi(kr[r][e / 2]);
            v[r][e] = bf16_lo(vr[r][e / 2]); v[r][e + 1] = bf16_hi(vr[r][e / 2]);
        }
    write_block<D, CODE>(k, v, a.c, (int64_t)page * a.Hk + kh, words, sm, tid);
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

// Sum over the workgroup's threads before this one, and over all; waves: one word for each wave, two of them in turn.
__device__ __forceinline__ uint2 count_before(uint32_t mine, uint32_t* waves, int lane, int wave) {
    uint32_t incl = mine;
#pragma unroll
    for (int off = 1; off < 64; off <<= 1) {
        const uint32_t up = __shfl_up(incl, off);
        if (lane >= off) incl += up;
    }
    if (lane == 63) waves[wave] = incl;
    __syncthreads();
    const uint32_t other = lane < kRankThreads / 64 ? waves[lane] : 0;
    uint32_t before = incl - mine, all = 0;
#pragma unroll
    for (int w = 0; w < kRankThreads / 64; ++w) {
        const uint32_t x = __builtin_amdgcn_readlane(other, w);
        before += w < wave ? x : 0;
        all += x;
    }
    return make_uint2(before, all);
}

// Workgroup (key head, sequence): the key of the last row kept by a radix search (11 + 11 + 10 bits), then the rows kept, their scores, and, of the rows
// with that last key, as many of the first as are wanted.  PER > 0: a thread holds PER rows that follow each other in registers (rows of up to 1024 PER);
// 0: rows of any length, read again in every pass.  Bound by its chain of passes: evictions of 8 strips of 1200 rows 8.5 us with PER = 0.
template <int PER>
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
    const bool all = n <= a.keep;
    float x[PER > 0 ? PER : 1];
    if constexpr (PER > 0) {
#pragma unroll
        for (int i = 0; i < PER; ++i) x[i] = tid * PER + i < n ? score[tid * PER + i] : 0.f;
    }
    uint32_t want = all ? 0 : a.keep - a.n_sink - a.n_recent;   // candidates wanted, at last of those with the last key
    uint32_t key = want > 0 ? 0 : 0xffffffffu, mask = 0;        // (no row has the key of all ones)
    for (int pass = 0; pass < 3 && want > 0; ++pass) {
        const int shift = pass == 0 ? 21 : pass == 1 ? 10 : 0, bits = pass == 2 ? 10 : 11;
        hist[tid] = 0;
        hist[tid + kRankThreads] = 0;
        __syncthreads();
        auto note = [&](int i, float s) {
            const uint32_t u = rank_key(s);
            if (i >= lo && i < hi && (u & mask) == key) atomicAdd(&hist[(u >> shift) & ((1u << bits) - 1)], 1u);
        };
        if constexpr (PER > 0) {
#pragma unroll
            for (int i = 0; i < PER; ++i) note(tid * PER + i, x[i]);
        } else {
            for (int i = lo + tid; i < hi; i += kRankThreads) note(i, score[i]);
        }
        __syncthreads();
        // bins from the top: thread t owns bins 2047 - 2 t and 2046 - 2 t
        const uint32_t h0 = hist[2047 - 2 * tid], h1 = hist[2046 - 2 * tid];
        const uint32_t before = count_before(h0 + h1, waves[0], lane, wave).x;
        if (before < want && before + h0 >= want) { found[0] = 2047 - 2 * tid; found[1] = want - before; }
        else if (before + h0 < want && before + h0 + h1 >= want) { found[0] = 2046 - 2 * tid; found[1] = want - before - h0; }
        __syncthreads();
        key |= found[0] << shift;
        mask |= ((1u << bits) - 1) << shift;
        want = found[1];
        __syncthreads();
    }
    auto safe = [&](int i) { return all || i < lo || i >= hi; };
    if constexpr (PER > 0) {
        uint32_t ties = 0, mine = 0;
#pragma unroll
        for (int i = 0; i < PER; ++i) { const int r = tid * PER + i; ties += r < n && !safe(r) && rank_key(x[i]) == key ? 1 : 0; }
        uint32_t tie = count_before(ties, waves[0], lane, wave).x;
        bool keep[PER];
#pragma unroll
        for (int i = 0; i < PER; ++i) {
            const int r = tid * PER + i;
            const uint32_t u = rank_key(x[i]);
            const bool is_tie = r < n && !safe(r) && u == key;
            keep[i] = r < n && (safe(r) || u > key || (is_tie && tie < want));
            tie += is_tie ? 1 : 0;
            mine += keep[i] ? 1 : 0;
        }
        uint32_t at = count_before(mine, waves[1], lane, wave).x;      // (every thread has read its scores: to_score may be score)
#pragma unroll
        for (int i = 0; i < PER; ++i)
            if (keep[i]) { kept[at] = tid * PER + i; to[at] = x[i]; ++at; }
    } else {
        uint32_t out = 0, ties = 0;             // rows written, rows with the last key met
        for (int i0 = 0; i0 < n; i0 += kRankThreads) {
            const int i = i0 + tid;
            const float s = i < n ? score[i] : 0.f;
            const uint32_t u = rank_key(s);
            const bool tie = i < n && !safe(i) && u == key;
            const uint2 t = count_before(tie ? 1 : 0, waves[0], lane, wave);
            const bool keep = i < n && (safe(i) || u > key || (tie && ties + t.x < want));
            const uint2 at = count_before(keep ? 1 : 0, waves[1], lane, wave);      // (the chunk's scores are read: to_score may be score)
            if (keep) { kept[out + at.x] = i; to[out + at.x] = s; }
            out += at.y;
            ties += t.y;
        }
    }
    for (int i = min(n, a.keep) + tid; i < a.keep; i += kRankThreads) kept[i] = -1;
}

// Workgroup (key head, new block, sequence).  K's rows are fetched one by one; any row of a page's V lies in all of its lines, so V comes as whole pages, one
// after the other (a block's rows ascend: a few pages that follow each other), and is picked from LDS.
template <int D, int CODE>
__global__ __launch_bounds__(kThreads) void block_move_kernel(EvictBlockArgs a) {
    using F = BlockCode<CODE>;
    constexpr int W = D / 16, kPiece = D * kBlk / 16 / kThreads;       // 16-byte pieces of a page a thread fetches
    __shared__ __attribute__((aligned(16))) uint32_t words[D * kWordRow];
    __shared__ __attribute__((aligned(16))) uint8_t page_v[D * kBlk];
    __shared__ float2 sm[4];
    const int tid = threadIdx.x, lane = tid & 63, x = tid & 15, y = tid >> 4;
    const int kh = blockIdx.x, j = blockIdx.y, b = blockIdx.z;
    const int n = min(a.from.len[b], a.max_len), count = min(n, a.keep);
    if (j * kBlk >= count) return;
    const int32_t* kept = a.kept + b * a.i_sb + kh * a.i_sh + j * kBlk;
    const bool whole = (j + 1) * kBlk <= count;
    const int to_page = whole ? page_of(a.to, b, j) : 0;
    if (to_page < 0) return;
    const int64_t strip = (int64_t)b * a.Hk + kh, to_at = (int64_t)to_page * a.Hk + kh;
    // lane i looks up row i (every wave all of them): its old block, -1 where it is in the tail, and that block's page
    const int row_l = kept[min(lane, count - 1 - j * kBlk)], blk_l = row_l < n / kBlk * kBlk ? row_l / kBlk : -1;
    const int page_l = blk_l >= 0 ? page_of(a.from, b, blk_l) : -1;
    const int64_t at_l = (int64_t)max(page_l, 0) * a.Hk + kh;
    const float ks_l = page_l >= 0 ? a.from.k_scale[at_l] : 0.f, vs_l = page_l >= 0 ? a.from.v_scale[at_l] : 0.f;
    const uint64_t in_place = __ballot(page_l >= 0 && row_l % kBlk == lane);
    if (whole && in_place == ~0ull && __ballot(blk_l == __builtin_amdgcn_readfirstlane(blk_l)) == ~0ull) {     // one whole old block
        for (int i = tid; i < D * kBlk / 16; i += kThreads) {
            reinterpret_cast<uint4*>(a.to.k_codes + to_at * (kBlk * D))[i] = reinterpret_cast<const uint4*>(a.from.k_codes + at_l * (kBlk * D))[i];
            reinterpret_cast<uint4*>(a.to.v_codes + to_at * (kBlk * D))[i] = reinterpret_cast<const uint4*>(a.from.v_codes + at_l * (kBlk * D))[i];
        }
        if (tid == 0) { a.to.k_scale[to_at] = ks_l; a.to.v_scale[to_at] = vs_l; }
        return;
    }
    // the pages that the rows lie in, from the first to the last (in every wave alike)
    uint64_t left = __ballot(page_l >= 0);
    uint4 piece[kPiece];
    auto fetch = [&](int first) {
        const int64_t at = (int64_t)__builtin_amdgcn_readlane(page_l, first) * a.Hk + kh;
        const uint4* src = reinterpret_cast<const uint4*>(a.from.v_codes + at * (kBlk * D));
#pragma unroll
        for (int i = 0; i < kPiece; ++i) piece[i] = src[tid + i * kThreads];
    };
    if (left != 0) fetch(__ffsll((unsigned long long)left) - 1);
    // this thread's rows: K as it is, V's rows of the tail
    float k[4][W], v[4][W];
    int row[4], blk[4];
#pragma unroll
    for (int r = 0; r < 4; ++r) {
        row[r] = __shfl(row_l, 4 * y + r) % kBlk;
        blk[r] = __shfl(blk_l, 4 * y + r);
        const int page = __shfl(page_l, 4 * y + r);
        const float ks = __shfl(ks_l, 4 * y + r);
        const int64_t at = (int64_t)max(page, 0) * a.Hk + kh;
        if (blk[r] >= 0) {
            uint32_t w[W / 4];
            const uint8_t* p = a.from.k_codes + at * (kBlk * D) + row[r] * D + W * x;
#pragma unroll
            for (int i = 0; i < W / 4; ++i) w[i] = page >= 0 ? reinterpret_cast<const uint32_t*>(p)[i] : 0u;
#pragma unroll
            for (int e = 0; e < W; ++e) { k[r][e] = F::value(w[e / 4] >> (8 * (e & 3)) & 0xffu) * ks; v[r][e] = 0.f; }
        } else {
            const uint16_t* kt = a.from.k_tail + strip * (kBlk * D) + row[r] * D + W * x;
            const uint16_t* vt = a.from.v_tail + strip * (kBlk * D) + row[r];
#pragma unroll
            for (int e = 0; e < W; ++e) {
                k[r][e] = __uint_as_float((uint32_t)kt[e] << 16);
                v[r][e] = __uint_as_float((uint32_t)vt[(W * x + e) * kBlk] << 16);
            }
        }
    }
    while (left != 0) {
        const int now = __builtin_amdgcn_readlane(blk_l, __ffsll((unsigned long long)left) - 1);
        __syncthreads();                                    // (the page before is not read any more)
#pragma unroll
        for (int i = 0; i < kPiece; ++i) reinterpret_cast<uint4*>(page_v)[tid + i * kThreads] = piece[i];
        left &= ~__ballot(blk_l == now);
        if (left != 0) fetch(__ffsll((unsigned long long)left) - 1);
        __syncthreads();
#pragma unroll
        for (int r = 0; r < 4; ++r) {
            const float vs = __shfl(vs_l, 4 * y + r);
            if (blk[r] == now) {
#pragma unroll
                for (int e = 0; e < W; ++e) v[r][e] = F::value(page_v[(W * x + e) * kBlk + row[r]]) * vs;
            }
        }
    }
    if (whole) write_block<D, CODE>(k, v, a.to, to_at, words, sm, tid);
    else write_tail<D>([&](int which, int r, int e) { return (uint16_t)f32_to_bf16_bits(which ? v[r][e] : k[r][e]); }, a.to, strip, count - j * kBlk, tid);
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
    if (max_len <= 4 * kRankThreads) block_rank_kernel<4><<<dim3(Hk, B), kRankThreads, 0, st>>>(a);
    else if (max_len <= 16 * kRankThreads) block_rank_kernel<16><<<dim3(Hk, B), kRankThreads, 0, st>>>(a);
    else block_rank_kernel<0><<<dim3(Hk, B), kRankThreads, 0, st>>>(a);
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
