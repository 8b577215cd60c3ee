// Causal attention of several new tokens over a cache of 8-bit blocks, with grouped heads and accumulated weights.
//
// Rows.  The G query heads that share a key head are rows of one matrix, as for packed prompts: row x of a (sequence, key head) pair is head x % G of new
// token x / G.  A workgroup's eight waves have up to 32 rows each (more would not fit the registers: 48 and 64 spill, and take 2 and 4 times as long) and
// walk the blocks of 64 keys together; 8-bit codes, loaded two blocks ahead into registers, become bf16 on their way into LDS, once for all rows (codes have
// at most 8 significant bits: exact), and the scale of a block multiplies the logits and the weights.  By waves of four the conversion costs twice as
// much: 1138 us against 1005 for 2048 tokens over 30000 rows (32 heads, 8 key heads, d = 128).
//   S^T = K Q^T    (A: lane (c, g) holds A[c][8g..8g+7], B: B[8g..8g+7][c], C: C[4g..4g+3][c]) product t of four: row 4g'+i of A is key 16 g' + 4 t + i, so
//                  that lane (c, g) of C ends with keys 16 g .. 16 g + 15 of row c.
//   O^T = V^T P^T  the lane's 16 keys are the contraction slots 8g..8g+7 of two steps: P^T is where S^T left it.
// No value crosses lanes but the maximum.  Where row tiles are too few to fill the card, a strip's blocks are cut into pieces, and a second launch joins them.
// What bounds it: the matrix units with many rows (2048 tokens over 30000 rows 895 to 930 us, 1140 to 1180 TFLOP/s); with few, the chain from a block's codes
// through both products to its barrier (1.3 us a block of 64 keys with 36 rows, 1.8 with 256), so that rows up to kFewRows go another way, below, bound by
// memory.
#include <algorithm>
#include <type_traits>

#include "st3_block.h"
#include "st3_block_few.h"

namespace st3 {
namespace {

constexpr int kChunkWaves = 8, kChunkThreads = 64 * kChunkWaves;

struct ChunkArgs {
    BlockPages c;
    const uint16_t* q; uint16_t* out;
    int64_t q_st, q_sh, o_st, o_sh;
    const int32_t* cu;
    int32_t B, total, max_new, max_len, H, Hk, G;
    int32_t tile;                   // rows of a row tile: a multiple of 16
    int32_t piece, pieces;          // blocks of a piece; pieces of the longest strip (1: whole strips)
    float scale_l2;
    float* score; int64_t s_sb, s_sh;
    int32_t window;
    float2* ml;                     // [total][H] maximum, and one over the sum; null: no score
    float* part_o;                  // [total][H][pieces][D]
    float2* part_ml;                // [total][H][pieces]
};

// A sequence's new rows, the rows in front of them (negative: an empty place), and what it attends.
struct Turn {
    int start, m, n;
    __device__ __forceinline__ int rows() const { return n < 0 ? 0 : n + m; }
    __device__ __forceinline__ int sees(int t) const { return n < 0 ? -1 : n + t; }        // the last row that new row t sees
};
__device__ __forceinline__ Turn turn_of(const ChunkArgs& a, int b) {
    const int s = max(0, min(a.cu[b], a.total)), e = max(s, min(a.cu[b + 1], a.total)), n = a.c.len[b];
    return Turn{s, min(min(e - s, a.max_new), n < 0 ? a.max_new : max(a.max_len - n, 0)), n};
}

// Workgroup -> (sequence, key head, row tile).  Key heads run fastest (they go round-robin to the 8 XCDs), longest sequences come first, so that the launch
// ends with its shortest workgroups; more than 64 keep their own order.  Lengths are known to the device only: every wave finds its place, a lane for
// each sequence.
__device__ __forceinline__ bool place(const ChunkArgs& a, int lane, int& b, int& kh, int& tile, Turn& sq) {
    kh = blockIdx.x % a.Hk;
    int x = blockIdx.x / a.Hk;
    Turn its = {0, 0, 0};
    auto tiles_of = [&](int i) {
        if (i < a.B) its = turn_of(a, i);
        return i < a.B ? (its.m * a.G + a.tile - 1) / a.tile : 0;
    };
    auto found = [&](int first, int at, int t) {        // (lane `at` has sequence first + at)
        at = __builtin_amdgcn_readfirstlane(at);
        b = first + at;
        tile = __builtin_amdgcn_readfirstlane(t);
        sq = Turn{__builtin_amdgcn_readlane(its.start, at), __builtin_amdgcn_readlane(its.m, at), __builtin_amdgcn_readlane(its.n, at)};
        return true;
    };
    if (a.B > kWave) {
        for (int i0 = 0; i0 < a.B; i0 += kWave) {
            const int mine = tiles_of(i0 + lane), upto = wave_prefix(mine), all = __builtin_amdgcn_readlane(upto, 63);
            if (x < all) {
                const int at = __ffsll((unsigned long long)__ballot(x < upto)) - 1;
                return found(i0, at, __builtin_amdgcn_readlane(upto, at) - 1 - x);
            }
            x -= all;
        }
        return false;
    }
    const int mine = tiles_of(lane), rows = its.rows();
    if (x >= wave_total(mine)) return false;
    int before = 0;                     // tiles of the sequences in front of this one
    for (int i = 0; i < a.B; ++i) {
        const int other = __builtin_amdgcn_readlane(rows, i);
        before += other > rows || (other == rows && i < lane) ? __builtin_amdgcn_readlane(mine, i) : 0;
    }
    const int at = __ffsll((unsigned long long)__ballot(mine > 0 && before <= x && x < before + mine)) - 1;
    return found(0, at, __builtin_amdgcn_readlane(before + mine, at) - 1 - x);
}

// A block in LDS: K as 64 rows of D bf16, V as D rows (columns of V) of 64.  Unit u (16 bytes) of a row r of K lies at u ^ k_swz(r), of V at v_place(u) ^ v_swz(r):
// lanes that are served together (16 of them, of rows 0 .. 3 and 12 .. 15 of one g and 4 .. 11 of the next) read 16 different units of the banks.
template <int D> struct Tile {
    static constexpr int K = kBlk * D, BYTES = 4 * K;       // elements of K, and of V; bytes of both
    __device__ static __forceinline__ int k_swz(int row) {
        return D == 128 ? (row >> 4 & 3) << 2 | (row & 3) : (row >> 4 & 3) << 1 | (row >> 1 & 1);
    }
    __device__ static __forceinline__ int v_swz(int row) { return row >> 1 & 7; }
    __device__ static __forceinline__ int v_place(int unit) { return unit >> 1 | (unit & 1) << 2; }
};

__device__ __forceinline__ void lds_write16(uint32_t at, u32x4 x) { *reinterpret_cast<__attribute__((address_space(3))) u32x4*>(at) = x; }

// A block's codes on their way from memory to LDS: pieces of 16 bytes, those of K and then those of V, dealt to the threads.
template <int D, int CODE, int THREADS>
struct Codes {
    static constexpr int PIECES = kBlk * D / 16, N = 2 * PIECES / THREADS;
    static_assert(N * THREADS == 2 * PIECES && PIECES % kWave == 0, "whole waves take pieces of K, or of V");
    u32x4 w[N];
    __device__ __forceinline__ void load(const BlockPages& c, int64_t at, int tid) {
#pragma unroll
        for (int i = 0; i < N; ++i) {
            const int p = tid + i * THREADS;
            const uint8_t* codes = p < PIECES ? c.k_codes : c.v_codes;
            w[i] = reinterpret_cast<const u32x4*>(codes + at * (kBlk * D))[p < PIECES ? p : p - PIECES];
        }
    }
    // half a piece: 8 codes
    static constexpr int HALVES = 2 * N;
    __device__ __forceinline__ void store_half(int h, uint32_t lds, int tid) const {
        using F = BlockCode<CODE>;
        const int i = h / 2, p = tid + i * THREADS, kr = p / (D / 16), vr = (p - PIECES) / (kBlk / 16);
        const uint32_t row_at = p < PIECES ? 2 * D * kr : 2 * Tile<D>::K + 2 * kBlk * vr;
        const int swz = p < PIECES ? Tile<D>::k_swz(kr) : Tile<D>::v_swz(vr);
        const int first = p < PIECES ? 2 * (p % (D / 16)) : p % (kBlk / 16), second = first + (p < PIECES ? 1 : 4);       // (v_place of 2 u and 2 u + 1)
        const uint2 a = F::to_bf16(h & 1 ? w[i].z : w[i].x), b = F::to_bf16(h & 1 ? w[i].w : w[i].y);
        lds_write16(lds + (row_at + 16 * ((h & 1 ? second : first) ^ swz)), u32x4{a.x, a.y, b.x, b.y});
    }
    __device__ __forceinline__ void store(uint32_t lds, int tid) const {
#pragma unroll
        for (int h = 0; h < HALVES; ++h) store_half(h, lds, tid);
    }
};

// The tail, `rows` rows in 16 bits, into LDS; the rows behind them are zeros, whatever their bits are.
template <int D, int THREADS>
__device__ __forceinline__ void tail_to_lds(const BlockPages& c, int64_t strip, int rows, uint32_t lds, int tid) {
    asm volatile("" : "+v"(tid));                           // (opaque, as below: else what follows from it is kept in registers through a walk that needs it once)
    const u32x4* kp = reinterpret_cast<const u32x4*>(c.k_tail + strip * (kBlk * D));
    const u32x4* vp = reinterpret_cast<const u32x4*>(c.v_tail + strip * (kBlk * D));
    constexpr int N = kBlk * D / 8 / THREADS;
    static_assert(N * THREADS == kBlk * D / 8, "all of the tail");
#pragma unroll
    for (int i = 0; i < N; ++i) {
        const int p = tid + i * THREADS, kr = p / (D / 8), vr = p / (kBlk / 8);
        const u32x4 k = kp[p];
        lds_write16(lds + 2 * D * kr + 16 * (p % (D / 8) ^ Tile<D>::k_swz(kr)), kr < rows ? k : u32x4{0, 0, 0, 0});
        Frag f;
        f.u4 = vp[p];
        const int key = 8 * (p % (kBlk / 8));
#pragma unroll
        for (int j = 0; j < 4; ++j) f.w[j] &= (key + 2 * j < rows ? 0xffffu : 0u) | (key + 2 * j + 1 < rows ? 0xffff0000u : 0u);
        lds_write16(lds + 2 * Tile<D>::K + 2 * kBlk * vr + 16 * (Tile<D>::v_place(p % (kBlk / 8)) ^ Tile<D>::v_swz(vr)), f.u4);
    }
}

// A wave's 16 QC rows, as QC columns of 16: lane (c, g) holds row 16 qc + c of each, and of its output the columns 16 dt + 4 g .. + 3.
template <int D, int QC>
struct Rows {
    f32x4 o[D / 16][QC];
    float m[QC], l[QC];
    int pos[QC];            // the last of the sequence's rows that the row sees
    __device__ __forceinline__ void init() {
#pragma unroll
        for (int qc = 0; qc < QC; ++qc) {
#pragma unroll
            for (int dt = 0; dt < D / 16; ++dt) o[dt][qc] = f32x4{0.f, 0.f, 0.f, 0.f};
            m[qc] = -3.402823466e38f; l[qc] = 0.f;
        }
    }
};

// A wave's products, O^T += V^T P^T of one block and S^T = K Q^T of the next; fragments are read from LDS a few products ahead (and no more: the scheduling
// barriers keep the compiler from holding more of them than there are registers for).
template <int D, int QC>
struct Products {
    static constexpr int KS = D / 32, DT = D / 16, kAhead = 2;
    Frag va[kAhead + 1][2], ka[2][KS];
    __device__ __forceinline__ void read_v(int dt, uint32_t v_at) {
#pragma unroll
        for (int x = 0; x < 2; ++x) va[dt % (kAhead + 1)][x].u4 = lds_read16((v_at ^ (64 * x)) + 32 * kBlk * dt);
    }
    __device__ __forceinline__ void read_k(int t, uint32_t k_at) {
#pragma unroll
        for (int x = 0; x < KS; ++x) ka[t & 1][x].u4 = lds_read16((k_at ^ (64 * x)) + 8 * D * t);
    }
    __device__ __forceinline__ void values(uint32_t v_at, const Frag (&pb)[2][QC], Rows<D, QC>& st) {
#pragma unroll
        for (int dt = 0; dt < kAhead; ++dt) read_v(dt, v_at);
#pragma unroll
        for (int dt = 0; dt < DT; ++dt) {
            if (dt + kAhead < DT) read_v(dt + kAhead, v_at);
            __builtin_amdgcn_sched_barrier(0);
#pragma unroll
            for (int x = 0; x < 2; ++x)
#pragma unroll
                for (int qc = 0; qc < QC; ++qc) st.o[dt][qc] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(va[dt % (kAhead + 1)][x].v, pb[x][qc].v, st.o[dt][qc], 0, 0, 0);
            __builtin_amdgcn_sched_barrier(0);
        }
    }
    // beside(t): what else is done between the products, a quarter of it (VALU instructions and a write to LDS)
    template <typename Beside>
    __device__ __forceinline__ void logits(uint32_t k_at, const Frag (&qf)[QC][KS], f32x4 (&s)[4][QC], const Beside& beside) {
        read_k(0, k_at);
#pragma unroll
        for (int t = 0; t < 4; ++t) {
            if (t + 1 < 4) read_k(t + 1, k_at);
            __builtin_amdgcn_sched_barrier(0);
            beside(t);
#pragma unroll
            for (int x = 0; x < KS; ++x)
#pragma unroll
                for (int qc = 0; qc < QC; ++qc)
                    s[t][qc] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(ka[t & 1][x].v, qf[qc][x].v, x == 0 ? f32x4{0.f, 0.f, 0.f, 0.f} : s[t][qc], 0, 0, 0);
#pragma unroll
            for (int i = 0; i < KS * QC; ++i) {
                __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);          // a product, two others
                __builtin_amdgcn_sched_group_barrier(0x002, 2, 0);
            }
            __builtin_amdgcn_sched_barrier(0);
        }
    }
};

// Weights of 64 keys, some of which some row may not see; ks: the block's scale of K times that of the logits (in the log2 domain), vs: of V.
// A weight times V's scale is rounded to bf16 once, to nearest: an error of 2^-8 of it at most and without bias, beside the output's own rounding by as
// much; the sum is of the unrounded ones.
template <int D, int QC>
__device__ __forceinline__ void chunk_weights(f32x4 (&s)[4][QC], Rows<D, QC>& st, float ks, float vs, int g, int k0, Frag (&pb)[2][QC]) {
    asm volatile("" : "+v"(g));
    // (a block's scale may be 0, and -infinity times 0 is no number: masks come behind the scale)
#pragma unroll
    for (int t = 0; t < 4; ++t)
#pragma unroll
        for (int qc = 0; qc < QC; ++qc) {
            s[t][qc] *= ks;
#pragma unroll
            for (int i = 0; i < 4; ++i)
                if (k0 + 16 * g + 4 * t + i > st.pos[qc]) s[t][qc][i] = -INFINITY;
        }
    // the reference point of the exponents follows the maximum only when that has moved by more than kLazy
    constexpr float kLazy = 8.0f;
    float mx[QC];
    bool moved = false;
#pragma unroll
    for (int qc = 0; qc < QC; ++qc) {
        mx[qc] = -INFINITY;
#pragma unroll
        for (int t = 0; t < 4; ++t) mx[qc] = fmaxf(mx[qc], fmaxf(fmaxf(s[t][qc][0], s[t][qc][1]), fmaxf(s[t][qc][2], s[t][qc][3])));
        moved |= mx[qc] - st.m[qc] > kLazy;
    }
    if (__any(moved)) {
#pragma unroll
        for (int qc = 0; qc < QC; ++qc) {
            const float cand = fmaxf(st.m[qc], wave_max_from<16>(mx[qc]));
            const float m_new = cand - st.m[qc] > kLazy ? cand : st.m[qc];
            const float alpha = exp2_fast(st.m[qc] - m_new);
            st.m[qc] = m_new;
            st.l[qc] *= alpha;
#pragma unroll
            for (int dt = 0; dt < D / 16; ++dt) st.o[dt][qc] *= alpha;
        }
    }
#pragma unroll
    for (int qc = 0; qc < QC; ++qc)
#pragma unroll
        for (int x = 0; x < 2; ++x)
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const f32x4 y = s[2 * x + j / 2][qc];
                const float p0 = exp2_fast(y[2 * (j & 1)] - st.m[qc]), p1 = exp2_fast(y[2 * (j & 1) + 1] - st.m[qc]);
                st.l[qc] += p0 + p1;
                pb[x][qc].w[j] = bf16_pair(p0 * vs, p1 * vs);
            }
}

// The same of a block that every row sees whole, nearly all of them.  The reference point stays where it is (weights are floating point, in bf16 too: nothing is
// lost as long as none of them grows large), and V's scale comes with the exponent: exp2(s ks - m + log2 vs); what a lane adds to the sum is that
// divided by vs.  False, and nothing done, where weights have grown above kMost, are no numbers, or vs has no logarithm (lvs is NaN then).
template <int D, int QC>
__device__ __forceinline__ bool chunk_weights_whole(const f32x4 (&s)[4][QC], Rows<D, QC>& st, float ks, float lvs, float rvs, Frag (&pb)[2][QC]) {
    constexpr float kMost = 4096.0f;
    float sum[QC];
    bool large = false;
#pragma unroll
    for (int qc = 0; qc < QC; ++qc) {
        const float off = lvs - st.m[qc];
        sum[qc] = 0.f;
#pragma unroll
        for (int x = 0; x < 2; ++x)
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const f32x4 y = s[2 * x + j / 2][qc];
                const float w0 = exp2_fast(fmaf(y[2 * (j & 1)], ks, off)), w1 = exp2_fast(fmaf(y[2 * (j & 1) + 1], ks, off));
                sum[qc] += w0 + w1;
                pb[x][qc].w[j] = bf16_pair(w0, w1);
            }
        sum[qc] *= rvs;
        large |= !(sum[qc] <= kMost);
    }
    if (__any(large)) return false;
#pragma unroll
    for (int qc = 0; qc < QC; ++qc) st.l[qc] += sum[qc];
    return true;
}

// 64 keys for one wave where V may hold infinities or NaN, which a weight of 0 does not silence: row by row, V's keys that the row does not see count as 0.
template <int D, int QC>
__device__ __forceinline__ void chunk_step_careful(uint32_t k_at, uint32_t v_at, const Frag (&qf)[QC][D / 32], Rows<D, QC>& st, float ks, float vs, int g, int k0) {
    f32x4 s[4][QC];
    Frag pb[2][QC];
    Products<D, QC>{}.logits(k_at, qf, s, [](int) {});
    chunk_weights<D, QC>(s, st, ks, vs, g, k0, pb);
    const int c = threadIdx.x & 15;
#pragma unroll
    for (int qc = 0; qc < QC; ++qc)
#pragma unroll 1
        for (int row = 0; row < 16; ++row) {
            const int pos = __builtin_amdgcn_readlane(st.pos[qc], row);
#pragma unroll
            for (int x = 0; x < 2; ++x) {
                Frag seen;
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    const int key = k0 + 16 * g + 8 * x + 2 * j;
                    seen.w[j] = (key <= pos ? 0xffffu : 0u) | (key < pos ? 0xffff0000u : 0u);
                }
#pragma unroll
                for (int dt = 0; dt < D / 16; ++dt) {
                    Frag va;
                    va.u4 = lds_read16((v_at ^ (64 * x)) + 32 * kBlk * dt);
#pragma unroll
                    for (int j = 0; j < 4; ++j) va.w[j] &= seen.w[j];
                    const f32x4 o = __builtin_amdgcn_mfma_f32_16x16x32_bf16(va.v, pb[x][qc].v, st.o[dt][qc], 0, 0, 0);
                    st.o[dt][qc] = c == row ? o : st.o[dt][qc];
                    __builtin_amdgcn_sched_barrier(0);
                }
            }
        }
}

// A barrier that nothing is moved across.
__device__ __forceinline__ void meet() {
    __builtin_amdgcn_sched_barrier(0);
    __syncthreads();
    __builtin_amdgcn_sched_barrier(0);
}

// What a workgroup works on.
struct Work {
    Turn sq;
    int64_t strip;
    int kh, ch, b, rows, u_begin, u_end;
};

// One wave's part of it: 16 QC rows from row r0 on (idle: none).  Every wave of a workgroup meets the same barriers, whatever its QC.
template <int D, int CODE, int QC, int COLS>
__device__ __forceinline__ void chunk_wave(const ChunkArgs& a, const Work& w, uint8_t* buf, int* redo, int r0, bool idle) {
    constexpr int kThr = kChunkThreads, KS = D / 32, DT = D / 16, OSTR = D + 8;
    using L = Tile<D>;
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), g = lane >> 4, c = lane & 15;
    const int rows = w.rows, kh = w.kh, b = w.b, ch = w.ch, u_begin = w.u_begin, u_end = w.u_end, blocks = w.sq.rows() / kBlk;
    const Turn& sq = w.sq;
    const int64_t strip = w.strip;
    const uint32_t lds0 = lds_addr(buf);
    Rows<D, QC> st;
    st.init();
    Frag qf[QC][KS];
#pragma unroll
    for (int qc = 0; qc < QC; ++qc) {
        const int r = min(r0 + 16 * qc + c, rows - 1), t = r / a.G;
        st.pos[qc] = sq.sees(t);
        const uint16_t* row = a.q + (int64_t)(sq.start + t) * a.q_st + (int64_t)(kh * a.G + r - t * a.G) * a.q_sh;
#pragma unroll
        for (int s = 0; s < KS; ++s) qf[qc][s].u4 = *reinterpret_cast<const u32x4*>(row + 32 * s + 8 * g);
    }
    const int p_first = sq.sees(min(r0, rows - 1) / a.G), p_last = sq.sees((min(r0 + 16 * QC, rows) - 1) / a.G);      // what the wave's first and last rows see
    const int krow = 16 * (c >> 2) + (c & 3);
    const uint32_t k_lane = (uint32_t)(2 * D * krow + 16 * (g ^ L::k_swz(krow))), v_lane = (uint32_t)(2 * L::K + 2 * kBlk * c + 16 * (g ^ L::v_swz(c)));
    // lane i has the page and the scales of block `base` + i
    int base = 0, page_l = -1;
    float ks_l = 0.f, vs_l = 0.f, lvs_l = 0.f, rvs_l = 0.f;
    auto look_up = [&](int from) {
        base = from;
        const int u = from + lane;
        page_l = u < u_end && u < blocks ? page_of(a.c, b, u) : -1;
        ks_l = vs_l = 0.f;
        if (page_l >= 0) {
            const int64_t at = (int64_t)page_l * a.Hk + kh;
            ks_l = a.c.k_scale[at] * a.scale_l2;
            vs_l = a.c.v_scale[at];
        }
        // (0, and scales so small or large that weights times them leave the normal range, have no logarithm here)
        lvs_l = vs_l > 0x1p-90f && vs_l < 0x1p90f ? __builtin_amdgcn_logf(vs_l) : __uint_as_float(0x7fc00000u);
        rvs_l = 1.0f / vs_l;
    };
    auto lane_value = [](float x, int i) { return __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(x), i)); };
    const int u_stop = min(u_end, blocks), units = max(u_end - u_begin, 0);     // (one behind u_stop: the rows in 16 bits)
    // A block's scales, and whether there is one.
    struct Scales { bool there; float ks, vs, lvs, rvs; };
    auto scales_of = [&](int u) {
        if (u >= u_stop) return Scales{u < u_end, a.scale_l2, 1.0f, 0.0f, 1.0f};
        if (u >= base + kWave) look_up(u);
        const int i = u - base;
        return Scales{__builtin_amdgcn_readlane(page_l, i) >= 0, lane_value(ks_l, i), lane_value(vs_l, i), lane_value(lvs_l, i), lane_value(rvs_l, i)};
    };
    // Blocks' codes on their way: codes[x] and page[x] those of the i-th from u_begin on, x = i & 1.
    Codes<D, CODE, kThr> codes[2];
    int page[2] = {-1, -1};
    int ahead = 0, page_ahead = -1;                         // lane i has the page of block `ahead` + i (codes are fetched further ahead than scales)
    auto fetch = [&](int i, int x) {
        const int u = u_begin + i;
        if (u >= ahead + kWave) {
            ahead = u;
            page_ahead = u + lane < u_stop ? page_of(a.c, b, u + lane) : -1;
        }
        page[x] = __builtin_amdgcn_readlane(page_ahead, u - ahead);
        codes[x].load(a.c, (int64_t)max(page[x], 0) * a.Hk + kh, tid);     // (always: where loads hang on a condition, those behind them are waited for too)
    };
    // The i-th block into LDS; what is no block of codes comes behind it, and the codes (those of page 0) then go where nothing is yet, into the next one's place.
    auto place_of = [&](int i, int x) { return lds0 + ((page[x] >= 0 ? i : i + 1) & 3) * L::BYTES; };
    auto others_of = [&](int i, int x) {
        const int u = u_begin + i;
        if (page[x] < 0 && u < u_end) tail_to_lds<D, kThr>(a.c, strip, u >= u_stop ? sq.rows() % kBlk : 0, lds0 + (i & 3) * L::BYTES, tid);    // (a block without a page: zeros, without weight)
    };
    auto store = [&](int i, int x) {
        codes[x].store(place_of(i, x), tid);
        others_of(i, x);
    };
    // A step of a wave is a half on the matrix units (the values of one block and the logits of the next; beside them codes of the one behind go into
    // LDS) and one on the others (weights).  The two waves of a SIMD are half a step apart: while one keeps the matrix units busy, the other
    // computes weights (2048 tokens over 30000 rows: 1045 us in step, 958 so; with the codes' conversion between the products 895).
    const int mine = idle || p_last < u_begin * kBlk ? 0 : min(units, p_last / kBlk - u_begin + 1);     // steps in which this wave has rows that see something
    auto v_of = [&](int i) { return lds0 + (i & 3) * L::BYTES + v_lane; };
    auto k_of = [&](int i) { return lds0 + (i & 3) * L::BYTES + k_lane; };
    look_up(u_begin);
    ahead = u_begin;
    page_ahead = page_l;
    fetch(0, 0);
    fetch(1, 1);
    store(0, 0);
    fetch(2, 0);
    meet();
    const bool second = wave >= kChunkWaves / 2;
    if (second) meet();
    if (mine > 0) {
        f32x4 s[4][QC];
        Frag pb[2][QC];
        Products<D, QC> products;
        auto multiply = [&](int i, int x) {                 // logits of the i-th block; codes[x]: those of the next
            const uint32_t at = place_of(i + 1, x);
            products.logits(k_of(i), qf, s, [&](int t) {
                constexpr int H = Codes<D, CODE, kThr>::HALVES;
                if (t < H) codes[x].store_half(t, at, tid);
            });
            others_of(i + 1, x);
            fetch(i + 3, x);
        };
        multiply(0, 1);
        meet();
        auto step = [&](int i, int x) {
            const int u = u_begin + i;
            const Scales w = scales_of(u);
            if (u >= u_stop || !w.there || u * kBlk + kBlk - 1 > p_first || !chunk_weights_whole<D, QC>(s, st, w.ks, w.lvs, w.rvs, pb))
                chunk_weights<D, QC>(s, st, w.ks, w.vs, g, w.there ? u * kBlk : 0x7fffff00, pb);        // (a block without a page lies behind all rows)
            meet();
            __builtin_amdgcn_s_setprio(1);
            products.values(v_of(i), pb, st);
            if (i + 1 == mine) return false;
            multiply(i + 1, x);
            __builtin_amdgcn_s_setprio(0);
            meet();
            return true;
        };
        for (int i = 0; step(i, 0) && step(i + 1, 1); i += 2) {}
        __builtin_amdgcn_s_setprio(0);
    }
    auto idle_step = [&](int i, int x) {                    // codes[x]: those of block i + 1
        store(i + 1, x);
        fetch(i + 3, x);
        meet();
        meet();
    };
    int i = mine;
    if (i < units && (i & 1)) idle_step(i++, 0);
    for (; i < units; i += 2) {
        idle_step(i, 1);
        if (i + 1 < units) idle_step(i + 1, 0);
    }
    if (!second) meet();
    // Anything but finite: it may be from V of keys that a row does not see (0 times infinity).  Once more, such V left out.
    float odd = 0.f;
#pragma unroll
    for (int dt = 0; dt < DT; ++dt)
#pragma unroll
        for (int qc = 0; qc < QC; ++qc)
#pragma unroll
            for (int i = 0; i < 4; ++i) odd = fmaf(st.o[dt][qc][i], 0.f, odd);
    if (odd != 0.f) *redo = 1;
    __syncthreads();
    if (*redo) {
        st.init();
        look_up(u_begin);
        for (int u = u_begin; u < u_end; ++u) {
            __syncthreads();
            const Scales x = scales_of(u);
            if (u >= u_stop) tail_to_lds<D, kThr>(a.c, strip, sq.rows() % kBlk, lds0, tid);
            else if (x.there) {
                codes[0].load(a.c, (int64_t)__builtin_amdgcn_readlane(page_l, u - base) * a.Hk + kh, tid);
                codes[0].store(lds0, tid);
            }
            __syncthreads();
            if (x.there && !idle && u * kBlk <= p_last) chunk_step_careful<D, QC>(lds0 + k_lane, lds0 + v_lane, qf, st, x.ks, x.vs, g, u * kBlk);
        }
        __syncthreads();
    }
    if (a.pieces > 1) {
#pragma unroll
        for (int qc = 0; qc < QC; ++qc) {
            const float l = wave_sum_from<16>(st.l[qc]);
            const int r = r0 + 16 * qc + c, t = r / a.G;
            if (r >= rows || idle) continue;
            const int64_t part = ((int64_t)(sq.start + t) * a.H + kh * a.G + r - t * a.G) * a.pieces + ch;
#pragma unroll
            for (int dt = 0; dt < DT; ++dt) *reinterpret_cast<f32x4*>(a.part_o + part * D + 16 * dt + 4 * g) = st.o[dt][qc];
            if (g == 0) a.part_ml[part] = make_float2(st.m[qc], l);
        }
        return;
    }
    // ---- normalise; the block of outputs goes through LDS and leaves as whole rows ----------------------------------------------
    if (idle) return;
    uint16_t* ob = reinterpret_cast<uint16_t*>(buf) + wave * 16 * COLS * OSTR;
    constexpr int VPR = D / 8, RPI = 64 / VPR;
#pragma unroll
    for (int qc = 0; qc < QC; ++qc) {
        const float l = wave_sum_from<16>(st.l[qc]), rl = l == 0.f ? 0.f : 1.0f / l;      // (a sum of NaN stays one)
#pragma unroll
        for (int dt = 0; dt < DT; ++dt) {
            const f32x4 o = st.o[dt][qc] * rl;
            uint2 pk;
            pk.x = bf16_pair(o[0], o[1]);
            pk.y = bf16_pair(o[2], o[3]);
            *reinterpret_cast<uint2*>(ob + (16 * qc + c) * OSTR + 16 * dt + 4 * g) = pk;
        }
        const int r = r0 + 16 * qc + c, t = r / a.G;
        if (a.ml != nullptr && g == 0 && r < rows) a.ml[(int64_t)(sq.start + t) * a.H + kh * a.G + r - t * a.G] = make_float2(st.m[qc], rl);
    }
#pragma unroll
    for (int i = 0; i < 16 * QC / RPI; ++i) {
        const int x = i * RPI + lane / VPR, r = r0 + x;
        const u32x4 val = *reinterpret_cast<const u32x4*>(ob + x * OSTR + (lane % VPR) * 8);
        if (r < rows) {
            const int t = r / a.G;
            *reinterpret_cast<u32x4*>(a.out + (int64_t)(sq.start + t) * a.o_st + (int64_t)(kh * a.G + r - t * a.G) * a.o_sh + (lane % VPR) * 8) = val;
        }
    }
}

// A tile's columns of 16 rows are dealt to the waves as evenly as they go: one column a wave (COLS 1), or one or two.
template <int D, int CODE, int COLS>
__global__ __launch_bounds__(kChunkThreads, 2) void block_chunk_kernel(ChunkArgs a) {
    constexpr int kOut = 2 * kChunkWaves * 16 * COLS * (D + 8), kTiles = 4 * Tile<D>::BYTES;        // bytes
    __shared__ __attribute__((aligned(1024))) uint8_t buf[kTiles > kOut ? kTiles : kOut];
    __shared__ int redo;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    Work w;
    int tile;
    if (!place(a, lane, w.b, w.kh, tile, w.sq)) return;
    w.ch = blockIdx.y;
    w.rows = w.sq.m * a.G;
    const int first = tile * a.tile, cols = (min(a.tile, w.rows - first) + 15) / 16;
    const int last = w.sq.sees((min(w.rows, first + a.tile) - 1) / a.G);                     // the last row that the workgroup sees (-1: none)
    w.u_begin = w.ch * a.piece;
    w.u_end = min((last + kBlk) / kBlk, w.u_begin + a.piece);
    if (w.ch > 0 && w.u_begin >= w.u_end) return;
    w.strip = (int64_t)w.b * a.Hk + w.kh;
    if (threadIdx.x == 0) redo = 0;
    const int from = wave * cols / kChunkWaves, n = (wave + 1) * cols / kChunkWaves - from, r0 = first + 16 * from;
    if constexpr (COLS == 2) {
        if (n == 2) {
            chunk_wave<D, CODE, 2, COLS>(a, w, buf, &redo, r0, false);
            return;
        }
    }
    chunk_wave<D, CODE, 1, COLS>(a, w, buf, &redo, r0, n == 0);
}

// ---------------------------------------------------------------------------------------------------------------------------------
// Few rows (a token or a few drafted ones; a workgroup has 16 QC of them at most): every wave has them all, and takes the blocks in turn, each by itself, as the
// attention of single tokens does: K straight to its own LDS, V straight into registers, 16 codes of a lane's operand at once, the rows in 16 bits by the
// first waves, 32 keys at a time.  The waves' parts are joined in LDS.  WHOLE: a workgroup takes a whole strip; with room for the logits in LDS (stage:
// rows of a strip there; 0: none) it adds the weights too.
// ---------------------------------------------------------------------------------------------------------------------------------
constexpr float kNoPage = -3.402823466e38f;     // in place of a logit: no page, no weight

template <int D, int CODE, int QC, int WAVES, bool WHOLE, bool TWO>
__global__ __launch_bounds__(WAVES * 64, QC == 1 ? 3 : 2) void chunk_few_kernel(ChunkArgs a, int stage) {
    using F = BlockCode<CODE>;
    using L = KeyTile<D>;
    constexpr int KS = D / 32, DT = D / 16, KH = D / 64, kThr = WAVES * 64, OS = D + 4;
    extern __shared__ __attribute__((aligned(16))) float few[];
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), g = lane >> 4, c = lane & 15;
    const int kh = blockIdx.x % a.Hk, ch = blockIdx.y, b = blockIdx.z, cols = a.tile, r0 = blockIdx.x / a.Hk * cols;
    const Turn got = turn_of(a, b);
    const Turn sq{__builtin_amdgcn_readfirstlane(got.start), __builtin_amdgcn_readfirstlane(got.m), __builtin_amdgcn_readfirstlane(got.n)};
    if (sq.m * a.G <= r0) return;
    const int rows = min(sq.m * a.G - r0, cols), keys = sq.rows(), blocks = keys / kBlk, units = (keys + kBlk - 1) / kBlk;
    const int u_begin = WHOLE ? 0 : ch * a.piece, u_end = WHOLE ? units : min(units, u_begin + a.piece);
    if (!WHOLE && ch > 0 && u_begin >= units) return;
    const FewLds<D> at(WAVES, cols);
    float* sm_o = few;
    float* sm_m = few + at.maxima;
    float* sm_l = few + at.sums;
    float* sm_h = few + at.heads;                           // a row's maximum, and one over its sum
    float* staged = few + at.staged;                        // [cols][stage]
    const int64_t strip = (int64_t)b * a.Hk + kh;
    const int krow = 16 * (c >> 2) + (c & 3);               // + 4 t: the key of row c of product t
    const uint32_t v_lane = (uint32_t)(c * kBlk + 16 * g);
    uint8_t* own = reinterpret_cast<uint8_t*>(few) + wave * (kBlk * D);
    const uint32_t k_lane = (uint32_t)(lane / L::UPR * D + 16 * ((lane % L::UPR) ^ L::swz(lane / L::UPR)));
    const uint32_t own_at = __builtin_amdgcn_readfirstlane(lds_addr(own));
    u32x4 vr[DT];
    auto load_k = [&](int page) {
        const uint8_t* p = a.c.k_codes + ((int64_t)page * a.Hk + kh) * (kBlk * D);
#pragma unroll
        for (int i = 0; i < L::NI; ++i)                     // (what the first row adds to the permutation of a lane's row comes on top of it)
            direct_load16_stream(p + 1024 * i, k_lane ^ (16 * L::swz(i * L::RPI)), own_at + 1024 * i);
    };
    auto load_v = [&](int page) {
        const auto rsrc = __builtin_amdgcn_make_buffer_rsrc(a.c.v_codes + ((int64_t)page * a.Hk + kh) * (kBlk * D), 0, kBlk * D, 0x00020000);
#pragma unroll
        for (int dt = 0; dt < DT; ++dt) vr[dt] = __builtin_amdgcn_raw_buffer_load_b128(rsrc, v_lane, 16 * dt * kBlk, 2);       // (nt: read once)
    };
    // Position i of a wave: first the halves of the tail, where it belongs to the piece, then the piece's blocks.  Lane i has the page and the scales of
    // the block at the wave's i-th position (the launcher sees to it that there are no more of them).
    const bool with_tail = units > blocks && blocks >= u_begin && blocks < u_end;
    const int tail_rows = keys % kBlk, halves = !with_tail ? 0 : tail_rows > 32 ? 2 : 1, u_stop = min(u_end, blocks);
    auto unit_at = [&](int i) { return u_begin + wave + WAVES * i - halves; };
    int page_l = -1;
    float ks_l = 0.f, vs_l = 0.f;
    {
        const int u = unit_at(lane);
        page_l = u >= u_begin && u < u_stop ? page_of(a.c, b, u) : -1;
        if (page_l >= 0) {
            const int64_t at = (int64_t)page_l * a.Hk + kh;
            ks_l = a.c.k_scale[at] * a.scale_l2;
            vs_l = a.c.v_scale[at];
        }
    }
    Frag qf[QC][KS];
    Rows<D, QC> st;
    st.init();
#pragma unroll
    for (int qc = 0; qc < QC; ++qc) {
        const int r = r0 + min(16 * qc + c, rows - 1), t = r / a.G;
        st.pos[qc] = sq.sees(t);
        const uint16_t* row = a.q + (int64_t)(sq.start + t) * a.q_st + (int64_t)(kh * a.G + r - t * a.G) * a.q_sh;
#pragma unroll
        for (int s = 0; s < KS; ++s) qf[qc][s].u4 = *reinterpret_cast<const u32x4*>(row + 64 * (s / 2) + 16 * g + 8 * (s & 1));
    }
    auto keep = [&](int qc, const f32x4& s, int key) {      // logits of keys key .. + 3, of those of the strip
        if (WHOLE && stage > 0 && 16 * qc + c < rows) *reinterpret_cast<f32x4*>(staged + (16 * qc + c) * stage + key) = s;
    };
    // the reference point of the exponents: follows the maximum only when that has moved by more than kLazy
    auto follow = [&](const float (&mx)[QC]) {
        constexpr float kLazy = 8.0f;
        bool moved = false;
#pragma unroll
        for (int qc = 0; qc < QC; ++qc) moved |= mx[qc] - st.m[qc] > kLazy;
        if (!__any(moved)) return;
#pragma unroll
        for (int qc = 0; qc < QC; ++qc) {
            const float cand = fmaxf(st.m[qc], wave_max_from<16>(mx[qc])), m_new = cand - st.m[qc] > kLazy ? cand : st.m[qc];
            const float alpha = exp2_fast(st.m[qc] - m_new);
            st.m[qc] = m_new;
            st.l[qc] *= alpha;
#pragma unroll
            for (int dt = 0; dt < DT; ++dt) st.o[dt][qc] *= alpha;
        }
    };
    // Weights times V's scale.  TWO, rows of one group: as two bf16 terms, cut off at 8 significant bits and the rest rounded to nearest: what is left out is
    // 2^-16 of a weight at most, as for single tokens (five tokens over 739 rows 16.2 us, with one term 15.2; four of 32 sequences 27.5 and 26.3, of E4M3 24.8 and
    // 24.4).  Two groups, whose matrix instructions are what their time goes into, have one, rounded to nearest (16 tokens of eight sequences over 20000 to
    // 30000 rows 127 us, with two 141), as tiles have.
    auto weigh = [&](int qc, const f32x4& s0, const f32x4& s1, float vs, Frag& hi, Frag& lo) {
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const f32x4& y = j < 2 ? s0 : s1;
            const float p0 = exp2_fast(y[2 * (j & 1)] - st.m[qc]), p1 = exp2_fast(y[2 * (j & 1) + 1] - st.m[qc]);
            st.l[qc] += p0 + p1;
            const float w0 = p0 * vs, w1 = p1 * vs;
            if constexpr (TWO) {
                const uint32_t b0 = __float_as_uint(w0), b1 = __float_as_uint(w1);
                hi.w[j] = __builtin_amdgcn_perm(b1, b0, 0x07060302u);
                lo.w[j] = bf16_pair(w0 - __uint_as_float(b0 & 0xffff0000u), w1 - __uint_as_float(b1 & 0xffff0000u));
            } else {
                hi.w[j] = bf16_pair(w0, w1);
            }
        }
    };
    // O^T += V^T P^T where V of keys that a row does not see may be infinite or no number: row by row, such V left out.  f: keys key .. + 7.
    auto careful = [&](int dt, const Frag& f, const Frag (&hi)[QC], const Frag (&lo)[QC], int key) {
#pragma unroll
        for (int qc = 0; qc < QC; ++qc)
#pragma unroll 1
            for (int row = 0; row < 16; ++row) {
                const int pos = __builtin_amdgcn_readlane(st.pos[qc], row);
                Frag v;
#pragma unroll
                for (int j = 0; j < 4; ++j) v.w[j] = f.w[j] & ((key + 2 * j <= pos ? 0xffffu : 0u) | (key + 2 * j < pos ? 0xffff0000u : 0u));
                f32x4 o = __builtin_amdgcn_mfma_f32_16x16x32_bf16(v.v, hi[qc].v, st.o[dt][qc], 0, 0, 0);
                if constexpr (TWO) o = __builtin_amdgcn_mfma_f32_16x16x32_bf16(v.v, lo[qc].v, o, 0, 0, 0);
                st.o[dt][qc] = c == row ? o : st.o[dt][qc];
            }
    };
    // bytes 0x7f and 0xff of four codes, by their highest bits
    auto no_numbers = [](uint32_t w) { return ((w & 0x7f7f7f7fu) + 0x01010101u) & 0x80808080u; };
    uint64_t odd_at = 0;                                    // positions of masked blocks with such codes among V's
    uint64_t left = __ballot(page_l >= 0);                  // the wave's positions whose blocks are to come
    if (left != 0) load_k(__builtin_amdgcn_readlane(page_l, __ffsll((unsigned long long)left) - 1));     // (on its way beside the tail)
    __builtin_amdgcn_sched_barrier(0);
    if (wave < halves) {                                    // product t of two: row 4g'+i of A is key 8 g' + 4 t + i
        const int first = 32 * wave, key0 = blocks * kBlk + first;
        const uint16_t* kt = a.c.k_tail + strip * (kBlk * D);
        const uint16_t* vt = a.c.v_tail + strip * (kBlk * D);
        Frag tk[2][KS], tv[DT];
#pragma unroll
        for (int t = 0; t < 2; ++t)
#pragma unroll
            for (int i = 0; i < KS; ++i)
                tk[t][i].u4 = *reinterpret_cast<const u32x4*>(kt + (first + 8 * (c >> 2) + (c & 3) + 4 * t) * D + 64 * (i / 2) + 16 * g + 8 * (i & 1));
#pragma unroll
        for (int dt = 0; dt < DT; ++dt) tv[dt].u4 = *reinterpret_cast<const u32x4*>(vt + (16 * dt + c) * kBlk + first + 8 * g);
        __builtin_amdgcn_sched_barrier(0);                  // (all of that is on its way)
        f32x4 s[2][QC];
        float mx[QC];
#pragma unroll
        for (int qc = 0; qc < QC; ++qc) {
            mx[qc] = -INFINITY;
#pragma unroll
            for (int t = 0; t < 2; ++t) {
                f32x4 y = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
                for (int i = 0; i < KS; ++i) y = __builtin_amdgcn_mfma_f32_16x16x32_bf16(tk[t][i].v, qf[qc][i].v, y, 0, 0, 0);
                y *= a.scale_l2;
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    if (key0 + 8 * g + 4 * t + i > st.pos[qc]) y[i] = -INFINITY;       // (rows that hold nothing lie behind all rows)
                    mx[qc] = fmaxf(mx[qc], y[i]);
                }
                s[t][qc] = y;
                keep(qc, y, key0 + 8 * g + 4 * t);
            }
        }
        follow(mx);
        Frag hi[QC], lo[QC];
#pragma unroll
        for (int qc = 0; qc < QC; ++qc) weigh(qc, s[0][qc], s[1][qc], 1.0f, hi[qc], lo[qc]);
        bool odd = false;
#pragma unroll
        for (int dt = 0; dt < DT; ++dt)
#pragma unroll
            for (int j = 0; j < 4; ++j) {                   // rows that hold nothing weigh nothing, whatever their bits are
                const int row = first + 8 * g + 2 * j;
                tv[dt].w[j] &= (row < tail_rows ? 0xffffu : 0u) | (row + 1 < tail_rows ? 0xffff0000u : 0u);
                odd |= (tv[dt].w[j] & 0x7f80u) == 0x7f80u || (tv[dt].w[j] & 0x7f800000u) == 0x7f800000u;
            }
        if (__any(odd)) {
#pragma unroll
            for (int dt = 0; dt < DT; ++dt) careful(dt, tv[dt], hi, lo, key0 + 8 * g);
        } else {
#pragma unroll
            for (int dt = 0; dt < DT; ++dt)
#pragma unroll
                for (int qc = 0; qc < QC; ++qc) {
                    st.o[dt][qc] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(tv[dt].v, hi[qc].v, st.o[dt][qc], 0, 0, 0);
                    if constexpr (TWO) st.o[dt][qc] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(tv[dt].v, lo[qc].v, st.o[dt][qc], 0, 0, 0);
                }
        }
        __builtin_amdgcn_sched_barrier(0);
    }
    auto lane_value = [](float x, int i) { return __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(x), i)); };
    if (WHOLE && stage > 0) {
        const int unit_l = unit_at(lane);
        for (uint64_t gone = __ballot(page_l < 0 && unit_l >= u_begin && unit_l < u_stop); gone != 0; gone &= gone - 1) {
            const int u = unit_at(__ffsll((unsigned long long)gone) - 1);
#pragma unroll
            for (int qc = 0; qc < QC; ++qc)
#pragma unroll
                for (int t = 0; t < 4; ++t) keep(qc, f32x4{kNoPage, kNoPage, kNoPage, kNoPage}, u * kBlk + 16 * g + 4 * t);
        }
    }
    if (left != 0) {
        int i = __ffsll((unsigned long long)left) - 1;
        load_v(__builtin_amdgcn_readlane(page_l, i));
        while (true) {
            left &= left - 1;
            const int next = left != 0 ? __ffsll((unsigned long long)left) - 1 : -1;
            const int k0 = unit_at(i) * kBlk;
            wait_direct_loads_but<DT>();                    // K is there: all of the wave's loads but V's, which came behind
            asm volatile("" ::: "memory");
            f32x4 s[4][QC];
            u32x4 kr[2][4];
            auto fetch = [&](int x) {
#pragma unroll
                for (int t = 0; t < 4; ++t) kr[x & 1][t] = *reinterpret_cast<const u32x4*>(own + (krow + 4 * t) * D + 16 * ((4 * x + g) ^ L::swz(krow)));
            };
            fetch(0);
#pragma unroll
            for (int t = 0; t < 4; ++t)
#pragma unroll
                for (int qc = 0; qc < QC; ++qc) s[t][qc] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int x = 0; x < KH; ++x) {
                if (x + 1 < KH) fetch(x + 1);
                __builtin_amdgcn_sched_barrier(0);
#pragma unroll
                for (int t = 0; t < 4; ++t) {
                    const u32x4 w = kr[x & 1][t];
                    const uint2 w0 = F::to_bf16(w.x), w1 = F::to_bf16(w.y), w2 = F::to_bf16(w.z), w3 = F::to_bf16(w.w);
                    Frag f0, f1;
                    f0.u4 = u32x4{w0.x, w0.y, w1.x, w1.y};
                    f1.u4 = u32x4{w2.x, w2.y, w3.x, w3.y};
#pragma unroll
                    for (int qc = 0; qc < QC; ++qc) s[t][qc] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(f0.v, qf[qc][2 * x].v, s[t][qc], 0, 0, 0);
#pragma unroll
                    for (int qc = 0; qc < QC; ++qc) s[t][qc] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(f1.v, qf[qc][2 * x + 1].v, s[t][qc], 0, 0, 0);
                    if (t & 1) __builtin_amdgcn_sched_barrier(0);   // (else all codes are converted ahead, into more registers than there are)
                }
            }
            const float ks = lane_value(ks_l, i), vs = lane_value(vs_l, i);
            const bool masked = k0 + kBlk - 1 > sq.n;       // (row n is the first token's own)
            float mx[QC];
#pragma unroll
            for (int qc = 0; qc < QC; ++qc) {
                mx[qc] = -INFINITY;
#pragma unroll
                for (int t = 0; t < 4; ++t) {
                    s[t][qc] *= ks;
                    if (masked) {
#pragma unroll
                        for (int j = 0; j < 4; ++j)
                            if (k0 + 16 * g + 4 * t + j > st.pos[qc]) s[t][qc][j] = -INFINITY;
                    }
                    mx[qc] = fmaxf(mx[qc], fmaxf(fmaxf(s[t][qc][0], s[t][qc][1]), fmaxf(s[t][qc][2], s[t][qc][3])));
                    keep(qc, s[t][qc], k0 + 16 * g + 4 * t);
                }
            }
            follow(mx);
            // V is there.  Only now may the next K follow it: the compiler does not see direct loads, and would wait for them where it waits for V.
            wait_direct_loads();
            __builtin_amdgcn_sched_barrier(0);
            if (next >= 0) load_k(__builtin_amdgcn_readlane(page_l, next));
            __builtin_amdgcn_sched_barrier(0);
            if (CODE == ST3_BLOCK_E4M3 && masked) {         // codes that are no numbers count as 0 here, and below for the rows that see them
                bool odd = false;
#pragma unroll
                for (int dt = 0; dt < DT; ++dt)
#pragma unroll
                    for (int j = 0; j < 4; ++j) odd |= no_numbers(vr[dt][j]) != 0;
                if (__any(odd)) {
                    odd_at |= 1ull << i;
#pragma unroll
                    for (int dt = 0; dt < DT; ++dt)
#pragma unroll
                        for (int j = 0; j < 4; ++j) {
                            const uint32_t top = no_numbers(vr[dt][j]);
                            vr[dt][j] &= ~(top | (top - (top >> 7)));
                        }
                }
            }
#pragma unroll
            for (int x = 0; x < 2; ++x) {
                Frag hi[QC], lo[QC];
#pragma unroll
                for (int qc = 0; qc < QC; ++qc) weigh(qc, s[2 * x][qc], s[2 * x + 1][qc], vs, hi[qc], lo[qc]);
                __builtin_amdgcn_sched_barrier(0);
#pragma unroll
                for (int d2 = 0; d2 < DT; d2 += 2) {        // two chains of products at a time
                    Frag f[2];
#pragma unroll
                    for (int y = 0; y < 2; ++y) {
                        const uint2 w0 = F::to_bf16(vr[d2 + y][2 * x]), w1 = F::to_bf16(vr[d2 + y][2 * x + 1]);
                        f[y].u4 = u32x4{w0.x, w0.y, w1.x, w1.y};
                    }
#pragma unroll
                    for (int y = 0; y < 2; ++y)
#pragma unroll
                        for (int qc = 0; qc < QC; ++qc) st.o[d2 + y][qc] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(f[y].v, hi[qc].v, st.o[d2 + y][qc], 0, 0, 0);
                    if constexpr (TWO) {
#pragma unroll
                        for (int y = 0; y < 2; ++y)
#pragma unroll
                            for (int qc = 0; qc < QC; ++qc) st.o[d2 + y][qc] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(f[y].v, lo[qc].v, st.o[d2 + y][qc], 0, 0, 0);
                    }
                    __builtin_amdgcn_sched_barrier(0);
                }
            }
            if (next < 0) break;
            load_v(__builtin_amdgcn_readlane(page_l, next));
            __builtin_amdgcn_sched_barrier(0);
            i = next;
        }
    }
    // Such blocks once more, behind the loop: a row's output is NaN in a column whose first such code it sees.  (Products row by row within the loop cost it its
    // registers, 5 to 29 spilled at d = 128: four tokens of 32 sequences over 611 to 3136 rows 29.7 us, 24.4 so; 8 of eight over 20000 to 30000 rows 188 and 115.)
    for (; odd_at != 0; odd_at &= odd_at - 1) {
        const int i = __ffsll((unsigned long long)odd_at) - 1, k0 = unit_at(i) * kBlk;
        const uint8_t* v = a.c.v_codes + ((int64_t)__builtin_amdgcn_readlane(page_l, i) * a.Hk + kh) * (kBlk * D);
#pragma unroll
        for (int dt = 0; dt < DT; ++dt)
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const uint32_t* col = reinterpret_cast<const uint32_t*>(v + (16 * dt + 4 * g + j) * kBlk);
                int from = 0x7fffffff;
#pragma unroll 1
                for (int w = kBlk / 4 - 1; w >= 0; --w) {
                    const uint32_t top = no_numbers(col[w]);
                    from = top != 0 ? k0 + 4 * w + (__ffs(top) - 1) / 8 : from;
                }
#pragma unroll
                for (int qc = 0; qc < QC; ++qc)
                    if (from <= st.pos[qc]) st.o[dt][qc][j] = __uint_as_float(0x7fc00000u);
            }
    }
    // what the first rows have received so far, on its way while the waves' parts are joined
    constexpr int kAhead = 4;
    float* score = a.score + b * a.s_sb + kh * a.s_sh;
    float old[kAhead] = {};
    if (WHOLE && stage > 0 && sq.n > 0) {
#pragma unroll
        for (int j = 0; j < kAhead; ++j) old[j] = score[min(tid + j * kThr, sq.n - 1)];
    }
    // ---- the waves' parts ---------------------------------------------------------------------------------------------------------
    __syncthreads();                                        // (no wave reads its keys any more)
#pragma unroll
    for (int qc = 0; qc < QC; ++qc) {
        const float l = wave_sum_from<16>(st.l[qc]);
        const int col = 16 * qc + c;
        if (col >= rows) continue;
        if (g == 0) { sm_m[wave * cols + col] = st.m[qc]; sm_l[wave * cols + col] = l; }
#pragma unroll
        for (int dt = 0; dt < DT; ++dt) *reinterpret_cast<f32x4*>(sm_o + (wave * cols + col) * OS + 16 * dt + 4 * g) = st.o[dt][qc];
    }
    __syncthreads();
    for (int e = tid; e < rows * (D / 2); e += kThr) {      // two columns of a row
        const int col = e / (D / 2), dim = 2 * (e % (D / 2)), t = (r0 + col) / a.G, h = kh * a.G + r0 + col - t * a.G;
        float top = sm_m[col];
#pragma unroll
        for (int w = 1; w < WAVES; ++w) top = fmaxf(top, sm_m[w * cols + col]);
        float sum = 0.f, x = 0.f, y = 0.f;
#pragma unroll
        for (int w = 0; w < WAVES; ++w) {
            const float f = exp2_fast(sm_m[w * cols + col] - top);
            const f32x2 o = *reinterpret_cast<const f32x2*>(sm_o + (w * cols + col) * OS + dim);
            sum = fmaf(sm_l[w * cols + col], f, sum);
            x = fmaf(o.x, f, x);
            y = fmaf(o.y, f, y);
        }
        const int64_t row = (int64_t)(sq.start + t) * a.H + h;
        if constexpr (WHOLE) {
            const float rl = sum == 0.f ? 0.f : 1.0f / sum;     // (a sum of NaN stays one)
            *reinterpret_cast<uint32_t*>(a.out + (int64_t)(sq.start + t) * a.o_st + (int64_t)h * a.o_sh + dim) = bf16_pair(x * rl, y * rl);
            if (dim == 0) {
                sm_h[2 * col] = top;
                sm_h[2 * col + 1] = rl;
                if (stage == 0 && a.ml != nullptr) a.ml[row] = make_float2(top, rl);
            }
        } else {
            *reinterpret_cast<f32x2*>(a.part_o + (row * a.pieces + ch) * D + dim) = f32x2{x, y};
            if (dim == 0) a.part_ml[row * a.pieces + ch] = make_float2(top, sum);
        }
    }
    if (!WHOLE || stage == 0) return;
    __syncthreads();
    const int first = max(0, sq.m - a.window) * a.G;
    auto weight = [&](int key) {
        const int from = (key - sq.n) * a.G;                // (the rows of the tokens that see the key)
        float w = 0.f;
#pragma unroll 4
        for (int col = first; col < rows; ++col) {
            const float s = staged[col * stage + key];
            const f32x2 h = *reinterpret_cast<const f32x2*>(sm_h + 2 * col);
            const float p = exp2_fast(s - h.x) * h.y;
            w += col < from || s == kNoPage ? 0.f : p;
        }
        return w;
    };
#pragma unroll
    for (int j = 0; j < kAhead; ++j) {
        const int key = tid + j * kThr;
        if (key < keys) score[key] = (key < sq.n ? old[j] : 0.f) + weight(key);
    }
    for (int key = tid + kAhead * kThr; key < keys; key += kThr) score[key] = (key < sq.n ? score[key] : 0.f) + weight(key);
}

// ---------------------------------------------------------------------------------------------------------------------------------
// Behind the pieces: a wave joins a row's parts, eight loads on their way (1952 rows of up to 16 parts: 9.8 us).
// ---------------------------------------------------------------------------------------------------------------------------------
template <int D>
__global__ __launch_bounds__(256) void chunk_join_kernel(ChunkArgs a) {
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int64_t x = (int64_t)blockIdx.x * 4 + wave;
    const int row = (int)(x / a.H), h = (int)(x % a.H);
    if (row >= a.total) return;
    // whose row it is: the sequence that begins last among those that begin at it or before (empty ones begin where the next one does)
    int b = -1, start = 0;
    for (int i0 = 0; i0 < a.B; i0 += kWave) {
        const int s = i0 + lane < a.B ? max(0, min(a.cu[i0 + lane], a.total)) : 0x7fffffff;
        const uint64_t before = __ballot(s <= row);
        if (before == 0) break;
        b = i0 + 63 - __clzll(before);
        start = __builtin_amdgcn_readlane(s, 63 - __clzll(before));
        if (before != ~0ull) break;
    }
    if (b < 0) return;
    const Turn sq = turn_of(a, b);
    if (row - start >= sq.m) return;
    const int units = (sq.sees(row - start) + kBlk) / kBlk, parts = max(1, (units + a.piece - 1) / a.piece);
    const int64_t at = ((int64_t)row * a.H + h) * a.pieces;
    float top = -3.402823466e38f;
    for (int i = lane; i < parts; i += kWave) top = fmaxf(top, a.part_ml[at + i].x);
    top = wave_max_from<1>(top);
    constexpr int PER = D / 64;
    float sum = 0.f, v[PER] = {};
    for (int i0 = 0; i0 < parts; i0 += kWave) {             // lane i has part i0 + i's factor; the parts' loads go out eight at a time
        const int here = min(kWave, parts - i0);
        const float2 ml = lane < here ? a.part_ml[at + i0 + lane] : make_float2(top, 0.f);
        const float f_l = exp2_fast(ml.x - top);
        sum = fmaf(ml.y, f_l, sum);
        const float* from = a.part_o + (at + i0) * D + PER * lane;
#pragma unroll 8
        for (int i = 0; i < here; ++i) {
            const float f = __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(f_l), i));
#pragma unroll
            for (int e = 0; e < PER; ++e) v[e] = fmaf(from[(int64_t)i * D + e], f, v[e]);
        }
    }
    sum = wave_sum_from<1>(sum);
    const float rl = sum == 0.f ? 0.f : 1.0f / sum;
    uint16_t* out = a.out + (int64_t)row * a.o_st + (int64_t)h * a.o_sh + PER * lane;
    if constexpr (PER == 2) *reinterpret_cast<uint32_t*>(out) = bf16_pair(v[0] * rl, v[1] * rl);
    else *out = (uint16_t)bf16_pair(v[0] * rl, 0.f);
    if (a.ml != nullptr && lane == 0) a.ml[(int64_t)row * a.H + h] = make_float2(top, rl);
}

// ---------------------------------------------------------------------------------------------------------------------------------
// Scores: the logits of the window's rows are formed again.  Workgroup (key head, strip of 4 x rounds blocks, sequence): the rows, up to kScoreRows of them,
// lie in LDS; a wave has the 64 keys of a block in registers, meets 16 rows at a time, and a lane adds up what its 16 keys get.  SHARED: a workgroup has one
// block, and its waves every fourth 16 of the rows; their sums are added in one order.  Three waves of a SIMD hide
// each other's loads of codes better than two that have the next block's codes on their way (those need the registers): a call with 16 tokens' windows over
// 202000 rows took 303 us so and 314 with two, before its other launches became as fast as they are (274).  At d = 128 LDS has room for three workgroups of up to
// 192 rows each; with more, as in windows of 64 tokens of groups of 4, there are two (2048 tokens over 30000 rows: 31 to 36 us of scores).
// ---------------------------------------------------------------------------------------------------------------------------------
constexpr int kScoreRows = 256;         // rows in LDS at a time: 64 KB at d = 128

// Rows in LDS, of a launch whose windows hold `rows` at most.
inline int score_rows(int64_t rows) { return (int)std::min<int64_t>((rows + 15) / 16 * 16, kScoreRows); }

template <int D, int CODE, bool SHARED>
__global__ __launch_bounds__(256, 3) void chunk_score_kernel(ChunkArgs a, int rounds, int fit) {
    using F = BlockCode<CODE>;
    constexpr int KS = D / 32, KH = D / 64, UPR = D / 8;    // contraction steps; 16-byte pieces of codes in a key's row for a lane; units of a row
    extern __shared__ __attribute__((aligned(16))) uint8_t lds[];
    __shared__ float part[4][kBlk];
    u32x4* sm_q = reinterpret_cast<u32x4*>(lds);            // [fit][UPR], unit u of row r at u ^ r: 16 rows' units lie in 16 units of the banks
    float2* sm_ml = reinterpret_cast<float2*>(lds + (size_t)fit * 2 * D);
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), g = lane >> 4, c = lane & 15;
    const int kh = blockIdx.x, n_units = SHARED ? 1 : 4 * rounds, u0 = blockIdx.y * n_units, b = blockIdx.z;
    const Turn sq = turn_of(a, b);
    const int keys = sq.rows(), blocks = keys / kBlk, units = (keys + kBlk - 1) / kBlk;
    if (sq.n < 0 || sq.m <= 0 || u0 >= units) return;
    const int64_t strip = (int64_t)b * a.Hk + kh;
    const int u_end = min(units, u0 + n_units);
    // lane i has the page and the scale of the wave's i-th block
    int page_l = -1;
    float ks_l = 0.f;
    {
        const int u = SHARED ? u0 : u0 + wave + 4 * lane;
        if (lane < rounds && u < u_end && u < blocks) page_l = page_of(a.c, b, u);
        if (page_l >= 0) ks_l = a.c.k_scale[(int64_t)page_l * a.Hk + kh];
    }
    // key 16 x + c; a lane's columns are 64 y + 16 g .. + 15, in two steps
    u32x4 raw[4][KH];
    const uint32_t k_lane = (uint32_t)(c * D + 16 * g);
    auto fetch = [&](int i) {                               // (page -1: whatever; it is not used)
        const int page = max(__builtin_amdgcn_readlane(page_l, i), 0);
        const auto rsrc = __builtin_amdgcn_make_buffer_rsrc(a.c.k_codes + ((int64_t)page * a.Hk + kh) * (kBlk * D), 0, kBlk * D, 0x00020000);
#pragma unroll
        for (int x = 0; x < 4; ++x)
#pragma unroll
            for (int y = 0; y < KH; ++y) raw[x][y] = __builtin_amdgcn_raw_buffer_load_b128(rsrc, k_lane, 16 * x * D + 64 * y, 0);
    };
    const int rows = sq.m * a.G, first = max(0, sq.m - a.window) * a.G;
    auto stage = [&](int r0) {                              // rows r0 .. into LDS
#pragma unroll 4
        for (int e = tid; e < fit * UPR; e += 256) {
            const int x = e / UPR, r = min(r0 + x, rows - 1), t = r / a.G;
            const uint16_t* row = a.q + (int64_t)(sq.start + t) * a.q_st + (int64_t)(kh * a.G + r - t * a.G) * a.q_sh;
            sm_q[x * UPR + (e % UPR ^ (D == 128 ? x & 15 : x >> 1 & 7))] = reinterpret_cast<const u32x4*>(row)[e % UPR];
        }
#pragma unroll 1
        for (int x = tid; x < fit; x += 256) {
            const int r = min(r0 + x, rows - 1), t = r / a.G;
            sm_ml[x] = r0 + x < rows ? a.ml[(int64_t)(sq.start + t) * a.H + kh * a.G + r - t * a.G] : make_float2(0.f, 0.f);
        }
    };
    stage(first);
    __syncthreads();
    const bool all_fit = rows - first <= fit;               // (else every round takes the rows piece by piece)
#pragma unroll 1
    for (int i = 0; i < rounds; ++i) {
        const int u = SHARED ? u0 : u0 + wave + 4 * i;
        if (all_fit && u >= u_end) break;
        const bool tail = u == blocks && u < u_end, there = tail || __builtin_amdgcn_readlane(page_l, i) >= 0;
        const float ks = tail ? a.scale_l2 : __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(ks_l), i)) * a.scale_l2;
        fetch(i);
        Frag kf[4][KS];
        if (tail) {
            const uint16_t* from = a.c.k_tail + strip * (kBlk * D);
#pragma unroll
            for (int x = 0; x < 4; ++x)
#pragma unroll
                for (int s = 0; s < KS; ++s) kf[x][s].u4 = *reinterpret_cast<const u32x4*>(from + (16 * x + c) * D + 64 * (s / 2) + 16 * g + 8 * (s & 1));
        } else {
#pragma unroll
            for (int x = 0; x < 4; ++x)
#pragma unroll
                for (int y = 0; y < KH; ++y) {
                    const u32x4 w = raw[x][y];
                    const uint2 w0 = F::to_bf16(w.x), w1 = F::to_bf16(w.y), w2 = F::to_bf16(w.z), w3 = F::to_bf16(w.w);
                    kf[x][2 * y].u4 = u32x4{w0.x, w0.y, w1.x, w1.y};
                    kf[x][2 * y + 1].u4 = u32x4{w2.x, w2.y, w3.x, w3.y};
                }
        }
        __builtin_amdgcn_sched_barrier(0);
        const int key = u * kBlk + lane;
        float* to = a.score + b * a.s_sb + kh * a.s_sh + key;
        const float old = u < u_end && key < sq.n && (!SHARED || wave == 0) ? *to : 0.f;
        __builtin_amdgcn_sched_barrier(0);
        f32x4 sum[4];
#pragma unroll
        for (int x = 0; x < 4; ++x) sum[x] = f32x4{0.f, 0.f, 0.f, 0.f};
        for (int r0 = first;;) {
            const int here = min(fit, rows - r0);
            if (there) {
                // 16 rows, this lane's the one of column c: logits, weights
                auto add = [&](int x0, auto masked) {
                    const float2 ml = sm_ml[x0 + c];
                    // keys of the block that the row sees, those of this lane's first (a row that does not exist sees none)
                    const int seen = !decltype(masked)::value ? 0 : x0 + c < here ? sq.n + (r0 + x0 + c) / a.G + 1 - u * kBlk - 4 * g : -kBlk;
                    Frag qf[KS];
#pragma unroll
                    for (int s = 0; s < KS; ++s)
                        qf[s].u4 = sm_q[(x0 + c) * UPR + ((8 * (s / 2) + 2 * g + (s & 1)) ^ (D == 128 ? c : (x0 + c) >> 1 & 7))];
#pragma unroll
                    for (int x = 0; x < 4; ++x) {
                        f32x4 y = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
                        for (int s = 0; s < KS; ++s) y = __builtin_amdgcn_mfma_f32_16x16x32_bf16(kf[x][s].v, qf[s].v, y, 0, 0, 0);
#pragma unroll
                        for (int j = 0; j < 4; ++j) {
                            const float p = exp2_fast(fmaf(y[j], ks, -ml.x));
                            if constexpr (decltype(masked)::value) {
                                sum[x][j] += 16 * x + j < seen ? p * ml.y : 0.f;
                            } else {
                                sum[x][j] = fmaf(p, ml.y, sum[x][j]);
                            }
                        }
                        if (x & 1) __builtin_amdgcn_sched_barrier(0);       // (else all products are kept at once)
                    }
                };
                int x0 = SHARED ? 16 * wave : 0;
                constexpr int kStep = SHARED ? 64 : 16;
                if (u * kBlk + kBlk - 1 <= sq.n + r0 / a.G) {       // every row sees the whole block
#pragma unroll 1
                    for (; x0 + 16 <= here; x0 += kStep) add(x0, std::false_type{});
                }
#pragma unroll 1
                for (; x0 < here; x0 += kStep) add(x0, std::true_type{});
            }
            r0 += fit;
            if (r0 >= rows) break;
            __syncthreads();
            stage(r0);
            __syncthreads();
        }
        if (!all_fit && i + 1 < rounds) {                   // the next round begins with the first rows again
            __syncthreads();
            stage(first);
            __syncthreads();
        }
        if (u >= u_end) continue;
#pragma unroll
        for (int x = 0; x < 4; ++x)
#pragma unroll
            for (int j = 0; j < 4; ++j) sum[x][j] = group_sum<16>(sum[x][j]);
        if (c == 0) {
#pragma unroll
            for (int x = 0; x < 4; ++x) *reinterpret_cast<f32x4*>(&part[wave][16 * x + 4 * g]) = sum[x];
        }
        if constexpr (SHARED) {
            __syncthreads();
            if (wave == 0 && key < keys) *to = old + ((part[0][lane] + part[1][lane]) + (part[2][lane] + part[3][lane]));
        } else {
            __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
            if (key < keys) *to = old + part[wave][lane];   // (written by this wave)
        }
    }
}

// How a call is cut: rows of a tile, blocks of a piece, pieces; waves of a workgroup where rows are few (else 0), and rows of a strip whose logits fit in LDS.
// No more workgroups than compute units: a second one would wait for the first, with products of its own to begin and to join (33 tokens over 131072 rows:
// 178 us with 512 of them, 158 with 256; 64 over 30000: 91 and 68).
struct ChunkCut { int rows, piece, pieces, few, stage, groups; };
constexpr int kMostRowsOfTile = 32 * kChunkWaves;
constexpr int kWanted = 256;            // workgroups that a cut aims at: one has a compute unit's LDS to itself
constexpr int kLeastPiece = 4;
// Few rows, up to kFewRows: every wave has those of its group, kFewGroup at most (8 key heads, d = 128: 4 tokens of 32 sequences over 611 to 3136 rows 27 us,
// by tiles 56; 8 of one over 30000 rows 23 and 37).  Two groups read a strip twice, the second time from L2: 16 tokens (64 rows) of 8 sequences over 20000 to
// 30000 rows 127 us, by tiles 159; three would not pay (24 tokens of them 199, by tiles 155).
//   whole strips, without a join, and with one group's weights added at once, where there are kWholeStrips of them or they have no more than kShortUnits
//     blocks: 4 tokens of 64 sequences of 1000 to 3000 rows 51 us, in pieces 57; 5 of one of 744 rows 16.2 and 19.3; 4 of 16 sequences 36.3, in pieces 34.4.
//     By 12 waves (8 with more than 16 rows), by 4 where there are more than kManyStrips: 32 sequences 27.5 us by 12 and 28.6 by 4, 64 sequences 52.3 and
//     51.0, with 8 tokens 65 and 61.
//   pieces by 4 waves: of no more than kWanted / 4 strips one for each compute unit (8 tokens over 30000 rows 23 us, three times as many pieces 40; of eight
//     sequences 82 and 95), of more strips, whose lengths differ, three times as many (4 tokens of 15 sequences of 1000 to 9000 rows 38.8 us, two pieces each 39.7).
//     A wave's blocks are lanes of a register, no more than kMostPiece; longer strips in twice, three times as many pieces (4 tokens of 8 sequences over
//     70000 to 131072 rows 276 us, in as few as hold them 302, measured with one term of weights).
constexpr int kFewGroup = 32, kFewRows = 64, kWholeStrips = 192, kShortUnits = 20, kManyStrips = 256, kMostPiece = 4 * kWave - 2;

// Room for as many parts as a launch of these or any smaller sizes may leave.  Tiles hold all rows, so kWanted / tiles pieces are no more than kWanted tiles
// of parts (with few rows: than three times as many of kFewGroup, or a few for every kMostPiece blocks); nor are there more than one for every kLeastPiece
// blocks.  (Where that is not enough, as for a batch with many more rows than its sequences have, there are fewer pieces.)
inline int64_t chunk_parts(int64_t rows, int64_t units) {
    return std::min((int64_t)kWanted * kMostRowsOfTile + rows * (1 + (units + kMostPiece - 1) / kMostPiece), rows * ((units + kLeastPiece - 1) / kLeastPiece));
}

// most_pieces: that there is room for
template <int D>
inline ChunkCut few_cut(int64_t strips, int most, int max_len, bool scored, int64_t most_pieces) {
    constexpr size_t kLds = 160 << 10;
    const int64_t units = max_len / kBlk + 1;
    const int groups = (most + kFewGroup - 1) / kFewGroup, cols = (most + groups - 1) / groups;
    strips *= groups;                       // (workgroups of a whole launch)
    const int waves = strips > kManyStrips ? 4 : cols <= 16 ? 12 : 8;
    if (units + 2 <= waves * kWave && (strips >= kWholeStrips || units <= kShortUnits)) {
        const bool staged = scored && groups == 1 && FewLds<D>(waves, cols).bytes(cols, units * kBlk) <= kLds;
        return ChunkCut{cols, (int)units, 1, waves, staged ? (int)units * kBlk : 0, groups};
    }
    const int64_t even = strips <= kWanted / 4 ? kWanted / strips : (3 * kWanted + strips - 1) / strips, pieces = even * ((units + even * kMostPiece - 1) / (even * kMostPiece));
    const int64_t piece = std::max((int64_t)kLeastPiece, (units + std::min(pieces, most_pieces) - 1) / std::min(pieces, most_pieces));
    return ChunkCut{cols, (int)piece, (int)((units + piece - 1) / piece), 4, 0, groups};
}

// No more row tiles than this, whatever the lengths are: each sequence has one that is not full.
inline int64_t chunk_tiles(const st3_gqa_shape* s, int total, int max_new, int rows) {
    const int G = s->heads / s->kv_heads;
    return std::min((int64_t)total * G / rows + std::min(s->batch, total), ((int64_t)max_new * G + rows - 1) / rows * s->batch);
}
// The longest sequence's rows in as few tiles as hold them, all alike.
inline int tile_rows(int64_t most) {
    const int64_t tiles = (most + kMostRowsOfTile - 1) / kMostRowsOfTile;
    return tiles == 0 ? 16 : (int)((most + 16 * tiles - 1) / (16 * tiles) * 16);
}
// (total and max_new above zero)
inline ChunkCut chunk_cut(const st3_gqa_shape* s, int total, int max_new, int max_len, bool scored) {
    const int64_t most = (int64_t)max_new * (s->heads / s->kv_heads), strips = (int64_t)s->batch * s->kv_heads;
    const int64_t units = max_len / kBlk + 1, most_pieces = chunk_parts((int64_t)total * s->heads, units) / ((int64_t)total * s->heads);
    if (most <= kFewRows) return s->head_dim == 128 ? few_cut<128>(strips, (int)most, max_len, scored, most_pieces) : few_cut<64>(strips, (int)most, max_len, scored, most_pieces);
    const int rows = tile_rows(most);
    const int64_t tiles = chunk_tiles(s, total, max_new, rows) * s->kv_heads;
    if (2 * tiles >= kWanted) return ChunkCut{rows, (int)units, 1, 0, 0, 0};
    const int64_t pieces = std::min({kWanted / tiles, (units + kLeastPiece - 1) / kLeastPiece, most_pieces});
    const int64_t piece = (units + pieces - 1) / pieces;
    return ChunkCut{rows, (int)piece, (int)((units + piece - 1) / piece), 0, 0, 0};
}

// Blocks that a wave of the scores' launch takes one behind the other: as many as leave three workgroups for each compute unit, which hold its registers
// (9 to 33 tokens over 70000 to 131072 rows 274 us, with four 284, with two 286); their pages are lanes of a register (4 x 130000 rows 297 us, no more
// than 16 blocks a wave 311).
// Where there are fewer blocks than compute units, a workgroup's waves share one and deal out the rows (7 x 626 tokens, 1024 rows of each in the window: the
// call 62 us, 85 by a block a wave; 100 tokens behind 1000 rows 29.4 and 31.0; with 576 blocks 41.1 and 40.1).
constexpr int kScoreWgs = 768, kMostRounds = kWave;
inline int score_rounds(int64_t units, int Hk, int B) {
    const int64_t want = units * Hk * B / (4 * kScoreWgs);
    return (int)std::max<int64_t>(1, std::min<int64_t>(want, kMostRounds));
}

struct ChunkWs { size_t ml, part_o, part_ml, total; };
inline ChunkWs chunk_ws(const st3_gqa_shape* s, int total, int max_len) {
    const int64_t rows = (int64_t)total * s->heads, parts = chunk_parts(rows, max_len / kBlk + 1);
    ChunkWs w{};
    size_t off = 0;
    w.ml = off;      off = align_up(off + rows * sizeof(float2), 256);
    w.part_o = off;  off = align_up(off + parts * s->head_dim * sizeof(float), 256);
    w.part_ml = off; off = align_up(off + parts * sizeof(float2), 256);
    w.total = off;
    return w;
}

template <int D, int CODE, int QC, bool TWO>
void launch_few(const ChunkArgs& a, const ChunkCut& cut, hipStream_t st) {
    const size_t lds = FewLds<D>(cut.few, a.tile).bytes(a.tile, cut.stage);
    const dim3 grid(a.Hk * cut.groups, a.pieces, a.B);
    constexpr int kMost = QC == 1 ? 12 : 8;
    if (a.pieces > 1) chunk_few_kernel<D, CODE, QC, 4, false, TWO><<<grid, 256, lds, st>>>(a, 0);
    else if (cut.few == kMost) chunk_few_kernel<D, CODE, QC, kMost, true, TWO><<<grid, 64 * kMost, lds, st>>>(a, cut.stage);
    else chunk_few_kernel<D, CODE, QC, 4, true, TWO><<<grid, 256, lds, st>>>(a, cut.stage);
}

template <int D, int CODE>
void launch_chunk(const ChunkArgs& a, const ChunkCut& cut, unsigned grid, hipStream_t st) {
    if (cut.few > 0 && a.tile <= 16) launch_few<D, CODE, 1, true>(a, cut, st);          // (two groups have more than 16 each)
    else if (cut.few > 0) cut.groups == 1 ? launch_few<D, CODE, 2, true>(a, cut, st) : launch_few<D, CODE, 2, false>(a, cut, st);
    else if (a.tile <= 16 * kChunkWaves) block_chunk_kernel<D, CODE, 1><<<dim3(grid, a.pieces), kChunkThreads, 0, st>>>(a);
    else block_chunk_kernel<D, CODE, 2><<<dim3(grid, a.pieces), kChunkThreads, 0, st>>>(a);
    if (a.pieces > 1) chunk_join_kernel<D><<<(unsigned)(((int64_t)a.total * a.H + 3) / 4), 256, 0, st>>>(a);
    if (!a.score || a.max_len == 0 || cut.stage > 0) return;
    const int fit = score_rows((int64_t)std::min(a.window, a.max_new) * a.G), units = (a.max_len + kBlk - 1) / kBlk, rounds = score_rounds(units, a.Hk, a.B);
    const size_t lds = fit * (2 * D + sizeof(float2));
    if ((int64_t)units * a.Hk * a.B <= kWanted && fit > 16) chunk_score_kernel<D, CODE, true><<<dim3(a.Hk, units, a.B), 256, lds, st>>>(a, 1, fit);
    else chunk_score_kernel<D, CODE, false><<<dim3(a.Hk, (units + 4 * rounds - 1) / (4 * rounds), a.B), 256, lds, st>>>(a, rounds, fit);
}

}  // namespace
}  // namespace st3

extern "C" size_t st3_block_attend_workspace_bytes(const st3_gqa_shape* shape, int32_t total, int32_t max_new, int32_t max_len) {
    if (st3::check_gqa_shape(shape) != ST3_OK || total < 0 || max_new < 0 || max_len < 0) return 0;
    return std::max<size_t>(256, st3::chunk_ws(shape, total, max_len).total);
}

extern "C" st3_status st3_block_attend(const st3_gqa_shape* shape, const st3_rows* q, const int32_t* cu_len, int32_t total, int32_t max_new,
                                       const st3_block_cache* cache, int32_t max_len, const st3_rows* out, int32_t window, float* score,
                                       int64_t score_stride_b, int64_t score_stride_h, void* workspace, size_t workspace_bytes, void* stream) {
    using namespace st3;
    st3_status s = check_gqa_shape(shape);
    if (s != ST3_OK) return s;
    if ((s = check_block_cache(shape, cache)) != ST3_OK) return s;
    const int B = shape->batch, H = shape->heads, Hk = shape->kv_heads, D = shape->head_dim, G = H / Hk;
    if (!cu_len || total < 0 || max_new < 0 || max_new > total || max_len < 0 || window < 0) return ST3_ERR_INVALID_ARG;
    if (max_len > kMostRows || (int64_t)max_new * G > kMostRows) return ST3_ERR_UNSUPPORTED;
    if (total == 0) return ST3_OK;          // (an empty tensor may have no address)
    if ((s = check_rows(q, D, 2)) != ST3_OK || (s = check_output(out, H, total, D, 2)) != ST3_OK) return s;
    if (max_new == 0) return ST3_OK;
    if (cache->table_blocks < max_len / kBlk) return ST3_ERR_INVALID_ARG;
    if (packed_rows_meet(q, H, out, H, total, D, 2)) return ST3_ERR_INVALID_ARG;
    if (score && (window < 1 || score_stride_h < max_len || (B > 1 && score_stride_b < max_len))) return ST3_ERR_INVALID_ARG;
    if (!workspace || !aligned16(workspace)) return ST3_ERR_INVALID_ARG;
    const ChunkCut cut = chunk_cut(shape, total, max_new, max_len, score != nullptr);
    const int64_t grid = cut.few > 0 ? Hk * cut.groups : chunk_tiles(shape, total, max_new, cut.rows) * Hk;
    if (!grid_fits(grid, kChunkThreads, cut.pieces) || (cut.pieces > 1 && !grid_fits(((int64_t)total * H + 3) / 4, 256, 1)) || (score && (max_len + 4 * kBlk - 1) / (4 * kBlk) > 65535)) return ST3_ERR_UNSUPPORTED;
    const ChunkWs wl = chunk_ws(shape, total, max_len);
    if (workspace_bytes < st3_block_attend_workspace_bytes(shape, total, max_new, max_len)) return ST3_ERR_WORKSPACE_TOO_SMALL;
    char* ws = reinterpret_cast<char*>(workspace);
    ChunkArgs a{};
    a.c = block_pages(cache);
    a.q = reinterpret_cast<const uint16_t*>(q->data); a.out = reinterpret_cast<uint16_t*>(out->data);
    a.q_st = q->stride_t; a.q_sh = q->stride_h; a.o_st = out->stride_t; a.o_sh = out->stride_h;
    a.cu = cu_len; a.B = B; a.total = total; a.max_new = max_new; a.max_len = max_len; a.H = H; a.Hk = Hk; a.G = G;
    a.tile = cut.rows; a.piece = cut.piece; a.pieces = cut.pieces;
    a.scale_l2 = gqa_scale_log2(shape);
    a.score = score; a.s_sb = score_stride_b; a.s_sh = score_stride_h; a.window = window;
    a.ml = score ? reinterpret_cast<float2*>(ws + wl.ml) : nullptr;
    a.part_o = reinterpret_cast<float*>(ws + wl.part_o);
    a.part_ml = reinterpret_cast<float2*>(ws + wl.part_ml);
    hipStream_t st = reinterpret_cast<hipStream_t>(stream);
    if (cache->code == ST3_BLOCK_INT8) {
        if (D == 128) launch_chunk<128, ST3_BLOCK_INT8>(a, cut, (unsigned)grid, st);
        else launch_chunk<64, ST3_BLOCK_INT8>(a, cut, (unsigned)grid, st);
    } else {
        if (D == 128) launch_chunk<128, ST3_BLOCK_E4M3>(a, cut, (unsigned)grid, st);
        else launch_chunk<64, ST3_BLOCK_E4M3>(a, cut, (unsigned)grid, st);
    }
    return check_launch();
}
