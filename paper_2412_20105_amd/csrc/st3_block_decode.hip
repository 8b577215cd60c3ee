// Attention of single tokens over a cache of 8-bit blocks, with grouped heads, appended rows and accumulated weights.
//
// A workgroup of four or twelve waves takes a chunk of the blocks of one (sequence, key head), or the whole strip; a wave takes a block of 64 keys at
// a time, with v_mfma_f32_16x16x32_bf16 (A: lane (c, g) holds A[c][8g..8g+7], B: B[8g..8g+7][c], C: C[4g..4g+3][c]); the group's query heads are the
// columns (up to 16; a larger group is several workgroups).  8-bit codes have at most 8 significant bits: exact in bf16, so the products are exact,
// and the block's scale multiplies the finished sums.
//   S^T = K Q^T    product t of four: row 4g'+i of A is key 16 g' + 4 t + i, so that lane (c, g) of C ends with keys 16 g .. 16 g + 15 of query c.
//                  A lane reads 16 codes of its row at once: columns 64 x + 16 g .. + 15, contraction steps 2 x and 2 x + 1.
//   O^T = V^T P^T  the lane's 16 keys are the contraction slots 8g..8g+7 of two steps: P^T is where S^T left it, and V^T, whose rows lie in
//                  memory, is read 16 codes at a time too.  P is two bf16 terms (16 significant bits: what is left out is 2^-16 of a weight at most).
// No value crosses lanes but the maximum.  Bound by memory: K goes straight to LDS, a block ahead, V into registers.  2 sequences of 70000 and
// 131072 rows, 32 heads over 8 of 128: 489 MB in 107 us, 4.6 TB/s (a large copy: 4.8); 32 of 611 to 3136 rows, 114 MB in 28.5 us.
#include <algorithm>

#include "st3_block.h"

namespace st3 {
namespace {

constexpr int kCols = 16;               // query heads of a workgroup
constexpr int kStream = 2;              // cache policy of a load: read once, "nt"

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

// A block's K lies in a wave's own LDS, rows of D bytes, the 16-byte units of a row permuted: unit u of row r is at u ^ swz(r), so that the 16 rows
// that a fragment's lanes read (16 (c / 4) + c % 4 + 4 t) lie in 16 different units of the banks.
template <int D> struct KeyTile {
    static constexpr int UPR = D / 16, RPI = 1024 / D, NI = kBlk / RPI;     // units of a row; rows of a wave-wide load; loads of a block
    __device__ static __forceinline__ int swz(int row) { return D == 128 ? ((row >> 4 & 3) << 1 | (row >> 1 & 1)) : row >> 4 & 3; }
};

// Dynamic LDS: the waves' K blocks, and where those were the waves' outputs [waves][columns][D + 4], their maxima and sums [2][waves][16], the heads'
// [2][16], and in a launch of whole strips the logits [columns][rows].
template <int D>
inline size_t attend_lds(int waves, int cols, int64_t staged_rows) {
    const size_t keys = (size_t)waves * kBlk * D, parts = sizeof(float) * waves * cols * (D + 4);
    return std::max(keys, parts) + sizeof(float) * (2 * waves * kCols + 2 * kCols + (size_t)cols * staged_rows);
}

// WHOLE: a workgroup takes the whole strip, writes the output itself and, from logits that it kept in LDS, the weights.  Else it takes a chunk, and
// leaves a part of the output and the logits of its keys for the launch behind.
template <int D, int CODE, int WAVES, bool WHOLE>
__global__ __launch_bounds__(WAVES * 64, 3) void block_attend_kernel(BlockDecodeArgs a) {
    using F = BlockCode<CODE>;
    constexpr int KS = D / 32, DT = D / 16, KH = D / 64;    // contraction steps of S, row tiles of O, 16-byte pieces of a K row per lane
    constexpr int kThr = WAVES * 64, OS = D + 4;
    extern __shared__ __attribute__((aligned(16))) float lds[];
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), g = lane >> 4, c = lane & 15;
    const int kh = blockIdx.x / a.QG, q0 = (blockIdx.x % a.QG) * kCols, b = blockIdx.z, ch = blockIdx.y;
    const int nq = min(kCols, a.G - q0), cols = min(kCols, a.G);     // query heads of this workgroup, of the fullest
    float* sm_o = lds;
    constexpr int kKeys = WAVES * kBlk * D / 4;             // floats
    float* sm_m = lds + max(kKeys, WAVES * cols * OS);
    float* sm_l = sm_m + WAVES * kCols;
    float* sm_h = sm_l + WAVES * kCols;                     // a head's maximum, and one over its sum
    float* staged = sm_h + 2 * kCols;                       // [cols][stage_rows]
    const bool fresh = a.k_new != nullptr, scored = a.score != nullptr;
    const int n = __builtin_amdgcn_readfirstlane(min(a.c.len[b], a.max_len));
    const int units = n < 0 ? 0 : units_of(n, fresh), blocks = max(n, 0) / kBlk;
    if (!WHOLE && ch > 0 && ch * a.chunk >= units) return;
    const int h0 = kh * a.G + q0, u_begin = WHOLE ? 0 : ch * a.chunk, u_end = WHOLE ? units : min(units, (ch + 1) * a.chunk);
    const int hq = h0 + min(c, nq - 1);                     // this lane's query head (columns past the last repeat it)

    using L = KeyTile<D>;
    const int krow = 16 * (c >> 2) + (c & 3);               // + 4 t: the key of row c of product t
    const uint32_t v_lane = (uint32_t)(c * kBlk + 16 * g);
    uint8_t* keys = reinterpret_cast<uint8_t*>(lds) + wave * (kBlk * D);
    u32x4 vr[DT];
    // Direct loads (st3_mfma.h): 1 KB of consecutive rows each, in which a lane chooses the unit that belongs where its 16 bytes land.
    const uint32_t k_lane = (uint32_t)(lane / L::UPR * D + 16 * ((lane % L::UPR) ^ L::swz(lane / L::UPR)));
    const uint32_t keys_at = __builtin_amdgcn_readfirstlane(lds_addr(keys));
    auto load_k = [&](int page) {
        const uint8_t* p = a.c.k_codes + ((int64_t)page * a.Hk + kh) * (kBlk * D);
#pragma unroll
        for (int i = 0; i < L::NI; ++i)                     // (what the first row adds to the permutation of a lane's row comes on top of it)
            direct_load16_stream(p + 1024 * i, k_lane ^ (16 * L::swz(i * L::RPI)), keys_at + 1024 * i);
    };
    // (buffer loads: one base for the block in scalar registers, 32 bits of offset a lane; read once, so past the caches)
    auto load_v = [&](int page) {
        const auto rsrc = __builtin_amdgcn_make_buffer_rsrc(a.c.v_codes + ((int64_t)page * a.Hk + kh) * (kBlk * D), 0, kBlk * D, 0x00020000);
#pragma unroll
        for (int dt = 0; dt < DT; ++dt) vr[dt] = __builtin_amdgcn_raw_buffer_load_b128(rsrc, v_lane, 16 * dt * kBlk, kStream);
    };
    // A wave's work is at the positions wave, wave + WAVES, ...: first the halves of the tail, where it belongs to the chunk, then the chunk's blocks
    // in order.  Lane i has the page and the scales of the block at the wave's i-th position (a chunk has no more than 64 of them; fetched one by one
    // they had to be waited for, and with them every load in flight).  A block without a page is passed over: whatever lies elsewhere is not read.
    const int u_most = WHOLE ? a.max_len / kBlk : min((ch + 1) * a.chunk, a.max_len / kBlk);       // (known before the length has arrived)
    const int u_stop = min(u_end, blocks);
    const bool with_tail = units > blocks && blocks >= u_begin && blocks < u_end;
    const int tail_rows = n % kBlk + (fresh ? 1 : 0), halves = !with_tail ? 0 : tail_rows > 32 ? 2 : 1;
    auto unit_at = [&](int i) { return u_begin + wave + WAVES * i - halves; };      // (less than u_begin: a half of the tail)
    int page_l = -1;
    float ks_l = 0.f, vs_l = 0.f;
    {
        const int unit = unit_at(lane);
        page_l = unit >= u_begin && unit < u_most ? page_of(a.c, b, unit) : -1;
        if (page_l >= 0) {
            const int64_t at = (int64_t)page_l * a.Hk + kh;
            ks_l = a.c.k_scale[at];
            vs_l = a.c.v_scale[at];
        }
    }
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
    // (a chunk's logits wait in LDS too, and leave as whole lines: from the registers they would go 16 bytes a head at a time)
    const int stage_rows = (WHOLE ? a.max_len / kBlk + 1 : a.chunk) * kBlk;
    float* logit = scored && c < nq ? staged + c * stage_rows : nullptr;

    // softmax of 64 keys (s[t][i]: key 16 g + 4 t + i, in the log2 domain) and the weights of V, times vs, as two bf16 terms
    auto keep_logits = [&](const f32x4 (&s)[4], int unit) {
        if (logit != nullptr) {
#pragma unroll
            for (int t = 0; t < 4; ++t) *reinterpret_cast<f32x4*>(logit + (unit - u_begin) * kBlk + 16 * g + 4 * t) = s[t];
        }
    };
    auto follow = [&](const f32x4 (&s)[4]) {                // the reference point of the exponents
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
    };
    auto weigh = [&](const f32x4 &s0, const f32x4 &s1, float scale, Frag& hi, Frag& lo) {
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const float p0 = exp2_fast((j < 2 ? s0 : s1)[2 * (j & 1)] - m), p1 = exp2_fast((j < 2 ? s0 : s1)[2 * (j & 1) + 1] - m);
            l += p0 + p1;
            const float w0 = p0 * scale, w1 = p1 * scale;
            const uint32_t b0 = __float_as_uint(w0), b1 = __float_as_uint(w1);
            hi.w[j] = __builtin_amdgcn_perm(b1, b0, 0x07060302u);
            const f32x2 rest = {w0 - __uint_as_float(b0 & 0xffff0000u), w1 - __uint_as_float(b1 & 0xffff0000u)};
            lo.w[j] = __builtin_bit_cast(uint32_t, __builtin_convertvector(rest, bf16x2));
        }
    };
    const int unit_l = unit_at(lane);
    uint64_t left = __ballot(page_l >= 0 && unit_l < u_stop);          // the wave's positions whose blocks are to come
    if (left != 0) load_k(__builtin_amdgcn_readlane(page_l, __ffsll((unsigned long long)left) - 1));     // (on its way beside the tail)
    __builtin_amdgcn_sched_barrier(0);
    // The rows in 16 bits, and the new one, 32 at a time (product t of two: row 4g'+i of A is key 8 g' + 4 t + i), by the first waves while the
    // others have begun with the blocks.
    if (wave < halves) {
        const int r = n % kBlk, first = 32 * wave;          // rows in the tail, the new row's place; the half's first row
        const int64_t at = ((int64_t)b * a.Hk + kh) * kBlk * D;
        const uint16_t* kt = a.c.k_tail + at;
        const uint16_t* vt = a.c.v_tail + at;
        // (without a new row: any row that exists; what it says is masked)
        const uint16_t* kn = fresh ? a.k_new + (int64_t)b * a.k_st + (int64_t)kh * a.k_sh : kt;
        const uint16_t* vn = fresh ? a.v_new + (int64_t)b * a.v_st + (int64_t)kh * a.v_sh : vt;
        Frag tk[2][KS], tv[DT];
        uint32_t fresh_v[DT];
#pragma unroll
        for (int t = 0; t < 2; ++t) {
            const int key = first + 8 * (c >> 2) + (c & 3) + 4 * t;
            const uint16_t* row = key >= r ? kn : kt + key * D;
#pragma unroll
            for (int i = 0; i < KS; ++i) tk[t][i].u4 = *reinterpret_cast<const u32x4*>(row + 64 * (i / 2) + 16 * g + 8 * (i & 1));
        }
#pragma unroll
        for (int dt = 0; dt < DT; ++dt) {
            fresh_v[dt] = vn[16 * dt + c];
            tv[dt].u4 = *reinterpret_cast<const u32x4*>(vt + (16 * dt + c) * kBlk + first + 8 * g);
        }
        __builtin_amdgcn_sched_barrier(0);                  // (all of that is on its way)
        f32x4 s[4];
        s[2] = s[3] = f32x4{-INFINITY, -INFINITY, -INFINITY, -INFINITY};
#pragma unroll
        for (int t = 0; t < 2; ++t) {
            s[t] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int i = 0; i < KS; ++i) s[t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(tk[t][i].v, qf[i].v, s[t], 0, 0, 0);
            s[t] *= a.scale_l2;
#pragma unroll
            for (int i = 0; i < 4; ++i)
                if (first + 8 * g + 4 * t + i >= tail_rows) s[t][i] = -INFINITY;    // whatever lies there
            if (logit != nullptr) *reinterpret_cast<f32x4*>(logit + (blocks - u_begin) * kBlk + first + 8 * g + 4 * t) = s[t];
        }
        follow(s);
        Frag hi, lo;
        weigh(s[0], s[1], 1.0f, hi, lo);
#pragma unroll
        for (int dt = 0; dt < DT; ++dt) {
            Frag f = tv[dt];
#pragma unroll
            for (int i = 0; i < 8; ++i) {                   // rows that hold nothing weigh nothing, whatever their bits are
                const int key = first + 8 * g + i;
                const uint32_t keep = i & 1 ? 0x0000ffffu : 0xffff0000u;
                if (key >= r) f.w[i / 2] = (f.w[i / 2] & keep) | (key < tail_rows ? fresh_v[dt] << (16 * (i & 1)) : 0u);
            }
            o[dt] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(f.v, hi.v, o[dt], 0, 0, 0);
            o[dt] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(f.v, lo.v, o[dt], 0, 0, 0);
        }
        __builtin_amdgcn_sched_barrier(0);
        if (fresh && q0 == 0 && r / 32 == wave) {
            for (int e = lane; e < D; e += kWave) {
                a.c.k_tail[at + r * D + e] = kn[e];
                a.c.v_tail[at + e * kBlk + r] = vn[e];
            }
        }
    }
    auto lane_value = [](float x, int i) { return __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(x), i)); };
    for (uint64_t gone = __ballot(page_l < 0 && unit_l >= u_begin && unit_l < u_stop); gone != 0; gone &= gone - 1) {
        const f32x4 none = {-INFINITY, -INFINITY, -INFINITY, -INFINITY}, s[4] = {none, none, none, none};
        keep_logits(s, unit_at(__ffsll((unsigned long long)gone) - 1));
    }
    if (left != 0) {
        int i = __ffsll((unsigned long long)left) - 1;
        load_v(__builtin_amdgcn_readlane(page_l, i));
        while (true) {
            left &= left - 1;
            const int next = left != 0 ? __ffsll((unsigned long long)left) - 1 : -1;
            wait_direct_loads_but<DT>();                    // K is there: all of the wave's loads but V's, which came behind
            asm volatile("" ::: "memory");
            f32x4 s[4];
            u32x4 kr[2][4];
            auto fetch = [&](int x) {
#pragma unroll
                for (int t = 0; t < 4; ++t)
                    kr[x & 1][t] = *reinterpret_cast<const u32x4*>(keys + (krow + 4 * t) * D + 16 * ((4 * x + g) ^ L::swz(krow)));
            };
            fetch(0);
#pragma unroll
            for (int t = 0; t < 4; ++t) s[t] = f32x4{0.f, 0.f, 0.f, 0.f};
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
                    s[t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(f0.v, qf[2 * x].v, s[t], 0, 0, 0);
                    s[t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(f1.v, qf[2 * x + 1].v, s[t], 0, 0, 0);
                    if (t & 1) __builtin_amdgcn_sched_barrier(0);   // (else all codes are converted ahead, into more registers than there are)
                }
            }
            const float ks = lane_value(ks_l, i) * a.scale_l2, vs = lane_value(vs_l, i);
#pragma unroll
            for (int t = 0; t < 4; ++t) s[t] *= ks;
            keep_logits(s, unit_at(i));
            follow(s);
            // V is there.  Only now may the next K follow it: the compiler does not see direct loads, and would wait for them where it waits for V.
            wait_direct_loads();
            __builtin_amdgcn_sched_barrier(0);
            if (next >= 0) load_k(__builtin_amdgcn_readlane(page_l, next));
            __builtin_amdgcn_sched_barrier(0);
#pragma unroll
            for (int x = 0; x < 2; ++x) {
                Frag hi, lo;
                weigh(s[2 * x], s[2 * x + 1], vs, hi, lo);
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
                    for (int y = 0; y < 2; ++y) o[d2 + y] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(f[y].v, hi.v, o[d2 + y], 0, 0, 0);
#pragma unroll
                    for (int y = 0; y < 2; ++y) o[d2 + y] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(f[y].v, lo.v, o[d2 + y], 0, 0, 0);
                    __builtin_amdgcn_sched_barrier(0);
                }
            }
            if (next < 0) break;
            load_v(__builtin_amdgcn_readlane(page_l, next));
            __builtin_amdgcn_sched_barrier(0);
            i = next;
        }
    }
    // what the first rows have received so far, on its way while the waves' parts are joined
    constexpr int kAhead = 4;
    float old[kAhead] = {};
    if constexpr (WHOLE) {
        if (scored && n > 0) {
            const float* score = a.score + b * a.s_sb + kh * a.s_sh;
#pragma unroll
            for (int j = 0; j < kAhead; ++j) old[j] = score[min(tid + j * kThr, n - 1)];
        }
    }
    // ---- the waves' parts ---------------------------------------------------------------------------------------------------------
    l = wave_sum_from<16>(l);
    __syncthreads();                                        // (no wave reads its keys any more)
    if (g == 0) { sm_m[wave * kCols + c] = m; sm_l[wave * kCols + c] = l; }
    if (c < nq) {
#pragma unroll
        for (int dt = 0; dt < DT; ++dt) *reinterpret_cast<f32x4*>(sm_o + (wave * cols + c) * OS + 16 * dt + 4 * g) = o[dt];
    }
    __syncthreads();
    for (int e = tid; e < nq * D; e += kThr) {
        const int col = e / D, dim = e % D;
        float top = sm_m[col];
#pragma unroll
        for (int w = 1; w < WAVES; ++w) top = fmaxf(top, sm_m[w * kCols + col]);
        float sum = 0.f, x = 0.f;
#pragma unroll
        for (int w = 0; w < WAVES; ++w) {
            const float f = exp2_fast(sm_m[w * kCols + col] - top);
            sum = fmaf(sm_l[w * kCols + col], f, sum);
            x = fmaf(sm_o[(w * cols + col) * OS + dim], f, x);
        }
        if constexpr (WHOLE) {
            const float rl = sum == 0.f ? 0.f : 1.0f / sum;      // (a sum of NaN stays one)
            a.out[(int64_t)b * a.o_st + (int64_t)(h0 + col) * a.o_sh + dim] = (uint16_t)f32_to_bf16_bits(x * rl);
            if (dim == 0) { sm_h[col] = top; sm_h[kCols + col] = rl; }
        } else {
            const int64_t part = ((int64_t)b * a.H + h0 + col) * a.nsplit + ch;
            a.part_o[part * D + dim] = x;
            if (dim == 0) { a.part_ml[2 * part] = top; a.part_ml[2 * part + 1] = sum; }
        }
    }
    if constexpr (!WHOLE) {
        if (scored) {
            const int quads = (u_end - u_begin) * (kBlk / 4);
            for (int e = tid; e < nq * quads; e += kThr) {
                const int col = e / quads, at = e - col * quads;
                __builtin_nontemporal_store(reinterpret_cast<const f32x4*>(staged + col * stage_rows)[at],
                                            reinterpret_cast<f32x4*>(a.logits + ((int64_t)b * a.H + h0 + col) * a.logit_stride + u_begin * kBlk) + at);
            }
        }
    }
    if constexpr (WHOLE) {
        if (scored && n >= 0) {                             // (one workgroup holds all heads of the group: the launcher sees to it)
            __syncthreads();
            float* score = a.score + b * a.s_sb + kh * a.s_sh;
            auto weight = [&](int key) {
                float w = 0.f;
                for (int col = 0; col < nq; ++col) w = fmaf(exp2_fast(staged[col * stage_rows + key] - sm_h[col]), sm_h[kCols + col], w);
                return w;
            };
            const int rows = n + (fresh ? 1 : 0);
#pragma unroll
            for (int j = 0; j < kAhead; ++j) {
                const int key = tid + j * kThr;
                if (key < rows) score[key] = (key < n ? old[j] : 0.f) + weight(key);
            }
            for (int key = tid + kAhead * kThr; key < rows; key += kThr) score[key] = (key < n ? score[key] : 0.f) + weight(key);
        }
    }
    // ---- a block that is whole now -------------------------------------------------------------------------------------------------
    if (with_tail && fresh && q0 == 0 && n % kBlk == kBlk - 1) {
        const int to = page_of(a.c, b, n / kBlk);
        __syncthreads();                                    // (the new row is written, sm_m is free)
        if (to < 0) return;
        const int64_t at = (int64_t)to * a.Hk + kh, tail = ((int64_t)b * a.Hk + kh) * kBlk * D;
        for (int which = 0; which < 2; ++which) {
            const uint16_t* src = (which ? a.c.v_tail : a.c.k_tail) + tail;     // (codes lie in the tails' own order)
            uint8_t* dst = (which ? a.c.v_codes : a.c.k_codes) + at * (kBlk * D);
            auto largest = [&](uint32_t below, uint32_t* words) {
                uint32_t mx = 0;
                for (int e = tid; e < kBlk * D; e += kThr) {
                    const uint32_t m = magnitude(__uint_as_float((uint32_t)src[e] << 16));
                    mx = max(mx, m < below ? m : 0u);
                }
                return largest_of<WAVES>(mx, words, tid);
            };
            uint32_t* words = reinterpret_cast<uint32_t*>(sm_m) + 2 * which * WAVES;
            uint32_t top = largest(0xffffffffu, words);
            const bool all_finite = top < kInfinity;
            if (!all_finite) top = largest(kInfinity, words + WAVES);
            const float scale = __uint_as_float(top) * F::kUnit;
            const Divider divide(scale, __uint_as_float(top), all_finite);
            for (int e = 4 * tid; e < kBlk * D; e += 4 * kThr) {
                const uint2 raw = *reinterpret_cast<const uint2*>(src + e);
                float x[4] = {bf16_lo(raw.x), bf16_hi(raw.x), bf16_lo(raw.y), bf16_hi(raw.y)};
                if (divide.care) {
#pragma unroll
                    for (int i = 0; i < 4; ++i) x[i] = divide.careful(x[i], F::nan_code(), F::kMost);
                }
                *reinterpret_cast<uint32_t*>(dst + e) = F::code4(x, divide);
            }
            if (tid == 0) (which ? a.c.v_scale : a.c.k_scale)[at] = scale;
        }
    }
}

// Maximum, and one over the sum, of a head over its chunks.
__device__ __forceinline__ float2 head_sum(const BlockDecodeArgs& a, int64_t part, int chunks, int lane) {
    float top = -3.402823466e38f, sum = 0.f;
    for (int i = lane; i < chunks; i += kWave) {
        const float2 ml = reinterpret_cast<const float2*>(a.part_ml)[part + i];
        const float m = fmaxf(top, ml.x);
        sum = sum * exp2_fast(top - m) + ml.y * exp2_fast(ml.x - m);
        top = m;
    }
    const float m = wave_max_from<1>(top);
    sum = wave_sum_from<1>(sum * exp2_fast(top - m));
    return make_float2(m, sum == 0.f ? 0.f : 1.0f / sum);
}

constexpr int kFinishThreads = 256, kScoreKeys = 4 * kFinishThreads;

// Behind the chunks: workgroups [0, H) merge a head's parts, the rest add the weights of 1024 keys of a key head.
template <int D>
__global__ __launch_bounds__(kFinishThreads) void block_finish_kernel(BlockDecodeArgs a) {
    constexpr int kGroups = kFinishThreads / D;             // chunks are dealt to groups of D threads
    __shared__ float sm[kFinishThreads + 2 * 1024];
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, b = blockIdx.y;
    const bool fresh = a.k_new != nullptr;
    const int n = min(a.c.len[b], a.max_len);
    const int units = n < 0 ? 0 : units_of(n, fresh), chunks = max(1, (units + a.chunk - 1) / a.chunk);
    int x = blockIdx.x;
    if (x < a.H) {
        const int64_t part = ((int64_t)b * a.H + x) * a.nsplit;
        const float2 hs = head_sum(a, part, chunks, lane);
        const int dim = tid % D, grp = tid / D;
        float v = 0.f;
#pragma unroll 4
        for (int i = grp; i < chunks; i += kGroups) v = fmaf(a.part_o[(part + i) * D + dim], exp2_fast(a.part_ml[2 * (part + i)] - hs.x), v);
        sm[tid] = v;
        __syncthreads();
        if (grp == 0) {
#pragma unroll
            for (int i = 1; i < kGroups; ++i) v += sm[i * D + dim];
            a.out[(int64_t)b * a.o_st + (int64_t)x * a.o_sh + dim] = (uint16_t)f32_to_bf16_bits(v * hs.y);
        }
        return;
    }
    x -= a.H;
    const int kh = x % a.Hk, first = x / a.Hk * kScoreKeys, rows = n + (fresh ? 1 : 0);
    if (n < 0 || first >= rows) return;
    float2* heads = reinterpret_cast<float2*>(sm);
    for (int i = wave; i < a.G; i += kFinishThreads / kWave) {
        const float2 hs = head_sum(a, ((int64_t)b * a.H + kh * a.G + i) * a.nsplit, chunks, lane);
        if (lane == 0) heads[i] = hs;
    }
    __syncthreads();
    const int key = first + 4 * tid;
    if (key >= rows) return;
    const float* logit = a.logits + ((int64_t)b * a.H + kh * a.G) * a.logit_stride + key;
    f32x4 w = {0.f, 0.f, 0.f, 0.f};
#pragma unroll 4
    for (int i = 0; i < a.G; ++i) {
        const f32x4 s = *reinterpret_cast<const f32x4*>(logit + i * a.logit_stride);
        const float2 hs = heads[i];
#pragma unroll
        for (int j = 0; j < 4; ++j) w[j] = fmaf(exp2_fast(s[j] - hs.x), hs.y, w[j]);
    }
    float* score = a.score + b * a.s_sb + kh * a.s_sh + key;
#pragma unroll
    for (int j = 0; j < 4; ++j)
        if (key + j < rows) score[j] = key + j < n ? score[j] + w[j] : w[j];
}

// How a call is cut: waves of a workgroup, blocks of a chunk (0: whole strips, one launch).
//   Whole strips while there are enough to fill the card, or while they are so short that the second launch of a cut costs more than it
//   brings (with their logits in LDS, up to what there is of it).  us a call, whole / cut: 64 strips of 32 blocks 18.3 / 14.2, 8 strips of 12 blocks
//   10.0 / 12.6, 256 strips of 10 to 49 blocks 28.5 / 36.9.  Lengths are known to the device only, so the rule goes by the longest that may come and
//   takes strips for equal: that holds at 256 of 49 blocks (38.8 / 42.5, with scores 42.5 / 52.3) and of 188 (136 / 140), not where one sequence is far
//   longer than the others, whose strips are then walked by one unit each.  248 strips of 11 blocks and 8 of 63: 29.5 / 23.7, of 125 48.9 / 31.3, of
//   250 87.5 / 47.1, of 625 204 / 96; 280 of 11 and 40 of 49, with scores, 35.7 / 30.3, 40 of 250 127 / 58.
//   Workgroups of 12 waves, one on a compute unit, where strips are no more than compute units, else of 4 waves, three on a unit.  12 / 4: 256 strips
//   28.5 / 31.7, 320 strips of 11 to 20 blocks 22.6 / 19.2.
//   Chunks for about three workgroups on a unit; where logits are kept, no longer than leaves room for three in LDS.  16 strips of 1100 to 2049 blocks: 20
//   blocks (20 KB) 107, 10 blocks 115, 40 blocks 109; 512 / 768 / 1536 workgroups without logits 79.9 / 81.4 / 89.1.
struct Cut { int waves, chunk, most; };      // most: chunks of a strip, at any length up to this one
constexpr int kWholeStrips = 192, kShortUnits = 20, kManyStrips = 256, kStageBytes = 20 << 10, kChunkWgs = 768;

template <int D>
inline Cut cut_of(int B, int Hk, int G, int max_len, bool scored) {
    constexpr size_t kLds = 160 << 10;
    const int QG = (G + kCols - 1) / kCols, cols = std::min(G, kCols);
    const int64_t units = max_len / kBlk + 1, strips = (int64_t)B * Hk * QG;
    const int waves = strips > kManyStrips ? 4 : 12;
    const bool fits = units + 2 <= waves * kWave && (!scored || (QG == 1 && attend_lds<D>(waves, cols, units * kBlk) <= kLds));
    if (fits && (strips >= kWholeStrips || units <= kShortUnits)) return Cut{waves, 0, 0};
    constexpr int kLeast = 4;
    int64_t top = 4 * kWave - 2;
    if (scored) top = std::min<int64_t>(top, std::max<int64_t>(8, kStageBytes / (cols * kBlk * (int)sizeof(float))));
    const int64_t chunk = std::min<int64_t>({std::max<int64_t>(kLeast, (units * strips + kChunkWgs - 1) / kChunkWgs), top, units});
    const int64_t most = std::max<int64_t>(std::min<int64_t>((units + kLeast - 1) / kLeast, (kChunkWgs + strips - 1) / strips), (units + top - 1) / top);
    return Cut{4, (int)chunk, (int)most};
}
inline Cut cut_of(const st3_gqa_shape* s, int max_len, bool scored) {
    const int G = s->heads / s->kv_heads;
    return s->head_dim == 128 ? cut_of<128>(s->batch, s->kv_heads, G, max_len, scored) : cut_of<64>(s->batch, s->kv_heads, G, max_len, scored);
}

struct BlockWs { size_t part_o, part_ml, logits, total; int64_t logit_stride; int nsplit; };

inline BlockWs block_ws(const st3_gqa_shape* s, int max_len, bool scored) {
    const Cut cut = cut_of(s, max_len, scored);
    const int64_t units = max_len / kBlk + 1;
    BlockWs w{};
    if (cut.chunk == 0) return w;
    w.nsplit = (int)((units + cut.chunk - 1) / cut.chunk);
    w.logit_stride = units * kBlk;
    const size_t BH = (size_t)s->batch * s->heads;
    size_t off = 0;                     // (room for cut.most chunks: shorter lengths may be cut into more, and what is enough here is enough for them)
    w.part_o = off;  off = align_up(off + BH * cut.most * s->head_dim * sizeof(float), 256);
    w.part_ml = off; off = align_up(off + BH * cut.most * 2 * sizeof(float), 256);
    w.logits = off;  if (scored) off = align_up(off + BH * w.logit_stride * sizeof(float), 256);
    w.total = off;
    return w;
}

// Workgroups of the launch behind the chunks, for a sequence.
inline int64_t finish_groups(int H, int Hk, int max_len, bool scored) { return H + (scored ? (int64_t)Hk * ((max_len + kScoreKeys) / kScoreKeys) : 0); }

template <int D, int CODE>
void launch_decode(const BlockDecodeArgs& a, int B, int waves, hipStream_t st) {
    const int cols = std::min(kCols, a.G);
    if (a.chunk == 0) {
        const size_t lds = attend_lds<D>(waves, cols, a.score ? (a.max_len / kBlk + 1) * kBlk : 0);
        const dim3 grid(a.Hk * a.QG, 1, B);
        if (waves == 12) block_attend_kernel<D, CODE, 12, true><<<grid, 768, lds, st>>>(a);
        else block_attend_kernel<D, CODE, 4, true><<<grid, 256, lds, st>>>(a);
        return;
    }
    block_attend_kernel<D, CODE, 4, false><<<dim3(a.Hk * a.QG, a.nsplit, B), 256, attend_lds<D>(4, cols, a.score ? a.chunk * kBlk : 0), st>>>(a);
    block_finish_kernel<D><<<dim3((unsigned)finish_groups(a.H, a.Hk, a.max_len, a.score != nullptr), B), kFinishThreads, 0, st>>>(a);
}

}  // namespace
}  // namespace st3

extern "C" size_t st3_block_workspace_bytes(const st3_gqa_shape* shape, int32_t max_len) {
    if (st3::check_gqa_shape(shape) != ST3_OK || max_len < 0) return 0;
    return std::max<size_t>(256, std::max(st3::block_ws(shape, max_len, true).total, st3::block_ws(shape, max_len, false).total));
}

extern "C" st3_status st3_block_decode(const st3_gqa_shape* shape, const st3_rows* q, const st3_rows* k_new, const st3_rows* v_new,
                                       const st3_block_cache* cache, int32_t max_len, const st3_rows* out, float* score, int64_t score_stride_b,
                                       int64_t score_stride_h, void* workspace, size_t workspace_bytes, void* stream) {
    using namespace st3;
    st3_status s = check_gqa_shape(shape);
    if (s != ST3_OK) return s;
    if ((s = check_block_cache(shape, cache)) != ST3_OK) return s;
    const int B = shape->batch, H = shape->heads, Hk = shape->kv_heads, D = shape->head_dim, G = H / Hk;
    if ((s = check_rows(q, D, 2)) != ST3_OK || (s = check_output(out, H, B, D, 2)) != ST3_OK) return s;
    if (!k_new != !v_new) return ST3_ERR_INVALID_ARG;
    if (k_new && ((s = check_rows(k_new, D, 2)) != ST3_OK || (s = check_rows(v_new, D, 2)) != ST3_OK)) return s;
    if (max_len < 0 || max_len > kMostRows) return ST3_ERR_INVALID_ARG;
    // (a row that fills its block needs that block's page)
    if (cache->table_blocks < (max_len + (k_new ? 1 : 0)) / kBlk) return ST3_ERR_INVALID_ARG;
    if (score && (score_stride_h < (int64_t)max_len + 1 || (B > 1 && score_stride_b < (int64_t)max_len + 1))) return ST3_ERR_INVALID_ARG;
    if (!workspace || !aligned16(workspace)) return ST3_ERR_INVALID_ARG;
    const Cut cut = cut_of(shape, max_len, score != nullptr);
    const BlockWs wl = block_ws(shape, max_len, score != nullptr);
    if (cut.chunk > 0 && !(grid_fits(1, 1, wl.nsplit) && grid_fits(finish_groups(H, Hk, max_len, score != nullptr), kFinishThreads, B)))
        return ST3_ERR_UNSUPPORTED;
    if (workspace_bytes < st3_block_workspace_bytes(shape, max_len)) return ST3_ERR_WORKSPACE_TOO_SMALL;
    // (a workgroup's output may be written before another has read the new row, or queries that are not the first one's own)
    if (k_new && (packed_rows_meet(k_new, Hk, out, H, B, D, 2) || packed_rows_meet(v_new, Hk, out, H, B, D, 2))) return ST3_ERR_INVALID_ARG;
    const bool in_place = q->data == out->data && (B == 1 || q->stride_t == out->stride_t) && (H == 1 || q->stride_h == out->stride_h);
    if (!in_place && packed_rows_meet(q, H, out, H, B, D, 2)) return ST3_ERR_INVALID_ARG;
    char* ws = reinterpret_cast<char*>(workspace);
    auto bits = [](const st3_rows* r) { return r ? reinterpret_cast<uint16_t*>(r->data) : nullptr; };
    BlockDecodeArgs a{};
    a.c = block_pages(cache);
    a.q = bits(q); a.k_new = bits(k_new); a.v_new = bits(v_new); a.out = bits(out);
    a.q_st = q->stride_t; a.q_sh = q->stride_h; a.o_st = out->stride_t; a.o_sh = out->stride_h;
    if (k_new) { a.k_st = k_new->stride_t; a.k_sh = k_new->stride_h; a.v_st = v_new->stride_t; a.v_sh = v_new->stride_h; }
    a.max_len = max_len; a.H = H; a.Hk = Hk; a.G = G; a.QG = (G + kCols - 1) / kCols;
    a.chunk = cut.chunk; a.nsplit = wl.nsplit;
    a.scale_l2 = gqa_scale_log2(shape);
    a.score = score; a.s_sb = score_stride_b; a.s_sh = score_stride_h;
    a.part_o = reinterpret_cast<float*>(ws + wl.part_o);
    a.part_ml = reinterpret_cast<float*>(ws + wl.part_ml);
    a.logits = reinterpret_cast<float*>(ws + wl.logits);
    a.logit_stride = wl.logit_stride;
    hipStream_t st = reinterpret_cast<hipStream_t>(stream);
    if (cache->code == ST3_BLOCK_INT8) {
        if (D == 128) launch_decode<128, ST3_BLOCK_INT8>(a, B, cut.waves, st);
        else launch_decode<64, ST3_BLOCK_INT8>(a, B, cut.waves, st);
    } else {
        if (D == 128) launch_decode<128, ST3_BLOCK_E4M3>(a, B, cut.waves, st);
        else launch_decode<64, ST3_BLOCK_E4M3>(a, B, cut.waves, st);
    }
    return check_launch();
}
