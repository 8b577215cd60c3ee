// Causal attention over packed prompts with grouped heads (Eq. 2), and the weight that the last W rows of each prompt give to every key.
//
// Rows.  The G query heads that share a key head are rows of ONE matrix: row x of a (sequence, key head) pair is head x % G of position x / G,
// so a group's queries meet a K and V tile together, any G fills the MFMA's columns, and a tile of rows spans few positions (the
// causal edge wastes little).  A workgroup takes kRows such rows of a pair and walks the key tiles up to its last position.
#include <algorithm>
#include <type_traits>

#include "st3_block.h"

namespace st3 {
namespace {

struct PackedArgs {
    const void* q; const void* k; const void* v; void* out;
    int64_t q_st, q_sh, k_st, k_sh, v_st, v_sh, o_st, o_sh;     // strides in elements
    const int32_t* cu;
    int32_t B, total, max_len, H, Hk, G;
    int32_t levels;                 // row tiles of the longest prompt that may come
    int32_t spread;                 // row tiles dealt together at the end of the launch
    float scale_l2;
    float* score; int64_t s_sb, s_sh;
    float2* ml;                     // [total][H] maximum and sum of the rows whose weights count; null: no score
    int32_t window;
};

struct Seq { int start, n; };
__device__ __forceinline__ Seq sequence(const PackedArgs& a, int b) {
    const int s = max(0, min(a.cu[b], a.total)), e = max(s, min(a.cu[b + 1], a.total));
    return Seq{s, min(e - s, a.max_len)};
}

// Workgroup -> (sequence, key head, row tile).  Key heads run fastest: workgroups go round-robin to the 8 XCDs, so with a multiple of 8 key heads a
// pair's K and V stay in one XCD's L2, and a sequence's tiles follow each other, heaviest (last) first, longest sequences first, so that they are
// there when the next tile wants them.  A tile costs in proportion to its index: the last sequences' tiles (a.spread of them, or so) are dealt
// together, heaviest first over all of them, so that the launch ends with its shortest workgroups.  Lengths are known to the device only: every wave
// finds its place, a lane for each of up to 64 sequences; more keep their own order.
template <int ROWS>
__device__ __forceinline__ bool place(const PackedArgs& a, int lane, int& b, int& kh, int& tile, Seq& sq) {
    kh = blockIdx.x % a.Hk;
    int x = blockIdx.x / a.Hk;
    Seq its = {0, 0};               // this lane's sequence
    auto tiles_of = [&](int i) {
        if (i < a.B) its = sequence(a, i);
        return i < a.B ? (int)(((int64_t)its.n * a.G + ROWS - 1) / ROWS) : 0;
    };
    auto found = [&](int first, int at, int t) {        // (lane `at` has sequence first + at)
        at = __builtin_amdgcn_readfirstlane(at);
        b = first + at;
        tile = __builtin_amdgcn_readfirstlane(t);
        sq = Seq{__builtin_amdgcn_readlane(its.start, at), __builtin_amdgcn_readlane(its.n, at)};
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
    const int mine = tiles_of(lane);
    const int total = wave_total(mine);
    if (x >= total) return false;
    int dealt = mine;
    if (total > a.spread) {
        int before = 0;                 // tiles of the sequences in front of this one, longest first
        for (int i = 0; i < a.B; ++i) {
            const int other = __builtin_amdgcn_readlane(mine, i);
            before += other > mine || (other == mine && i < lane) ? other : 0;
        }
        // the sequences in front of `apart` have their tiles to themselves
        const int end = before + mine, apart = wave_most(mine > 0 && end <= total - a.spread ? end : 0);
        if (x < apart) {
            const int at = __ffsll((unsigned long long)__ballot(mine > 0 && before <= x && x < end)) - 1;
            return found(0, at, __builtin_amdgcn_readlane(end, at) - 1 - x);
        }
        x -= apart;
        dealt = before >= apart ? mine : 0;
    }
    auto from = [&](int t) { return wave_total(max(0, dealt - t)); };      // tiles of index t or more
    int lo = 0, hi = a.levels, above = 0;                                  // from(lo) > x >= from(hi)
    while (hi - lo > 1) {
        const int mid = (lo + hi) / 2, s = from(mid);
        if (s > x) lo = mid;
        else { hi = mid; above = s; }
    }
    const uint64_t who = __ballot(dealt > lo);
    const uint64_t me = __ballot(dealt > lo && __popcll(who & ((1ull << lane) - 1)) == x - above);
    return found(0, __ffsll((unsigned long long)me) - 1, lo);
}

// ---------------------------------------------------------------------------------------------------------------------------------
// bf16
// ---------------------------------------------------------------------------------------------------------------------------------

// A wave's 16 QC rows, as QC columns of 16: lane (c, g) holds row 16 qc + c of each, and of its output the columns 16 dt + 4 g .. + 3.
template <int D, int QC>
struct Rows {
    f32x4 o[D / 16][QC];
    float m[QC];
    float l[QC];
    int pos[QC];            // position of the row: the last key that it sees
    __device__ __forceinline__ void init() {
#pragma unroll
        for (int qc = 0; qc < QC; ++qc) {
#pragma unroll
            for (int dt = 0; dt < D / 16; ++dt) o[dt][qc] = f32x4{0.f, 0.f, 0.f, 0.f};
            m[qc] = -3.402823466e38f; l[qc] = 0.f;
        }
    }
};

// 32 keys for one wave: S^T = K Q^T, one online-softmax update, O^T += V^T P^T.  MASKED: some row does not see some of the keys.
// CAREFUL: V may hold infinities or NaN, and a weight of 0 does not silence those; row by row, V's keys that the row does not see count as 0.
// (The scheduling barriers keep the compiler from holding more fragments than there are registers for.)
template <int D, int QC, bool MASKED, bool CAREFUL = false>
__device__ __forceinline__ void packed_step(uint32_t Kt, uint32_t Vt, const Frag (&qf)[QC][D / 32], Rows<D, QC>& st, float scale_l2, int g, int k0) {
    constexpr int KS = D / 32, DT = D / 16;
    f32x4 s[2][QC];
    Frag ka[2][KS];
    auto load_k = [&](int half) {
#pragma unroll
        for (int x = 0; x < KS; ++x) ka[half][x].u4 = lds_read16((Kt ^ (64 * x)) + 32 * half * D);
    };
    __builtin_amdgcn_s_setprio(1);
    load_k(0);
#pragma unroll
    for (int half = 0; half < 2; ++half) {
        if (half == 0) load_k(1);
        __builtin_amdgcn_sched_barrier(0);
#pragma unroll
        for (int qc = 0; qc < QC; ++qc) {
            f32x4 x = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int i = 0; i < KS; ++i) x = __builtin_amdgcn_mfma_f32_16x16x32_bf16(ka[half][i].v, qf[qc][i].v, x, 0, 0, 0);
            s[half][qc] = x;
            __builtin_amdgcn_sched_barrier(0);
        }
    }
    constexpr int VB = DT < 4 ? DT : 4;
    Frag va[VB];
    auto load_v = [&](int dt) {
        const uint32_t at = Vt ^ (32 * dt);
        va[dt % VB].h[0] = lds_read_tr(at);
        va[dt % VB].h[1] = lds_read_tr(at + 32 * D);
    };
#pragma unroll
    for (int i = 0; i < VB; ++i) load_v(i);
    __builtin_amdgcn_sched_barrier(0);
    __builtin_amdgcn_s_setprio(0);
    if (MASKED) {
#pragma unroll
        for (int half = 0; half < 2; ++half)
#pragma unroll
            for (int qc = 0; qc < QC; ++qc)
#pragma unroll
                for (int r = 0; r < 4; ++r)
                    if (k0 + 16 * half + 4 * g + r > st.pos[qc]) s[half][qc][r] = -INFINITY;
    }
    // the reference point of the exponents follows the maximum only when that has moved by more than kLazy (probabilities reach 2^kLazy at most)
    constexpr float kLazy = 8.0f;
    float mx[QC];
    bool moved = false;
#pragma unroll
    for (int qc = 0; qc < QC; ++qc) {
        mx[qc] = fmaxf(fmaxf(fmaxf(s[0][qc][0], s[0][qc][1]), fmaxf(s[0][qc][2], s[0][qc][3])),
                       fmaxf(fmaxf(s[1][qc][0], s[1][qc][1]), fmaxf(s[1][qc][2], s[1][qc][3]))) * scale_l2;
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
            for (int dt = 0; dt < DT; ++dt) st.o[dt][qc] *= alpha;
        }
    }
    // P is rounded to bf16 once, to nearest: an error of 2^-8 of a probability at most and without bias, beside the output's own rounding by as
    // much; the sum is of the unrounded ones.  (Two terms, as the prefill's kernel has them: the outputs' rms error is 0.00163 of their rms, the
    // rounding's own, for 0.00207 with one; 304 us for 245 at the mixed prompts, 2265 for 1691 at the long ones.)
    Frag pb[QC];
#pragma unroll
    for (int qc = 0; qc < QC; ++qc)
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const f32x2 p = {exp2_fast(fmaf(s[j / 2][qc][2 * (j & 1)], scale_l2, -st.m[qc])),
                             exp2_fast(fmaf(s[j / 2][qc][2 * (j & 1) + 1], scale_l2, -st.m[qc]))};
            st.l[qc] += p.x + p.y;
            pb[qc].w[j] = __builtin_bit_cast(uint32_t, __builtin_convertvector(p, bf16x2));
        }
    if constexpr (CAREFUL) {
#pragma unroll
        for (int qc = 0; qc < QC; ++qc)
            for (int x = 0; x < 16; ++x) {
                const int pos = __builtin_amdgcn_readlane(st.pos[qc], x), c = threadIdx.x & 15;
                Frag seen;
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    const int key = k0 + 16 * (j / 2) + 4 * g + 2 * (j & 1);
                    seen.w[j] = (key <= pos ? 0xffffu : 0u) | (key < pos ? 0xffff0000u : 0u);
                }
#pragma unroll
                for (int dt = 0; dt < DT; ++dt) {
                    load_v(dt);
#pragma unroll
                    for (int j = 0; j < 4; ++j) va[dt % VB].w[j] &= seen.w[j];
                    const f32x4 o = __builtin_amdgcn_mfma_f32_16x16x32_bf16(va[dt % VB].v, pb[qc].v, st.o[dt][qc], 0, 0, 0);
                    st.o[dt][qc] = c == x ? o : st.o[dt][qc];
                    __builtin_amdgcn_sched_barrier(0);
                }
            }
        return;
    }
#pragma unroll
    for (int dt = 0; dt < DT; ++dt) {
        if (dt > 0 && dt + VB - 1 < DT) load_v(dt + VB - 1);
        __builtin_amdgcn_sched_barrier(0);
#pragma unroll
        for (int qc = 0; qc < QC; ++qc) st.o[dt][qc] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(va[dt % VB].v, pb[qc].v, st.o[dt][qc], 0, 0, 0);
        __builtin_amdgcn_sched_barrier(0);
    }
}

// Starts the direct loads of the tile of 32 keys at k0 (rows past the last are clamped: no row sees them).  k_lane, v_lane: byte offset of
// this lane's 16 bytes in a tile's first 1 KB; the 1 KB pieces of a tile lie RPI * 4 rows apart.
template <int D>
__device__ __forceinline__ void load_tile(uint32_t lds, const uint16_t* K, const uint16_t* V, int64_t k_st, int64_t v_st, int k0, int n, uint32_t k_lane,
                                          uint32_t v_lane, int row0, int wave_s) {
    using L = TileLayout<D, 32>;
    if (k0 + 32 <= n) {
#pragma unroll
        for (int i = 0; i < L::NI; ++i) {
            const uint32_t dst = lds + (4 * i + wave_s) * 1024;
            direct_load16(uniform_ptr(K + (k0 + 4 * i * L::RPI) * k_st), k_lane, dst);
            direct_load16(uniform_ptr(V + (k0 + 4 * i * L::RPI) * v_st), v_lane, dst + 2 * L::TILE);
        }
    } else {
        const uint16_t* kp = uniform_ptr(K + k0 * k_st);
        const uint16_t* vp = uniform_ptr(V + k0 * v_st);
#pragma unroll
        for (int i = 0; i < L::NI; ++i) {
            const uint32_t dst = lds + (4 * i + wave_s) * 1024;
            const int back = min(row0 + 4 * i * L::RPI, n - 1 - k0) - row0;          // rows from where k_lane points
            direct_load16(kp, k_lane + (uint32_t)(back * (int)(2 * k_st)), dst);
            direct_load16(vp, v_lane + (uint32_t)(back * (int)(2 * v_st)), dst + 2 * L::TILE);
        }
    }
}

// A workgroup's four waves have 16 QC rows each and share the K and V tiles, which go straight from memory to LDS, two tiles ahead.
// SPLIT: as many groups of four waves take the same rows and every SPLIT-th tile, and join their sums in LDS at the end.
// Bound by the matrix instructions' power at long prompts (clock 1.76 GHz, the matrix units busy for 59 % of it, the vector units for 68 %): 21300 tokens
// of 32 heads over 8 of 128 in 1.64 to 1.77 ms with their scores, 1080 to 1170 TF/s of the 1500 that a large product reaches; by a step's chain of products, maximum, exponentials and products at short ones: 1 us for 32 keys and 128 rows alone
// on a unit. Two columns of rows leave registers for 3 waves a SIMD; three columns with 2 waves take 1.66 ms there, but 395 us for 368 at 32 x 739
// tokens of 40 key heads.
template <int D, int QC, int SPLIT>
__global__ __launch_bounds__(256 * SPLIT, SPLIT == 1 ? 3 : SPLIT) void packed_kernel(PackedArgs a) {
    using L = TileLayout<D, 32>;
    constexpr int kRows = 64 * QC, KS = D / 32, DT = D / 16, kRing = 3, OSTR = D + 8;
    constexpr int kTiles = kRing * 2 * L::TILE, kOut = 4 * 16 * QC * OSTR;
    __shared__ __attribute__((aligned(1024))) uint16_t buf[SPLIT * kTiles > kOut ? SPLIT * kTiles : kOut];
    __shared__ int redo;
    const int lane = threadIdx.x & 63, wave_s = __builtin_amdgcn_readfirstlane((threadIdx.x >> 6) & 3), wave = wave_s;
    const int part = SPLIT == 1 ? 0 : __builtin_amdgcn_readfirstlane(threadIdx.x >> 8);
    const int g = lane >> 4, c = lane & 15;
    int b, kh, tile;
    Seq sq;
    if (!place<kRows>(a, lane, b, kh, tile, sq)) return;
    if (threadIdx.x == 0) redo = 0;
    const int n = sq.n, rows = n * a.G;
    // row tiles are cut from the end, in whole columns: a prompt's first tile, the cheapest, is the one that is not full
    const int tiles = (rows + kRows - 1) / kRows, shift = (tiles * kRows - rows) / (16 * QC) * (16 * QC);
    const int r0 = tile * kRows - shift + wave * 16 * QC;            // the wave's first row; < 0 or >= rows: it has none
    const uint16_t* K = reinterpret_cast<const uint16_t*>(a.k) + (int64_t)sq.start * a.k_st + kh * a.k_sh;
    const uint16_t* V = reinterpret_cast<const uint16_t*>(a.v) + (int64_t)sq.start * a.v_st + kh * a.v_sh;
    const uint32_t lds0 = lds_addr(buf) + part * (2 * kTiles);
    constexpr int kBuf = 4 * L::TILE;
    const int last = min(rows, (tile + 1) * kRows - shift) - 1;      // the workgroup's last row
    const int nt = last / a.G / 32 + 1;
    const int row0 = wave * L::RPI + lane / L::UPR;
    const uint32_t k_lane = (uint32_t)(2 * (row0 * (int)a.k_st + (lane % L::UPR ^ L::k_swz(row0)) * 8));
    const uint32_t v_lane = (uint32_t)(2 * (row0 * (int)a.v_st + (lane % L::UPR ^ L::v_swz(row0)) * 8));
    auto issue = [&](int t, int slot) { load_tile<D>(lds0 + slot * kBuf, K, V, a.k_st, a.v_st, t * 32, n, k_lane, v_lane, row0, wave_s); };
    if (SPLIT == 1 || part < nt) issue(part, 0);
    Rows<D, QC> st;
    st.init();
    Frag qf[QC][KS];
#pragma unroll
    for (int qc = 0; qc < QC; ++qc) {
        const int r = max(0, min(r0 + 16 * qc + c, rows - 1)), p = r / a.G;
        st.pos[qc] = p;
        const uint16_t* row = reinterpret_cast<const uint16_t*>(a.q) + (int64_t)(sq.start + p) * a.q_st + (int64_t)(kh * a.G + r - p * a.G) * a.q_sh;
#pragma unroll
        for (int s = 0; s < KS; ++s) qf[qc][s].u4 = *reinterpret_cast<const u32x4*>(row + 32 * s + 8 * g);
    }
    const int p_last = __builtin_amdgcn_readfirstlane(min(r0 + 16 * QC, rows) - 1) / a.G;        // (a wave without rows has none or works on its neighbour's)
    uint32_t k_at, v_at;                                             // this lane's operands in a tile (as in the prefill's kernel)
    {
        k_at = (uint32_t)(2 * (c * D + (g ^ L::k_swz(c)) * 8));
        const int row = 4 * g + (c >> 2);
        v_at = (uint32_t)(2 * (row * D + (((c & 3) >> 1) ^ L::v_swz(row)) * 8 + 4 * (c & 1))) + 2 * L::TILE;
    }
    if (part + SPLIT < nt) { issue(part + SPLIT, 1); wait_direct_loads_but<2 * L::NI>(); }
    else wait_direct_loads();
    __syncthreads();
    // Tiles that every row of the workgroup sees whole come first, in a loop without conditions (with both kinds in one loop the accumulators were
    // moved between the two forms' registers, and spilled); the few at the edge follow.
    int t = part, slot = 0, next = 2;
    auto advance = [&]() {
        if (t + 2 * SPLIT < nt) { issue(t + 2 * SPLIT, next); wait_direct_loads_but<2 * L::NI>(); }
        else wait_direct_loads();
        __syncthreads();
        slot = slot == kRing - 1 ? 0 : slot + 1;
        next = next == kRing - 1 ? 0 : next + 1;
        t += SPLIT;
    };
    for (int whole = (max(tile * kRows - shift, 0) / a.G + 1) / 32 / SPLIT; whole > 0; --whole) {
        const uint32_t at = lds0 + slot * kBuf;
        packed_step<D, QC, false>(at + k_at, at + v_at, qf, st, a.scale_l2, g, 32 * t);
        advance();
    }
    while (t - part < nt) {
        const uint32_t at = lds0 + slot * kBuf;
        if (32 * t <= p_last) packed_step<D, QC, true>(at + k_at, at + v_at, qf, st, a.scale_l2, g, 32 * t);
        advance();
    }
    // Anything but finite: it may be from V of keys that a row does not see (0 times infinity).  Once more, such V left out.
    f32x4 odd = {0.f, 0.f, 0.f, 0.f};                                // (four chains of sums: none waits for the one before it)
#pragma unroll
    for (int dt = 0; dt < DT; ++dt)
#pragma unroll
        for (int qc = 0; qc < QC; ++qc)
#pragma unroll
            for (int i = 0; i < 4; ++i) odd[i] = fmaf(st.o[dt][qc][i], 0.f, odd[i]);
    if ((odd[0] + odd[1]) + (odd[2] + odd[3]) != 0.f) redo = 1;
    __syncthreads();
    if (redo) {
        st.init();
        for (t = part; t - part < nt; t += SPLIT) {
            if (t < nt) issue(t, 0);
            wait_direct_loads();
            __syncthreads();
            if (32 * t <= p_last) packed_step<D, QC, true, true>(lds0 + k_at, lds0 + v_at, qf, st, a.scale_l2, g, 32 * t);
            __syncthreads();
        }
    }
    uint16_t* ob = buf + wave * 16 * QC * OSTR;
    if constexpr (SPLIT > 1) {                                       // join the parts' sums: lane for lane the same rows and columns
        constexpr int kLane = DT * QC * 256;                         // floats of a wave's accumulators
        static_assert((SPLIT - 1) * 4 * (4 * kLane + 512 * QC) <= (int)sizeof(buf), "parts in LDS");
        float* acc = reinterpret_cast<float*>(buf) + wave * (kLane + 128 * QC);
        constexpr int kPart = 4 * (kLane + 128 * QC);
        if (part > 0) {
            float* to = acc + (part - 1) * kPart;
#pragma unroll
            for (int qc = 0; qc < QC; ++qc) {
#pragma unroll
                for (int dt = 0; dt < DT; ++dt) *reinterpret_cast<f32x4*>(to + (qc * DT + dt) * 256 + 4 * lane) = st.o[dt][qc];
                to[kLane + 128 * qc + lane] = st.m[qc];
                to[kLane + 128 * qc + 64 + lane] = st.l[qc];
            }
        }
        __syncthreads();
        if (part > 0) return;
#pragma unroll
        for (int x = 0; x < SPLIT - 1; ++x) {
            const float* from = acc + x * kPart;
#pragma unroll
            for (int qc = 0; qc < QC; ++qc) {
                const float m = from[kLane + 128 * qc + lane], top = fmaxf(m, st.m[qc]), f = exp2_fast(m - top), mine = exp2_fast(st.m[qc] - top);
                st.m[qc] = top;
                st.l[qc] = st.l[qc] * mine + from[kLane + 128 * qc + 64 + lane] * f;
#pragma unroll
                for (int dt = 0; dt < DT; ++dt) st.o[dt][qc] = st.o[dt][qc] * mine + *reinterpret_cast<const f32x4*>(from + (qc * DT + dt) * 256 + 4 * lane) * f;
            }
        }
        ob = reinterpret_cast<uint16_t*>(acc);                       // (read by this wave only)
    }
    // ---- normalise; the block of outputs goes through LDS and leaves as whole rows ----------------------------------------------
    constexpr int VPR = D / 8, RPI = 64 / VPR;
#pragma unroll
    for (int qc = 0; qc < QC; ++qc) {
        const float l = wave_sum_from<16>(st.l[qc]), rl = 1.0f / l;
#pragma unroll
        for (int dt = 0; dt < DT; ++dt) {
            const f32x4 o = st.o[dt][qc] * rl;
            const f32x2 o01 = {o[0], o[1]}, o23 = {o[2], o[3]};
            uint2 pk;
            pk.x = __builtin_bit_cast(uint32_t, __builtin_convertvector(o01, bf16x2));
            pk.y = __builtin_bit_cast(uint32_t, __builtin_convertvector(o23, bf16x2));
            *reinterpret_cast<uint2*>(ob + (16 * qc + c) * OSTR + 16 * dt + 4 * g) = pk;
        }
        int col = c;
        asm volatile("" : "+v"(col));                                // (formed again: kept from the start, rows and addresses were spilled)
        const int r = r0 + 16 * qc + col, p = r / a.G;
        if (a.ml != nullptr && g == 0 && r >= 0 && r < rows && p >= n - a.window)
            a.ml[(int64_t)(sq.start + p) * a.H + kh * a.G + r - p * a.G] = make_float2(st.m[qc], rl);
    }
    uint16_t* O = reinterpret_cast<uint16_t*>(a.out);
#pragma unroll
    for (int i = 0; i < 16 * QC / RPI; ++i) {
        const int x = i * RPI + lane / VPR, r = r0 + x;
        const u32x4 val = *reinterpret_cast<const u32x4*>(ob + x * OSTR + (lane % VPR) * 8);
        if (r >= 0 && r < rows) {
            const int p = r / a.G;
            *reinterpret_cast<u32x4*>(O + (int64_t)(sq.start + p) * a.o_st + (int64_t)(kh * a.G + r - p * a.G) * a.o_sh + (lane % VPR) * 8) = val;
        }
    }
}

// ---------------------------------------------------------------------------------------------------------------------------------
// A row's operand of a product over d, straight from memory: lane (c, g) holds elements of row c, in the same order for both operands.
// ---------------------------------------------------------------------------------------------------------------------------------
template <typename T, int D> struct RowFrag;
template <int D> struct RowFrag<bf16_t, D> {
    Frag f[D / 32];
    __device__ __forceinline__ void set(int s, u32x4 unit) { f[s].u4 = unit; }      // the 16 bytes 4 s + g of the row
    __device__ __forceinline__ void load(const bf16_t* row, int g) {
#pragma unroll
        for (int s = 0; s < D / 32; ++s) f[s].u4 = *reinterpret_cast<const u32x4*>(row + 32 * s + 8 * g);
    }
    __device__ __forceinline__ f32x4 dot(const RowFrag& o) const {      // [row of this][row of o]
        f32x4 x = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int s = 0; s < D / 32; ++s) x = __builtin_amdgcn_mfma_f32_16x16x32_bf16(f[s].v, o.f[s].v, x, 0, 0, 0);
        return x;
    }
};
template <int D> struct RowFrag<float, D> {
    f32x4 f[D / 16];
    __device__ __forceinline__ void set(int s, u32x4 unit) { f[s] = __builtin_bit_cast(f32x4, unit); }
    __device__ __forceinline__ void load(const float* row, int g) {
#pragma unroll
        for (int s = 0; s < D / 16; ++s) f[s] = *reinterpret_cast<const f32x4*>(row + 16 * s + 4 * g);
    }
    __device__ __forceinline__ f32x4 dot(const RowFrag& o) const {
        f32x4 x = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int s = 0; s < D / 16; ++s)
#pragma unroll
            for (int e = 0; e < 4; ++e) x = __builtin_amdgcn_mfma_f32_16x16x4f32(f[s][e], o.f[s][e], x, 0, 0, 0);
        return x;
    }
};

// ---------------------------------------------------------------------------------------------------------------------------------
// float32: the same rows on v_mfma_f32_16x16x4f32 (A: lane (c, g) holds A[c][g]).  A workgroup has 16 rows; its four waves take the key tiles of 16
// in turn, operands straight from memory, a wave's next tile on its way, and join their parts through LDS.  Bound by the latency of a tile's loads
// (600 rows of 300 keys: 10.2 us; eight waves for 16 rows 11.1, one 22).
// ---------------------------------------------------------------------------------------------------------------------------------
template <int D>
__global__ __launch_bounds__(256) void packed_f32_kernel(PackedArgs a) {
    constexpr int DT = D / 16, kRows = 16;
    __shared__ __attribute__((aligned(16))) float sm_o[4][16][D + 4];
    __shared__ float sm_m[4][16], sm_l[4][16];
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), g = lane >> 4, c = lane & 15;
    int b, kh, tile;
    Seq sq;
    if (!place<kRows>(a, lane, b, kh, tile, sq)) return;
    const int n = sq.n, rows = n * a.G, r0 = tile * kRows;
    const float* K = reinterpret_cast<const float*>(a.k) + (int64_t)sq.start * a.k_st + kh * a.k_sh;
    const float* V = reinterpret_cast<const float*>(a.v) + (int64_t)sq.start * a.v_st + kh * a.v_sh;
    const int r = min(r0 + c, rows - 1), pos = r / a.G, head = kh * a.G + r - pos * a.G;
    const int tiles = (min(r0 + 15, rows - 1) / a.G) / 16 + 1;
    RowFrag<float, D> kf, qf;
    float vf[DT][4];                                        // contraction slot g of product i is key 4 g + i, the one whose weight this lane holds
    auto load_k = [&](int t) { kf.load(K + (int64_t)min(16 * t + c, n - 1) * a.k_st, g); };
    auto load_v = [&](int t) {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const float* row = V + (int64_t)min(16 * t + 4 * g + i, n - 1) * a.v_st + c;
#pragma unroll
            for (int dt = 0; dt < DT; ++dt) vf[dt][i] = row[16 * dt];
        }
    };
    if (wave < tiles) { load_k(wave); load_v(wave); }
    qf.load(reinterpret_cast<const float*>(a.q) + (int64_t)(sq.start + pos) * a.q_st + (int64_t)head * a.q_sh, g);
    f32x4 o[DT];
    float m, l;
    // (CAREFUL as in packed_step)
    auto walk = [&](auto careful) {
#pragma unroll
        for (int dt = 0; dt < DT; ++dt) o[dt] = f32x4{0.f, 0.f, 0.f, 0.f};
        m = -3.402823466e38f; l = 0.f;
        for (int t = wave; t < tiles; t += 4) {
            f32x4 s = kf.dot(qf) * a.scale_l2;
            if (t + 4 < tiles) load_k(t + 4);
#pragma unroll
            for (int i = 0; i < 4; ++i)
                if (16 * t + 4 * g + i > pos) s[i] = -INFINITY;
            const float mx = fmaxf(m, wave_max_from<16>(fmaxf(fmaxf(s[0], s[1]), fmaxf(s[2], s[3]))));
            const float alpha = exp2_fast(m - mx);
            m = mx;
            l *= alpha;
            float p[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) { p[i] = exp2_fast(s[i] - m); l += p[i]; }
#pragma unroll
            for (int dt = 0; dt < DT; ++dt) {
                o[dt] *= alpha;
                if constexpr (decltype(careful)::value) {
                    for (int x = 0; x < 16; ++x) {
                        const int seen = __builtin_amdgcn_readlane(pos, x) - 16 * t - 4 * g;
                        f32x4 y = o[dt];
#pragma unroll
                        for (int i = 0; i < 4; ++i) y = __builtin_amdgcn_mfma_f32_16x16x4f32(i <= seen ? vf[dt][i] : 0.f, p[i], y, 0, 0, 0);
                        o[dt] = c == x ? y : o[dt];
                    }
                } else {
#pragma unroll
                    for (int i = 0; i < 4; ++i) o[dt] = __builtin_amdgcn_mfma_f32_16x16x4f32(vf[dt][i], p[i], o[dt], 0, 0, 0);
                }
            }
            if (t + 4 < tiles) load_v(t + 4);
        }
    };
    walk(std::false_type{});
    float odd = 0.f;
#pragma unroll
    for (int dt = 0; dt < DT; ++dt)
#pragma unroll
        for (int i = 0; i < 4; ++i) odd = fmaf(o[dt][i], 0.f, odd);
    if (__any(odd != 0.f)) {                                // not finite: V of keys that a row does not see?
        load_k(wave);
        load_v(wave);
        walk(std::true_type{});
    }
    // ---- join the waves' parts (one without tiles has sum 0 at the lowest float) -------------------------------------------------
    l = wave_sum_from<16>(l);
    if (g == 0) { sm_m[wave][c] = m; sm_l[wave][c] = l; }
#pragma unroll
    for (int dt = 0; dt < DT; ++dt) *reinterpret_cast<f32x4*>(&sm_o[wave][c][16 * dt + 4 * g]) = o[dt];
    __syncthreads();
    for (int e = tid; e < 16 * (D / 4); e += 256) {
        const int x = e / (D / 4), col = e % (D / 4) * 4;
        if (r0 + x >= rows) continue;
        float top = fmaxf(fmaxf(sm_m[0][x], sm_m[1][x]), fmaxf(sm_m[2][x], sm_m[3][x])), sum = 0.f;
        f32x4 v = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int w = 0; w < 4; ++w) {
            const float f = exp2_fast(sm_m[w][x] - top);
            sum = fmaf(sm_l[w][x], f, sum);
            v += *reinterpret_cast<const f32x4*>(&sm_o[w][x][col]) * f;
        }
        const float rl = 1.0f / sum;
        const int p = (r0 + x) / a.G, hd = kh * a.G + r0 + x - p * a.G;
        *reinterpret_cast<f32x4*>(reinterpret_cast<float*>(a.out) + (int64_t)(sq.start + p) * a.o_st + (int64_t)hd * a.o_sh + col) = v * rl;
        if (a.ml != nullptr && col == 0 && p >= n - a.window) a.ml[(int64_t)(sq.start + p) * a.H + hd] = make_float2(top, rl);
    }
}

// ---------------------------------------------------------------------------------------------------------------------------------
// score[b,kh,j] = sum over the rows of the window of exp2(logit - maximum) / sum.  The logits are formed again: a wave has 64 keys in registers and
// meets the rows 16 at a time; a lane adds up what its 16 keys get.
// ---------------------------------------------------------------------------------------------------------------------------------
template <typename T, int D>
struct ScoreKeys {
    RowFrag<T, D> k[4];
    f32x4 sum[4];
    __device__ __forceinline__ void load(const PackedArgs& a, const Seq& sq, int kh, int k0, int g, int c) {
#pragma unroll
        for (int x = 0; x < 4; ++x) {
            k[x].load(reinterpret_cast<const T*>(a.k) + (int64_t)(sq.start + min(k0 + 16 * x + c, sq.n - 1)) * a.k_st + kh * a.k_sh, g);
            sum[x] = f32x4{0.f, 0.f, 0.f, 0.f};
        }
    }
    // 16 rows, this lane's at position pos (ml: maximum, one over the sum); MASKED: some may not see all of the keys k0 ..
    template <bool MASKED>
    __device__ __forceinline__ void add(const RowFrag<T, D>& q, float2 ml, int pos, float scale_l2, int k0, int g) {
#pragma unroll
        for (int x = 0; x < 4; ++x) {
            const f32x4 s = k[x].dot(q);
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const float p = exp2_fast(fmaf(s[i], scale_l2, -ml.x)) * ml.y;
                sum[x][i] += MASKED && k0 + 16 * x + 4 * g + i > pos ? 0.f : p;
            }
        }
    }
    __device__ __forceinline__ void finish(float* part, int g, int c) {
#pragma unroll
        for (int x = 0; x < 4; ++x)
#pragma unroll
            for (int i = 0; i < 4; ++i) sum[x][i] = group_sum<16>(sum[x][i]);
        if (c == 0) {
#pragma unroll
            for (int x = 0; x < 4; ++x) *reinterpret_cast<f32x4*>(part + 16 * x + 4 * g) = sum[x];
        }
    }
};

// The workgroup's four waves have the same keys and take the rows in turn, straight from memory, the next ones on their way: the shorter way where
// workgroups are few.
template <typename T, int D>
__global__ __launch_bounds__(256) void packed_score_deal_kernel(PackedArgs a) {
    __shared__ float part[4][64];
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), g = lane >> 4, c = lane & 15;
    const int kh = blockIdx.x, b = blockIdx.z, k0 = blockIdx.y * 64;
    const Seq sq = sequence(a, b);
    const int n = sq.n;
    if (k0 >= n) return;
    ScoreKeys<T, D> keys;
    keys.load(a, sq, kh, k0, g, c);
    const int from = max(max(0, n - a.window), k0), rows = n * a.G;     // (rows in front of the first key see none of them)
    RowFrag<T, D> qf, next;
    float2 ml, ml_next;
    int pos, pos_next;
    auto fetch = [&](int r0) {
        const int r = min(r0 + c, rows - 1);
        pos_next = r / a.G;
        const int head = kh * a.G + r - pos_next * a.G;
        next.load(reinterpret_cast<const T*>(a.q) + (int64_t)(sq.start + pos_next) * a.q_st + (int64_t)head * a.q_sh, g);
        ml_next = a.ml[(int64_t)(sq.start + pos_next) * a.H + head];
        if (r0 + c >= rows) pos_next = -1;                             // (a row that does not exist)
    };
    int r0 = from * a.G + 16 * wave;
    if (r0 < rows) fetch(r0);
    for (; r0 < rows; r0 += 64) {
        qf = next; pos = pos_next; ml = ml_next;
        if (r0 + 64 < rows) fetch(r0 + 64);
        keys.template add<true>(qf, ml, pos, a.scale_l2, k0, g);
    }
    keys.finish(part[wave], g, c);
    __syncthreads();
    if (tid < 64 && k0 + tid < n)
        a.score[b * a.s_sb + kh * a.s_sh + k0 + tid] = (part[0][tid] + part[1][tid]) + (part[2][tid] + part[3][tid]);
}

// The workgroup has 256 keys; all of its waves take all rows, which come through LDS, 16 KB of them at a time, the next ones on their way in registers.
// Bound by the exponentials and products of as many waves as the fullest SIMD has, and by the start.  16 prompts of 35 to 3136 tokens, windows of 32, 4
// heads of 128 a key head: 15.0 us; 2 of 6000 and 12288, windows of 64: 26.2.  (Each wave fetching rows for itself, 16 at a time: 21.8 and 33.9; 32 KB at
// a time: 17.5 and 32.5, more registers and fewer waves.)
template <typename T, int D>
__global__ __launch_bounds__(256, sizeof(T) == 2 ? 3 : 1) void packed_score_kernel(PackedArgs a) {
    constexpr int UPR = D * (int)sizeof(T) / 16, PER = 4, kRows = 256 * PER / UPR;       // 16-byte units of a row; rows in LDS; units a thread fetches
    __shared__ u32x4 sm_q[256 * PER];
    __shared__ float2 sm_ml[kRows];
    __shared__ float part[4][64];
    // unit u of row r lies at u ^ swz(r): the 16 rows that a fragment's lanes read lie in 16 different units of the banks
    auto swz = [](int row) { return UPR == 8 ? row >> 1 & 7 : row & 15; };
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), g = lane >> 4, c = lane & 15;
    const int kh = blockIdx.x, b = blockIdx.z, k_first = blockIdx.y * 256, k0 = k_first + wave * 64;
    const Seq sq = sequence(a, b);
    const int n = sq.n;
    if (k_first >= n) return;
    const int rows = n * a.G;
    int r0 = max(max(0, n - a.window), k_first) * a.G;                  // (rows in front of the first key see none of them)
    u32x4 raw[PER];
    float2 ml_raw;
    auto fetch = [&]() {
#pragma unroll
        for (int i = 0; i < PER; ++i) {
            const int e = tid + i * 256, r = min(r0 + e / UPR, rows - 1), p = r / a.G;
            const T* row = reinterpret_cast<const T*>(a.q) + (int64_t)(sq.start + p) * a.q_st + (int64_t)(kh * a.G + r - p * a.G) * a.q_sh;
            raw[i] = reinterpret_cast<const u32x4*>(row)[e % UPR];
        }
        if (tid < kRows) {
            const int r = min(r0 + tid, rows - 1), p = r / a.G;
            ml_raw = a.ml[(int64_t)(sq.start + p) * a.H + kh * a.G + r - p * a.G];
        }
    };
    fetch();
    ScoreKeys<T, D> keys;
    keys.load(a, sq, kh, k0, g, c);
    while (true) {
#pragma unroll
        for (int i = 0; i < PER; ++i) {
            const int e = tid + i * 256, row = e / UPR;
            sm_q[row * UPR + (e % UPR ^ swz(row))] = raw[i];
        }
        if (tid < kRows) sm_ml[tid] = ml_raw;
        __syncthreads();
        const int first = r0, here = min(kRows, rows - r0);
        r0 += kRows;
        if (r0 < rows) fetch();
#pragma unroll 1
        for (int x = 0; x < here; x += 16) {
            const int row = x + c;
            RowFrag<T, D> q;
#pragma unroll
            for (int s = 0; s < D * (int)sizeof(T) / 64; ++s) q.set(s, sm_q[row * UPR + ((4 * s + g) ^ swz(row))]);
            if (x + 16 > here || first + x < (k0 + 63) * a.G)
                keys.template add<true>(q, sm_ml[row], row < here ? (first + row) / a.G : -1, a.scale_l2, k0, g);
            else
                keys.template add<false>(q, sm_ml[row], 0, a.scale_l2, k0, g);
        }
        if (r0 >= rows) break;
        __syncthreads();
    }
    keys.finish(part[wave], g, c);
    if (k0 + lane < n) a.score[b * a.s_sb + kh * a.s_sh + k0 + lane] = part[wave][lane];     // (written by this wave)
}

// Dealt or not, in us, by blocks of 64 keys over all prompts.  128 rows: 40 5.0 / 7.4, 160 5.4 / 7.6, 352 8.4 / 8.8, 512 8.6 / 8.6, 704 11.1 / 8.5,
// 1024 14.3 / 9.6; 700 rows, whose steps weigh more than the start: 1024 25 / 31; 1600 rows: 96 17 / 53.
constexpr int kDealTiles = 512, kDealTilesOfManyRows = 1024, kManyRows = 256;
template <typename T, int D>
void launch_score(const PackedArgs& a, hipStream_t st) {
    const int64_t strips = (int64_t)a.Hk * a.B, tiles = (a.max_len + 63) / 64;
    const int deal = (int64_t)a.window * a.G > kManyRows ? kDealTilesOfManyRows : kDealTiles;
    if (tiles * strips <= deal) packed_score_deal_kernel<T, D><<<dim3(a.Hk, (unsigned)tiles, a.B), 256, 0, st>>>(a);
    else packed_score_kernel<T, D><<<dim3(a.Hk, (unsigned)((tiles + 3) / 4), a.B), 256, 0, st>>>(a);
}

// How a launch is cut, by the number of row tiles of 64 over all key heads and by the longest prompt.  Few tiles: one column of rows a wave, twice
// the workgroups, each with the shorter step; and where the walk over the keys is long, two groups of waves share it.  us with 1 / 1 shared / 2 / 2
// shared columns:
//   tiles  104   1 x 200   14.1  14.2  17.0  17.5          704   2 x 700   26.7  34.7  31.1  29.7
//          152   1 x 300   15.0  14.3  18.4  17.9          752   1 x 1500  43.2  50.3  50.6  39.5
//          256   1 x 500   20.1  17.6  24.3  22.1         1000   1 x 2000  57.7  72.5  63.9  55.6
//          504   1 x 1000  31.6  29.4  38.0  31.0         1408   4 x 700   39.9  62.6  36.9  49.6
//          512   8 x 120   14.5  20.1  16.5  17.5         1568   1 x 3136   109   151   104   114
//          600   3 x 400   20.9  28.6  23.8  26.2         1920   4 x 739   59.5  89.1  50.7  70.3
//   (32 heads over 8 of 128, the last row 40 over 40.  Three groups: within 1 us of two.)
struct PackedCut { int cols, split; };
inline PackedCut packed_cut(int64_t tiles64, int max_len) {
    if (tiles64 <= 512) return PackedCut{1, max_len > 256 ? 2 : 1};
    if (tiles64 <= 1024) return max_len > 1024 ? PackedCut{2, 2} : PackedCut{1, 1};
    return PackedCut{2, 1};
}
// No more row tiles than this, whatever the lengths are: each sequence has one that is not full.
inline int64_t packed_tiles(const st3_gqa_shape* s, int total, int max_len, int rows) {
    const int G = s->heads / s->kv_heads;
    return std::min((int64_t)total * G / rows + std::min(s->batch, total), ((int64_t)max_len * G + rows - 1) / rows * s->batch);
}
// Row tiles dealt over the prompts at a launch's end, as workgroups: all the tiles of 32 x 739 tokens, 40 key heads, in order of their length 499 us,
// no dealing 368, 768 to 3000 364 to 380; 4 x 700 42 without, 36 with; 8 x 3136, 32 key heads, 809 / 722 / 710 at 1536.
constexpr int kSpread = 1536;
template <int D>
void launch_packed(const PackedArgs& a, PackedCut cut, unsigned grid, hipStream_t st) {
    if (cut.cols == 1 && cut.split == 1) packed_kernel<D, 1, 1><<<grid, 256, 0, st>>>(a);
    else if (cut.cols == 1) packed_kernel<D, 1, 2><<<grid, 512, 0, st>>>(a);
    else if (cut.split == 2) packed_kernel<D, 2, 2><<<grid, 512, 0, st>>>(a);
    else packed_kernel<D, 2, 1><<<grid, 256, 0, st>>>(a);
}

}  // namespace
}  // namespace st3

extern "C" size_t st3_packed_workspace_bytes(const st3_gqa_shape* shape, int32_t total) {
    if (st3::check_gqa_shape(shape) != ST3_OK || total < 0) return 0;
    return st3::align_up((size_t)total * shape->heads * sizeof(float2), 256);
}

extern "C" st3_status st3_packed_attention(const st3_gqa_shape* shape, const st3_rows* q, const st3_rows* k, const st3_rows* v,
                                           const int32_t* cu_len, int32_t total, int32_t max_len, const st3_rows* out, int32_t window,
                                           float* score, int64_t score_stride_b, int64_t score_stride_h, void* workspace,
                                           size_t workspace_bytes, void* stream) {
    using namespace st3;
    st3_status s = check_gqa_shape(shape);
    if (s != ST3_OK) return s;
    const int H = shape->heads, Hk = shape->kv_heads, D = shape->head_dim, eb = elem_bytes(shape->dtype), G = H / Hk;
    if (!cu_len || total < 0 || max_len < 0 || max_len > total || window < 0) return ST3_ERR_INVALID_ARG;
    if (total == 0) return ST3_OK;          // (an empty tensor may have no address)
    for (const st3_rows* r : {q, k, v})
        if ((s = check_rows(r, D, eb)) != ST3_OK) return s;
    if ((s = check_output(out, H, total, D, eb)) != ST3_OK) return s;
    if ((int64_t)max_len * G > kMostRows || k->stride_t * eb * 32 >= (int64_t)1 << 31 || v->stride_t * eb * 32 >= (int64_t)1 << 31) return ST3_ERR_UNSUPPORTED;
    if (max_len == 0) return ST3_OK;
    if (packed_rows_meet(q, H, out, H, total, D, eb) || packed_rows_meet(k, Hk, out, H, total, D, eb) || packed_rows_meet(v, Hk, out, H, total, D, eb))
        return ST3_ERR_INVALID_ARG;
    if (score) {
        if (window < 1 || score_stride_h < max_len || (shape->batch > 1 && score_stride_b < max_len)) return ST3_ERR_INVALID_ARG;
        if (!workspace || !aligned16(workspace)) return ST3_ERR_INVALID_ARG;
        if (workspace_bytes < st3_packed_workspace_bytes(shape, total)) return ST3_ERR_WORKSPACE_TOO_SMALL;
    }
    hipStream_t st = reinterpret_cast<hipStream_t>(stream);
    PackedArgs a{q->data, k->data, v->data, out->data, q->stride_t, q->stride_h, k->stride_t, k->stride_h, v->stride_t, v->stride_h, out->stride_t,
                 out->stride_h, cu_len, shape->batch, total, max_len, H, Hk, G, 0, 0, gqa_scale_log2(shape), score, score_stride_b, score_stride_h,
                 score ? reinterpret_cast<float2*>(workspace) : nullptr, window};
    const PackedCut cut = packed_cut(packed_tiles(shape, total, max_len, 64) * Hk, max_len);
    const int rows = shape->dtype == ST3_BF16 ? 64 * cut.cols : 16;
    a.levels = (int)(((int64_t)max_len * G + rows - 1) / rows);
    a.spread = (kSpread + Hk - 1) / Hk;
    const int64_t tiles = packed_tiles(shape, total, max_len, rows);
    if (!grid_fits(tiles * Hk, shape->dtype == ST3_BF16 ? 256 * cut.split : 256, 1)) return ST3_ERR_UNSUPPORTED;
    if (score && (max_len + 63) / 64 > 65535) return ST3_ERR_UNSUPPORTED;
    const unsigned grid = (unsigned)(tiles * Hk);
    if (shape->dtype == ST3_BF16) {
        if (D == 128) launch_packed<128>(a, cut, grid, st);
        else launch_packed<64>(a, cut, grid, st);
    } else {
        if (D == 128) packed_f32_kernel<128><<<grid, 256, 0, st>>>(a);
        else packed_f32_kernel<64><<<grid, 256, 0, st>>>(a);
    }
    if (score) {
        if (shape->dtype == ST3_BF16) {
            if (D == 128) launch_score<bf16_t, 128>(a, st);
            else launch_score<bf16_t, 64>(a, st);
        } else {
            if (D == 128) launch_score<float, 128>(a, st);
            else launch_score<float, 64>(a, st);
        }
    }
    return check_launch();
}
