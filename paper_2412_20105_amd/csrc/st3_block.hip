// The cache of 8-bit blocks: packed prompts into pages, further rows behind them, and eviction by accumulated weight into other pages.
//
// A workgroup of 256 threads makes K or V of one block of one key head.  A thread holds four rows that follow each other and d / 16 columns that do
// (Place): for K 16 threads in a row have a row group's columns, so that they read and write whole rows; for V they have a column's rows, so that
// four codes make a word and 16 words a column of the page, without a trip through LDS.  Bound by memory: both read and write what they must once,
// but for the lines of a page's V of which an eviction keeps a part.  A workgroup is a chain of a few trips to memory; with K and V in workgroups of
// their own there are twice as many, of half the registers, beside each other.
#include <algorithm>
#include <utility>

#include "st3_block.h"
#include "st3_rotary.h"

namespace st3 {
namespace {

constexpr int kThreads = 256;
constexpr int kRankThreads = 1024;         // (by the radix alone, 8 strips of 1200 rows: 512 as long as 1024, 256 a third longer)

// A thread's part of a block: rows row .. + 3, columns col .. + d / 16 - 1.
template <int D, bool COLUMNS>
struct Place {
    int row, col;
    __device__ __forceinline__ explicit Place(int tid) {
        const int fast = tid & 15, slow = tid >> 4;
        row = 4 * (COLUMNS ? fast : slow);
        col = D / 16 * (COLUMNS ? slow : fast);
    }
};

// Codes a block of K (COLUMNS: of V) from the threads' values v [row][column] into a page (past the caches: 16 prompts into pages 20.3 -> 18.7 us).
// SPLIT (K only): the thread's columns are two runs, from `first` and from `second` on.
template <int D, int CODE, bool COLUMNS, bool SPLIT = false>
__device__ __forceinline__ void write_block(float (&v)[4][D / 16], const BlockPages& c, int64_t at, uint32_t* sm, int tid, int first = 0, int second = 0) {
    using F = BlockCode<CODE>;
    constexpr int W = D / 16;
    const Place<D, COLUMNS> my(tid);
    uint32_t mx = 0;
#pragma unroll
    for (int r = 0; r < 4; ++r)
#pragma unroll
        for (int e = 0; e < W; ++e) mx = max(mx, magnitude(v[r][e]));
    uint32_t top = largest_of<kThreads / 64>(mx, sm, tid);
    const bool all_finite = top < kInfinity;
    if (!all_finite) {                                      // (rare: without the magnitudes from above, which would wait in registers)
        float f = 0.f;
#pragma unroll
        for (int r = 0; r < 4; ++r)
#pragma unroll
            for (int e = 0; e < W; ++e) f = fmaxf(f, fabsf(v[r][e]) <= 3.402823466e38f ? fabsf(v[r][e]) : 0.f);
        top = largest_of<kThreads / 64>(__float_as_uint(f), sm + kThreads / 64, tid);
    }
    const Divider divide(__uint_as_float(top) * F::kUnit, __uint_as_float(top), all_finite);
    if (tid == 0) (COLUMNS ? c.v_scale : c.k_scale)[at] = divide.scale;
    if (divide.care) {
#pragma unroll
        for (int r = 0; r < 4; ++r)
#pragma unroll
            for (int e = 0; e < W; ++e) v[r][e] = divide.careful(v[r][e], F::nan_code(), F::kMost);
    }
    uint8_t* codes = (COLUMNS ? c.v_codes : c.k_codes) + at * (kBlk * D);
    if constexpr (COLUMNS) {
#pragma unroll
        for (int e = 0; e < W; ++e) {
            const float x[4] = {v[0][e], v[1][e], v[2][e], v[3][e]};
            __builtin_nontemporal_store(F::code4(x, divide), reinterpret_cast<uint32_t*>(codes + (my.col + e) * kBlk + my.row));
        }
    } else if constexpr (SPLIT) {
#pragma unroll
        for (int r = 0; r < 4; ++r) {
            uint8_t* to = codes + (my.row + r) * D;
            const float rear[4] = {v[r][W / 2], v[r][W / 2 + 1], W == 8 ? v[r][W - 2] : 0.f, W == 8 ? v[r][W - 1] : 0.f};
            if constexpr (W == 8) {
                __builtin_nontemporal_store(F::code4(v[r], divide), reinterpret_cast<uint32_t*>(to + first));
                __builtin_nontemporal_store(F::code4(rear, divide), reinterpret_cast<uint32_t*>(to + second));
            } else {                                        // two codes each
                const uint32_t w = F::code4(v[r], divide);
                *reinterpret_cast<uint16_t*>(to + first) = (uint16_t)w;
                *reinterpret_cast<uint16_t*>(to + second) = (uint16_t)(w >> 16);
            }
        }
    } else {
#pragma unroll
        for (int r = 0; r < 4; ++r) {
            uint8_t* to = codes + (my.row + r) * D + my.col;
            if constexpr (W == 8) {
                const u32x2 w = {F::code4(v[r], divide), F::code4(v[r] + 4, divide)};
                __builtin_nontemporal_store(w, reinterpret_cast<u32x2*>(to));
            } else {
                __builtin_nontemporal_store(F::code4(v[r], divide), reinterpret_cast<uint32_t*>(to));
            }
        }
    }
}

// The rows [0, rows) of a partial block into a tail; bits(r, e): the thread's row r, column e.
template <int D, bool COLUMNS, typename Bits>
__device__ __forceinline__ void write_tail(const Bits& bits, const BlockPages& c, int64_t strip, int rows, int tid) {
    const Place<D, COLUMNS> my(tid);
    uint16_t* tail = (COLUMNS ? c.v_tail : c.k_tail) + strip * (kBlk * D);
#pragma unroll
    for (int r = 0; r < 4; ++r) {
        if (my.row + r >= rows) continue;
#pragma unroll
        for (int e = 0; e < D / 16; ++e) tail[COLUMNS ? (my.col + e) * kBlk + my.row + r : (my.row + r) * D + my.col + e] = bits(r, e);
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
// prompts into pages: workgroup (K or V of a key head, block, sequence).  16 prompts of 35 to 3136 tokens, 8 key heads of 128: 76 MB in 16.5 us, 4.6
// TB/s.
// ---------------------------------------------------------------------------------------------------------------------------------
struct StoreArgs {
    BlockPages c;
    const uint16_t* k; const uint16_t* v;
    int64_t k_st, k_sh, v_st, v_sh;
    const int32_t* cu;
    int32_t total, max_len, Hk;
};

template <int D, int CODE, bool COLUMNS>
__device__ __forceinline__ void store_block(const StoreArgs& a, int kh, int j, int b, uint32_t* sm) {
    constexpr int W = D / 16;
    const int tid = threadIdx.x;
    const Place<D, COLUMNS> my(tid);
    const int page = page_of(a.c, b, j);                    // (on its way beside the lengths)
    const int start = max(0, min(a.cu[b], a.total)), n = min(max(start, min(a.cu[b + 1], a.total)) - start, a.max_len);
    if (j * kBlk >= n) return;
    const uint16_t* src = (COLUMNS ? a.v + kh * a.v_sh : a.k + kh * a.k_sh) + my.col;
    const int64_t stride = COLUMNS ? a.v_st : a.k_st;
    uint32_t raw[4][W / 2];
#pragma unroll
    for (int r = 0; r < 4; ++r) load_bf16<W>(src + (start + min(j * kBlk + my.row + r, n - 1)) * stride, raw[r]);
    if ((j + 1) * kBlk > n) {
        write_tail<D, COLUMNS>([&](int r, int e) { return (uint16_t)(raw[r][e / 2] >> (16 * (e & 1))); }, a.c, (int64_t)b * a.Hk + kh, n - j * kBlk, tid);
        return;
    }
    if (page < 0) return;
    float v[4][W];
#pragma unroll
    for (int r = 0; r < 4; ++r)
#pragma unroll
        for (int e = 0; e < W; e += 2) { v[r][e] = bf16_lo(raw[r][e / 2]); v[r][e + 1] = bf16_hi(raw[r][e / 2]); }
    write_block<D, CODE, COLUMNS>(v, a.c, (int64_t)page * a.Hk + kh, sm, tid);
}

template <int D, int CODE>
__global__ __launch_bounds__(kThreads, 8) void block_store_kernel(StoreArgs a) {
    __shared__ uint32_t sm[2 * kThreads / 64];
    const int kh = blockIdx.x % a.Hk;
    if ((int)blockIdx.x < a.Hk) store_block<D, CODE, false>(a, kh, blockIdx.y, blockIdx.z, sm);
    else store_block<D, CODE, true>(a, kh, blockIdx.y, blockIdx.z, sm);
}

// ---------------------------------------------------------------------------------------------------------------------------------
// further rows: workgroup (K or V of a key head, block from the first that takes new rows on, sequence).  The first one alone reads the tail, and so it
// also writes what is the tail afterwards.
// ---------------------------------------------------------------------------------------------------------------------------------
struct AppendArgs {
    BlockPages c;
    const uint16_t* k; const uint16_t* v;
    int64_t k_st, k_sh, v_st, v_sh;
    const int32_t* cu;
    Rotation r;
    int32_t total, max_new, max_len, Hk;
};

// A thread's columns, two runs of D / 32.  Where the halves of a row turn against each other they are a pair's two sides, and those of the last threads
// the columns that do not turn; else they follow each other.
enum Turn { kStill, kHalves, kAdjacent };
template <int D, int TURN>
struct Runs {
    static constexpr int R = D / 32;
    int first, second;
    __device__ __forceinline__ Runs(int fast, int pairs) {
        if (TURN == kHalves && fast < pairs / R) {
            first = R * fast;
            second = first + pairs;
        } else {
            first = 2 * R * fast;
            second = first + R;
        }
    }
};

// Four rows of a thread's columns on their way, with the cosines and sines that turn them; rows outside [0, m) are the nearest.
template <int D, bool COLUMNS, int TURN>
struct NewRows {
    static constexpr int R = D / 32;                        // columns of a run, pairs of a thread
    uint32_t raw[4][R];                                     // two bf16 each: the first run, the second
    float4 cs[4][R / 2];
    bool turns;
    __device__ __forceinline__ void load(const AppendArgs& a, const Runs<D, TURN>& my, int kh, int start, int m, int row) {
        const uint16_t* src = COLUMNS ? a.v + kh * a.v_sh : a.k + kh * a.k_sh;
        const int64_t stride = COLUMNS ? a.v_st : a.k_st;
        turns = TURN != kStill && !COLUMNS && my.first < (TURN == kHalves ? a.r.pairs : 2 * a.r.pairs);
#pragma unroll
        for (int r = 0; r < 4; ++r) {
            const int t = start + max(0, min(row + r, m - 1));
            const uint16_t* at = src + t * stride;
            if constexpr (TURN == kHalves && !COLUMNS) {
                run(at + my.first, raw[r]);
                run(at + my.second, raw[r] + R / 2);
            } else {
                load_bf16<2 * R>(at + my.first, raw[r]);
            }
            if constexpr (TURN != kStill && !COLUMNS) {
                const float4* from = reinterpret_cast<const float4*>(a.r.table + t * a.r.stride + (turns ? (TURN == kHalves ? 2 * my.first : my.first) : 0));
#pragma unroll
                for (int e = 0; e < R / 2; ++e) cs[r][e] = from[e];
            }
        }
    }
    __device__ __forceinline__ static void run(const uint16_t* p, uint32_t* to) {
        if constexpr (R == 4) {
            const uint2 q = *reinterpret_cast<const uint2*>(p);
            to[0] = q.x;
            to[1] = q.y;
        } else {
            to[0] = *reinterpret_cast<const uint32_t*>(p);
        }
    }
    __device__ __forceinline__ void turn_all() {
        if (!turns) return;
#pragma unroll
        for (int r = 0; r < 4; ++r)
#pragma unroll
            for (int e = 0; e < R / 2; ++e) {               // two pairs
                const float4 x = cs[r][e];
                uint32_t& u = raw[r][TURN == kHalves ? e : 2 * e];
                uint32_t& w = raw[r][TURN == kHalves ? R / 2 + e : 2 * e + 1];
                float p[4] = {bf16_lo(u), bf16_hi(u), bf16_lo(w), bf16_hi(w)};
                if constexpr (TURN == kHalves) {
                    turn(p[0], p[2], x.x, x.y);
                    turn(p[1], p[3], x.z, x.w);
                } else {
                    turn(p[0], p[1], x.x, x.y);
                    turn(p[2], p[3], x.z, x.w);
                }
                u = bf16_pair(p[0], p[1]);
                w = bf16_pair(p[2], p[3]);
            }
    }
    __device__ __forceinline__ uint16_t bits(int r, int e) const { return (uint16_t)(raw[r][e / 2] >> (16 * (e & 1))); }
};

template <int D, int CODE, bool COLUMNS, int TURN>
__device__ __forceinline__ void append_block(const AppendArgs& a, int kh, int j, int b, uint32_t* sm) {
    constexpr int W = D / 16, R = W / 2, kTurn = COLUMNS ? kStill : TURN;
    const int tid = threadIdx.x;
    const int row = 4 * (COLUMNS ? tid & 15 : tid >> 4);    // (Place)
    const Runs<D, kTurn> my(COLUMNS ? tid >> 4 : tid & 15, a.r.pairs);
    auto column = [&](int e) { return e < R ? my.first + e : my.second + e - R; };
    const int n = a.c.len[b], start = max(0, min(a.cu[b], a.total));
    const int m = min(min(max(start, min(a.cu[b + 1], a.total)) - start, a.max_new), a.max_len - n);
    if (n < 0 || n >= a.max_len || m <= 0) return;
    const int first = n / kBlk, at = (first + j) * kBlk, total = n + m, rest = total % kBlk, held = j == 0 ? n % kBlk : 0;
    const int64_t strip = (int64_t)b * a.Hk + kh;
    if (at >= total || (j > 0 && at + kBlk > total)) return;        // (the last, partial block is the first workgroup's)
    const bool whole = at + kBlk <= total, more = j == 0 && whole && rest > 0;
    const int page = whole ? page_of(a.c, b, first + j) : -1;
    uint16_t* tail = (COLUMNS ? a.c.v_tail : a.c.k_tail) + strip * (kBlk * D);
    NewRows<D, COLUMNS, kTurn> now, behind;
    now.load(a, my, kh, start, m, at + row - n);
    if (more) behind.load(a, my, kh, start, m, total - rest + row - n);
    uint32_t old[4][R];
    if (whole && row < held) {                              // the block's rows that are in the tail
        if constexpr (COLUMNS) {
            uint32_t pair[W][2];
#pragma unroll
            for (int e = 0; e < W; ++e) {
                const uint2 x = *reinterpret_cast<const uint2*>(tail + column(e) * kBlk + row);
                pair[e][0] = x.x;
                pair[e][1] = x.y;
            }
#pragma unroll
            for (int r = 0; r < 4; ++r)
#pragma unroll
                for (int e = 0; e < W; e += 2)
                    old[r][e / 2] = __builtin_amdgcn_perm(pair[e + 1][r / 2], pair[e][r / 2], r & 1 ? 0x07060302u : 0x05040100u);
        } else {
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                NewRows<D, COLUMNS, kTurn>::run(tail + (row + r) * D + my.first, old[r]);
                NewRows<D, COLUMNS, kTurn>::run(tail + (row + r) * D + my.second, old[r] + R / 2);
            }
        }
    }
    now.turn_all();
    if (whole) {
        if (row < held) {
#pragma unroll
            for (int r = 0; r < 4; ++r)
#pragma unroll
                for (int e = 0; e < R; ++e) now.raw[r][e] = row + r < held ? old[r][e] : now.raw[r][e];
        }
        if (page >= 0) {
            float v[4][W];
#pragma unroll
            for (int r = 0; r < 4; ++r)
#pragma unroll
                for (int e = 0; e < W; e += 2) { v[r][e] = bf16_lo(now.raw[r][e / 2]); v[r][e + 1] = bf16_hi(now.raw[r][e / 2]); }
            write_block<D, CODE, COLUMNS, kTurn == kHalves>(v, a.c, (int64_t)page * a.Hk + kh, sm, tid, my.first, my.second);
        }
        if (!more) return;
        behind.turn_all();
        __syncthreads();                                    // (all have read the tail)
    }
    const NewRows<D, COLUMNS, kTurn>& x = more ? behind : now;      // rows of the tail, behind those that stay
    const int from = more ? 0 : held;
#pragma unroll
    for (int r = 0; r < 4; ++r) {
        if (row + r < from || row + r >= rest) continue;
#pragma unroll
        for (int e = 0; e < W; ++e) tail[COLUMNS ? column(e) * kBlk + row + r : (row + r) * D + column(e)] = x.bits(r, e);
    }
}

template <int D, int CODE, int TURN>
__global__ __launch_bounds__(kThreads) void block_append_kernel(AppendArgs a) {
    __shared__ uint32_t sm[2 * kThreads / 64];
    const int kh = blockIdx.x % a.Hk;
    if ((int)blockIdx.x < a.Hk) append_block<D, CODE, false, TURN>(a, kh, blockIdx.y, blockIdx.z, sm);
    else append_block<D, CODE, true, TURN>(a, kh, blockIdx.y, blockIdx.z, sm);
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

// Greater means better; NaN below everything, -0 as +0.  0 is left for rows that do not exist, what is above kRankTop for rows kept whatever their score.
constexpr uint32_t kRankTop = 0xff800000u;      // (an infinity)
__device__ __forceinline__ uint32_t rank_key(float x) {
    if (!(x == x)) return 1;
    const uint32_t u = __float_as_uint(x == 0.f ? 0.f : x);
    return u & 0x80000000u ? ~u : u | 0x80000000u;
}

// Sums over the workgroup's waves before this one, and over all, of a value that is the same in a wave's lanes; waves: a word for each wave.
__device__ __forceinline__ uint2 waves_before(uint32_t mine, uint32_t* waves, int lane, int wave) {
    constexpr int kWaves = kRankThreads / 64;
    if (lane == 0) waves[wave] = mine;
    __syncthreads();
    const int upto = wave_prefix(lane < kWaves ? (int)waves[lane] : 0);     // (each wave for itself; picked one by one they took 0.5 us)
    return make_uint2(wave > 0 ? __builtin_amdgcn_readlane(upto, wave - 1) : 0, __builtin_amdgcn_readlane(upto, kWaves - 1));
}

// Workgroup (key head, sequence): the key of the last row kept by a radix search (12 + 10 + 10 bits; as soon as a bin holds kFew rows or less, their
// places among each other are counted instead), then the rows kept, their scores, and, of the rows with that last key, as many of the first as
// are wanted.  A wave holds 64 PER rows that follow each other, lane by lane, so that loads and stores are whole lines and places are counts of
// ballots; LONG: any number of rows, 1024 PER at a time, read again in every pass.  Bound by its chain of passes and barriers: 8 strips
// of 1200 rows 5.8 us (7.9 by the radix alone, 11 + 11 + 10 bits, with threads that hold rows in a row), 256 of up to 3136 6.9 (9.5), 40 of 12596 12.7
// (20.1), 40 of up to 18347 20.3 (LONG 30.3).
constexpr int kFew = 128;
template <int PER, bool LONG>
__global__ __launch_bounds__(kRankThreads) void block_rank_kernel(EvictBlockArgs a) {
    constexpr int kTop = 4096, kBins = kTop / kRankThreads, kRows = PER * kRankThreads;
    static_assert(kRows <= 32768, "counts of a chunk's rows in 16 bits");
    __shared__ uint32_t hist[kTop];
    __shared__ uint32_t waves[2][kRankThreads / 64];
    __shared__ uint32_t found[3];
    __shared__ uint32_t few[kFew], n_few;
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), kh = blockIdx.x, b = blockIdx.y;
    const float* score = a.score + b * a.s_sb + kh * a.s_sh;
    const int mine = wave * (64 * PER) + lane;              // + 64 i: this thread's rows of a chunk
    float x[PER];
    uint32_t u[PER];
    auto load = [&](int base) {
#pragma unroll
        for (int i = 0; i < PER; ++i) x[i] = base + mine + 64 * i < a.max_len ? score[base + mine + 64 * i] : 0.f;
    };
    if constexpr (!LONG) load(0);                           // (on their way beside the length)
    const int n = min(a.from.len[b], a.max_len);
    if (n < 0) return;
    float* to = a.to_score + b * a.t_sb + kh * a.t_sh;
    int32_t* kept = a.kept + b * a.i_sb + kh * a.i_sh;
    const int lo = a.n_sink, hi = n - a.n_recent;
    const bool all = n <= a.keep;
    uint32_t want = all ? 0 : a.keep - a.n_sink - a.n_recent;   // candidates wanted, at last of those with the last key
    uint32_t key = want > 0 ? 0 : kRankTop, mask = 0;
    auto rank = [&](int base) {
#pragma unroll
        for (int i = 0; i < PER; ++i) {
            const int r = base + mine + 64 * i;
            u[i] = r >= n ? 0 : all || r < lo || r >= hi ? 0xffffffffu : rank_key(x[i]);
        }
    };
    if constexpr (!LONG) rank(0);
    auto each = [&](auto f) {                                   // the candidates that share the key's leading bits
        for (int base = 0; base < (LONG ? n : 1); base += kRows) {
            if constexpr (LONG) { load(base); rank(base); }
#pragma unroll
            for (int i = 0; i < PER; ++i)
                if (u[i] - 1 < kRankTop && (u[i] & mask) == key) f(u[i]);
        }
    };
    for (int pass = 0; pass < 3 && want > 0; ++pass) {
        const int shift = pass == 0 ? 20 : pass == 1 ? 10 : 0;
        const uint32_t low = pass == 0 ? 0xfff : 0x3ff;
#pragma unroll
        for (int i = 0; i < kBins; ++i) hist[tid + i * kRankThreads] = 0;
        if (tid == 0) n_few = 0;
        __syncthreads();
        each([&](uint32_t u) {
            atomicAdd(&hist[(u >> shift) & low], 1u);
        });
        __syncthreads();
        // bins from the top: thread t owns kBins of them
        uint32_t h[kBins], sum = 0;
#pragma unroll
        for (int i = 0; i < kBins; ++i) { h[i] = hist[kTop - 1 - kBins * tid - i]; sum += h[i]; }
        const uint32_t incl = wave_prefix((int)sum);
        uint32_t before = incl - sum + waves_before(__builtin_amdgcn_readlane(incl, 63), waves[0], lane, wave).x;
#pragma unroll
        for (int i = 0; i < kBins; ++i) {
            if (before < want && before + h[i] >= want) { found[0] = kTop - 1 - kBins * tid - i; found[1] = want - before; found[2] = h[i]; }
            before += h[i];
        }
        __syncthreads();
        key |= found[0] << shift;
        mask |= low << shift;
        want = found[1];
        const uint32_t here = found[2];
        __syncthreads();
        if (here <= kFew && pass < 2) {
            each([&](uint32_t u) {
                few[atomicAdd(&n_few, 1u)] = u;             // (in any order: only values are compared)
            });
            __syncthreads();
            constexpr int kTeam = kRankThreads / kFew;          // threads that count for one of them
            const uint32_t one = tid / kTeam;
            if (one < here) {
                const uint32_t u = few[one];
                uint32_t more = 0, same = 0;
                for (uint32_t i = tid % kTeam; i < here; i += kTeam) { more += few[i] > u ? 1 : 0; same += few[i] == u ? 1 : 0; }
#pragma unroll
                for (int off = 1; off < kTeam; off <<= 1) { more += __shfl_xor(more, off); same += __shfl_xor(same, off); }
                if (more < want && more + same >= want) { found[0] = u; found[1] = want - more; }       // (equal ones write the same)
            }
            __syncthreads();
            key = found[0];
            want = found[1];
            break;
        }
    }
    // Rows written and rows with the last key met, by the chunks before.  (A chunk's scores are read before any of its rows is written, and a row moves
    // to the front if at all: to_score may be score.)
    uint32_t out = 0, ties = 0;
    for (int base = 0, turn = 0; base < (LONG ? n : 1); base += kRows, turn ^= 1) {
        if constexpr (LONG) { load(base); rank(base); }
        uint32_t count = 0;                                 // the wave's rows above the key, and from bit 16 on those with it
#pragma unroll
        for (int i = 0; i < PER; ++i) count += __popcll(__ballot(u[i] > key)) + (__popcll(__ballot(want > 0 && u[i] == key)) << 16);
        const uint2 sums = waves_before(count, waves[turn], lane, wave);
        uint32_t at = out + (sums.x & 0xffff), met = ties + (sums.x >> 16);     // of ties, the first `want` of all are kept
        at += min(met, want) - min(ties, want);
#pragma unroll
        for (int i = 0; i < PER; ++i) {
            const uint64_t tied = __ballot(want > 0 && u[i] == key), below = (1ull << lane) - 1;
            const bool keep = u[i] > key || (want > 0 && u[i] == key && met + __popcll(tied & below) < want);
            const uint64_t all_kept = __ballot(keep);
            if (keep) {
                const uint32_t place = at + __popcll(all_kept & below);
                kept[place] = base + mine + 64 * i;
                to[place] = x[i];
            }
            at += __popcll(all_kept);
            met += __popcll(tied);
        }
        const uint32_t ties_now = ties + (sums.y >> 16);
        out += (sums.y & 0xffff) + min(ties_now, want) - min(ties, want);
        ties = ties_now;
    }
    for (int i = min(n, a.keep) + tid; i < a.keep; i += kRankThreads) kept[i] = -1;
}

// Workgroup (K or V of a key head, new block, sequence).  K's rows are fetched one by one; any row of a page lies in all lines of its V, so V comes
// as whole pages, two at a time (a block's rows ascend: a few pages that follow each other), and is picked from LDS.  (Picked byte by byte from
// memory it kept the address units busy: 32 caches 84 us.)  32 caches of 611 to 3136 rows to 1500 rows: 189 MB in 52 us, 3.6 TB/s, the vector units
// busy for 51 % of the cycles with codes, values and quotients; with registers for 5 waves a SIMD instead of 6 it takes 59.
constexpr int kPageRow = kBlk + 8;          // bytes: the 4 columns that a wave picks at a time, 8 apart, are 16 banks apart
template <int D, int CODE, bool COLUMNS>
__device__ __forceinline__ void move_block(const EvictBlockArgs& a, int kh, int j, int b, uint8_t* pages, uint32_t* sm) {
    using F = BlockCode<CODE>;
    constexpr int W = D / 16, kPage = D * kBlk, kPiece = kPage / 16 / kThreads;       // 16-byte pieces of a page a thread fetches
    const int tid = threadIdx.x, lane = tid & 63;
    const Place<D, COLUMNS> my(tid);
    // lane i looks up row i (every wave all of them): its old block, and that block's page (what stands there for rows that are not kept is not used)
    const int32_t* kept = a.kept + b * a.i_sb + kh * a.i_sh;
    const int first = j * kBlk, raw_l = kept[min(first + lane, a.keep - 1)];
    const int to_page_any = page_of(a.to, b, j);
    int row_l = max(0, min(raw_l, a.max_len - 1));
    int page_l = page_of(a.from, b, row_l / kBlk);
    const int n = min(a.from.len[b], a.max_len), count = min(n, a.keep);
    if (first >= count) return;
    const bool whole = first + kBlk <= count;
    const int to_page = whole ? to_page_any : 0;
    if (to_page < 0) return;
    const int last = count - 1 - first;                     // (lanes past the last row repeat it)
    const int row_last = __shfl(row_l, min(last, 63)), page_last = __shfl(page_l, min(last, 63));
    if (lane > last) { row_l = row_last; page_l = page_last; }
    const int blk_l = row_l < n / kBlk * kBlk ? row_l / kBlk : -1;      // -1: in the tail
    if (blk_l < 0) page_l = -1;
    const float* scales = COLUMNS ? a.from.v_scale : a.from.k_scale;
    const uint8_t* codes = COLUMNS ? a.from.v_codes : a.from.k_codes;
    const int64_t strip = (int64_t)b * a.Hk + kh, to_at = (int64_t)to_page * a.Hk + kh, at_l = (int64_t)max(page_l, 0) * a.Hk + kh;
    const float scale_l = page_l >= 0 ? scales[at_l] : 0.f;
    if (whole && __ballot(page_l >= 0 && row_l % kBlk == lane && blk_l == __builtin_amdgcn_readfirstlane(blk_l)) == ~0ull) {     // one whole old block
        uint8_t* to = (COLUMNS ? a.to.v_codes : a.to.k_codes) + to_at * kPage;
        for (int i = tid; i < kPage / 16; i += kThreads) reinterpret_cast<uint4*>(to)[i] = reinterpret_cast<const uint4*>(codes + at_l * kPage)[i];
        if (tid == 0) (COLUMNS ? a.to.v_scale : a.to.k_scale)[to_at] = scale_l;
        return;
    }
    float v[4][W], scale[4];
    int row[4], blk[4];
#pragma unroll
    for (int r = 0; r < 4; ++r) {
        row[r] = __shfl(row_l, my.row + r) % kBlk;
        blk[r] = __shfl(blk_l, my.row + r);
        scale[r] = __shfl(scale_l, my.row + r);
    }
    if constexpr (COLUMNS) {
        uint64_t left = __ballot(page_l >= 0);              // rows whose pages are still to come (in every wave alike)
        u32x4 piece[2][kPiece];
        int now[2];
        auto fetch = [&]() {
#pragma unroll
            for (int p = 0; p < 2; ++p) {
                const int lead = left != 0 ? __ffsll((unsigned long long)left) - 1 : 0;
                now[p] = left != 0 ? __builtin_amdgcn_readlane(blk_l, lead) : -2;
                const int64_t at = (int64_t)max(__builtin_amdgcn_readlane(page_l, lead), 0) * a.Hk + kh;
                const u32x4* src = reinterpret_cast<const u32x4*>(codes + at * kPage);
                if (now[p] >= 0) {
#pragma unroll
                    for (int i = 0; i < kPiece; ++i) piece[p][i] = src[tid + i * kThreads];
                }
                left &= ~__ballot(blk_l == now[p]);
            }
        };
        fetch();
        const uint16_t* tail = a.from.v_tail + strip * kPage + my.col * kBlk;
#pragma unroll
        for (int r = 0; r < 4; ++r) {
#pragma unroll
            for (int e = 0; e < W; ++e) v[r][e] = 0.f;      // (a row whose page does not exist)
            if (blk[r] < 0) {
#pragma unroll
                for (int e = 0; e < W; ++e) v[r][e] = __uint_as_float((uint32_t)tail[e * kBlk + row[r]] << 16);
            }
        }
        while (now[0] >= 0) {
            __syncthreads();                                // (the pages before are not read any more)
#pragma unroll
            for (int p = 0; p < 2; ++p)
#pragma unroll
                for (int i = 0; i < kPiece; ++i) {
                    if (now[p] < 0) continue;
                    const int unit = tid + i * kThreads;
                    u32x2* to = reinterpret_cast<u32x2*>(pages + (p * D + (unit >> 2)) * kPageRow + 16 * (unit & 3));
                    to[0] = u32x2{piece[p][i].x, piece[p][i].y};
                    to[1] = u32x2{piece[p][i].z, piece[p][i].w};
                }
            const int here0 = now[0], here1 = now[1];
            fetch();
            __syncthreads();
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                if (blk[r] != here0 && blk[r] != here1) continue;
                const uint8_t* at = pages + ((blk[r] == here0 ? 0 : D) + my.col) * kPageRow + row[r];
#pragma unroll
                for (int e = 0; e < W; ++e) v[r][e] = F::value(at[e * kPageRow]) * scale[r];
            }
        }
    } else {
        uint32_t raw[4][W / 2];                             // (codes, or the tail's 16 bits)
#pragma unroll
        for (int r = 0; r < 4; ++r) {
            const int page = __shfl(page_l, my.row + r);
#pragma unroll
            for (int i = 0; i < W / 2; ++i) raw[r][i] = 0;
            if (page >= 0) {
                const uint32_t* p = reinterpret_cast<const uint32_t*>(codes + ((int64_t)page * a.Hk + kh) * kPage + row[r] * D + my.col);
#pragma unroll
                for (int i = 0; i < W / 4; ++i) raw[r][i] = p[i];
            } else if (blk[r] < 0) {
                load_bf16<W>(a.from.k_tail + strip * kPage + row[r] * D + my.col, raw[r]);
            }
        }
        if (__ballot(blk_l < 0) == 0) {                     // (in all waves alike; nearly every block)
#pragma unroll
            for (int r = 0; r < 4; ++r)
#pragma unroll
                for (int e = 0; e < W; ++e) v[r][e] = F::value4(raw[r][e / 4])[e & 3] * scale[r];
        } else {
#pragma unroll
            for (int r = 0; r < 4; ++r)
#pragma unroll
                for (int e = 0; e < W; ++e)
                    v[r][e] = blk[r] >= 0 ? F::value(raw[r][e / 4] >> (8 * (e & 3)) & 0xffu) * scale[r]
                                          : __uint_as_float((raw[r][e / 2] >> (16 * (e & 1))) << 16);
        }
    }
    if (whole) write_block<D, CODE, COLUMNS>(v, a.to, to_at, sm, tid);
    else write_tail<D, COLUMNS>([&](int r, int e) { return (uint16_t)f32_to_bf16_bits(v[r][e]); }, a.to, strip, count - first, tid);
}

template <int D, int CODE>
__global__ __launch_bounds__(kThreads, 6) void block_move_kernel(EvictBlockArgs a) {
    __shared__ __attribute__((aligned(16))) uint8_t pages[2 * D * kPageRow];
    __shared__ uint32_t sm[2 * kThreads / 64];
    const int kh = blockIdx.x % a.Hk;
    if ((int)blockIdx.x < a.Hk) move_block<D, CODE, false>(a, kh, blockIdx.y, blockIdx.z, pages, sm);
    else move_block<D, CODE, true>(a, kh, blockIdx.y, blockIdx.z, pages, sm);
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
    if (!cu_len || total < 0 || max_len < 0 || max_len > total) return ST3_ERR_INVALID_ARG;
    if (total == 0) return ST3_OK;          // (an empty tensor may have no address)
    if ((s = check_rows(k, D, 2)) != ST3_OK || (s = check_rows(v, D, 2)) != ST3_OK) return s;
    if (max_len == 0) return ST3_OK;
    const int blocks = (max_len - 1) / kBlk + 1;
    if (blocks > 65535) return ST3_ERR_UNSUPPORTED;
    if (cache->table_blocks < max_len / kBlk) return ST3_ERR_INVALID_ARG;
    const StoreArgs a{block_pages(cache), reinterpret_cast<const uint16_t*>(k->data), reinterpret_cast<const uint16_t*>(v->data), k->stride_t, k->stride_h,
                      v->stride_t, v->stride_h, cu_len, total, max_len, Hk};
    const dim3 grid(2 * Hk, blocks, shape->batch);
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

extern "C" st3_status st3_block_append(const st3_gqa_shape* shape, const st3_rows* k, const st3_rows* v, const int32_t* cu_len, int32_t total,
                                       int32_t max_new, const st3_block_cache* cache, int32_t max_len, const st3_rotary* rotary, void* stream) {
    using namespace st3;
    st3_status s = check_gqa_shape(shape);
    if (s != ST3_OK) return s;
    if ((s = check_block_cache(shape, cache)) != ST3_OK) return s;
    const int Hk = shape->kv_heads, D = shape->head_dim;
    if (!cu_len || total < 0 || max_new < 0 || max_new > total || max_len < 0) return ST3_ERR_INVALID_ARG;
    if (max_len > kMostRows) return ST3_ERR_UNSUPPORTED;
    if (total == 0) return ST3_OK;          // (an empty tensor may have no address)
    if (rotary && (s = check_rotary(rotary, D)) != ST3_OK) return s;
    if ((s = check_rows(k, D, 2)) != ST3_OK || (s = check_rows(v, D, 2)) != ST3_OK) return s;
    if (max_new == 0) return ST3_OK;
    const int blocks = (int)(((int64_t)max_new + kBlk - 2) / kBlk) + 1;     // (new rows may begin with a block's last)
    if (blocks > 65535) return ST3_ERR_UNSUPPORTED;
    if (cache->table_blocks < max_len / kBlk) return ST3_ERR_INVALID_ARG;
    const AppendArgs a{block_pages(cache), reinterpret_cast<const uint16_t*>(k->data), reinterpret_cast<const uint16_t*>(v->data), k->stride_t, k->stride_h,
                       v->stride_t, v->stride_h, cu_len, rotation(rotary), total, max_new, max_len, Hk};
    const dim3 grid(2 * Hk, blocks, shape->batch);
    hipStream_t st = reinterpret_cast<hipStream_t>(stream);
    auto launch = [&](auto kernel) { kernel<<<grid, kThreads, 0, st>>>(a); };
    auto turned = [&](auto still, auto halves, auto adjacent) {
        if (!rotary) launch(still);
        else if (rotary->layout == ST3_ROTARY_HALVES) launch(halves);
        else launch(adjacent);
    };
    if (cache->code == ST3_BLOCK_INT8) {
        if (D == 128) turned(block_append_kernel<128, ST3_BLOCK_INT8, kStill>, block_append_kernel<128, ST3_BLOCK_INT8, kHalves>, block_append_kernel<128, ST3_BLOCK_INT8, kAdjacent>);
        else turned(block_append_kernel<64, ST3_BLOCK_INT8, kStill>, block_append_kernel<64, ST3_BLOCK_INT8, kHalves>, block_append_kernel<64, ST3_BLOCK_INT8, kAdjacent>);
    } else {
        if (D == 128) turned(block_append_kernel<128, ST3_BLOCK_E4M3, kStill>, block_append_kernel<128, ST3_BLOCK_E4M3, kHalves>, block_append_kernel<128, ST3_BLOCK_E4M3, kAdjacent>);
        else turned(block_append_kernel<64, ST3_BLOCK_E4M3, kStill>, block_append_kernel<64, ST3_BLOCK_E4M3, kHalves>, block_append_kernel<64, ST3_BLOCK_E4M3, kAdjacent>);
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
    if (max_len > kMostRows) return ST3_ERR_UNSUPPORTED;
    const int blocks = (most + kBlk - 1) / kBlk;
    if (blocks > 65535) return ST3_ERR_UNSUPPORTED;
    const bool in_place = score == to_score && (B == 1 || score_stride_b == to_score_stride_b) && (Hk == 1 || score_stride_h == to_score_stride_h);
    const st3_rows old_scores{const_cast<float*>(score), score_stride_b, score_stride_h}, new_scores{to_score, to_score_stride_b, to_score_stride_h};
    if (most > 0 && !in_place && packed_rows_meet(&old_scores, Hk, &new_scores, Hk, B, max_len, 4, most)) return ST3_ERR_INVALID_ARG;
    const EvictBlockArgs a{block_pages(from), block_pages(to), max_len, keep, n_sink, n_recent, Hk, score, score_stride_b, score_stride_h, to_score,
                           to_score_stride_b, to_score_stride_h, kept, kept_stride_b, kept_stride_h};
    hipStream_t st = reinterpret_cast<hipStream_t>(stream);
    const dim3 strips(Hk, B);
    if (max_len <= 4 * kRankThreads) block_rank_kernel<4, false><<<strips, kRankThreads, 0, st>>>(a);
    else if (max_len <= 8 * kRankThreads) block_rank_kernel<8, false><<<strips, kRankThreads, 0, st>>>(a);
    else if (max_len <= 16 * kRankThreads) block_rank_kernel<16, false><<<strips, kRankThreads, 0, st>>>(a);
    else if (max_len <= 32 * kRankThreads) block_rank_kernel<32, false><<<strips, kRankThreads, 0, st>>>(a);
    else block_rank_kernel<16, true><<<strips, kRankThreads, 0, st>>>(a);
    if (blocks == 0) return check_launch();
    const dim3 grid(2 * Hk, blocks, B);
    if (from->code == ST3_BLOCK_INT8) {
        if (D == 128) block_move_kernel<128, ST3_BLOCK_INT8><<<grid, kThreads, 0, st>>>(a);
        else block_move_kernel<64, ST3_BLOCK_INT8><<<grid, kThreads, 0, st>>>(a);
    } else {
        if (D == 128) block_move_kernel<128, ST3_BLOCK_E4M3><<<grid, kThreads, 0, st>>>(a);
        else block_move_kernel<64, ST3_BLOCK_E4M3><<<grid, kThreads, 0, st>>>(a);
    }
    return check_launch();
}
