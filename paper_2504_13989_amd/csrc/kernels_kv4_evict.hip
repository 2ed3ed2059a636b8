// Which positions of a cached sequence are kept, and the kept rows moved together (kv4_layout.h).
//
// select: a workgroup takes a row of weights, as integers in the order of the numbers, in registers up to 57344 of them.  The k-th largest is found
// in up to four passes of eight bits: how many there are of each digit among those whose bits before it are the ones found so far, until
// all that are left of a digit are wanted.  Weights crowd in a few digits, so each has sixteen counters, one for every fourth lane of a
// wave (2048 of one counter each: bound by lanes that wait for each other's additions, 4096 rows of 8192 in 101 us).  So 48, of which reading and
// writing are 10 and 5: LDS additions and the waits between passes; 32 rows of 4099 in 7.9, four passes one after the other.
// evict: codes and parameters move as they are, nothing is quantized again.  Bound by the lines of 128 bytes that are touched: a token's key codes
// are 64 bytes (128 elements), its value codes a quarter of four tokens'.  1024 rows of 4096 positions to 1024, in place: 96 us for 443 MB that move
// (4.6 TB/s, a large copy 4.9), 294 of them wanted; 32 rows to 1000 in other pages 5.5 us, a chain of loads (index, table, codes).
#include "kv4_layout.h"
#include "wave_common.h"

namespace rq {
namespace {

// Numbers as integers of the same order: -infinity .. infinity (0xff800000) above NaN, which is 1; 0 is none of them, and 0xffffffff what is kept in any
// case.  Both zeros are one.
__device__ __forceinline__ uint32_t ordered(float x) {
    uint32_t u = __float_as_uint(x);
    if ((u << 1) > 0xff000000u) return 1u;
    if ((u << 1) == 0u) u = 0u;
    return u ^ ((uint32_t)((int32_t)u >> 31) | 0x80000000u);
}

__device__ __forceinline__ int below(uint64_t mask) {                // set bits of lower lanes
    return (int)__builtin_amdgcn_mbcnt_hi((uint32_t)(mask >> 32), __builtin_amdgcn_mbcnt_lo((uint32_t)mask, 0u));
}

constexpr int kPasses = 4, kCopies = 16;
struct Digits {
    uint32_t count[2][256 * kCopies];             // [digit][copy]; passes in turn
    uint32_t found[kPasses][4];                   // the threshold's digit, how many are above it, how many have it
};

// Sums over the lanes up to this one.
template <int CTRL, int ROWS>
__device__ __forceinline__ int plus_dpp(int x) { return x + __builtin_amdgcn_update_dpp(0, x, CTRL, ROWS, 0xf, true); }
__device__ __forceinline__ int wave_prefix(int x) {
    x = plus_dpp<0x118, 0xf>(plus_dpp<0x114, 0xf>(plus_dpp<0x112, 0xf>(plus_dpp<0x111, 0xf>(x))));   // row_shr:1, 2, 4, 8
    return plus_dpp<0x143, 0xc>(plus_dpp<0x142, 0xa>(x));            // row_bcast:15, 31
}

// What is taken of a row: keys >= `least`, and of those that are least - 1 the first `ties`.
struct Threshold {
    uint32_t least;
    int ties;
};
// The `want` (at least 1) largest of more keys.  each(f): f(key) for the thread's keys, 0 where there is none.
template <int W, typename EACH>
__device__ __forceinline__ Threshold find_threshold(Digits& d, int want, EACH each) {
    const int lane = threadIdx.x & 63;
    const auto clear = [&](uint32_t* count) {
        for (int i = threadIdx.x; i < 256 * kCopies / 4; i += 64 * W) reinterpret_cast<u32x4*>(count)[i] = u32x4{0, 0, 0, 0};
    };
    clear(d.count[0]);
    __syncthreads();
    uint32_t found = 0;                           // the bits of the threshold so far
#pragma unroll
    for (int pass = 0; pass < kPasses; ++pass) {
        const int shift = 24 - 8 * pass;
        uint32_t* count = d.count[pass % 2];
        each([&](uint32_t key) {
            if (pass == 0 || (key >> (shift + 8)) == found) atomicAdd(&count[(key >> shift & 255u) * kCopies + (lane & (kCopies - 1))], 1u);
        });
        if (pass + 1 < kPasses) clear(d.count[(pass + 1) % 2]);      // (read before the barrier that the last pass ended with)
        __syncthreads();
        if (W == 1 || threadIdx.x < 64) {         // a wave's work, and the others' meanwhile would be the same
            // from the largest digit down, four a lane: 64 counters, from another one on in each lane, so that lanes use all banks
            int sum = 0;
#pragma unroll
            for (int i = 0; i < 16; ++i) {
                const u32x4 x = reinterpret_cast<const u32x4*>(count)[(63 - lane) * 16 + ((i + lane) & 15)];
                sum += (int)(x[0] + x[1] + x[2] + x[3]);
            }
            int upto = wave_prefix(sum);
            const int at = __builtin_ctzll(__ballot(upto >= want));  // (there are as many)
            const int before = __builtin_amdgcn_readlane(upto - sum, at);
            // its four digits, sixteen lanes each, the largest first
            const int mine = (int)count[(63 - at) * 64 + (63 - lane)];
            upto = wave_prefix(mine);
            const int s0 = __builtin_amdgcn_readlane(upto, 15), s1 = __builtin_amdgcn_readlane(upto, 31), s2 = __builtin_amdgcn_readlane(upto, 47),
                      s3 = __builtin_amdgcn_readlane(upto, 63), left = want - before;
            const int i = left <= s0 ? 0 : left <= s1 ? 1 : left <= s2 ? 2 : 3;
            const int above = i == 0 ? 0 : i == 1 ? s0 : i == 2 ? s1 : s2, to = i == 0 ? s0 : i == 1 ? s1 : i == 2 ? s2 : s3;
            if (lane == 0) *reinterpret_cast<u32x4*>(d.found[pass]) = u32x4{(uint32_t)((63 - at) * 4 + 3 - i), (uint32_t)(before + above), (uint32_t)(to - above), 0u};
        }
        __syncthreads();
        const u32x4 x = *reinterpret_cast<const u32x4*>(d.found[pass]);
        found = (found << 8) | (uint32_t)__builtin_amdgcn_readfirstlane((int)x[0]);
        want -= __builtin_amdgcn_readfirstlane((int)x[1]);
        if (want == __builtin_amdgcn_readfirstlane((int)x[2])) return Threshold{found << shift, 0};  // all of them
    }
    return Threshold{found + 1, want};
}

// Which row a workgroup has, and what of it is kept in any case: before lo, from hi on.
struct SelectRow {
    const float* w;
    int32_t* out;
    int len, lo, hi;
    __device__ __forceinline__ SelectRow(const Kv4Select& a, int64_t row) {
        const int head = (int)(row % a.kv_heads);
        const int64_t rest = row / a.kv_heads, layer = rest / a.batch;
        const int seq = (int)(rest - layer * a.batch);
        w = a.weights + layer * a.w_layer + seq * a.w_seq + head * a.w_head;
        out = a.index + row * a.keep;
        const int n = a.kv_lens[seq];
        len = n < 0 ? 0 : n > a.n ? a.n : n;
        lo = a.sinks;
        hi = len - a.recent;
    }
    __device__ __forceinline__ uint32_t key(int64_t j, float x) const { return j >= len ? 0u : j < lo || j >= hi ? 0xffffffffu : ordered(x); }
    // All of a row that has no more than are kept.
    __device__ __forceinline__ bool whole(const Kv4Select& a, int threads) const {
        if (len > a.keep) return false;
        for (int i = threadIdx.x; i < a.keep; i += threads) out[i] = i < len ? i : -1;
        return true;
    }
};

// The keys of a wave's 64 R weights x, from position `begin` on.  Weights are seldom anything but 0 .. infinity, whose bits have their order: two
// instructions each for fourteen, which bind where a row is long (one of 131072: 120 and 87 us).
template <int R>
__device__ __forceinline__ void to_keys(uint32_t (&key)[R], const SelectRow& at, const float (&x)[R], int begin, int lane) {
    bool plain = begin >= at.lo && begin + 64 * R <= at.hi;
#pragma unroll
    for (int r = 0; r < R; ++r) plain = plain && __float_as_uint(x[r]) <= 0x7f800000u;
    if (__all(plain)) {
#pragma unroll
        for (int r = 0; r < R; ++r) key[r] = __float_as_uint(x[r]) | 0x80000000u;
    } else {
#pragma unroll
        for (int r = 0; r < R; ++r) key[r] = at.key(begin + lane + 64 * r, x[r]);
    }
}

// A row of at most 64 W R weights.  Wave w has the R * 64 from 64 R w on, lane by lane.
template <int W, int R>
__global__ __launch_bounds__(64 * W) void k_kv4_select(Kv4Select a, int64_t rows) {
    __shared__ __attribute__((aligned(16))) Digits digits;
    __shared__ int taken_of[W], equal_of[W];
    const int64_t row = group_index();
    if (row >= rows) return;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const SelectRow at(a, row);
    if (at.whole(a, 64 * W)) return;
    const int len = at.len, first = wave * (64 * R) + lane;
    // (range-checked, 0 behind the last one: no 64 bits of address for each.  The check is of the vector offset and the instruction's alone, so that
    // nothing stands in the scalar one.)
    const auto weights = __builtin_amdgcn_make_buffer_rsrc(const_cast<float*>(at.w), 0, 4 * len, 0x00020000);
    float x[R];
#pragma unroll
    for (int r = 0; r < R; ++r) x[r] = __uint_as_float(__builtin_amdgcn_raw_buffer_load_b32(weights, 4 * first + 256 * r, 0, 0));
    uint32_t key[R];
    to_keys<R>(key, at, x, first - lane, lane);
    const Threshold t = find_threshold<W>(digits, a.keep, [&](auto count) {
#pragma unroll
        for (int r = 0; r < R; ++r) count(key[r]);
    });
    int n = 0, e = 0;
#pragma unroll
    for (int r = 0; r < R; ++r) n += __builtin_popcountll(__ballot(key[r] >= t.least));
    if (t.ties)
#pragma unroll
        for (int r = 0; r < R; ++r) e += __builtin_popcountll(__ballot(key[r] == t.least - 1));
    if (lane == 0) {
        taken_of[wave] = n;
        equal_of[wave] = e;
    }
    __syncthreads();
    n = e = 0;                                    // those of the waves before
#pragma unroll
    for (int x = 0; x < W; ++x) {
        n += x < wave ? taken_of[x] : 0;
        e += x < wave ? equal_of[x] : 0;
    }
    uint32_t least = t.least;                     // (the compiler would keep the masks of the count, in more registers than there are)
    asm volatile("" : "+s"(least));
    int32_t* out = at.out + n;
    if (t.ties == 0) {
#pragma unroll
        for (int r = 0; r < R; ++r) {
            const uint64_t taken = __ballot(key[r] >= least);
            if (key[r] >= least) out[below(taken)] = first + 64 * r;
            out += __builtin_popcountll(taken);
        }
        return;
    }
#pragma unroll
    for (int r = 0; r < R; ++r) {
        const bool mine = key[r] >= least, tie = key[r] == least - 1;
        const uint64_t taken = __ballot(mine), equal = __ballot(tie);
        const int rank = e + below(equal), before = rank < t.ties ? rank : t.ties;                   // ties before this one; those of them that are taken
        if (mine || (tie && rank < t.ties)) out[below(taken) + before] = first + 64 * r;
        out += __builtin_popcountll(taken);
        e += __builtin_popcountll(equal);
    }
}

// Rows of any length: the same, with the row read again for every pass, kLong weights a thread at once.  (One row of 131072: 87 us; with one at once 295.)
constexpr int kLongWaves = 16, kLong = 8;
__global__ __launch_bounds__(64 * kLongWaves) void k_kv4_select_long(Kv4Select a, int64_t rows) {
    constexpr int W = kLongWaves, S = 64 * W * kLong;
    __shared__ __attribute__((aligned(16))) Digits digits;
    __shared__ int taken_of[2][W], equal_of[2][W];
    const int64_t row = group_index();
    if (row >= rows) return;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const SelectRow at(a, row);
    if (at.whole(a, 64 * W)) return;
    const int len = at.len, first = wave * (64 * kLong) + lane;
    const auto read = [&](uint32_t (&key)[kLong], int from) {        // the stretch of S weights from there on
        float x[kLong];
#pragma unroll
        for (int r = 0; r < kLong; ++r) {
            const int j = from + first + 64 * r;
            x[r] = at.w[j < len ? j : len - 1];
        }
        to_keys<kLong>(key, at, x, from + wave * (64 * kLong), lane);
    };
    const Threshold t = find_threshold<W>(digits, a.keep, [&](auto count) {
        for (int from = 0; from < len; from += S) {
            uint32_t key[kLong];
            read(key, from);
#pragma unroll
            for (int r = 0; r < kLong; ++r) count(key[r]);
        }
    });
    int n = 0, e = 0, turn = 0;                   // written, and ties met, before the stretch in hand
    for (int from = 0; from < len; from += S, turn ^= 1) {
        uint32_t key[kLong];
        read(key, from);
        int mine = 0, ties = 0;
#pragma unroll
        for (int r = 0; r < kLong; ++r) {
            mine += __builtin_popcountll(__ballot(key[r] >= t.least));
            ties += __builtin_popcountll(__ballot(key[r] == t.least - 1));
        }
        if (lane == 0) {
            taken_of[turn][wave] = mine;
            equal_of[turn][wave] = ties;
        }
        __syncthreads();
        int n0 = n, e0 = e;                       // ... and before this wave's part of it
#pragma unroll
        for (int x = 0; x < W; ++x) {
            const int cn = taken_of[turn][x], ce = equal_of[turn][x];
            n0 += x < wave ? cn : 0;
            e0 += x < wave ? ce : 0;
            n += cn;
            e += ce;
        }
#pragma unroll
        for (int r = 0; r < kLong; ++r) {
            const bool taken = key[r] >= t.least, tie = key[r] == t.least - 1;
            const uint64_t all = __ballot(taken), equal = __ballot(tie);
            const int rank = e0 + below(equal);
            if (taken || (tie && rank < t.ties)) at.out[n0 + below(all) + (rank < t.ties ? rank : t.ties)] = from + first + 64 * r;
            n0 += __builtin_popcountll(all);
            e0 += __builtin_popcountll(equal);
        }
    }
}

// ---- evict

constexpr int kTokens = 16;                       // of a wave that takes whole rows: they lie in one page where they go

// Where rows come from, a row a lane: the page (-1: there is none), the place in it.
struct Sources {
    int page, place;
};
__device__ __forceinline__ Sources find_sources(const Kv4& c, const Kv4Evict& a, const int32_t* index, const int32_t* table, int64_t i) {
    const int at = i < a.keep ? index[i] : -1;
    int page = at >= 0 && (at >> c.page_shift) < a.width ? table[at >> c.page_shift] : -1;
    if (page >= c.pages) page = -1;
    return Sources{page < 0 ? -1 : page, at & ((1 << c.page_shift) - 1)};
}

// What a wave holds of its kTokens * P tokens, of which it takes a P-th of the elements (part `part`), P 1 or 4.  Keys: a quarter of a token, of lane
// l quarter l % 4 of token l / 4, or `part` of token l.  Values: fours of tokens of a run, as the layout has them.  Parameters: lanes 0 .. 15
// keys', 16 .. 31 values'; P == 4: of token l, part 0 keys', 1 values'.
template <int D>
struct Held {
    uint32_t k[D / 32];
    uint32_t v[D / 64][4];
    uint32_t p;
    int from;                                     // of token `lane & 15`, or `lane`: its page; -1: none
};

// Tokens whose sources are those of lanes kTokens P n and on.  (Rows that are not there come from page 0, and go nowhere: no branch, behind which
// all loads would be waited for.)
template <int D, int P>
__device__ __forceinline__ void load_rows(Held<D>& t, const uint8_t* base, const Kv4& c, const Sources& s, int n, int head_at, int part, int lane) {
    typedef uint32_t words __attribute__((ext_vector_type(D / 32)));
    constexpr int cols = D / 4 / P;               // of a run of values
    const int p = 1 << c.page_shift, first = P == 1 ? kTokens * n : 0, mine = P == 1 ? lane & 15 : lane;
    t.from = P == 1 ? __shfl(s.page, first + mine) : s.page;
    const auto block = [&](int page) { return base + (uint64_t)(uint32_t)(page < 0 ? 0 : page) * (uint32_t)c.page_bytes + head_at; };
    {
        const int from = P == 1 ? __shfl(s.page, first + (lane >> 2)) : s.page, in = P == 1 ? __shfl(s.place, first + (lane >> 2)) : s.place;
        const words x = *reinterpret_cast<const words*>(block(from) + in * (D / 2) + (P == 1 ? lane & 3 : part) * (D / 8));
#pragma unroll
        for (int j = 0; j < D / 32; ++j) t.k[j] = x[j];
    }
#pragma unroll
    for (int r = 0; r < D / 64; ++r) {
        const int run = lane + 64 * r, four = run / cols, within = part * cols + run % cols;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const int from = __shfl(s.page, first + 4 * four + e), in = __shfl(s.place, first + 4 * four + e);
            t.v[r][e] = *reinterpret_cast<const uint16_t*>(block(from) + p * (D / 2) + (in >> 2) * (2 * D) + within * 8 + 2 * (in & 3));
        }
    }
    const int in = P == 1 ? __shfl(s.place, first + mine) : s.place, which = P == 1 ? lane >> 4 & 1 : part & 1;
    t.p = *reinterpret_cast<const uint32_t*>(block(t.from) + p * D + which * 4 * p + 4 * in);
}

// page: of the tokens, P == 4: of token `lane` (in the cache, or t.from is -1).
template <int D, int P>
__device__ __forceinline__ void store_rows(const Held<D>& t, uint8_t* base, const Kv4& c, int page, int i0, int head_at, int part, int lane) {
    typedef uint32_t words __attribute__((ext_vector_type(D / 32)));
    constexpr int cols = D / 4 / P;
    const int p = 1 << c.page_shift;
    const auto block = [&](int page) { return base + (uint64_t)(uint32_t)page * (uint32_t)c.page_bytes + head_at; };
    const int token = P == 1 ? lane >> 2 : lane;
    if ((P == 1 ? __shfl(t.from, token) : t.from) >= 0) {
        words x;
#pragma unroll
        for (int j = 0; j < D / 32; ++j) x[j] = t.k[j];
        *reinterpret_cast<words*>(block(page) + ((i0 + token) & (p - 1)) * (D / 2) + (P == 1 ? lane & 3 : part) * (D / 8)) = x;
    }
#pragma unroll
    for (int r = 0; r < D / 64; ++r) {
        const int run = lane + 64 * r, four = run / cols, within = part * cols + run % cols, to = P == 1 ? page : __shfl(page, 4 * four);
        bool there[4], all = true;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            there[e] = __shfl(t.from, 4 * four + e) >= 0;
            all = all && there[e];
        }
        uint16_t* v = reinterpret_cast<uint16_t*>(block(to) + p * (D / 2) + (((i0 >> 2) + four) & (p / 4 - 1)) * (2 * D) + within * 8);
        if (all) {
            *reinterpret_cast<u32x2*>(v) = u32x2{t.v[r][0] | (t.v[r][1] << 16), t.v[r][2] | (t.v[r][3] << 16)};
        } else {                                  // (rows that do not move leave others' bytes)
#pragma unroll
            for (int e = 0; e < 4; ++e)
                if (there[e]) v[e] = (uint16_t)t.v[r][e];
        }
    }
    const int mine = P == 1 ? lane & 15 : lane, which = P == 1 ? lane >> 4 : part;
    if (which < 2 && t.from >= 0) *reinterpret_cast<uint32_t*>(block(page) + p * D + which * 4 * p + 4 * ((i0 + mine) & (p - 1))) = t.p;
}

// A row of weights, in place, by a workgroup of T threads: stretch by stretch, each read before it is written.  (index[i] >= i: what is
// written has been read.)
template <int T>
__device__ __forceinline__ void move_weights(float* w, const int32_t* index, const Kv4Evict& a) {
    constexpr int N = 8;                          // of a thread at once
    for (int i0 = 0; i0 < a.keep; i0 += N * T) {
        int at[N];
        float x[N];
#pragma unroll
        for (int e = 0; e < N; ++e) {
            const int i = i0 + e * T + (int)threadIdx.x;
            at[e] = i < a.keep ? index[i] : -1;
        }
#pragma unroll
        for (int e = 0; e < N; ++e) x[e] = at[e] >= 0 && at[e] < a.n ? w[at[e]] : 0.0f;
        __builtin_amdgcn_s_waitcnt(0x0f70);       // vmcnt(0)
        __syncthreads();
#pragma unroll
        for (int e = 0; e < N; ++e) {
            const int i = i0 + e * T + (int)threadIdx.x;
            if (i < a.keep) w[i] = x[e];
        }
    }
    for (int i = a.keep + (int)threadIdx.x; i < a.n; i += T) w[i] = 0.0f;
}

// Which layer, sequence and head a workgroup has.
struct Row {
    int64_t layer;
    int seq, head;
    __device__ __forceinline__ Row(int64_t row, const Kv4& c, const Kv4Evict& a) {
        head = (int)(row % c.kv_heads);
        const int64_t rest = row / c.kv_heads;
        layer = rest / a.batch;
        seq = (int)(rest - layer * a.batch);
    }
};

// In place: a workgroup a row, stretch by stretch.  A position is read by stretches up to its own, which is written once all waves have
// read theirs; what the next one reads lies behind it, and is asked for before that.
//
// P: workgroups of a row, each with a P-th of every token's elements.  One a row moves lines whole; where rows are few their stretches follow one
// another too slowly (1.7 us), and four have a quarter of the stretches.  Positions 8192 to 4096, 8 heads of 128: 32 rows 54 us with one, 25 with
// four; 64 rows 55 and 42; 128 rows 55 and 70; 1024 rows of 4096 to 1024 96 and 171.  One row, 65536 to 32768: 421 and 152.
constexpr int kPlaceWaves = 8, kFewRows = 64;
template <int D, int P>
__global__ __launch_bounds__(64 * kPlaceWaves) void k_kv4_evict_in_place(Kv4 c, Kv4Evict a, int64_t rows) {
    constexpr int S = kPlaceWaves * kTokens * P, B = 4 / P;          // a stretch; stretches whose sources a wave holds
    const int64_t group = group_index(), row = group / P;
    const int part = (int)(group - row * P);
    if (row >= rows) return;
    const Row at(row, c, a);
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int32_t *index = a.index + row * a.keep, *table = a.table + (int64_t)at.seq * a.width;
    const int head_at = at.head * ((D + 8) << c.page_shift);
    uint8_t* base = c.data + at.layer * a.layer_bytes;
    // the wave's tokens of B stretches: a lane each
    const auto sources = [&](int first) {
        return find_sources(c, a, index, table, P == 1 ? (int64_t)first + (lane >> 4) * S + wave * kTokens + (lane & 15) : (int64_t)first + wave * 64 + lane);
    };
    Sources from = sources(0), later = sources(B * S);
    int n = 0;                                    // of the stretch that is asked for next, among those of `from`
    Held<D> even, odd;
    const auto ask = [&](Held<D>& t, int i0) {    // stretch i0
        if (n == B) {
            n = 0;
            from = later;
            later = sources(i0 + B * S);
        }
        load_rows<D, P>(t, base, c, from, n++, head_at, part, lane);
    };
    const auto move = [&](Held<D>& t, Held<D>& next, int i0) {
        const int i = i0 + wave * kTokens * P;
        int to = -1;                              // P == 4: the page that token `lane` goes to
        if constexpr (P == 4) to = i + lane < a.keep ? table[(i + lane) >> c.page_shift] : -1;
        ask(next, i0 + S);
        // what this stretch has asked for is here, and so it is in the other waves
#pragma unroll
        for (int j = 0; j < D / 32; ++j) asm volatile("" : "+v"(t.k[j]));
#pragma unroll
        for (int r = 0; r < D / 64; ++r) asm volatile("" : "+v"(t.v[r][0]), "+v"(t.v[r][1]), "+v"(t.v[r][2]), "+v"(t.v[r][3]));
        asm volatile("" : "+v"(t.p) : : "memory");
        __builtin_amdgcn_s_barrier();
        asm volatile("" : : : "memory");
        if (P == 1 && i < a.keep) {
            const int page = table[i >> c.page_shift];
            if (page >= 0 && page < c.pages) store_rows<D, P>(t, base, c, page, i, head_at, part, lane);
        }
        if (P == 4 && i < a.keep) {
            if (to < 0 || to >= c.pages) t.from = -1;
            store_rows<D, P>(t, base, c, to, i, head_at, part, lane);
        }
    };
    if (a.keep > 0 && c.pages > 0) {
        ask(even, 0);
        for (int64_t i0 = 0; i0 < a.keep; i0 += 2 * S) {
            move(even, odd, (int)i0);
            if (i0 + S < a.keep) move(odd, even, (int)i0 + S);
        }
    }
    if (a.weights && part == P - 1) move_weights<64 * kPlaceWaves>(a.weights + at.layer * a.w_layer + at.seq * a.w_seq + at.head * a.w_head, index, a);
}

// Into other pages: a wave sixteen tokens, and a workgroup for each row of weights.
constexpr int kMoveWaves = 4;
template <int D>
__global__ __launch_bounds__(64 * kMoveWaves) void k_kv4_evict(Kv4 c, Kv4Evict a, int parts, int64_t groups) {
    const int64_t group = group_index();
    if (group >= groups) return;
    const int64_t row = group / parts;
    const int part = (int)(group - row * parts);
    const Row at(row, c, a);
    const int32_t *index = a.index + row * a.keep, *table = a.table + (int64_t)at.seq * a.width;
    if (a.weights && part == parts - 1) {
        move_weights<64 * kMoveWaves>(a.weights + at.layer * a.w_layer + at.seq * a.w_seq + at.head * a.w_head, index, a);
        return;
    }
    const int lane = threadIdx.x & 63, i = (part * kMoveWaves + (int)(threadIdx.x >> 6)) * kTokens;
    if (i >= a.keep || c.pages == 0) return;
    const int head_at = at.head * ((D + 8) << c.page_shift);
    uint8_t* base = c.data + at.layer * a.layer_bytes;
    const int page = a.new_table[(int64_t)at.seq * a.new_width + (i >> c.page_shift)];
    Held<D> t;
    load_rows<D, 1>(t, base, c, find_sources(c, a, index, table, i + (lane & 15)), 0, head_at, 0, lane);
    if (page >= 0 && page < c.pages) store_rows<D, 1>(t, base, c, page, i, head_at, 0, lane);
}

template <int W, int R>
void launch_select(const Kv4Select& a, int64_t rows, hipStream_t s) {
    launch_kernel(k_kv4_select<W, R>, group_grid(rows, 64 * W), dim3(64 * W), 0, s, a, rows);
}

}  // namespace

int kv4_select(const Kv4Select& a, hipStream_t s) {
    const int64_t rows = (int64_t)a.layers * a.batch * a.kv_heads;
    if (a.n <= 1024) launch_select<4, 4>(a, rows, s);
    else if (a.n <= 4096) launch_select<4, 16>(a, rows, s);
    else if (a.n <= 8192) launch_select<8, 16>(a, rows, s);
    else if (a.n <= 16384) launch_select<16, 16>(a, rows, s);
    else if (a.n <= 32768) launch_select<16, 32>(a, rows, s);
    else if (a.n <= 57344) launch_select<16, 56>(a, rows, s);       // (as many as a wave's registers hold; a row of 40000 24 us, read again for every pass 31)
    else launch_kernel(k_kv4_select_long, group_grid(rows, 64 * kLongWaves), dim3(64 * kLongWaves), 0, s, a, rows);
    return launch_rc();
}

int kv4_evict(const Kv4& c, const Kv4Evict& a, hipStream_t s) {
    const int64_t rows = (int64_t)a.layers * a.batch * c.kv_heads;
    const bool wide = c.head_dim == 128;
    if (!a.new_table) {
        const dim3 block(64 * kPlaceWaves);
        if (rows <= kFewRows) launch_kernel(wide ? k_kv4_evict_in_place<128, 4> : k_kv4_evict_in_place<64, 4>, group_grid(4 * rows, 64 * kPlaceWaves), block, 0, s, c, a, rows);
        else launch_kernel(wide ? k_kv4_evict_in_place<128, 1> : k_kv4_evict_in_place<64, 1>, group_grid(rows, 64 * kPlaceWaves), block, 0, s, c, a, rows);
    } else {
        constexpr int S = kMoveWaves * kTokens;
        const int parts = (a.keep + S - 1) / S + (a.weights != nullptr);
        const int64_t groups = rows * parts;
        launch_kernel(wide ? k_kv4_evict<128> : k_kv4_evict<64>, group_grid(groups, 64 * kMoveWaves), dim3(64 * kMoveWaves), 0, s, c, a, parts, groups);
    }
    return launch_rc();
}

}  // namespace rq
