// Which positions of a cached sequence are kept, and the kept rows moved together (kv4_layout.h).
//
// select: a row of weights is held in registers by one workgroup, as integers in the order of the numbers; the k-th largest is found
// bit by bit, a count over the row each, until as many are at or above the threshold as are wanted.
// evict: codes and parameters move as they are, nothing is quantized again.
#include "kv4_layout.h"
#include "wave_common.h"

namespace rq {
namespace {

// Numbers as integers of the same order: -infinity .. infinity above NaN, which is 1, and 0 is none of them.  Both zeros are one.
__device__ __forceinline__ uint32_t ordered(float x) {
    uint32_t u = __float_as_uint(x);
    if ((u << 1) > 0xff000000u) return 1u;
    if ((u << 1) == 0u) u = 0u;
    return u ^ ((uint32_t)((int32_t)u >> 31) | 0x80000000u);
}

__device__ __forceinline__ int below(uint64_t mask) {                // set bits of lower lanes
    return (int)__builtin_amdgcn_mbcnt_hi((uint32_t)(mask >> 32), __builtin_amdgcn_mbcnt_lo((uint32_t)mask, 0u));
}

// A row of at most 64 W R weights.  Wave w has the R * 64 from 64 R w on, lane by lane.
template <int W, int R>
__global__ __launch_bounds__(64 * W) void k_kv4_select(Kv4Select a, int64_t rows) {
    __shared__ int counts[2][W], eq_counts[W];
    const int64_t row = group_index();
    if (row >= rows) return;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int head = (int)(row % a.kv_heads);
    const int64_t rest = row / a.kv_heads, layer = rest / a.batch;
    const int seq = (int)(rest - layer * a.batch);
    const float* w = a.weights + layer * a.w_layer + seq * a.w_seq + head * a.w_head;
    int32_t* out = a.index + row * a.keep;
    int len = a.kv_lens[seq];
    len = len < 0 ? 0 : len > a.n ? a.n : len;
    if (len <= a.keep) {                          // all of it
        for (int i = threadIdx.x; i < a.keep; i += 64 * W) out[i] = i < len ? i : -1;
        return;
    }
    const int lo = a.sinks, hi = len - a.recent, want = a.keep - a.sinks - a.recent, first = wave * (64 * R) + lane;
    uint32_t key[R];
#pragma unroll
    for (int r = 0; r < R; ++r) {
        const int j = first + 64 * r;
        key[r] = __float_as_uint(w[j < len ? j : len - 1]);
    }
#pragma unroll
    for (int r = 0; r < R; ++r) key[r] = (uint32_t)(first + 64 * r - lo) < (uint32_t)(hi - lo) ? ordered(__uint_as_float(key[r])) : 0u;
    int turn = 0;
    const auto count = [&](uint32_t t) {          // of keys at or above t, over the workgroup
        int n = 0;
#pragma unroll
        for (int r = 0; r < R; ++r) n += __builtin_popcountll(__ballot(key[r] >= t));
        if constexpr (W > 1) {
            if (lane == 0) counts[turn][wave] = n;
            __syncthreads();
            n = lane < W ? counts[turn][lane] : 0;
#pragma unroll
            for (int x = 1; x < W; x *= 2) n += __shfl_xor(n, x);
            n = __builtin_amdgcn_readfirstlane(n);
            turn ^= 1;
        }
        return n;
    };
    // keys >= `least` are taken, and the first `ties` that are least - 1
    uint32_t least = 0xffffffffu;
    int ties = 0;
    if (want > 0) {
        uint32_t t = 0;
        int n = 0;
        for (int bit = 31; bit >= 0; --bit) {
            const uint32_t to = t | (1u << bit);
            const int c = count(to);
            if (c < want) continue;
            t = to;
            n = c;
            if (c == want) break;
        }
        least = t;
        if (n != want) {                          // t is the last one that is taken, some of those equal to it are not
            least = t + 1;
            ties = want - count(least);
        }
    }
    int place = first;                            // (the compiler would keep the masks of the first pass for the second, in more registers than there are)
    const auto is_taken = [&](int r) {
        const int j = place + 64 * r;
        return key[r] >= least || (j < len && (j < lo || j >= hi));
    };
    const auto is_equal = [&](int r) { return ties && key[r] == least - 1; };
    int n = 0, e = 0;
#pragma unroll
    for (int r = 0; r < R; ++r) {
        n += __builtin_popcountll(__ballot(is_taken(r)));
        e += __builtin_popcountll(__ballot(is_equal(r)));
    }
    if constexpr (W > 1) {                        // those of the waves before
        if (lane == 0) {
            counts[turn][wave] = n;
            eq_counts[wave] = e;
        }
        __syncthreads();
        n = e = 0;
#pragma unroll
        for (int x = 0; x < W; ++x) {
            n += x < wave ? counts[turn][x] : 0;
            e += x < wave ? eq_counts[x] : 0;
        }
    } else {
        n = e = 0;
    }
    asm volatile("" : "+v"(place), "+s"(least));
#pragma unroll
    for (int r = 0; r < R; ++r) {
        const bool mine = is_taken(r), tie = is_equal(r);
        const uint64_t taken = __ballot(mine), equal = __ballot(tie);
        const int rank = e + below(equal);        // ties before this one
        if (mine || (tie && rank < ties)) out[n + below(taken) + (rank < ties ? rank : ties)] = place + 64 * r;
        n += __builtin_popcountll(taken);
        e += __builtin_popcountll(equal);
    }
}

// Rows of any length: the same, with the row read again for every count.
constexpr int kLongWaves = 16;
__global__ __launch_bounds__(64 * kLongWaves) void k_kv4_select_long(Kv4Select a, int64_t rows) {
    constexpr int W = kLongWaves, T = 64 * W;
    __shared__ int counts[2][W], eq_counts[2][W];
    const int64_t row = group_index();
    if (row >= rows) return;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int head = (int)(row % a.kv_heads);
    const int64_t rest = row / a.kv_heads, layer = rest / a.batch;
    const int seq = (int)(rest - layer * a.batch);
    const float* w = a.weights + layer * a.w_layer + seq * a.w_seq + head * a.w_head;
    int32_t* out = a.index + row * a.keep;
    int len = a.kv_lens[seq];
    len = len < 0 ? 0 : len > a.n ? a.n : len;
    if (len <= a.keep) {
        for (int i = threadIdx.x; i < a.keep; i += T) out[i] = i < len ? i : -1;
        return;
    }
    const int lo = a.sinks, hi = len - a.recent, want = a.keep - a.sinks - a.recent;
    int turn = 0;
    const auto count = [&](uint32_t t) {
        int n = 0;
        for (int j = lo + (int)threadIdx.x; j < hi; j += T) n += ordered(w[j]) >= t;
#pragma unroll
        for (int x = 1; x < 64; x *= 2) n += __shfl_xor(n, x);
        if (lane == 0) counts[turn][wave] = n;
        __syncthreads();
        n = lane < W ? counts[turn][lane] : 0;
#pragma unroll
        for (int x = 1; x < W; x *= 2) n += __shfl_xor(n, x);
        turn ^= 1;
        return __builtin_amdgcn_readfirstlane(n);
    };
    uint32_t least = 0xffffffffu;
    int ties = 0;
    if (want > 0) {
        uint32_t t = 0;
        int n = 0;
        for (int bit = 31; bit >= 0; --bit) {
            const uint32_t to = t | (1u << bit);
            const int c = count(to);
            if (c < want) continue;
            t = to;
            n = c;
            if (c == want) break;
        }
        least = t;
        if (n != want) {
            least = t + 1;
            ties = want - count(least);
        }
    }
    int n = 0, e = 0;                             // written, and ties met, before the stretch in hand
    for (int at = 0; at < len; at += T) {
        const int j = at + (int)threadIdx.x;
        const bool there = j < len, candidate = j >= lo && j < hi;
        const uint32_t key = candidate ? ordered(w[j]) : 0u;
        const uint64_t taken = __ballot(there && (!candidate || key >= least)), equal = __ballot(ties && candidate && key == least - 1);
        if (lane == 0) {
            counts[turn][wave] = __builtin_popcountll(taken);
            eq_counts[turn][wave] = __builtin_popcountll(equal);
        }
        __syncthreads();
        int n0 = n, e0 = e;                       // ... and before this wave's part of it
#pragma unroll
        for (int x = 0; x < W; ++x) {
            const int cn = counts[turn][x], ce = eq_counts[turn][x];
            n0 += x < wave ? cn : 0;
            e0 += x < wave ? ce : 0;
            n += cn;
            e += ce;
        }
        const uint64_t mine = (uint64_t)1 << lane;
        const int rank = e0 + below(equal);
        if ((taken & mine) || ((equal & mine) && rank < ties)) out[n0 + below(taken) + (rank < ties ? rank : ties)] = j;
        turn ^= 1;
    }
}

// ---- evict

constexpr int kTokens = 16;                       // of a wave: they lie in one page where they go

// What a wave holds of its tokens.  Keys: lane l has part l % 4 of token l / 4.  Values: fours of tokens of a run, as the layout has them.
// Parameters: lanes 0 .. 15 keys', 16 .. 31 values'.
template <int D>
struct Held {
    uint32_t k[D / 32];
    uint16_t v[D / 64][4];
    uint32_t p;
    int from;                                     // of token `lane & 15`: its page; -1: none
};

template <int D>
__device__ __forceinline__ void load_rows(Held<D>& t, const uint8_t* base, const Kv4& c, const Kv4Evict& a, const int32_t* index, const int32_t* table, int i0, int head_at,
                                          int lane) {
    typedef uint32_t words __attribute__((ext_vector_type(D / 32)));
    const int p = 1 << c.page_shift, i = i0 + (lane & 15);
    const int at = i < a.keep ? index[i] : -1;
    int page = at >= 0 && (at >> c.page_shift) < a.width ? table[at >> c.page_shift] : -1;
    if (page >= c.pages) page = -1;
    t.from = page < 0 ? -1 : page;
    const int place = at & (p - 1);
    const auto block = [&](int page) { return base + (uint64_t)(uint32_t)page * (uint32_t)c.page_bytes + head_at; };
    {
        const int from = __shfl(t.from, lane >> 2), in = __shfl(place, lane >> 2);
        words x{};
        if (from >= 0) x = *reinterpret_cast<const words*>(block(from) + in * (D / 2) + (lane & 3) * (D / 8));
#pragma unroll
        for (int j = 0; j < D / 32; ++j) t.k[j] = x[j];
    }
#pragma unroll
    for (int r = 0; r < D / 64; ++r) {
        const int run = lane + 64 * r, four = run / (D / 4), within = run % (D / 4);
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const int from = __shfl(t.from, 4 * four + e), in = __shfl(place, 4 * four + e);
            t.v[r][e] = 0;
            if (from >= 0) t.v[r][e] = *reinterpret_cast<const uint16_t*>(block(from) + p * (D / 2) + (in >> 2) * (2 * D) + within * 8 + 2 * (in & 3));
        }
    }
    t.p = 0;
    if (lane < 32 && t.from >= 0) t.p = *reinterpret_cast<const uint32_t*>(block(t.from) + p * D + (lane >> 4) * 4 * p + 4 * place);
}

template <int D>
__device__ __forceinline__ void store_rows(const Held<D>& t, uint8_t* base, const Kv4& c, int page, int i0, int head_at, int lane) {
    typedef uint32_t words __attribute__((ext_vector_type(D / 32)));
    const int p = 1 << c.page_shift, in = i0 & (p - 1);
    uint8_t* block = base + (uint64_t)(uint32_t)page * (uint32_t)c.page_bytes + head_at;
    if (__shfl(t.from, lane >> 2) >= 0) {
        words x;
#pragma unroll
        for (int j = 0; j < D / 32; ++j) x[j] = t.k[j];
        *reinterpret_cast<words*>(block + (in + (lane >> 2)) * (D / 2) + (lane & 3) * (D / 8)) = x;
    }
#pragma unroll
    for (int r = 0; r < D / 64; ++r) {
        const int run = lane + 64 * r, four = run / (D / 4), within = run % (D / 4);
        bool there[4], all = true;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            there[e] = __shfl(t.from, 4 * four + e) >= 0;
            all = all && there[e];
        }
        uint16_t* v = reinterpret_cast<uint16_t*>(block + p * (D / 2) + ((in >> 2) + four) * (2 * D) + within * 8);
        if (all) {
            *reinterpret_cast<u32x2*>(v) = u32x2{(uint32_t)t.v[r][0] | ((uint32_t)t.v[r][1] << 16), (uint32_t)t.v[r][2] | ((uint32_t)t.v[r][3] << 16)};
        } else {                                  // (rows that do not move leave others' bytes)
#pragma unroll
            for (int e = 0; e < 4; ++e)
                if (there[e]) v[e] = t.v[r][e];
        }
    }
    if (lane < 32 && t.from >= 0) *reinterpret_cast<uint32_t*>(block + p * D + (lane >> 4) * 4 * p + 4 * (in + (lane & 15))) = t.p;
}

// A row of weights, in place, by a workgroup of T threads: stretch by stretch, each read before it is written.  (index[i] >= i: what is
// written has been read.)
template <int T>
__device__ __forceinline__ void move_weights(float* w, const int32_t* index, const Kv4Evict& a) {
    for (int i0 = 0; i0 < a.keep; i0 += T) {
        const int i = i0 + (int)threadIdx.x, at = i < a.keep ? index[i] : -1;
        const float x = at >= 0 && at < a.n ? w[at] : 0.0f;
        __builtin_amdgcn_s_waitcnt(0x0f70);       // vmcnt(0)
        __syncthreads();
        if (i < a.keep) w[i] = x;
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
// read theirs; what the next one reads lies behind it.
constexpr int kPlaceWaves = 8;
template <int D>
__global__ __launch_bounds__(64 * kPlaceWaves) void k_kv4_evict_in_place(Kv4 c, Kv4Evict a, int64_t rows) {
    constexpr int S = kPlaceWaves * kTokens;
    const int64_t row = group_index();
    if (row >= rows) return;
    const Row at(row, c, a);
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int32_t *index = a.index + row * a.keep, *table = a.table + (int64_t)at.seq * a.width;
    const int head_at = at.head * ((D + 8) << c.page_shift);
    uint8_t* base = c.data + at.layer * a.layer_bytes;
    for (int i0 = 0; i0 < a.keep; i0 += S) {
        const int i = i0 + wave * kTokens;
        Held<D> t;
        load_rows<D>(t, base, c, a, index, table, i, head_at, lane);
        __builtin_amdgcn_s_waitcnt(0x0f70);       // vmcnt(0)
        __syncthreads();
        if (i < a.keep) {
            const int page = table[i >> c.page_shift];
            if (page >= 0 && page < c.pages) store_rows<D>(t, base, c, page, i, head_at, lane);
        }
    }
    if (a.weights) move_weights<64 * kPlaceWaves>(a.weights + at.layer * a.w_layer + at.seq * a.w_seq + at.head * a.w_head, index, a);
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
    if (i >= a.keep) return;
    const int head_at = at.head * ((D + 8) << c.page_shift);
    uint8_t* base = c.data + at.layer * a.layer_bytes;
    const int page = a.new_table[(int64_t)at.seq * a.new_width + (i >> c.page_shift)];
    Held<D> t;
    load_rows<D>(t, base, c, a, index, table, i, head_at, lane);
    if (page >= 0 && page < c.pages) store_rows<D>(t, base, c, page, i, head_at, lane);
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
    else launch_kernel(k_kv4_select_long, group_grid(rows, 64 * kLongWaves), dim3(64 * kLongWaves), 0, s, a, rows);
    return launch_rc();
}

int kv4_evict(const Kv4& c, const Kv4Evict& a, hipStream_t s) {
    const int64_t rows = (int64_t)a.layers * a.batch * c.kv_heads;
    const bool wide = c.head_dim == 128;
    if (!a.new_table) {
        launch_kernel(wide ? k_kv4_evict_in_place<128> : k_kv4_evict_in_place<64>, group_grid(rows, 64 * kPlaceWaves), dim3(64 * kPlaceWaves), 0, s, c, a, rows);
    } else {
        constexpr int S = kMoveWaves * kTokens;
        const int parts = (a.keep + S - 1) / S + (a.weights != nullptr);
        const int64_t groups = rows * parts;
        launch_kernel(wide ? k_kv4_evict<128> : k_kv4_evict<64>, group_grid(groups, 64 * kMoveWaves), dim3(64 * kMoveWaves), 0, s, c, a, parts, groups);
    }
    return launch_rc();
}

}  // namespace rq
