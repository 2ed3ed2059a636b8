// How much attention the positions of cached sequences receive: w_j <- decay * w_j + sum_i exp(scale q_i . k_j - lse_i), over the
// queries i that see position j, of all heads that share its kv head.
//
// Products are queries x keys: a key is a column, column n the lanes n, n + 16, n + 32, n + 48, of which lane g has rows 4 g + 0 .. 3.  A
// key's step and centre and its sum stay in its lanes, and the sum over a tile's rows is three additions.
//   - Codes are exact operands: c - 8 for few rows, whose half the accumulator starts from, half the sum of the row's elements; c - 7.5 for
//     many.  (Attention has 1024 + c, and takes the 1024 off the sums: they are good to 2^-12 then, and weights are 32 bits.)
//   - Queries are two fp16 numbers each (kv4_attention.h): 22 bits.
#include "kv4_attention.h"

#include <type_traits>

namespace rq {
namespace {

constexpr int kWaves = 4;
typedef float f32x16 __attribute__((ext_vector_type(16)));

// A tile's key codes and parameters (of key 16 i + lane % 16; F == 4: of key `lane`), and the weight of the key that the lane writes.
template <int D, int F>
struct KeyCodes {
    float old;
    uint32_t k[4][D / 32], kp[F == 4 ? 1 : 4];
};
template <int D, int F, bool PAGED>
__device__ __forceinline__ void load_keys(KeyCodes<D, F>& t, const Kv4& c, int pages, int n, int head_at, int k0, int lane) {
    typedef uint32_t words __attribute__((ext_vector_type(D / 32)));
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const uint8_t* block = block_of<PAGED>(c, pages, n, PAGED ? i : 0, head_at);
        const int at = PAGED ? place_of(c, k0, i) : place_of(c, k0, 0) + 16 * i;
        const words x = __builtin_nontemporal_load(reinterpret_cast<const words*>(block + at * (D / 2) + (uint32_t)((lane & 15) * (D / 2) + (lane >> 4) * (D / 8))));
#pragma unroll
        for (int j = 0; j < D / 32; ++j) t.k[i][j] = x[j];
        if constexpr (F != 4) t.kp[i] = __builtin_nontemporal_load(reinterpret_cast<const uint32_t*>(block + ((D << c.page_shift) + 4 * at) + (uint32_t)(4 * (lane & 15))));
    }
    if constexpr (F == 4) {
        const uint8_t* w;
        if constexpr (PAGED) {
            const int mine = lane >> 4;
            const uint8_t* block = nullptr;
            int at = 0;
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                block = mine == i ? block_of<PAGED>(c, pages, n, i, head_at) : block;
                at = mine == i ? place_of(c, k0, i) : at;
            }
            w = block + (uint32_t)((D << c.page_shift) + 4 * (at + (lane & 15)));
        } else {
            w = block_of<PAGED>(c, pages, n, 0, head_at) + ((D << c.page_shift) + 4 * place_of(c, k0, 0)) + (uint32_t)(4 * lane);
        }
        t.kp[0] = __builtin_nontemporal_load(reinterpret_cast<const uint32_t*>(w));
    }
}

// Eight codes less 8, in the order (0, 4), (1, 5), (2, 6), (3, 7).  (A code's bits by themselves are an fp16 number below the normal ones, c 2^-24,
// four instructions fewer a dword: right, but the matrix cores then keep some bits less of the sums, 1e-5 of a weight.)
__device__ __forceinline__ f16x8 key_operand(uint32_t w, const CodeBits& bits) {
    const f16x2 low{(_Float16)-1032.0f, (_Float16)-1032.0f}, high{(_Float16)-72.0f, (_Float16)-72.0f};
    const uint32_t h = w >> 8;
    const auto f = [](uint32_t x, f16x2 less) { return __builtin_bit_cast(uint32_t, as_f16(x) + less); };
    return __builtin_bit_cast(f16x8, u32x4{f(bits.low(w), low), f(bits.high(w), high), f(bits.low(h), low), f(bits.high(h), high)});
}

// Eight codes less 7.5.
__device__ __forceinline__ f16x8 key_codes(uint32_t w, const CodeBits& bits) {
    const f16x2 less{(_Float16)-71.5f, (_Float16)-71.5f};
    const auto f = [&](uint32_t x) { return __builtin_bit_cast(uint32_t, as_f16(bits.high(x)) + less); };
    return __builtin_bit_cast(f16x8, u32x4{f(w << 4), f(w), f(w >> 4), f(w >> 8)});
}

// What a row needs besides its operand, in the lanes of the row's results.
struct RowTerms {
    float f;                                      // log2 of the weight for a unit of the product, a power of two
    float sum;                                    // of the row's elements
    float lse;                                    // log2 of the softmax's sum; infinity where there is no row
};
struct Rows {
    float f[4], sum[4], lse[4];
};
__device__ __forceinline__ void spread(Rows& r, const RowTerms& t, int lane) {
#pragma unroll
    for (int e = 0; e < 4; ++e) {
        const int from = 4 * (lane >> 4) + e;     // (row `from` is column `from` of the operand: lanes 0 .. 15)
        r.f[e] = __shfl(t.f, from);
        r.sum[e] = __shfl(t.sum, from);
        r.lse[e] = __shfl(t.lse, from);
    }
}

// One query a sequence, at most sixteen heads a kv head.  F: copies of 16 / F rows among the sixteen, of which each takes every F-th 16 keys.
// A wave takes every fourth tile of 64 keys of the workgroup's chunk, and asks for the next one before this one's work.  Bound by memory: 16
// sequences x 32 heads x 8192 positions, 319 MB, 60 us (5.4 TB/s; the keys alone 44, stores mixed with reads cost the rest); vector issue
// 53 %, matrix cores 24 %.  1025 positions, 32 heads to 8: 5 us, launch and dependent loads.
template <int D, int F, bool F16, bool PAGED>
__global__ __launch_bounds__(64 * kWaves, 2) void k_kv4_weights(KvJob job, Kv4Weights out) {
    constexpr int C = 16 / F;
    const Kv4Attention& a = job.a;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int item = item_number(), seq = item / job.chunks, chunk = item - seq * job.chunks, head = blockIdx.x;
    if (seq >= a.batch) return;
    const int copy = (lane >> 4) * 4 / C, g = lane >> 4;
    const int head_at = head * ((D + 8) << job.cache.page_shift);
    int len = a.kv_lens[seq];
    len = len < 0 ? 0 : len > a.max_len ? (int)a.max_len : len;
    const int begin = chunk * job.chunk, end = begin + job.chunk < len ? begin + job.chunk : len;
    constexpr int stride = kWaves * kTile;
    int k0 = begin + wave * kTile;
    if (k0 >= end) return;
    const int lo = a.window && len > a.window ? len - a.window : 0;          // the first position that the query sees: it stands at the last
    float* weights = out.weights + seq * out.w_seq + head * out.w_head;
    const int of_lane = F == 2 ? 16 * (2 * (g & 1) + copy) + (lane & 15) : lane;            // of a tile's keys, the one that the lane writes
    // keys before the window: the weights decay
    for (; k0 + kTile <= lo; k0 += stride) {
        if (k0 >= end) return;
        if (out.decay != 1.0f && k0 + of_lane < end) weights[k0 + of_lane] = out.decay == 0.0f ? 0.0f : out.decay * weights[k0 + of_lane];
    }
    if (k0 >= end) return;
    const CodeBits bits;
    const int32_t* table = a.table + (int64_t)seq * a.width;
    int pages = load_pages<PAGED>(job.cache, table, a.width, k0, stride, lane), number_of = 0;
    // Weights of a tile, those behind the end out of range: loads and stores without a branch, after which all that is under way would be waited
    // for (16 sequences x 32 heads x 8192: 62.5 us with one).  The old ones first: what may not be asked for comes before what is.
    const auto weights_of = [&](int k0) { return __builtin_amdgcn_make_buffer_rsrc(weights + k0, 0, 4 * (end - k0 < kTile ? end - k0 : kTile), 0x00020000); };
    const auto load = [&](KeyCodes<D, F>& t, int k0) {
        if (out.decay != 0.0f) t.old = __uint_as_float(__builtin_amdgcn_raw_buffer_load_b32(weights_of(k0), 4 * of_lane, 0, 2));
        load_keys<D, F, PAGED>(t, job.cache, pages, number_of, head_at, k0, lane);
    };
    KeyCodes<D, F> even, odd;
    load(even, k0);
    Query<D, 16> q;
    Rows r;
    const int n = (lane & 15) % C;
    const bool there = n < job.group;
    {
        const int x = head * job.group + (there ? n : 0);
        const RawQuery<D, 16> raw = load_query<D, 16>(job, there, seq, x, lane);
        const float lse = there ? a.lse[(int64_t)seq * a.heads + x] : 0.0f;
        take_query<D, 16, F16, true>(q, job, raw, lane);
        spread(r, RowTerms{q.f, q.even + q.odd, there ? lse * kLog2e : INFINITY}, lane);
    }
    f32x4 start;                                  // the accumulator's first value
#pragma unroll
    for (int e = 0; e < 4; ++e) start[e] = 0.5f * r.sum[e];
    // The tile `t`, and the next one asked for.
    const auto take = [&](KeyCodes<D, F>& t, KeyCodes<D, F>& next, auto more) __attribute__((always_inline)) {
        if constexpr (more) {
            if (++number_of == kPagesOf<PAGED>) {
                pages = load_pages<PAGED>(job.cache, table, a.width, k0 + stride, stride, lane);
                number_of = 0;
            }
            load(next, k0 + stride);
            RQ_FENCE();                           // (the compiler would ask for them behind half of this tile's work)
        }
        float sums[4 / F] = {};
#pragma unroll
        for (int u = 0; u < 4 / F; ++u) {
            f32x4 s{};
            uint32_t p = t.kp[0];
#pragma unroll
            for (int f = 0; f < F; ++f) {
                const int i = u * F + f;
                f32x4 acc = start;
#pragma unroll
                for (int j = 0; j < D / 32; ++j) {
                    const f16x8 b = key_operand(t.k[i][j], bits);
                    acc = __builtin_amdgcn_mfma_f32_16x16x32_f16(q.hi[j], b, acc, 0, 0, 0);
                    acc = __builtin_amdgcn_mfma_f32_16x16x32_f16(q.lo[j], b, acc, 0, 0, 0);
                }
                const bool mine = F == 1 || copy == f;
#pragma unroll
                for (int e = 0; e < 4; ++e) s[e] = mine ? acc[e] : s[e];
                if constexpr (F != 4) p = mine ? t.kp[i] : p;
            }
            const float step = __uint_as_float(p << 16), mid = __uint_as_float(p & 0xffff0000u);
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const float x = fmaf(step, r.f[e] * s[e], fmaf(mid, r.f[e] * r.sum[e], -r.lse[e]));
                sums[u] += __builtin_amdgcn_exp2f(x);
            }
        }
        // a key's sum is in the lanes of its column that have rows of its copy
        float total = 0.0f;
#pragma unroll
        for (int u = 0; u < 4 / F; ++u) {
            float x = sums[u], b;
            if constexpr (F <= 2) {
                other_rows(x, false, x, b);
                x += b;
            }
            if constexpr (F == 1) {
                other_rows(x, true, x, b);
                x += b;
            }
            // (F == 2: block 2 u + copy, in lanes 2 copy, 2 copy + 1)
            total = F == 4 || (F == 2 ? (g & 1) == u : g == u) ? x : total;
        }
        total = k0 + of_lane >= lo ? total : 0.0f;
        __builtin_amdgcn_raw_buffer_store_b32(__float_as_uint(out.decay == 0.0f ? total : fmaf(out.decay, t.old, total)), weights_of(k0), 4 * of_lane, 0, 2);
        k0 += stride;
    };
    while (true) {
        if (k0 + stride >= end) {
            take(even, odd, std::false_type{});
            return;
        }
        take(even, odd, std::true_type{});
        if (k0 + stride >= end) {
            take(odd, even, std::false_type{});
            return;
        }
        take(odd, even, std::true_type{});
    }
}

// ---- many rows

// Row tile `tile` of 32 as the matrix cores take it, for every kv head: [tile][kv head][step][high, low][lane] sixteens of bytes, as
// Query<D, 32> has them, and [tile][kv head] terms of its rows.
struct TileTerms {
    float f[32], shift[32], lse[32];              // f as in RowTerms, f times the sum of the row's elements, -lse
    int at[32];                                   // the row's query among its sequence's; the last one where there is no row
};
template <int D>
constexpr int kTileBytes = 32 * D * 4;
template <int D>
__device__ __forceinline__ uint8_t* tile_at(const KvJob& job, int tile, int head) {
    return reinterpret_cast<uint8_t*>(job.part) + ((int64_t)tile * job.cache.kv_heads + head) * (kTileBytes<D> + (int)sizeof(TileTerms));
}

template <int D, bool F16>
__global__ __launch_bounds__(64 * kWaves) void k_kv4_weights_rows(KvJob job) {
    const Kv4Attention& a = job.a;
    const int lane = threadIdx.x & 63, tile = item_number() * kWaves + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), head = blockIdx.x;
    Place at;
    if (tile >= job.tiles || !find_rows<32>(job, tile, at)) return;
    const int n = at.base + (lane & 31);
    const bool there = n < at.nq * job.group;
    const int token = there ? token_of(job, at, n) : 0, x = head * job.group + (there ? n - token * job.group : 0);
    const RawQuery<D, 32> raw = load_query<D, 32>(job, there, at.q0 + token, x, lane);
    const float lse = there ? a.lse[(int64_t)(at.q0 + token) * a.heads + x] : 0.0f;
    Query<D, 32> q;
    take_query<D, 32, F16, true>(q, job, raw, lane);
    uint8_t* to = tile_at<D>(job, tile, head);
    u32x4* w = reinterpret_cast<u32x4*>(to);
#pragma unroll
    for (int j = 0; j < D / 16; ++j) {
        w[(2 * j) * 64 + lane] = __builtin_bit_cast(u32x4, q.hi[j]);
        w[(2 * j + 1) * 64 + lane] = __builtin_bit_cast(u32x4, q.lo[j]);
    }
    TileTerms* terms = reinterpret_cast<TileTerms*>(to + kTileBytes<D>);
    if (lane < 32) {
        terms->f[lane] = q.f;
        terms->shift[lane] = q.f * (q.even + q.odd);
        terms->lse[lane] = there ? -lse * kLog2e : -INFINITY;
        terms->at[lane] = there ? token : at.nq - 1;
    }
}

// A workgroup takes 256 keys, 64 a wave, unpacked once into registers, and a share of the row tiles that see some of them; row tiles come
// through LDS, the next one while this one is multiplied, and a tile's products stand between the exponentials of the one before.  Bound by
// issue: 64 queries of 32 heads on 8 against 16384 positions 20 us of 25.5 (one after the other 31); two prompts of 4000 queries, 5003 positions,
// window 1024, 14 heads of 64 on 2: 65 - 69 us in all, vector issue 50 %, matrix cores 23 %, 12 of them for laying queries out.
template <int D, bool PAGED>
__global__ __launch_bounds__(64 * kWaves, 2) void k_kv4_weights_many(KvJob job, Kv4Weights out, float* parts) {
    constexpr int S = D / 16, N = 2 * S * 64 / (64 * kWaves);        // steps; sixteens of bytes of a tile that a thread brings
    struct Staged {
        u32x4 q[2 * S * 64];
        TileTerms terms;
    };
    __shared__ __attribute__((aligned(16))) Staged staged[3];        // the tile being multiplied, the one whose terms are in use, the next
    static_assert(sizeof(TileTerms) == 16 * 32, "half a wave brings the terms");
    const Kv4Attention& a = job.a;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), half = lane >> 5;
    // (the last keys of a causal sequence are seen least: the first begin first)
    const int per = job.chunks * job.workers, item = item_number(), seq = item / per, rest = item - seq * per, chunk = rest / job.workers, share = rest - chunk * job.workers;
    const int head = blockIdx.x;
    if (seq >= a.batch) return;
    const int first_key = chunk * (kWaves * kTile), k0 = first_key + wave * kTile;
    const int head_at = head * ((D + 8) << job.cache.page_shift);
    // (asked for before the length is known)
    const int pages = load_pages<PAGED>(job.cache, a.table + (int64_t)seq * a.width, a.width, k0, kTile, lane);
    const int len = own_len(job, seq);
    int q0 = seq, nq = 1;
    if (a.q_start) {
        q0 = a.q_start[seq];
        int q1 = a.q_start[seq + 1];
        q0 = q0 < 0 ? 0 : q0 > a.tokens ? a.tokens : q0;
        q1 = q1 < q0 ? q0 : q1 > a.tokens ? a.tokens : q1;
        nq = q1 - q0;
    }
    if (first_key >= len) return;
    const int first_pos = len - nq;               // of the sequence's first query
    const int first_tile = a.q_start ? (int)((int64_t)q0 * job.group / 32) + seq : seq * ((job.group + 31) / 32);
    // queries that see some of the workgroup's keys: those from the first key on, if causal, and before the window has passed the last
    int from = 0, to = nq;
    if (a.causal && first_key > first_pos) from = first_key - first_pos;
    const int last_key = first_key + kWaves * kTile - 1 < len - 1 ? first_key + kWaves * kTile - 1 : len - 1;
    if (a.window && (int64_t)last_key + a.window - first_pos < to) to = last_key + a.window - first_pos;
    int t0 = from * job.group / 32, t1 = to > from ? (to * job.group + 31) / 32 : t0;
    {
        const int each = (t1 - t0 + job.workers - 1) / job.workers;
        t0 += share * each;
        t1 = t1 < t0 + each ? t1 : t0 + each;
    }
    // the wave's keys: lane n of a block of 32 has the half-row `half` of key n
    f16x8 keys[2][S];
    float step[2], mid[2], sum[2] = {};
    // the row tile under way (the last one again at the end: where a load may be left out, all before it is waited for)
    u32x4 brought[N], brought_terms;
    const auto bring = [&](int tile) __attribute__((always_inline)) {
        const u32x4* x = reinterpret_cast<const u32x4*>(tile_at<D>(job, first_tile + (tile < t1 ? tile : t1 - 1), head));
#pragma unroll
        for (int i = 0; i < N; ++i) brought[i] = x[threadIdx.x + 64 * kWaves * i];
        brought_terms = x[2 * S * 64 + (threadIdx.x & 31)];
    };
    const auto put = [&](Staged& to) __attribute__((always_inline)) {
#pragma unroll
        for (int i = 0; i < N; ++i) to.q[threadIdx.x + 64 * kWaves * i] = brought[i];
        reinterpret_cast<u32x4*>(&to.terms)[threadIdx.x & 31] = brought_terms;   // (eight threads the same: no branch, behind which all loads were waited for)
    };
    if (t0 < t1) bring(t0);
    {
        const CodeBits bits;
        uint32_t raw[2][S], kp[2];
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            const int n = 32 * i + (lane & 31);   // (a half of 32 lies in one page, or two quarters do)
            const uint8_t* block;
            int at;
            if constexpr (PAGED) {
                const bool second = (n >> 4) & 1;
                block = second ? block_of<PAGED>(job.cache, pages, 0, 2 * i + 1, head_at) : block_of<PAGED>(job.cache, pages, 0, 2 * i, head_at);
                at = (second ? place_of(job.cache, k0, 2 * i + 1) : place_of(job.cache, k0, 2 * i)) + (n & 15);
            } else {
                block = block_of<PAGED>(job.cache, pages, 0, 0, head_at);
                at = place_of(job.cache, k0, 0) + n;
            }
            const u32x4* x = reinterpret_cast<const u32x4*>(block + at * (D / 2) + half * (D / 4));
#pragma unroll
            for (int j = 0; j < S / 4; ++j) {
                const u32x4 y = x[j];
#pragma unroll
                for (int e = 0; e < 4; ++e) raw[i][4 * j + e] = y[e];
            }
            kp[i] = *reinterpret_cast<const uint32_t*>(block + ((D << job.cache.page_shift) + 4 * at));
        }
#pragma unroll
        for (int i = 0; i < 2; ++i) {
#pragma unroll
            for (int j = 0; j < S; ++j) keys[i][j] = key_codes(raw[i][j], bits);
            step[i] = __uint_as_float(kp[i] << 16);
            mid[i] = __uint_as_float(kp[i] & 0xffff0000u);
        }
    }
    // what four rows (e: of the lane's sixteen) need besides their products; MASKED: and where they stand
    struct Four {
        f32x4 f, shift, lse;
        u32x4 at;
    };
    const auto terms_of = [&](const Staged& of, int e, auto masked) __attribute__((always_inline)) {
        const int row = 2 * e + 4 * half;
        const auto four = [&](const void* x) { return reinterpret_cast<const u32x4*>(x)[row / 4]; };
        Four t{__builtin_bit_cast(f32x4, four(of.terms.f)), __builtin_bit_cast(f32x4, four(of.terms.shift)), __builtin_bit_cast(f32x4, four(of.terms.lse)), u32x4{}};
        if constexpr (masked) t.at = four(of.terms.at);
        return t;
    };
    // Their weights for both blocks; MASKED: of keys that they see.  The key at place i of the sequence is seen by queries i - first_pos and on, if
    // causal, and by no later one than i - first_pos + window - 1.
    // (`most` queries from `sees` on; not causal: from 2^30 before that on)
    uint32_t sees[2];
#pragma unroll
    for (int i = 0; i < 2; ++i) sees[i] = a.causal || a.window ? (uint32_t)(k0 + 32 * i + (lane & 31) - first_pos) - (a.causal ? 0u : 1u << 30) : 0u;
    const uint32_t most = !a.window ? 0x7fffffffu : (uint32_t)a.window + (a.causal ? 0u : 1u << 30);
    const auto weigh = [&](f32x16 (&s)[2], const Four& t, int e, auto masked) __attribute__((always_inline)) {
#pragma unroll
        for (int u = 0; u < 4; ++u)
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                float x = fmaf(step[i], t.f[u] * s[i][e + u], fmaf(mid[i], t.shift[u], t.lse[u]));
                if constexpr (masked) x = t.at[u] - sees[i] < most ? x : -INFINITY;
                sum[i] += __builtin_amdgcn_exp2f(x);
            }
    };
    f16x8 q[2][4];
    const auto read = [&](const Staged& of, int g) __attribute__((always_inline)) {
#pragma unroll
        for (int i = 0; i < 4; ++i) q[g % 2][i] = __builtin_bit_cast(f16x8, of.q[(4 * g + i) * 64 + lane]);
    };
    const auto multiply = [&](f32x16 (&s)[2], int g) __attribute__((always_inline)) {
#pragma unroll
        for (int j = 0; j < 2; ++j)
#pragma unroll
            for (int part = 0; part < 2; ++part)
#pragma unroll
                for (int i = 0; i < 2; ++i) s[i] = __builtin_amdgcn_mfma_f32_32x32x16_f16(q[g % 2][2 * j + part], keys[i][2 * g + j], s[i], 0, 0, 0);
    };
    // A row tile's products, and beside them the weights of the one before it; the next tile goes into LDS, the one after it is asked for.
    // (Operands are read a group of products ahead; nothing moves from group to group.)
    constexpr int G = S / 2;
    Staged *last = &staged[2], *now = &staged[0], *then = &staged[1];
    bool whole = true;                            // all rows of the tile before see all of the wave's keys
    const auto take = [&](int tile, f32x16 (&s)[2], f32x16 (&before)[2]) __attribute__((always_inline)) {
        put(*then);
        bring(tile + 2);
        read(*now, 0);
        const int first_at = __builtin_amdgcn_readfirstlane(now->terms.at[0]), last_at = __builtin_amdgcn_readfirstlane(now->terms.at[31]);
        s[0] = s[1] = f32x16{};
        const auto both = [&](auto masked) __attribute__((always_inline)) {
            constexpr int E = 4 / G;              // fours of rows beside a group
            constexpr int P = masked ? 1 : 2;     // (masked: registers are too few for the next group's)
            Four t[P][E];
            const auto read_terms = [&](int g) __attribute__((always_inline)) {
#pragma unroll
                for (int e = 0; e < E; ++e) t[g % P][e] = terms_of(*last, 4 * (E * g + e), masked);
            };
            if (P == 2) read_terms(0);
#pragma unroll
            for (int g = 0; g < G; ++g) {
                RQ_FENCE();
                if (P == 1) read_terms(g);
                if (g + 1 < G) read(*now, g + 1);
                if (P == 2 && g + 1 < G) read_terms(g + 1);
                multiply(s, g);
#pragma unroll
                for (int e = 0; e < E; ++e) weigh(before, t[g % P][e], 4 * (E * g + e), masked);
                if (g + 1 < G) RQ_NEXT(kLdsRead, 4 + (P == 1 ? 4 : 3) * E);
                else if (P == 1) RQ_NEXT(kLdsRead, 4 * E);
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    RQ_NEXT(kMfma, 1);
                    RQ_NEXT(kValu, (masked ? 8 : 5) * E);
                }
            }
            RQ_FENCE();
        };
        if (whole) both(std::false_type{});
        else both(std::true_type{});
        // (from the last one's window on to the first one's position)
        whole = (!a.causal || k0 + kTile - 1 <= first_pos + first_at) && (!a.window || k0 > first_pos + last_at - a.window);
        Staged* free = last;
        last = now;
        now = then;
        then = free;
        lds_barrier();                            // (one a tile: what goes into LDS next takes the place of terms that were read before it)
    };
    if (t0 < t1) {
        f32x16 even[2], odd[2];
        odd[0] = odd[1] = f32x16{};               // before the first tile: rows of no weight
        last->terms.f[lane & 31] = last->terms.shift[lane & 31] = 0.0f;
        last->terms.lse[lane & 31] = -INFINITY;
        put(*now);
        bring(t0 + 1);
        lds_barrier();
        for (int tile = t0; tile < t1; tile += 2) {
            take(tile, even, odd);
            if (tile == t0) sum[0] = sum[1] = 0.0f;        // (of the rows before the first tile: NaN for a key that is not finite, seen or not)
            take(tile + 1, odd, even);            // (where there is no such tile, the last one again, whose weights are not taken)
        }
        if ((t1 - t0) % 2 == 0)
#pragma unroll
            for (int e = 0; e < 16; e += 4) weigh(odd, terms_of(*last, e, std::true_type{}), e, std::true_type{});
    }
    float x, y;
    other_rows(sum[0], true, x, y);
    const float first = x + y;
    other_rows(sum[1], true, x, y);
    const float total = half ? x + y : first;
    const int key = k0 + lane;
    if (key >= len) return;
    if (job.workers > 1) {
        parts[(((int64_t)share * a.batch + seq) * job.cache.kv_heads + head) * a.max_len + key] = total;
    } else {
        float* w = out.weights + seq * out.w_seq + head * out.w_head + key;
        *w = out.decay == 0.0f ? total : fmaf(out.decay, *w, total);
    }
}

// Shares of rows added up.
__global__ __launch_bounds__(256) void k_kv4_weights_join(KvJob job, Kv4Weights out, const float* parts) {
    const Kv4Attention& a = job.a;
    const int64_t item = group_index(), per = (a.max_len + 255) / 256, row = item / per;
    if (row >= (int64_t)a.batch * job.cache.kv_heads) return;
    const int seq = (int)(row / job.cache.kv_heads), head = (int)(row - (int64_t)seq * job.cache.kv_heads);
    const int key = (int)(item - row * per) * 256 + (int)threadIdx.x;
    if (key >= own_len(job, seq)) return;
    const int64_t rows = (int64_t)a.batch * job.cache.kv_heads;
    float total = 0.0f;
#pragma unroll 8
    for (int i = 0; i < job.workers; ++i) total += parts[(i * rows + row) * a.max_len + key];
    float* w = out.weights + seq * out.w_seq + head * out.w_head + key;
    *w = out.decay == 0.0f ? total : fmaf(out.decay, *w, total);
}

// ---- launches

bool few(const Kv4& c, const Kv4Attention& a) { return !a.q_start && a.heads / c.kv_heads <= 16; }

// Many rows: row tiles, chunks of 256 keys, shares of the rows.
struct Plan {
    int tiles, chunks, shares;
    size_t rows_bytes, bytes;
};
Plan plan(const Kv4& c, const Kv4Attention& a, int num_cu) {
    const int64_t group = a.heads / c.kv_heads, rows = (int64_t)a.tokens * group;
    Plan p{};
    p.tiles = (int)(a.q_start ? rows / 32 + a.batch : (int64_t)a.batch * ((group + 31) / 32));
    p.chunks = (int)((a.max_len + kWaves * kTile - 1) / (kWaves * kTile));
    // Shares of a workgroup's rows, by what they cost in row tiles: two workgroups a compute unit, each as long as its row tiles and two more;
    // what all of them take together, and one of them, which is what the last ones take (causal masks and windows make them unlike);
    // adding the shares up, a launch more, four.  Two prompts of 5003, window 1024, 14 heads to 2: 20 or 30 shares 65 us, 7: 74; 64 queries
    // against 16384 positions: one share 25, two 29.
    const int64_t wgs = (int64_t)a.batch * c.kv_heads * p.chunks, seen = a.window ? ((int64_t)a.window + kWaves * kTile) * group / 32 + 1 : INT64_MAX;
    const int64_t mean = rows / 32 / a.batch + 1, tiles = mean < seen ? mean : seen;
    double least = 0.0;
    for (int n = 1; n <= 64 && n <= tiles; ++n) {
        const double one = (double)((tiles + n - 1) / n + 2), cost = one * (double)(wgs * n) / (2.0 * num_cu) + one + (n > 1 ? 4.0 : 0.0);
        if (n > 1 && cost >= least) continue;
        least = cost;
        p.shares = n;
    }
    p.rows_bytes = (size_t)p.tiles * c.kv_heads * (32 * c.head_dim * 4 + sizeof(TileTerms));
    p.bytes = p.rows_bytes + (p.shares > 1 ? (size_t)p.shares * a.batch * c.kv_heads * a.max_len * sizeof(float) : 0);
    return p;
}

template <int D, int F, bool F16>
void launch_few(const KvJob& job, const Kv4Weights& w, hipStream_t s) {
    const dim3 grid = item_grid(job.cache.kv_heads, (int64_t)job.a.batch * job.chunks), block(64 * kWaves);
    if (job.cache.page_shift < 6) launch_kernel(k_kv4_weights<D, F, F16, true>, grid, block, 0, s, job, w);
    else launch_kernel(k_kv4_weights<D, F, F16, false>, grid, block, 0, s, job, w);
}
template <int D, bool F16>
void launch_few(const KvJob& job, const Kv4Weights& w, hipStream_t s) {
    if (job.group > 8) launch_few<D, 1, F16>(job, w, s);
    else if (job.group > 4) launch_few<D, 2, F16>(job, w, s);
    else launch_few<D, 4, F16>(job, w, s);
}
template <int D>
void launch_many(const KvJob& job, const Kv4Weights& w, const Plan& p, hipStream_t s) {
    const dim3 block(64 * kWaves);
    if (job.tiles > 0 && job.a.tokens > 0) {
        const dim3 grid = item_grid(job.cache.kv_heads, (job.tiles + kWaves - 1) / kWaves);
        if (job.a.dtype == RQ_F16) launch_kernel(k_kv4_weights_rows<D, true>, grid, block, 0, s, job);
        else launch_kernel(k_kv4_weights_rows<D, false>, grid, block, 0, s, job);
    }
    float* parts = reinterpret_cast<float*>(reinterpret_cast<uint8_t*>(job.part) + p.rows_bytes);
    const dim3 grid = item_grid(job.cache.kv_heads, (int64_t)job.a.batch * p.chunks * p.shares);
    if (job.cache.page_shift < 6) launch_kernel(k_kv4_weights_many<D, true>, grid, block, 0, s, job, w, parts);
    else launch_kernel(k_kv4_weights_many<D, false>, grid, block, 0, s, job, w, parts);
    if (p.shares > 1)
        launch_kernel(k_kv4_weights_join, group_grid((job.a.max_len + 255) / 256 * job.a.batch * job.cache.kv_heads, 256), dim3(256), 0, s, job, w, parts);
}

}  // namespace

size_t kv4_weights_workspace(const Kv4& c, const Kv4Attention& a, int num_cu) { return few(c, a) || a.tokens == 0 ? 0 : plan(c, a, num_cu).bytes; }

int kv4_weights(const Kv4& c, const Kv4Weights& w, int num_cu, void* workspace, hipStream_t s) {
    const Kv4Attention& a = w.a;
    const bool wide_q = reinterpret_cast<uintptr_t>(a.q) % 16 == 0 && a.q_token % 8 == 0 && a.q_head % 8 == 0;
    KvJob job{c, a, a.heads / c.kv_heads, 0, 0, 0, 0, wide_q, false, static_cast<float*>(workspace)};
    if (!few(c, a)) {
        const Plan p = plan(c, a, num_cu);
        job.tiles = p.tiles;
        job.workers = p.shares;
        job.chunks = p.chunks;
        c.head_dim == 128 ? launch_many<128>(job, w, p, s) : launch_many<64>(job, w, p, s);
        return launch_rc();
    }
    // workgroups of at least a tile a wave, eight a compute unit where there are as many
    const int64_t units = (a.max_len + kWaves * kTile - 1) / (kWaves * kTile), want = (8 * (int64_t)num_cu + (int64_t)a.batch * c.kv_heads - 1) / ((int64_t)a.batch * c.kv_heads);
    const int64_t chunks = want < units ? want : units;
    job.chunk = (int)((units + chunks - 1) / chunks) * kWaves * kTile;
    job.chunks = (int)((a.max_len + job.chunk - 1) / job.chunk);
    const bool f16 = a.dtype == RQ_F16;
    if (c.head_dim == 128) f16 ? launch_few<128, true>(job, w, s) : launch_few<128, false>(job, w, s);
    else f16 ? launch_few<64, true>(job, w, s) : launch_few<64, false>(job, w, s);
    return launch_rc();
}

}  // namespace rq
