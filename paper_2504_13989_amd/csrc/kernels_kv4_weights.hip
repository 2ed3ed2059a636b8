// How much attention the positions of cached sequences receive: w_j <- decay * w_j + sum_i exp(scale q_i . k_j - lse_i), over the
// queries i that see position j, of all heads that share its kv head.
//
// Products are queries x keys: a key is a column, column n the lanes n, n + 16, n + 32, n + 48, of which lane g has rows 4 g + 0 .. 3.  A
// key's step and centre and its sum stay in its lanes, and the sum over a tile's rows is three additions.
//   - Codes become fp16 numbers c - 8, exactly (mantissas of 1024 and 64, less 1032 and 72); the half that is missing is the sum of the
//     row's elements, which the accumulator starts from.  (The 1024 could be taken off there too, as attention does, but sums that
//     carry it are good to 2^-12, and weights are 32 bits.)
//   - Queries are two fp16 numbers each (kv4_attention.h): 22 bits.
#include "kv4_attention.h"

namespace rq {
namespace {

constexpr int kWaves = 4;

// A tile's key codes and parameters (of key 16 i + lane % 16).
template <int D>
struct KeyCodes {
    uint32_t k[4][D / 32], kp[4];
};
template <int D, bool PAGED>
__device__ __forceinline__ void load_keys(KeyCodes<D>& t, const Kv4& c, int pages, int n, int head_at, int k0, int lane) {
    typedef uint32_t words __attribute__((ext_vector_type(D / 32)));
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const uint8_t* block = block_of<PAGED>(c, pages, n, PAGED ? i : 0, head_at);
        const int at = PAGED ? place_of(c, k0, i) : place_of(c, k0, 0) + 16 * i;
        const words x = __builtin_nontemporal_load(reinterpret_cast<const words*>(block + at * (D / 2) + (uint32_t)((lane & 15) * (D / 2) + (lane >> 4) * (D / 8))));
#pragma unroll
        for (int j = 0; j < D / 32; ++j) t.k[i][j] = x[j];
        t.kp[i] = __builtin_nontemporal_load(reinterpret_cast<const uint32_t*>(block + ((D << c.page_shift) + 4 * at) + (uint32_t)(4 * (lane & 15))));
    }
}

// Eight codes less 8, in the order (0, 4), (1, 5), (2, 6), (3, 7).
__device__ __forceinline__ f16x8 key_operand(uint32_t w, const CodeBits& bits) {
    const f16x2 low{(_Float16)-1032.0f, (_Float16)-1032.0f}, high{(_Float16)-72.0f, (_Float16)-72.0f};
    const uint32_t h = w >> 8;
    const auto f = [](uint32_t x, f16x2 less) { return __builtin_bit_cast(uint32_t, as_f16(x) + less); };
    return __builtin_bit_cast(f16x8, u32x4{f(bits.low(w), low), f(bits.high(w), high), f(bits.low(h), low), f(bits.high(h), high)});
}

// What a row needs besides its operand, in the lanes of the row's results.
struct RowTerms {
    float f;                                      // log2 of the weight for a unit of the product, a power of two
    float sum;                                    // of the row's elements
    float lse;                                    // log2 of the softmax's sum; infinity where there is no row
    int lo, seen;                                 // the first position that it sees, how many
};
struct Rows {
    float f[4], sum[4], lse[4];
    int lo[4], seen[4];
};
__device__ __forceinline__ void spread(Rows& r, const RowTerms& t, int lane) {
#pragma unroll
    for (int e = 0; e < 4; ++e) {
        const int from = 4 * (lane >> 4) + e;     // (row `from` is column `from` of the operand: lanes 0 .. 15)
        r.f[e] = __shfl(t.f, from);
        r.sum[e] = __shfl(t.sum, from);
        r.lse[e] = __shfl(t.lse, from);
        r.lo[e] = __shfl(t.lo, from);
        r.seen[e] = __shfl(t.seen, from);
    }
}

// Weights of one block of 16 keys for the tile's rows, summed over the lane's four.
__device__ __forceinline__ float weigh(const f32x4& s, const Rows& r, float step, float mid, int key, bool whole) {
    float sum = 0.0f;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
        float x = fmaf(step, r.f[e] * s[e], fmaf(mid, r.f[e] * r.sum[e], -r.lse[e]));
        if (!whole) x = (uint32_t)(key - r.lo[e]) < (uint32_t)r.seen[e] ? x : -INFINITY;
        sum += __builtin_amdgcn_exp2f(x);
    }
    return sum;
}

// F: copies of 16 / F rows among the sixteen, of which each takes every F-th 16 keys (few rows: one tile of them a sequence).
// MANY: row tiles of 16 one after the other.  A wave takes every fourth tile of 64 keys of the workgroup's chunk.
template <int D, int F, bool F16, bool PAGED, bool MANY>
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
    int q0 = seq, nq = 1;
    if (a.q_start) {
        q0 = a.q_start[seq];
        int q1 = a.q_start[seq + 1];
        q0 = q0 < 0 ? 0 : q0 > a.tokens ? a.tokens : q0;
        q1 = q1 < q0 ? q0 : q1 > a.tokens ? a.tokens : q1;
        nq = q1 - q0;
    }
    const int rows = nq * job.group;
    const int begin = chunk * job.chunk, end = begin + job.chunk < len ? begin + job.chunk : len;
    constexpr int stride = kWaves * kTile;
    int k0 = begin + wave * kTile;
    if (k0 >= end) return;
    const CodeBits bits;
    const int32_t* table = a.table + (int64_t)seq * a.width;
    int pages = load_pages<PAGED>(job.cache, table, a.width, k0, stride, lane), number_of = 0;
    KeyCodes<D> t;
    load_keys<D, PAGED>(t, job.cache, pages, 0, head_at, k0, lane);
    Query<D, 16> q;
    Rows r;
    int all_lo = 0, all_hi = 0;                   // what all rows of the tile see
    const auto take_rows = [&](int base) {
        const int n = base + (lane & 15) % C;
        const bool there = n < rows;
        const int token = there ? (nq == 1 ? 0 : n / job.group) : 0, of = there ? n - token * job.group : 0;
        const RawQuery<D, 16> raw = load_query<D, 16>(job, there, q0 + token, head * job.group + of, lane);
        const float lse = there ? a.lse[(int64_t)(q0 + token) * a.heads + head * job.group + of] : 0.0f;
        take_query<D, 16, F16, true>(q, job, raw, lane);
        const int pos = len - nq + token;
        const int hi = !there ? 0 : a.causal ? (pos + 1 < len ? pos + 1 : len) : len;
        const int lo = a.window ? (pos - a.window + 1 > 0 ? pos - a.window + 1 : 0) : 0;
        spread(r, RowTerms{q.f, q.even + q.odd, there ? lse * kLog2e : INFINITY, lo, hi > lo ? hi - lo : 0}, lane);
        const int last = (base + C < rows ? base + C : rows) - 1;
        const int p0 = len - nq + (nq == 1 ? 0 : base / job.group), p1 = len - nq + (nq == 1 ? 0 : last / job.group);
        all_lo = a.window ? p1 - a.window + 1 : 0;
        all_hi = a.causal && p0 + 1 < len ? p0 + 1 : len;
    };
    if (!MANY) take_rows(0);
    for (; k0 < end; k0 += stride) {
        KeyCodes<D> next;
        if (k0 + stride < end) {
            if (++number_of == kPagesOf<PAGED>) {
                pages = load_pages<PAGED>(job.cache, table, a.width, k0 + stride, stride, lane);
                number_of = 0;
            }
            load_keys<D, PAGED>(next, job.cache, pages, number_of, head_at, k0 + stride, lane);
        }
        float sums[4 / F] = {};
        const auto take = [&] {
            const bool whole = k0 >= all_lo && k0 + kTile <= all_hi;
#pragma unroll
            for (int u = 0; u < 4 / F; ++u) {
                f32x4 s{};
                float step = 0.0f, mid = 0.0f;
#pragma unroll
                for (int f = 0; f < F; ++f) {
                    const int i = u * F + f;
                    f32x4 acc;
#pragma unroll
                    for (int e = 0; e < 4; ++e) acc[e] = 0.5f * r.sum[e];
#pragma unroll
                    for (int j = 0; j < D / 32; ++j) {
                        const f16x8 b = key_operand(t.k[i][j], bits);
                        acc = __builtin_amdgcn_mfma_f32_16x16x32_f16(q.hi[j], b, acc, 0, 0, 0);
                        acc = __builtin_amdgcn_mfma_f32_16x16x32_f16(q.lo[j], b, acc, 0, 0, 0);
                    }
                    const bool mine = F == 1 || copy == f;
#pragma unroll
                    for (int e = 0; e < 4; ++e) s[e] = mine ? acc[e] : s[e];
                    step = mine ? __uint_as_float(t.kp[i] << 16) : step;
                    mid = mine ? __uint_as_float(t.kp[i] & 0xffff0000u) : mid;
                }
                sums[u] += weigh(s, r, step, mid, k0 + 16 * (u * F + (F == 1 ? 0 : copy)) + (lane & 15), whole);
            }
        };
        if constexpr (MANY) {
            // the row tiles that see some of the tile: positions from k0 on if causal, and not behind the window's reach
            int first = 0, last = rows;
            if (a.causal && k0 - (len - nq) > 0) first = (k0 - (len - nq)) * job.group / C * C;
            if (a.window && k0 + kTile - 1 + a.window - (len - nq) < nq) last = (k0 + kTile - 1 + a.window - (len - nq)) * job.group;
            for (int base = first; base < last; base += C) {
                take_rows(base);
                take();
            }
        } else if (rows > 0) {
            take();
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
            // lane g writes keys 16 g ...
            if constexpr (F == 1) total = g == u ? x : total;
            else if constexpr (F == 2) {          // block 2 u + copy, in lanes 2 copy, 2 copy + 1
                total = (g & 1) == u ? x : total;
            } else total = x;
        }
        const int block = F == 2 ? 2 * (g & 1) + copy : g;
        const int key = k0 + 16 * block + (lane & 15);
        if (key < end) {
            float* w = out.weights + seq * out.w_seq + head * out.w_head + key;
            *w = out.decay == 0.0f ? total : fmaf(out.decay, *w, total);
        }
        t = next;
    }
}

template <int D, int F, bool F16, bool MANY>
void launch(const KvJob& job, const Kv4Weights& w, hipStream_t s) {
    const dim3 grid = item_grid(job.cache.kv_heads, (int64_t)job.a.batch * job.chunks), block(64 * kWaves);
    if (job.cache.page_shift < 6) launch_kernel(k_kv4_weights<D, F, F16, true, MANY>, grid, block, 0, s, job, w);
    else launch_kernel(k_kv4_weights<D, F, F16, false, MANY>, grid, block, 0, s, job, w);
}
template <int D, bool F16>
void launch(const KvJob& job, const Kv4Weights& w, hipStream_t s) {
    if (job.a.q_start || job.group > 16) launch<D, 1, F16, true>(job, w, s);
    else if (job.group > 8) launch<D, 1, F16, false>(job, w, s);
    else if (job.group > 4) launch<D, 2, F16, false>(job, w, s);
    else launch<D, 4, F16, false>(job, w, s);
}

}  // namespace

size_t kv4_weights_workspace(const Kv4&, const Kv4Attention&, int) { return 0; }

int kv4_weights(const Kv4& c, const Kv4Weights& w, int num_cu, void*, hipStream_t s) {
    const Kv4Attention& a = w.a;
    const bool wide_q = reinterpret_cast<uintptr_t>(a.q) % 16 == 0 && a.q_token % 8 == 0 && a.q_head % 8 == 0;
    // workgroups of at least a tile a wave, eight a compute unit where there are as many
    const int64_t units = (a.max_len + kWaves * kTile - 1) / (kWaves * kTile), want = (8 * (int64_t)num_cu + (int64_t)a.batch * c.kv_heads - 1) / ((int64_t)a.batch * c.kv_heads);
    const int64_t chunks = want < units ? want : units;
    const int chunk = (int)((units + chunks - 1) / chunks) * kWaves * kTile;
    const KvJob job{c, a, a.heads / c.kv_heads, 0, 0, chunk, (int)((a.max_len + chunk - 1) / chunk), wide_q, false, nullptr};
    const bool f16 = a.dtype == RQ_F16;
    if (c.head_dim == 128) f16 ? launch<128, true>(job, w, s) : launch<128, false>(job, w, s);
    else f16 ? launch<64, true>(job, w, s) : launch<64, false>(job, w, s);
    return launch_rc();
}

}  // namespace rq
