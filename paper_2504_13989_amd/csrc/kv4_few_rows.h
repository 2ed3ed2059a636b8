// Attention over the 4-bit paged cache (kv4_layout.h): o_i = sum_j p_ij v_j / sum_j p_ij, p_ij = exp(scale q_i . k_j - m_i), for few
// queries a sequence (a decode step): the kernel.
//
// With k_jd = (c_jd - 7.5) step_j + mid_j the scores are  q_i . k_j = step_j (q_i . c_j - 7.5 sum q_i) + mid_j sum q_i:  the codes
// themselves are an operand of the matrix cores and a key's step and centre are applied once a score, not once an element.  The
// values' side is alike: with p'_ij = p_ij step_j,  o_i = sum_j p'_ij (c_jd - 8 + mid_j / step_j + 1 / 2).
//   - A code becomes an fp16 number by masking it into the mantissa of 1024 or 64: two codes an instruction.  The constants' share
//     is known and taken off in fp32: for keys in the accumulator's initial value; for values, whose sums run over all keys and would lose
//     digits to it, tile by tile, by a second product with the constant.
//   - The query row is scaled by a power of two to at most 1 and rounded to fp16 (2^-11; bf16 would move a score of 10 by 0.02);
//     where that alone is more than an fp16 result's rounding, as rotated queries', it is two fp16 numbers.
//   - p' is rounded to fp16 too (bf16 would leave 1.4e-3 of error in outputs that fp16 holds to 2e-4): steps carry a power of two that
//     brings the largest seen so far to 2^7, so that p' neither overflows nor, down to 2^-21 of the largest, loses digits.  (They, and
//     not p: the sum of p is then the same however large or small values are.)
//     The centres' share is summed in fp32 from p' as it was rounded: what the codes and a centre make together is off by p's rounding.
//
// Products are taken transposed, keys x queries and elements x queries, so that a query is a column, column n the lanes n, n + 16,
// n + 32, n + 48: scores leave the matrix cores in the lanes in which p' enters them again (keys in an order of their own,
// which the values follow), and maxima, sums and factors of a query stay in its lanes.  Rows are the queries of all heads that
// share a kv head, token by token.  Where they fill only 16 / F columns, the columns are F copies of them, each of which takes
// every F-th 16 keys: a lane then works on 16 / F scores a tile and not on 16 (the matrix cores, which are idle most of the time,
// compute the rest for nothing), and the copies are joined at the end as waves are.
//
// What is bound here is the stream of codes.  A row tile is a workgroup's, of one, four or eight waves as there are many row tiles or
// few.  Where that leaves compute units empty for long, there are two workgroups of four waves a compute unit, and each takes
// the same number of tiles of 64 keys, which may be parts of several sequences (a workgroup costs 5 us beside its tiles: when that was settled, eight times as many of an eighth of the work took
// 141 us where two a unit took 109).  The waves take a workgroup's tiles in turn.  A tile's codes are read into the registers of the one before
// as soon as those are used up, keys during the softmax, values during the next keys' products.
// 16 sequences x 32 heads x 8192 positions of 128, bf16: 87 .. 90 us, 6.3 to 6.5 TB/s of codes and parameters (reading alone
// reaches 6.9); vector issue 44 %, matrix cores 24 %.  Six sequences of up to 65411 positions, 64 heads to 8, fp16: 46 us and 5.2.
// Five chunks of prompts, 14 heads of 64 to 2, window 1024, fp16: 44 us, vector issue 62 %.
#pragma once
#include "kv4_attention.h"

#include <type_traits>

namespace rq {
namespace {

constexpr int kWaves = 4, kMostWaves = 8;         // of a workgroup; of one that has a row tile to itself while the chip is not full (or one: plan())

// Eight key codes as fp16: elements (0, 4), (1, 5), (2, 6), (3, 7) of the dword, 1024 + c in the even ones, 64 + c in the odd ones.
__device__ __forceinline__ f16x8 key_operand(uint32_t w, const CodeBits& bits) {
    const uint32_t h = w >> 8;
    return __builtin_bit_cast(f16x8, u32x4{bits.low(w), bits.high(w), bits.low(h), bits.high(h)});
}
// Nibble J of both halves of a dword as fp16: 1024 + c for even J, 64 + c for odd J.
template <int J>
__device__ __forceinline__ uint32_t value_pair(uint32_t w, const CodeBits& bits) {
    const uint32_t x = J / 2 ? w >> 8 : w;
    return J % 2 ? bits.high(x) : bits.low(x);
}

// A tile's codes as they are stored, and its keys' parameters, a key a lane.
template <int D>
struct Codes {
    uint32_t k[4][D / 32], v[4][D / 32];          // [16 keys][dword]
    uint32_t kp, vp;
};
// Where a tile's codes and parameters lie: the head's block of its page, the place in the page; PAGED: of each 16 keys.
template <bool PAGED>
struct Source {
    const uint8_t* block[PAGED ? 4 : 1];
    int at[PAGED ? 4 : 1];
};
template <bool PAGED>
__device__ __forceinline__ Source<PAGED> find_tile(const Kv4& c, int pages, int n, int head_at, int k0) {
    Source<PAGED> s;
#pragma unroll
    for (int i = 0; i < (PAGED ? 4 : 1); ++i) {
        s.block[i] = block_of<PAGED>(c, pages, n, i, head_at);
        s.at[i] = place_of(c, k0, i);
    }
    return s;
}
template <int D, bool PAGED>
__device__ __forceinline__ void load_keys(Codes<D>& t, const Source<PAGED>& s, int page_shift, int lane) {
    typedef uint32_t words __attribute__((ext_vector_type(D / 32)));
    const uint32_t off = (uint32_t)((lane & 15) * (D / 2) + (lane >> 4) * (D / 8));
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const uint8_t* k = PAGED ? s.block[PAGED ? i : 0] + s.at[PAGED ? i : 0] * (D / 2) : s.block[0] + s.at[0] * (D / 2) + i * (8 * D);
        const words x = __builtin_nontemporal_load(reinterpret_cast<const words*>(k + off));
#pragma unroll
        for (int j = 0; j < D / 32; ++j) t.k[i][j] = x[j];
    }
    const uint8_t* w;
    if constexpr (PAGED) {
        const int i = lane >> 4;
        const uint8_t* block = i == 0 ? s.block[0] : i == 1 ? s.block[1] : i == 2 ? s.block[2] : s.block[3];
        const int at = i == 0 ? s.at[0] : i == 1 ? s.at[1] : i == 2 ? s.at[2] : s.at[3];
        w = block + (uint32_t)((D << page_shift) + 4 * (at + (lane & 15)));
    } else {
        w = s.block[0] + ((D << page_shift) + 4 * s.at[0]) + (uint32_t)(4 * lane);
    }
    t.kp = __builtin_nontemporal_load(reinterpret_cast<const uint32_t*>(w));
    t.vp = __builtin_nontemporal_load(reinterpret_cast<const uint32_t*>(w + (4 << page_shift)));
}
template <int D, bool PAGED>
__device__ __forceinline__ void load_values(Codes<D>& t, const Source<PAGED>& s, int page_shift, int lane) {
    typedef uint32_t words __attribute__((ext_vector_type(D / 32)));
    const uint32_t off = (uint32_t)((lane >> 4) * (2 * D) + (lane & 15) * (D / 8));
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const int at = (1 << page_shift) + s.at[PAGED ? i : 0];
        const uint8_t* v = s.block[PAGED ? i : 0] + at * (D / 2) + (PAGED ? 0 : i * (8 * D));
        const words x = __builtin_nontemporal_load(reinterpret_cast<const words*>(v + off));
#pragma unroll
        for (int j = 0; j < D / 32; ++j) t.v[i][j] = x[j];
    }
}

constexpr int kParameters = 5;                    // of a key in LDS

// The columns of a wave, and what it has summed up.
template <int D>
struct Columns {
    Query<D, 16> q;
    float sum, bias;                              // sum of q, what the accumulator starts from
    int lo, seen;                                 // the first key that the column's query sees, how many it sees
    float m, l, w;                                // running maximum; sums over the lane's keys of p, and of what centres and halves of steps add
    f32x4 o[D / 16];
    bool far;                                     // some centre of the tile goes with p
    float limit;                                  // a power of two that no step seen so far exceeds, nor 2^-64 of a centre that goes with p
    float factor;                                 // 2^7 / limit: in steps and in sums of values
};

// Sums of values times a factor of the column.
template <int D>
__device__ __forceinline__ void scale_sums(Columns<D>& r, float by) {
    r.w *= by;
#pragma unroll
    for (int j = 0; j < D / 16; ++j)
#pragma unroll
        for (int e = 0; e < 4; ++e) r.o[j][e] *= by;
}

// The parameters of a tile to LDS: keys' steps and centres, values' steps and what their centres + step / 2 add.  A value row that is not finite
// becomes zeros and its key NaN: columns that do not see it stay what they are.
template <int D>
__device__ __forceinline__ void take_parameters(Columns<D>& r, const Codes<D>& t, float* lds, bool there, int lane) {
    const uint32_t kp = there ? t.kp : 0u, vp = there ? t.vp : 0u;
    float ks = __uint_as_float(kp << 16), step = __uint_as_float(vp << 16), mid = __uint_as_float(vp & 0xffff0000u);
    if (!finite(step) || !finite(mid)) {
        step = mid = 0.0f;
        ks = __builtin_nanf("");
    }
    const Centre c = split_centre(step, mid);
    const auto put = [&] {
        lds[128 + lane] = step * r.factor;
        lds[256 + lane] = c.with_p * r.factor;
    };
    lds[lane] = ks;
    lds[64 + lane] = __uint_as_float(kp & 0xffff0000u);
    put_centre(lds + 192, lane, c.with_step + 0.5f);
    put();
    r.far = __any(c.with_p != 0.0f);
    float size = fmaxf(step, fabsf(c.with_p) * 0x1p-64f);
    if (__any(size > r.limit)) {
#pragma unroll
        for (int w = 1; w < 64; w *= 2) size = fmaxf(size, __shfl_xor(size, w));
        const int x = (int)(__float_as_uint(size) >> 23) - 126;      // size < 2^x
        const float limit = __uint_as_float((uint32_t)((x < -60 ? -60 : x > 127 ? 127 : x) + 127) << 23);
        if (limit > r.limit) {
            const float factor = 0x1p7f / limit;
            scale_sums(r, factor / r.factor);     // (0 where sums of values are lost beside the new ones)
            r.limit = limit;
            r.factor = factor;
            put();
        }
    }
}

// Scores of a tile: s[u], of 16 keys each that the lane's copy has.
template <int D, int F, bool F16>
__device__ __forceinline__ void take_keys(f32x4 (&s)[4 / F], const Columns<D>& r, const Codes<D>& t, const CodeBits& bits, int copy) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        f32x4 acc = f32x4{r.bias, r.bias, r.bias, r.bias};
#pragma unroll
        for (int j = 0; j < D / 32; ++j) {
            const f16x8 a = key_operand(t.k[i][j], bits);
            acc = __builtin_amdgcn_mfma_f32_16x16x32_f16(a, r.q.hi[j], acc, 0, 0, 0);
            if constexpr (F16) acc = __builtin_amdgcn_mfma_f32_16x16x32_f16(a, r.q.lo[j], acc, 0, 0, 0);
        }
#pragma unroll
        for (int e = 0; e < 4; ++e) s[i / F][e] = i % F == 0 || copy == i % F ? acc[e] : s[i / F][e];
    }
}

// Scores to p * step, and what goes with it.  k0: the tile's first key; `whole`: every column sees all of it.
template <int D, int F>
__device__ __forceinline__ void take_scores(uint32_t (&p)[4 / F][2], Columns<D>& r, f32x4 (&s)[4 / F], const float* lds, int k0, bool whole, int copy, int g) {
    constexpr int U = 4 / F;
#pragma unroll
    for (int u = 0; u < U; ++u) {
        const int key = 16 * (u * F + copy) + 4 * g;
        const f32x4 step = *reinterpret_cast<const f32x4*>(lds + key), mid = *reinterpret_cast<const f32x4*>(lds + 64 + key);
#pragma unroll
        for (int e = 0; e < 4; ++e) s[u][e] = fmaf(step[e], s[u][e], mid[e] * r.sum);
    }
    if (!whole) {
#pragma unroll
        for (int u = 0; u < U; ++u)
#pragma unroll
            for (int e = 0; e < 4; ++e) s[u][e] = (uint32_t)(k0 + 16 * (u * F + copy) + 4 * g + e - r.lo) < (uint32_t)r.seen ? s[u][e] : -INFINITY;
    }
    float mx = -INFINITY;
#pragma unroll
    for (int u = 0; u < U; ++u) mx = fmaxf(fmaxf(fmaxf(mx, s[u][0]), fmaxf(s[u][1], s[u][2])), s[u][3]);
    mx = column_max<16>(mx);
    // p may grow to 2^8 before the sums are scaled to a new maximum
    if (__any(r.q.f * (mx - r.m) > 8.0f)) {
        const float to = fmaxf(r.m, mx);
        const float by = to == -INFINITY ? 1.0f : __builtin_amdgcn_exp2f(r.q.f * (r.m - to));
        scale_sums(r, by);
        r.l *= by;
        r.m = to;
    }
    const float off = r.m == -INFINITY ? 0.0f : r.q.f * r.m;
#pragma unroll
    for (int u = 0; u < U; ++u) {
        const int key = 16 * (u * F + copy) + 4 * g;
        const f32x4 step = *reinterpret_cast<const f32x4*>(lds + 128 + key);
        const u32x4 with_step = *reinterpret_cast<const u32x4*>(lds + 192 + key);
        float x[4];
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            s[u][e] = __builtin_amdgcn_exp2f(fmaf(r.q.f, s[u][e], -off));
            r.l += s[u][e];
            x[e] = s[u][e] * step[e];
        }
#pragma unroll
        for (int e = 0; e < 2; ++e) {
            p[u][e] = pack_f16(x[2 * e], x[2 * e + 1]);
            r.w = add_centre(p[u][e], with_step[e], add_centre(p[u][e], with_step[2 + e], r.w));
        }
    }
    if (r.far)
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const f32x4 with_p = *reinterpret_cast<const f32x4*>(lds + 256 + 16 * (u * F + copy) + 4 * g);
#pragma unroll
            for (int e = 0; e < 4; ++e) r.w = fmaf(s[u][e], with_p[e], r.w);
        }
}

template <int D, int F>
__device__ __forceinline__ void take_values(Columns<D>& r, const Codes<D>& t, const uint32_t (&p)[4 / F][2], const CodeBits& bits, int copy) {
    const u32x4 less_even{0xe408e408u, 0xe408e408u, 0xe408e408u, 0xe408e408u}, less_odd{0xd480d480u, 0xd480d480u, 0xd480d480u, 0xd480d480u};   // -1032, -72
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        u32x4 b;
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            const int at = 2 * i + h;
#pragma unroll
            for (int e = 0; e < 2; ++e) b[2 * h + e] = F == 1 || copy == at % F ? p[at / F][e] : 0u;
        }
        const f16x8 x = __builtin_bit_cast(f16x8, b);
#define RQ_VALUES(J)                                                                                                            \
    {                                                                                                                           \
        constexpr int h = 2 * ((J) / 4);                                                                                        \
        const u32x4 a{value_pair<(J) % 4>(t.v[2 * i][h], bits), value_pair<(J) % 4>(t.v[2 * i][h + 1], bits),                               \
                      value_pair<(J) % 4>(t.v[2 * i + 1][h], bits), value_pair<(J) % 4>(t.v[2 * i + 1][h + 1], bits)};                      \
        r.o[J] = __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(f16x8, (J) % 2 ? less_odd : less_even), x, r.o[J], 0, 0, 0); \
        r.o[J] = __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(f16x8, a), x, r.o[J], 0, 0, 0);                      \
    }
        RQ_VALUES(0) RQ_VALUES(1) RQ_VALUES(2) RQ_VALUES(3)
        if constexpr (D == 128) { RQ_VALUES(4) RQ_VALUES(5) RQ_VALUES(6) RQ_VALUES(7) }
#undef RQ_VALUES
    }
}

// Shares of the row tiles' keys.  Row tile t has units begin[t] .. begin[t + 1] - 1: kStart for what a row tile costs besides its keys, then
// one for each 64 keys (and one where there are none: its results are zeros).  Worker i of a kv head takes units i * each on.  Its
// share of row tile t is number i + t of the partial results: no two shares have one number.
constexpr int kMostTiles = 1024;                  // row tiles that are shared out
struct Shares {
    int begin[kMostTiles + 1], len[kMostTiles];
    int wave_sum[kWaves];
};
constexpr int kStart = 2 * kWaves, kLeast = kStart + 2 * kWaves;     // kLeast: units of a worker, if there are as many

template <int C>
__device__ __forceinline__ int share_out(const KvJob& job, Shares& s) {
    constexpr int threads = 64 * kWaves;
    const int each = (job.tiles + threads - 1) / threads, lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    int count[kMostTiles / threads], sum = 0;
#pragma unroll
    for (int i = 0; i < kMostTiles / threads; ++i) {
        const int t = (int)threadIdx.x * each + i;
        Place p;
        count[i] = 0;
        if (i < each && t < job.tiles && find_rows<C>(job, t, p)) {
            find_keys<C>(job, p, job.a.kv_lens[p.b]);
            count[i] = kStart + (p.to > p.from ? (p.to - p.from + kTile - 1) / kTile : 1);
            s.len[t] = p.len;
        }
        sum += count[i];
    }
    int before = sum;
#pragma unroll
    for (int w = 1; w < 64; w *= 2) {
        const int x = __shfl_up(before, w);
        if (lane >= w) before += x;
    }
    if (lane == 63) s.wave_sum[wave] = before;
    __syncthreads();
    int at = before - sum;
    for (int w = 0; w < wave; ++w) at += s.wave_sum[w];
#pragma unroll
    for (int i = 0; i < kMostTiles / threads; ++i) {
        const int t = (int)threadIdx.x * each + i;
        if (i < each && t < job.tiles) s.begin[t] = at;
        at += count[i];
    }
    if (threadIdx.x == threads - 1) s.begin[job.tiles] = at;
    __syncthreads();
    const int total = s.begin[job.tiles], per = (total + job.workers - 1) / job.workers;
    return per < kLeast ? kLeast : per;
}

// Partial results: [workers + tiles][kv heads][C rows], D values each; behind them log2 of the sums, then for each row tile the first
// worker that has a share of it and the last one.
template <int D, int C>
__device__ __forceinline__ float* part_sums(const KvJob& job) { return job.part + (int64_t)(job.workers + job.tiles) * job.cache.kv_heads * C * D; }
template <int D, int C>
__device__ __forceinline__ int* part_workers(const KvJob& job) {
    return reinterpret_cast<int*>(part_sums<D, C>(job) + (int64_t)(job.workers + job.tiles) * job.cache.kv_heads * C);
}

// LDS of a workgroup.
template <int D, int W>
struct FewLds {
    __attribute__((aligned(16))) float params[W][kParameters * kTile];
    __attribute__((aligned(16))) float o[W][16][D + 4];
    float l[W][16];
};

// SHARED: workers share the keys out, else a workgroup takes a row tile, or (Part kShared, kOwn) a chunk of its keys.
// number: of the workgroup among those of a kv head.
template <int D, int F, bool F16, bool PAGED, int W, bool SHARED, Part PART>
__device__ __forceinline__ void few_rows(const std::conditional_t<PART == Part::kWhole, KvJob, PrefixJob>& job, int number, FewLds<D, W>& in_lds,
                                         std::conditional_t<SHARED, Shares, int>& shares) {
    static_assert(!SHARED || PART == Part::kWhole, "workers take whole sequences");
    constexpr bool CHUNKED = PART == Part::kShared || PART == Part::kOwn;
    constexpr int C = 16 / F, E = D / 4;          // rows of the workgroup; elements of a row in a lane
    auto& lds_params = in_lds.params;
    auto& lds_o = in_lds.o;
    auto& lds_l = in_lds.l;
    const Kv4Attention& a = job.a;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int copy = (lane & 15) / C, g = lane >> 4;
    const int kv = job.cache.kv_heads, head = blockIdx.x;
    const int head_at = head * ((D + 8) << job.cache.page_shift);    // of the kv head's block in a page
    const CodeBits bits;
    float* lds = lds_params[wave];
    int tile = number, share = 0, share_end = 1;  // SHARED: the workgroup's units
    int chunk = 0;
    if constexpr (CHUNKED) {
        tile = number / job.chunks;
        chunk = number - tile * job.chunks;
        tile += job.first_tile;
    }
    if constexpr (SHARED) {
        const int each = share_out<C>(job, shares);
        share = number * each;
        share_end = share + each < shares.begin[job.tiles] ? share + each : shares.begin[job.tiles];
        if (number == 0 && head == 0)
            for (int t = threadIdx.x; t < job.tiles; t += 64 * W) {
                const int begin = shares.begin[t], end = shares.begin[t + 1];
                int* w = part_workers<D, C>(job) + 2 * t;
                w[0] = end > begin ? (begin + kStart) / each : 0;
                w[1] = end > begin ? (end - 1) / each : 0;
            }
        if (share >= share_end) return;           // (also of workers that only fill the grid)
        int lo = 0, hi = job.tiles - 1;           // the last row tile that begins at or before the share
        while (lo < hi) {
            const int at = (lo + hi + 1) >> 1;
            if (shares.begin[at] <= share) lo = at; else hi = at - 1;
        }
        tile = lo;
    }
    // row tile by row tile; not SHARED: just the one
    for (; tile < job.tiles; ++tile) {
        Place at;
        int first = 0, count = 0;                 // of the row tile's tiles of 64 keys: those of this workgroup
        bool all = true;                          // it has all of them
        tile = __builtin_amdgcn_readfirstlane(tile);
        if constexpr (SHARED) {
            const int begin = shares.begin[tile], end = shares.begin[tile + 1], keys = begin + kStart;
            if (begin >= share_end) break;
            if (end == begin || share_end <= keys) continue;         // none of its keys
            first = share > keys ? share - keys : 0;
            count = (share_end < end ? share_end : end) - keys - first;
            all = count == end - keys;
        }
        if constexpr (PART == Part::kShared) {
            if (!find_group_rows<C>(job, tile, at)) return;
        } else {
            if (!find_rows<C>(job, tile, at)) return;                // (SHARED: such a tile has no units)
        }
        if constexpr (CHUNKED)
            if (!in_slice(job, at)) return;
        const int rows = at.nq * job.group, n = at.base + (lane & 15) % C;
        const bool there = n < rows;
        const int token = there ? token_of(job, at, n) : 0;
        // everything that does not depend on the length is asked for before it is known
        int len;
        if constexpr (SHARED) len = shares.len[tile];
        else if constexpr (PART == Part::kShared) len = prefix_len(job, at.b);
        else len = a.kv_lens[at.b];
        const RawQuery<D, 16> raw = load_query<D, 16>(job, there, at.q0 + token, head * job.group + (there ? n - token * job.group : 0), lane);
        const int32_t* table = a.table + (int64_t)at.b * a.width;
        int width = a.width;
        if constexpr (PART == Part::kShared) {
            width = job.p.width;
            table = job.p.table + (int64_t)at.b * width;
        }
        const int shift = job.cache.page_shift;
        constexpr int stride = W * kTile;
        int pages = 0, number_of = 0;             // of the tile in hand: number among those of `pages`
        if (PART != Part::kSeparate && a.window == 0 && width > 0)
            pages = load_pages<PAGED>(job.cache, table, width, (CHUNKED ? chunk * job.chunk : first * kTile) + wave * kTile, stride, lane);
        if constexpr (PART == Part::kShared) {
            at.len = len;
            at.from = 0;
            at.to = len;
        } else {
            find_keys<C>(job, at, len);
        }
        int from = at.from, to = at.to;
        if constexpr (SHARED) {
            from += first * kTile;
            if (to > from + count * kTile) to = from + count * kTile;
        }
        if constexpr (CHUNKED) {
            from += chunk * job.chunk;
            if (to > from + job.chunk) to = from + job.chunk;
        }
        // kSeparate: positions count from the end of the prefix; those of the prefix itself come first
        int behind = 0, own_from = 0, own_to = 0;
        [[maybe_unused]] const int32_t* own_table = table;
        if constexpr (PART == Part::kSeparate) {
            const int g = group_of(job, at.b), last = (at.base + C < rows ? at.base + C : rows) - 1;
            behind = prefix_len(job, g);
            own_from = from;
            own_to = to;
            const int p0 = behind + at.len - at.nq + token_of(job, at, at.base), p1 = behind + at.len - at.nq + token_of(job, at, last);
            from = a.window && p0 - a.window + 1 > 0 ? (p0 - a.window + 1) & ~(kTile - 1) : 0;
            to = a.causal && p1 + 1 < behind ? p1 + 1 : behind;
            width = job.p.width;
            table = job.p.table + (int64_t)g * width;
        }
        int k0 = from + wave * kTile;             // the tile in hand
        Codes<D> t;
        const auto begin = [&] {
            if (k0 < to) {
                if (PART == Part::kSeparate || a.window) pages = load_pages<PAGED>(job.cache, table, width, k0, stride, lane);
                number_of = 0;
                const Source<PAGED> s = find_tile<PAGED>(job.cache, pages, 0, head_at, k0);
                load_keys<D>(t, s, shift, lane);
                load_values<D>(t, s, shift, lane);
            }
        };
        begin();
        Columns<D> r;
        take_query<D, 16, F16, F16>(r.q, job, raw, lane);
        r.sum = r.q.even + r.q.odd;
        r.bias = -(1024.0f + 7.5f) * r.q.even - (64.0f + 7.5f) * r.q.odd;
        int all_lo, all_hi;                       // keys that all rows see
        // of the first `len` positions, `behind` of them before position 0 of the sequence
        const auto see = [&](int behind, int len) {
            int pos = behind + at.len - at.nq + token;               // the row's position in its sequence
            if constexpr (PART == Part::kShared) pos = there ? len + own_position(job, at.q0 + token) : 0;
            const int hi = !there ? 0 : a.causal ? (pos + 1 < len ? pos + 1 : len) : len;
            r.lo = a.window ? (pos - a.window + 1 > 0 ? pos - a.window + 1 : 0) : 0;
            r.seen = hi > r.lo ? hi - r.lo : 0;
            if constexpr (PART == Part::kShared) {                   // (rows of several sequences: none or all of the masks)
                const bool some = __any(there && hi < len);
                all_lo = 0;
                all_hi = some ? 0 : to;
            } else {
                const int last = (at.base + C < rows ? at.base + C : rows) - 1;
                const int p0 = behind + at.len - at.nq + token_of(job, at, at.base), p1 = behind + at.len - at.nq + token_of(job, at, last);
                all_lo = a.window ? p1 - a.window + 1 : 0;
                all_hi = a.causal && p0 + 1 < to ? p0 + 1 : to;
            }
        };
        see(behind, PART == Part::kSeparate ? behind : at.len);
        r.m = -INFINITY;
        r.l = r.w = r.limit = 0.0f;
        r.factor = 1.0f;
#pragma unroll
        for (int j = 0; j < D / 16; ++j) r.o[j] = f32x4{0, 0, 0, 0};
        // (the last tile by itself: where loads may be left out, all that was loaded before them is waited for)
        const auto step = [&](auto more) {
            const int next = k0 + stride;
            Source<PAGED> s;
            if constexpr (more) {
                if (++number_of == kPagesOf<PAGED>) {
                    pages = load_pages<PAGED>(job.cache, table, width, next, stride, lane);
                    number_of = 0;
                }
                s = find_tile<PAGED>(job.cache, pages, number_of, head_at, next);
            }
            take_parameters<D>(r, t, lds, k0 + lane < to, lane);
            f32x4 x[4 / F];
            take_keys<D, F, F16>(x, r, t, bits, copy);
            if constexpr (more) load_keys<D>(t, s, shift, lane);
            uint32_t p[4 / F][2];
            take_scores<D, F>(p, r, x, lds, k0, k0 >= all_lo && k0 + kTile <= all_hi, copy, g);
            take_values<D, F>(r, t, p, bits, copy);
            if constexpr (more) load_values<D>(t, s, shift, lane);
            k0 = next;
        };
        while (k0 + stride < to) step(std::true_type{});
        if (k0 < to) step(std::false_type{});
        if constexpr (PART == Part::kSeparate) {
            table = own_table;
            width = a.width;
            to = own_to;
            k0 = own_from + wave * kTile;
            begin();
            see(0, at.len);
            while (k0 + stride < to) step(std::true_type{});
            if (k0 < to) step(std::false_type{});
        }
        // a column's results: normalised, with log2 of the sum of e^(scale q.k)
        {
            const float l = column_sum<16>(r.l), w = column_sum<16>(r.w);
            const float by = (l > 0.0f ? 1.0f / l : (l == 0.0f ? 0.0f : l)) / r.factor;
            float* o = lds_o[wave][lane & 15] + E * g;
#pragma unroll
            for (int e = 0; e < 4; ++e)
#pragma unroll
                for (int j = 0; j < D / 16; j += 4)
                    *reinterpret_cast<f32x4*>(o + e * (D / 16) + j) =
                        f32x4{(r.o[j][e] + w) * by, (r.o[j + 1][e] + w) * by, (r.o[j + 2][e] + w) * by, (r.o[j + 3][e] + w) * by};
            if (lane < 16) lds_l[wave][lane] = l == 0.0f ? -INFINITY : fmaf(r.q.f, r.m, __builtin_amdgcn_logf(l));
        }
        // the waves' columns, and the copies among them, join in LDS
        __syncthreads();
        constexpr int per = C * D / (64 * W) > 0 ? C * D / (64 * W) : 1;  // results of a thread
        const int mine = threadIdx.x * per / D, d = threadIdx.x * per % D;
        if (mine < C && at.base + mine < rows) {
            float top = -INFINITY, sum = 0.0f, z[per] = {};
#pragma unroll
            for (int w = 0; w < W; ++w)
#pragma unroll
                for (int f = 0; f < F; ++f) top = fmaxf(top, lds_l[w][f * C + mine]);
#pragma unroll
            for (int w = 0; w < W; ++w)
#pragma unroll
                for (int f = 0; f < F; ++f) {
                    const float l = lds_l[w][f * C + mine];
                    const float by = l == -INFINITY ? 0.0f : __builtin_amdgcn_exp2f(l - top);        // (NaN goes on)
                    sum += by;
#pragma unroll
                    for (int e = 0; e < per; ++e) z[e] = fmaf(by, lds_o[w][f * C + mine][d + e], z[e]);
                }
            const float by = sum == 0.0f ? 0.0f : 1.0f / sum;
#pragma unroll
            for (int e = 0; e < per; ++e) z[e] *= by;
            const float total = top + __builtin_amdgcn_logf(sum);
            if constexpr (CHUNKED) {
                const int token_m = token_of(job, at, at.base + mine), h = head * job.group + at.base + mine - token_m * job.group, t = at.q0 + token_m;
                const int64_t rows_all = (int64_t)(job.slice_end - job.slice) * a.heads, part = (job.part_first + chunk) * rows_all + (int64_t)(t - job.slice) * a.heads + h;
                if (t >= job.slice && t < job.slice_end) {
                    float* o = job.part + part * D + d;
#pragma unroll
                    for (int e = 0; e < per; ++e) o[e] = z[e];
                    if (d == 0) job.part[job.part_chunks * rows_all * D + part] = total;
                }
            } else if (SHARED && !all) {
                const int64_t slot = ((int64_t)(number + tile) * kv + head) * C + mine;
                float* o = job.part + slot * D + d;
#pragma unroll
                for (int e = 0; e < per; ++e) o[e] = z[e];
                if (d == 0) part_sums<D, C>(job)[slot] = total;
            } else {
                const int token_m = token_of(job, at, at.base + mine), h = head * job.group + at.base + mine - token_m * job.group;
                store_row<per, F16>(static_cast<uint16_t*>(a.o) + (int64_t)(at.q0 + token_m) * a.o_token + (int64_t)h * a.o_head + d, z, job.wide_o);
                if (d == 0 && a.lse) a.lse[(int64_t)(at.q0 + token_m) * a.heads + h] = total * kLn2;
            }
        }
        if constexpr (!SHARED) return;
        __syncthreads();                          // (LDS is written again)
    }
}

template <int D, int F, bool F16, bool PAGED, int W, bool SHARED>
__global__ __launch_bounds__(64 * W, 2) void k_kv4_attention(KvJob job) {
    __shared__ FewLds<D, W> lds;
    __shared__ std::conditional_t<SHARED, Shares, int> shares;
    few_rows<D, F, F16, PAGED, W, SHARED, Part::kWhole>(job, item_number(), lds, shares);
}

}  // namespace
}  // namespace rq
