// Attention over the 4-bit paged cache (kv4_layout.h): o_i = sum_j p_ij v_j / sum_j p_ij, p_ij = exp(scale q_i . k_j - m_i).
//
// With k_jd = (c_jd - 7.5) step_j + mid_j the scores are  q_i . k_j = step_j (q_i . c_j - 7.5 sum q_i) + mid_j sum q_i:  the codes
// themselves are an operand of the matrix cores and a key's step and centre are applied once a score, not once an element.  The
// values' side is alike: with p'_ij = p_ij step_j,  o_i = sum_j p'_ij (c_jd - 8) + sum_j p_ij (mid_j + step_j / 2).
//   - A code becomes an fp16 number by masking it into the mantissa of 1024 or 64: two codes an instruction.  For keys the constants'
//     share of a score is known, sum q_i times the constant, and taken off in the accumulator's initial value; for values, whose
//     sums run over all keys and would lose digits to it, one more instruction takes it off the codes.
//   - The query row is scaled by a power of two to at most 1 and rounded to fp16 (2^-12; bf16 would move a score of 10 by 0.02).
//     p' is rounded to fp16 too (bf16 would leave 1.4e-3 of error in outputs that fp16 holds to 2e-4): p carries a power of two that
//     brings the largest step seen so far to 2^7, so that p' neither overflows nor, down to 2^-21 of the largest, loses
//     digits.  Everything else is fp32.
//
// A wave holds 16 R query rows and walks over the keys in tiles of 64.  Products are taken transposed, keys x queries and
// elements x queries, so that a query is a column, column n the lanes n, n + 16, n + 32, n + 48: scores leave the matrix
// cores in the lanes in which p' enters them again (keys in an order of their own, which the values follow), and maxima, sums and
// factors of a query stay in its lanes.  The parameters of a tile's keys, a key a lane, go to the lanes of its rows through LDS.
// Rows are the queries of all heads that share a kv head, token by token.
#include "kv4_layout.h"
#include "wave_common.h"

namespace rq {
namespace {

constexpr int kTile = 64;                         // keys a step
constexpr int kWaves = 4;
constexpr float kLog2e = 1.4426950408889634f, kLn2 = 0.6931471805599453f;

struct Job {
    Kv4 cache;
    Kv4Attention a;
    int group;                                    // query heads of a kv head
    int tiles;                                    // row tiles (bound)
    int chunk, chunks;                            // keys of a chunk, chunks (bound)
    bool wide_q, wide_o;                          // rows of q, of o begin on 16 bytes
    float* part;                                  // [chunks][tokens][heads][D], then [chunks][tokens][heads] log2 of the sums
};

__device__ __forceinline__ uint32_t pack16(float x, float y, bool f16) {
    return f16 ? (uint32_t)__builtin_bit_cast(uint16_t, (_Float16)x) | ((uint32_t)__builtin_bit_cast(uint16_t, (_Float16)y) << 16)
               : (uint32_t)__builtin_bit_cast(uint16_t, (__bf16)x) | ((uint32_t)__builtin_bit_cast(uint16_t, (__bf16)y) << 16);
}
__device__ __forceinline__ uint32_t and_or(uint32_t x, uint32_t mask, uint32_t bits) { return (x & mask) | bits; }

// Eight key codes as fp16: elements (0, 4), (1, 5), (2, 6), (3, 7) of the dword, 1024 + c in the even ones, 64 + c in the odd ones.
__device__ __forceinline__ f16x8 key_operand(uint32_t w) {
    const uint32_t h = w >> 8;
    const u32x4 x{and_or(w, 0x000f000fu, 0x64006400u), and_or(w, 0x00f000f0u, 0x54005400u), and_or(h, 0x000f000fu, 0x64006400u),
                  and_or(h, 0x00f000f0u, 0x54005400u)};
    return __builtin_bit_cast(f16x8, x);
}
// c - 8 of nibble J of both halves of a dword, as fp16.
template <int J>
__device__ __forceinline__ uint32_t value_pair(uint32_t w) {
    typedef _Float16 f16x2 __attribute__((ext_vector_type(2)));
    const uint32_t x = J % 2 ? and_or(J / 2 ? w >> 8 : w, 0x00f000f0u, 0x54005400u) : and_or(J / 2 ? w >> 8 : w, 0x000f000fu, 0x64006400u);
    const _Float16 off = J % 2 ? (_Float16)-72.0f : (_Float16)-1032.0f;
    return __builtin_bit_cast(uint32_t, __builtin_bit_cast(f16x2, x) + f16x2{off, off});
}

__device__ __forceinline__ float column_sum(float x) {
    x += __shfl_xor(x, 16);
    return x + __shfl_xor(x, 32);
}
__device__ __forceinline__ float column_max(float x) {
    x = fmaxf(x, __shfl_xor(x, 16));
    return fmaxf(x, __shfl_xor(x, 32));
}

// A tile's codes as they are stored, and its keys' parameters, a key a lane.
template <int D>
struct Codes {
    uint32_t k[4][D / 32], v[4][D / 32];          // [16 keys][dword]
    uint32_t kp, vp;
};

template <int D>
__device__ __forceinline__ Codes<D> load_tile(const Kv4& c, const int32_t* table, int head, int k0, int end, int lane) {
    typedef uint32_t words __attribute__((ext_vector_type(D / 32)));
    const int shift = c.page_shift, p = 1 << shift;
    Codes<D> t;
    const uint8_t* mine = nullptr;
    int mine_at = 0;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        int key = k0 + 16 * i;
        if (key >= end) key = (end - 1) & ~15;    // (those keys are masked)
        int page = table[key >> shift];
        if ((uint32_t)page >= (uint64_t)c.pages) page = 0;
        const uint8_t* block = c.data + (int64_t)page * c.page_bytes + (int64_t)head * (p * (D + 8));
        const int at = key & (p - 1);
        const words k = *reinterpret_cast<const words*>(block + at * (D / 2) + (lane & 15) * (D / 2) + (lane >> 4) * (D / 8));
        const words v = *reinterpret_cast<const words*>(block + (p + at) * (D / 2) + (lane >> 4) * (2 * D) + (lane & 15) * (D / 8));
#pragma unroll
        for (int j = 0; j < D / 32; ++j) t.k[i][j] = k[j], t.v[i][j] = v[j];
        if (lane >> 4 == i) {
            mine = block + p * D;
            mine_at = at + (lane & 15);
        }
    }
    const uint32_t* w = reinterpret_cast<const uint32_t*>(mine) + mine_at;
    t.kp = w[0];
    t.vp = w[p];
    return t;
}

// The queries of a wave, and what it has summed up.
template <int D, int R>
struct Rows {
    f16x8 q[R][D / 32];
    float sum[R], bias[R], f[R];                  // sum of q, what the accumulator starts from, log2 of e^(scale q.k) per unit
    int lo[R], hi[R];                             // keys that the row sees
    float m[R], l[R], w[R];                       // running maximum; sums over the lane's keys of p and p * (mid + step / 2)
    f32x4 o[R][D / 16];
    float limit, up;                              // a power of two that no step seen so far exceeds; log2 of the factor in p
};

// All sums times a factor of the row.
template <int D, int R>
__device__ __forceinline__ void scale_sums(Rows<D, R>& r, int n, float by) {
    r.l[n] *= by;
    r.w[n] *= by;
#pragma unroll
    for (int j = 0; j < D / 16; ++j)
#pragma unroll
        for (int e = 0; e < 4; ++e) r.o[n][j][e] *= by;
}

template <int D, int R, bool MASKED>
__device__ __forceinline__ void take_tile(Rows<D, R>& r, const Codes<D>& t, float* lds, int k0, int end, int lane) {
    const int g = lane >> 4;
    {
        const bool there = k0 + lane < end;
        const uint32_t kp = !MASKED || there ? t.kp : 0u, vp = !MASKED || there ? t.vp : 0u;
        lds[lane] = __uint_as_float(kp << 16);
        lds[64 + lane] = __uint_as_float(kp & 0xffff0000u);
        const float step = __uint_as_float(vp << 16);
        lds[128 + lane] = step;
        lds[192 + lane] = fmaf(0.5f, step, __uint_as_float(vp & 0xffff0000u));
        if (__any(step > r.limit && step < 0x1p127f)) {              // (NaN and infinity do not count)
            float most = step < 0x1p127f ? step : 0.0f;
#pragma unroll
            for (int w = 1; w < 64; w *= 2) most = fmaxf(most, __shfl_xor(most, w));
            const int x = (int)(__float_as_uint(most) >> 23) - 126;  // most < 2^x
            const float limit = __uint_as_float((uint32_t)((x < -60 ? -60 : x > 127 ? 127 : x) + 127) << 23);
            if (limit > r.limit) {
                const int up = 134 - (int)(__float_as_uint(limit) >> 23);
                const float by = __builtin_amdgcn_ldexpf(1.0f, up - (int)r.up);
#pragma unroll
                for (int n = 0; n < R; ++n) scale_sums(r, n, by);
                r.limit = limit;
                r.up = (float)up;
            }
        }
    }
    float s[R][16];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        f32x4 acc[R];
#pragma unroll
        for (int n = 0; n < R; ++n) acc[n] = f32x4{r.bias[n], r.bias[n], r.bias[n], r.bias[n]};
#pragma unroll
        for (int j = 0; j < D / 32; ++j) {
            const f16x8 a = key_operand(t.k[i][j]);
#pragma unroll
            for (int n = 0; n < R; ++n) acc[n] = __builtin_amdgcn_mfma_f32_16x16x32_f16(a, r.q[n][j], acc[n], 0, 0, 0);
        }
        const f32x4 step = *reinterpret_cast<const f32x4*>(lds + 16 * i + 4 * g), mid = *reinterpret_cast<const f32x4*>(lds + 64 + 16 * i + 4 * g);
#pragma unroll
        for (int n = 0; n < R; ++n)
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                float x = fmaf(step[e], acc[n][e], mid[e] * r.sum[n]);
                if constexpr (MASKED) {
                    const int key = k0 + 16 * i + 4 * g + e;
                    x = key >= r.lo[n] && key < r.hi[n] ? x : -INFINITY;
                }
                s[n][4 * i + e] = x;
            }
    }
#pragma unroll
    for (int n = 0; n < R; ++n) {
        float mx = s[n][0];
#pragma unroll
        for (int e = 1; e < 16; ++e) mx = fmaxf(mx, s[n][e]);
        mx = column_max(mx);
        // p may grow to 2^8 before the sums are scaled to a new maximum
        if (__any(r.f[n] * (mx - r.m[n]) > 8.0f)) {
            const float to = fmaxf(r.m[n], mx);
            const float by = to == -INFINITY ? 1.0f : __builtin_amdgcn_exp2f(r.f[n] * (r.m[n] - to));
            r.m[n] = to;
            scale_sums(r, n, by);
        }
    }
    u32x4 p[R][2];
#pragma unroll
    for (int n = 0; n < R; ++n) {
        const float off = (r.m[n] == -INFINITY ? 0.0f : r.f[n] * r.m[n]) - r.up;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const f32x4 step = *reinterpret_cast<const f32x4*>(lds + 128 + 16 * i + 4 * g);
            const f32x4 mid = *reinterpret_cast<const f32x4*>(lds + 192 + 16 * i + 4 * g);
            float x[4];
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const float y = __builtin_amdgcn_exp2f(fmaf(r.f[n], s[n][4 * i + e], -off));
                r.l[n] += y;
                if constexpr (MASKED) {           // a masked key's parameters may be infinite or NaN
                    const bool seen = s[n][4 * i + e] != -INFINITY;
                    x[e] = seen ? y * step[e] : 0.0f;
                    r.w[n] += seen ? y * mid[e] : 0.0f;
                } else {
                    x[e] = y * step[e];
                    r.w[n] = fmaf(y, mid[e], r.w[n]);
                }
            }
#pragma unroll
            for (int e = 0; e < 2; ++e)
                p[n][i / 2][2 * (i % 2) + e] = pack16(x[2 * e], x[2 * e + 1], true);
        }
    }
#pragma unroll
    for (int i = 0; i < 2; ++i) {
#define RQ_VALUES(J)                                                                                                            \
    {                                                                                                                           \
        constexpr int h = 2 * ((J) / 4);                                                                                        \
        const u32x4 a{value_pair<(J) % 4>(t.v[2 * i][h]), value_pair<(J) % 4>(t.v[2 * i][h + 1]),                               \
                      value_pair<(J) % 4>(t.v[2 * i + 1][h]), value_pair<(J) % 4>(t.v[2 * i + 1][h + 1])};                      \
        _Pragma("unroll") for (int n = 0; n < R; ++n) r.o[n][J] = __builtin_amdgcn_mfma_f32_16x16x32_f16(                        \
            __builtin_bit_cast(f16x8, a), __builtin_bit_cast(f16x8, p[n][i]), r.o[n][J], 0, 0, 0);                              \
    }
        RQ_VALUES(0) RQ_VALUES(1) RQ_VALUES(2) RQ_VALUES(3)
        if constexpr (D == 128) { RQ_VALUES(4) RQ_VALUES(5) RQ_VALUES(6) RQ_VALUES(7) }
#undef RQ_VALUES
    }
}

// The 16 R rows from `row` on of a sequence's rows at a kv head (`rows` of them), rotated, scaled and rounded.
template <int D, int R, bool F16>
__device__ __forceinline__ void load_rows(Rows<D, R>& r, const Job& job, int head, int row, int rows, int q0, int nq, int len, int lane) {
    const Kv4Attention& a = job.a;
    constexpr int E = D / 4;                      // elements of a row in a lane
#pragma unroll
    for (int n = 0; n < R; ++n) {
        const int mine = row + 16 * n + (lane & 15);
        const bool there = mine < rows;
        const int token = there ? mine / job.group : 0, of = there ? mine - token * job.group : 0;
        const uint16_t* x = static_cast<const uint16_t*>(a.q) + (int64_t)(q0 + token) * a.q_token + (int64_t)(head * job.group + of) * a.q_head + E * (lane >> 4);
        u32x4 raw[E / 8] = {};
        if (there) {
            if (job.wide_q) {
#pragma unroll
                for (int e = 0; e < E / 8; ++e) raw[e] = reinterpret_cast<const u32x4*>(x)[e];
            } else {
#pragma unroll
                for (int e = 0; e < E; e += 2) raw[e / 8][e / 2 % 4] = (uint32_t)x[e] | ((uint32_t)x[e + 1] << 16);
            }
        }
        float q[E];
#pragma unroll
        for (int e = 0; e < E; ++e) {
            const uint32_t u = raw[e / 8][e / 2 % 4];
            q[e] = F16 ? (float)__builtin_bit_cast(_Float16, (uint16_t)(e % 2 ? u >> 16 : u)) : __uint_as_float(e % 2 ? u & 0xffff0000u : u << 16);
        }
        if (a.rotate) {
#pragma unroll
            for (int w = 1; w < E; w *= 2)
#pragma unroll
                for (int e = 0; e < E; ++e)
                    if (!(e & w)) {
                        const float y = q[e], z = q[e + w];
                        q[e] = y + z;
                        q[e + w] = y - z;
                    }
#pragma unroll
            for (int w = 16; w < 64; w *= 2)
#pragma unroll
                for (int e = 0; e < E; ++e) {
                    const float z = __shfl_xor(q[e], w);
                    q[e] = lane & w ? z - q[e] : z + q[e];
                }
        }
        float most = 0.0f;
#pragma unroll
        for (int e = 0; e < E; ++e) most = fmaxf(most, fabsf(q[e]));
        most = column_max(most);
        // 2^-x with most < 2^x: 1 for rows of zeros; infinite rows stay what they are
        int x2 = (int)((__float_as_uint(most) >> 23) & 255) - 126;
        x2 = most == 0.0f || x2 > 128 ? 0 : x2 < -100 ? -100 : x2;
        const float by = __uint_as_float((uint32_t)(127 - (x2 > 126 ? 126 : x2)) << 23);
        r.f[n] = a.scale * kLog2e * (a.rotate ? (D == 128 ? 0.08838834764831845f : 0.125f) : 1.0f) / by;
        float even = 0.0f, odd = 0.0f;
#pragma unroll
        for (int j = 0; j < D / 32; ++j)
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                const _Float16 v = (_Float16)(q[8 * j + e / 2 + 4 * (e % 2)] * by);
                r.q[n][j][e] = v;
                (e / 2 % 2 ? odd : even) += (float)v;
            }
        even = column_sum(even);
        odd = column_sum(odd);
        r.sum[n] = even + odd;
        r.bias[n] = -(1024.0f + 7.5f) * even - (64.0f + 7.5f) * odd;
        const int pos = len - nq + token;         // the row's position in its sequence
        r.hi[n] = !there ? 0 : a.causal ? (pos + 1 < len ? pos + 1 : len) : len;
        r.lo[n] = a.window ? (pos - a.window + 1 > 0 ? pos - a.window + 1 : 0) : 0;
        r.m[n] = -INFINITY;
        r.l[n] = r.w[n] = 0.0f;
#pragma unroll
        for (int j = 0; j < D / 16; ++j) r.o[n][j] = f32x4{0, 0, 0, 0};
    }
}

// N consecutive results of a row.
template <int N, bool F16>
__device__ __forceinline__ void store_row(uint16_t* o, const float (&y)[N], bool wide) {
    uint32_t w[N / 2];
#pragma unroll
    for (int e = 0; e < N / 2; ++e) w[e] = pack16(y[2 * e], y[2 * e + 1], F16);
    if (wide) {
        if constexpr (N % 8 == 0) {
#pragma unroll
            for (int e = 0; e < N / 8; ++e) reinterpret_cast<u32x4*>(o)[e] = u32x4{w[4 * e], w[4 * e + 1], w[4 * e + 2], w[4 * e + 3]};
        } else {
#pragma unroll
            for (int e = 0; e < N / 4; ++e) reinterpret_cast<u32x2*>(o)[e] = u32x2{w[2 * e], w[2 * e + 1]};
        }
    } else {
#pragma unroll
        for (int e = 0; e < N / 2; ++e) {
            o[2 * e] = (uint16_t)w[e];
            o[2 * e + 1] = (uint16_t)(w[e] >> 16);
        }
    }
}

// SPLIT: the waves of a workgroup share 16 R rows and take the tiles in turn; else each has 16 R rows of its own.
template <int D, int R, bool F16, bool SPLIT>
__global__ __launch_bounds__(64 * kWaves) void k_kv4_attention(Job job) {
    constexpr int BM = SPLIT ? 16 * R : 16 * R * kWaves, E = D / 4;
    __shared__ __attribute__((aligned(16))) float lds_params[kWaves][4 * kTile];
    const Kv4Attention& a = job.a;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int64_t item = group_index();
    const int kv = job.cache.kv_heads;
    const int64_t tc = item / kv;
    const int head = (int)(item - tc * kv);
    const int tile_no = (int)(tc / job.chunks), chunk = (int)(tc - (int64_t)tile_no * job.chunks);
    if (tile_no >= job.tiles) return;
    const int tile = job.tiles - 1 - tile_no;     // the last rows of a causal prompt see most: they begin first
    // the sequence: its tiles begin at floor(q_start * group / BM) + its number
    int b = 0, q0 = 0, nq = 1, first = 0;
    if (a.q_start) {
        int lo = 0, hi = a.batch - 1;
        while (lo < hi) {
            const int at = (lo + hi + 1) >> 1;
            if ((int)((int64_t)a.q_start[at] * job.group / BM) + at <= tile) lo = at; else hi = at - 1;
        }
        b = lo;
        q0 = a.q_start[b];
        int q1 = a.q_start[b + 1];
        q0 = q0 < 0 ? 0 : q0 > a.tokens ? a.tokens : q0;
        q1 = q1 < q0 ? q0 : q1 > a.tokens ? a.tokens : q1;
        nq = q1 - q0;
        first = (int)((int64_t)q0 * job.group / BM) + b;
    } else {
        const int each = (job.group + BM - 1) / BM;
        b = tile / each;
        q0 = b;
        first = b * each;
    }
    const int rows = nq * job.group, base = (tile - first) * BM;
    if (base < 0 || base >= rows) return;
    int len = a.kv_lens[b];
    const int64_t most = (int64_t)a.width << job.cache.page_shift;
    len = len < 0 ? 0 : len > most ? (int)most : len;
    if (len > a.max_len) len = (int)a.max_len;

    Rows<D, R> r;
    r.limit = r.up = 0.0f;
    const int row = base + (SPLIT ? 0 : wave * 16 * R);
    load_rows<D, R, F16>(r, job, head, row, rows, q0, nq, len, lane);

    // the keys that the workgroup's rows see, and the chunk's and the wave's share of them
    int from, to;
    {
        const int last_row = (base + BM < rows ? base + BM : rows) - 1;
        const int p0 = len - nq + base / job.group, p1 = len - nq + last_row / job.group;
        from = a.window ? p0 - a.window + 1 : 0;
        from = (from < 0 ? 0 : from) & ~(kTile - 1);
        to = a.causal && p1 + 1 < len ? p1 + 1 : len;
    }
    from += chunk * job.chunk;
    if (to > from + job.chunk) to = from + job.chunk;
    const int32_t* table = a.table + (int64_t)b * a.width;
    // keys that all rows of the wave see need no mask
    int all_lo = 0, all_hi, my_to = to;
    {
        const int w_rows = SPLIT ? BM : 16 * R;
        const int last_row = (row + w_rows < rows ? row + w_rows : rows) - 1;
        const int p0 = len - nq + row / job.group, p1 = len - nq + (last_row < 0 ? 0 : last_row) / job.group;
        all_lo = a.window ? p1 - a.window + 1 : 0;
        all_hi = a.causal && p0 + 1 < len ? p0 + 1 : len;
        if (row >= rows) my_to = from;
        else if (a.causal && p1 + 1 < my_to) my_to = p1 + 1;
    }
    float* lds = lds_params[wave];
    constexpr int step = SPLIT ? kWaves * kTile : kTile;
    int k0 = from + (SPLIT ? wave * kTile : 0);
    if (k0 < my_to) {
        Codes<D> t = load_tile<D>(job.cache, table, head, k0, my_to, lane);
        while (true) {
            const int next = k0 + step;
            Codes<D> n;
            if (next < my_to) n = load_tile<D>(job.cache, table, head, next, my_to, lane);
            if (k0 >= all_lo && k0 + kTile <= (all_hi < my_to ? all_hi : my_to)) take_tile<D, R, false>(r, t, lds, k0, my_to, lane);
            else take_tile<D, R, true>(r, t, lds, k0, my_to, lane);
            if (next >= my_to) break;
            t = n;
            k0 = next;
        }
    }
    // a row's results: normalised, with log2 of the sum of e^(scale q.k)
    float lse[R];
#pragma unroll
    for (int n = 0; n < R; ++n) {
        const float l = column_sum(r.l[n]), w = column_sum(r.w[n]);
        const float by = l > 0.0f ? 1.0f / l : (l == 0.0f ? 0.0f : l);
        lse[n] = l == 0.0f ? -INFINITY : fmaf(r.f[n], r.m[n], __builtin_amdgcn_logf(l)) - r.up;
#pragma unroll
        for (int j = 0; j < D / 16; ++j)
#pragma unroll
            for (int e = 0; e < 4; ++e) r.o[n][j][e] = (r.o[n][j][e] + w) * by;
    }
    if constexpr (SPLIT) {
        // the four waves' results join in LDS
        __shared__ __attribute__((aligned(16))) float lds_o[kWaves][R][16][D + 4];
        __shared__ float lds_l[kWaves][R][16];
#pragma unroll
        for (int n = 0; n < R; ++n) {
            float* o = lds_o[wave][n][lane & 15] + E * (lane >> 4);
#pragma unroll
            for (int e = 0; e < 4; ++e)
#pragma unroll
                for (int j = 0; j < D / 16; j += 4)
                    *reinterpret_cast<f32x4*>(o + e * (D / 16) + j) = f32x4{r.o[n][j][e], r.o[n][j + 1][e], r.o[n][j + 2][e], r.o[n][j + 3][e]};
            if (lane < 16) lds_l[wave][n][lane] = lse[n];
        }
        __syncthreads();
        constexpr int per = 16 * R * D / (64 * kWaves);              // outputs of a thread
        const int at = threadIdx.x * per, mine = at / D, d = at % D;
        if (base + mine >= rows) return;
        float lw[kWaves], top = -INFINITY;
#pragma unroll
        for (int w = 0; w < kWaves; ++w) {
            lw[w] = lds_l[w][mine / 16][mine % 16];
            top = fmaxf(top, lw[w]);
        }
        float all = 0.0f;
#pragma unroll
        for (int w = 0; w < kWaves; ++w) {
            lw[w] = lw[w] == -INFINITY ? 0.0f : __builtin_amdgcn_exp2f(lw[w] - top);      // (NaN goes on)
            all += lw[w];
        }
        float y[per];
#pragma unroll
        for (int e = 0; e < per; ++e) {
            float sum = 0.0f;
#pragma unroll
            for (int w = 0; w < kWaves; ++w) sum = fmaf(lw[w], lds_o[w][mine / 16][mine % 16][d + e], sum);
            y[e] = all == 0.0f ? 0.0f : sum / all;
        }
        const float total = top + __builtin_amdgcn_logf(all);
        const int token = q0 + (base + mine) / job.group, h = head * job.group + (base + mine) % job.group;
        if (job.chunks > 1) {
            const int64_t at_row = ((int64_t)chunk * a.tokens + token) * a.heads + h;
            float* o = job.part + at_row * D + d;
#pragma unroll
            for (int e = 0; e < per; e += 4) *reinterpret_cast<f32x4*>(o + e) = f32x4{y[e], y[e + 1], y[e + 2], y[e + 3]};
            if (d == 0) job.part[(int64_t)job.chunks * a.tokens * a.heads * D + at_row] = total;
        } else {
            uint16_t* o = static_cast<uint16_t*>(a.o) + (int64_t)token * a.o_token + (int64_t)h * a.o_head + d;
            store_row<per, F16>(o, y, job.wide_o);
            if (d == 0 && a.lse) a.lse[(int64_t)token * a.heads + h] = total * kLn2;
        }
    } else {
#pragma unroll
        for (int n = 0; n < R; ++n) {
            const int mine = row + 16 * n + (lane & 15);
            if (mine >= rows) continue;
            const int token = q0 + mine / job.group, h = head * job.group + mine % job.group;
            float y[E];
#pragma unroll
            for (int e = 0; e < 4; ++e)
#pragma unroll
                for (int j = 0; j < D / 16; ++j) y[e * (D / 16) + j] = r.o[n][j][e];
            if (job.chunks > 1) {
                const int64_t at_row = ((int64_t)chunk * a.tokens + token) * a.heads + h;
                float* o = job.part + at_row * D + E * (lane >> 4);
#pragma unroll
                for (int e = 0; e < E; e += 4) *reinterpret_cast<f32x4*>(o + e) = f32x4{y[e], y[e + 1], y[e + 2], y[e + 3]};
                if (lane < 16) job.part[(int64_t)job.chunks * a.tokens * a.heads * D + at_row] = lse[n];
            } else {
                uint16_t* o = static_cast<uint16_t*>(a.o) + (int64_t)token * a.o_token + (int64_t)h * a.o_head + E * (lane >> 4);
                store_row<E, F16>(o, y, job.wide_o);
                if (lane < 16 && a.lse) a.lse[(int64_t)token * a.heads + h] = lse[n] * kLn2;
            }
        }
    }
}

// Joins the chunks of a row: a wave a row.
template <int D, bool F16>
__global__ __launch_bounds__(64 * kWaves) void k_kv4_join(Job job) {
    const Kv4Attention& a = job.a;
    const int lane = threadIdx.x & 63;
    const int64_t row = group_index() * kWaves + (threadIdx.x >> 6), rows = (int64_t)a.tokens * a.heads;
    if (row >= rows) return;
    const float* sums = job.part + (int64_t)job.chunks * rows * D;
    float top = -INFINITY;
    for (int c = lane; c < job.chunks; c += 64) top = fmaxf(top, sums[c * rows + row]);
#pragma unroll
    for (int w = 1; w < 64; w *= 2) top = fmaxf(top, __shfl_xor(top, w));
    float all = 0.0f, y[D / 64] = {};
    for (int c = 0; c < job.chunks; ++c) {
        const float l = sums[c * rows + row];
        const float by = l == -INFINITY ? 0.0f : __builtin_amdgcn_exp2f(l - top);
        if (by == 0.0f) continue;
        all += by;
#pragma unroll
        for (int e = 0; e < D / 64; ++e) y[e] = fmaf(by, job.part[(c * rows + row) * D + lane * (D / 64) + e], y[e]);
    }
    const int64_t token = row / a.heads;
    const int h = (int)(row - token * a.heads);
    uint16_t* o = static_cast<uint16_t*>(a.o) + token * a.o_token + (int64_t)h * a.o_head + lane * (D / 64);
#pragma unroll
    for (int e = 0; e < D / 64; ++e) o[e] = (uint16_t)pack16(all == 0.0f ? 0.0f : y[e] / all, 0.0f, F16);
    if (lane == 0 && a.lse) a.lse[row] = (all == 0.0f ? -INFINITY : top + __builtin_amdgcn_logf(all)) * kLn2;
}

// How a call is launched.
struct Plan {
    int r;                                        // row tiles of a wave
    bool split;                                   // waves share rows
    int tiles, chunk, chunks;
};

Plan plan(const Kv4& c, const Kv4Attention& a, int num_cu) {
    const int group = a.heads / c.kv_heads;
    const int64_t rows = (int64_t)a.tokens * group;
    const int64_t mean = rows / a.batch;
    Plan p{};
    // few rows: the waves share them; many: rows of their own, as many as the registers hold
    p.split = mean <= 64;
    p.r = p.split && mean <= 16 ? 1 : 2;
    const int bm = 16 * p.r * (p.split ? 1 : kWaves);
    p.tiles = a.q_start ? (int)(rows / bm) + a.batch : a.batch * ((group + bm - 1) / bm);
    // keys in chunks where the rows alone do not fill the chip, of four steps of a workgroup at least
    int64_t range = a.max_len;
    if (a.window) {
        const int64_t seen = (int64_t)a.window + bm / group + 2 + kTile;
        if (seen < range) range = seen;
    }
    const int64_t groups = (int64_t)p.tiles * c.kv_heads;
    const int64_t want = (4 * num_cu + groups - 1) / groups;
    const int64_t least = 4 * kTile * kWaves;
    int64_t chunk = (range + want - 1) / want;
    chunk = chunk < least ? least : chunk;
    chunk = (chunk + kTile * kWaves - 1) / (kTile * kWaves) * (kTile * kWaves);
    p.chunk = (int)chunk;
    p.chunks = (int)((range + chunk - 1) / chunk);
    if (p.chunks <= 1) {
        p.chunks = 1;
        p.chunk = 1 << 30;
    }
    return p;
}

template <int D, bool F16>
int launch_attention(const Job& job, const Plan& p, hipStream_t s) {
    const dim3 grid = group_grid((int64_t)p.tiles * job.cache.kv_heads * p.chunks, 64 * kWaves), block(64 * kWaves);
    if (p.split && p.r == 1) launch_kernel(k_kv4_attention<D, 1, F16, true>, grid, block, 0, s, job);
    else if (p.split) launch_kernel(k_kv4_attention<D, 2, F16, true>, grid, block, 0, s, job);
    else launch_kernel(k_kv4_attention<D, 2, F16, false>, grid, block, 0, s, job);
    if (p.chunks > 1)
        launch_kernel(k_kv4_join<D, F16>, group_grid(((int64_t)job.a.tokens * job.a.heads + kWaves - 1) / kWaves, 64 * kWaves), block, 0, s, job);
    return launch_rc();
}

}  // namespace

size_t kv4_attention_workspace(const Kv4& c, const Kv4Attention& a, int num_cu) {
    const Plan p = plan(c, a, num_cu);
    return p.chunks > 1 ? (size_t)p.chunks * a.tokens * a.heads * (c.head_dim + 1) * sizeof(float) : 0;
}

int kv4_attention(const Kv4& c, const Kv4Attention& a, int num_cu, float* workspace, hipStream_t s) {
    const Plan p = plan(c, a, num_cu);
    const auto wide = [](const void* x, int64_t token, int64_t head) {
        return reinterpret_cast<uintptr_t>(x) % 16 == 0 && token % 8 == 0 && head % 8 == 0;
    };
    const Job job{c, a, a.heads / c.kv_heads, p.tiles, p.chunk, p.chunks, wide(a.q, a.q_token, a.q_head), wide(a.o, a.o_token, a.o_head), workspace};
    const bool f16 = a.dtype == RQ_F16;
    if (c.head_dim == 128) return f16 ? launch_attention<128, true>(job, p, s) : launch_attention<128, false>(job, p, s);
    return f16 ? launch_attention<64, true>(job, p, s) : launch_attention<64, false>(job, p, s);
}

}  // namespace rq
