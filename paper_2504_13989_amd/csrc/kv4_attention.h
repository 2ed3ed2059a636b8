// What the kernels of attention over the 4-bit paged cache share (kv4_few_rows.h: few rows, kv4_many_rows.h: many).
#pragma once
#include "kv4_layout.h"
#include "wave_common.h"

namespace rq {

struct KvJob {
    Kv4 cache;
    Kv4Attention a;
    int group;                                    // query heads of a kv head
    int tiles;                                    // row tiles (bound)
    int workers;                                  // few rows: workgroups of a kv head that share its tiles out, 0: one a row tile
    int chunk, chunks;                            // many rows: keys of a chunk, chunks (bound)
    bool wide_q, wide_o;                          // rows of q, of o begin on 16 bytes
    float* part;                                  // workspace
    int first_token;                              // joining chunks: what has been taken off the tokens' numbers
};

// Which positions a launch takes.  kWhole: a sequence's.  Where sequences share a prefix: kShared: the prefixes, the rows of all sequences of a
// group against them, kOwn: those behind it, of a sequence at a time, both to partial results; kSeparate: one after the other.
enum class Part { kWhole, kShared, kOwn, kSeparate };
struct PrefixJob : KvJob {
    Kv4Prefix p;
    int part_first, part_chunks;                  // partial results [chunks][tokens][heads]: the launch's first, all there are
    int first_tile;                               // row tiles of the launch: from there to `tiles`
    int slice, slice_end;                         // tokens whose results it writes, which the partial results have
};

namespace {

typedef _Float16 f16x2 __attribute__((ext_vector_type(2)));

constexpr int kTile = 64;                         // keys a step
constexpr float kLog2e = 1.4426950408889634f, kLn2 = 0.6931471805599453f;

__device__ __forceinline__ uint32_t pack_f16(float x, float y) { return __builtin_bit_cast(uint32_t, f16x2{(_Float16)x, (_Float16)y}); }
template <bool F16>
__device__ __forceinline__ uint32_t pack16(float x, float y) {
    if constexpr (F16) return pack_f16(x, y);
    typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
    return __builtin_bit_cast(uint32_t, bf16x2{(__bf16)x, (__bf16)y});
}

// What makes codes fp16 numbers: x & even | e1024, x & odd | e64.  Held in registers of whose values the compiler knows nothing: with
// literals, of which a three-operand instruction takes none, it makes two instructions of each.
struct CodeBits {
    uint32_t even, odd, e1024, e64;
    __device__ __forceinline__ CodeBits() {
        asm("s_mov_b32 %0, 0x000f000f" : "=s"(even));
        asm("s_mov_b32 %0, 0x00f000f0" : "=s"(odd));
        asm("v_mov_b32 %0, 0x64006400" : "=v"(e1024));
        asm("v_mov_b32 %0, 0x54005400" : "=v"(e64));
    }
    // codes in bits 0 .. 3 (1024 + c), 4 .. 7 (64 + c) of both halves
    __device__ __forceinline__ uint32_t low(uint32_t x) const { return (x & even) | e1024; }
    __device__ __forceinline__ uint32_t high(uint32_t x) const { return (x & odd) | e64; }
};

// Sums and maxima over the lanes of a column: of 16 columns lanes n, n + 16, n + 32, n + 48, of 32 columns lanes n, n + 32.
__device__ __forceinline__ void other_rows(float x, bool far, float& a, float& b) {
    const uint32_t u = __float_as_uint(x);
    const auto r = far ? __builtin_amdgcn_permlane32_swap(u, u, false, false) : __builtin_amdgcn_permlane16_swap(u, u, false, false);
    a = __uint_as_float(r[0]);
    b = __uint_as_float(r[1]);
}
template <int COLUMNS>
__device__ __forceinline__ float column_sum(float x) {
    float a, b;
    if constexpr (COLUMNS == 16) {
        other_rows(x, false, a, b);
        x = a + b;
    }
    other_rows(x, true, a, b);
    return a + b;
}
template <int COLUMNS>
__device__ __forceinline__ float column_max(float x) {
    float a, b;
    if constexpr (COLUMNS == 16) {
        other_rows(x, false, a, b);
        x = fmaxf(a, b);
    }
    other_rows(x, true, a, b);
    return fmaxf(a, b);
}

// A query row as the matrix cores take it, over 64 / COLUMNS lanes: lane g of a column holds the g-th part of the row, eights of
// it in the order (0, 4), (1, 5), (2, 6), (3, 7) in which codes leave a dword.
template <int D, int COLUMNS>
struct Query {
    static constexpr int E = D * COLUMNS / 64;    // elements of a lane
    f16x8 hi[E / 8], lo[E / 8];                   // q = hi + lo; lo only where it is asked for
    float even, odd;                              // sums of elements 0, 2, 4, 6 and 1, 3, 5, 7 of the eights
    float f;                                      // log2 of e^(scale q.k) for a unit of hi.k, a power of two
};

// What a lane loads of a row.  Rows that are to be rotated are operands of products with H: lane g of a column has elements
// 8 L s + 8 g + 0 .. 7 (L lanes a column) for s = 0, 1 ...; others lie as Query wants them.  Zeros where there is no row.
template <int D, int COLUMNS>
struct RawQuery {
    u32x4 w[D * COLUMNS / 512];
};
template <int D, int COLUMNS>
__device__ __forceinline__ RawQuery<D, COLUMNS> load_query(const KvJob& job, bool there, int token, int head, int lane) {
    const Kv4Attention& a = job.a;
    constexpr int E = Query<D, COLUMNS>::E, L = 64 / COLUMNS;
    RawQuery<D, COLUMNS> raw{};
    const int g = lane / COLUMNS, first = a.rotate ? 8 * g : E * g, step = a.rotate ? 8 * L : 8;
    const uint16_t* x = static_cast<const uint16_t*>(a.q) + (int64_t)token * a.q_token + (int64_t)head * a.q_head + first;
    if (there) {
        if (job.wide_q) {
#pragma unroll
            for (int e = 0; e < E / 8; ++e) raw.w[e] = *reinterpret_cast<const u32x4*>(x + e * step);
        } else {
#pragma unroll
            for (int e = 0; e < E; e += 2) raw.w[e / 8][e / 2 % 4] = (uint32_t)x[e / 8 * step + e % 8] | ((uint32_t)x[e / 8 * step + e % 8 + 1] << 16);
        }
    }
    return raw;
}

// H x (fp32) of the columns' rows on the matrix cores, laid out as Query wants them.  H[i, j] = (-1)^popcount(i & j); an operand's signs
// are those of its eight elements' low bits times one sign for the rest of the index, which is a product of a part that
// depends on the step and one that depends on the tile.
template <int D, int COLUMNS, bool F16>
__device__ __forceinline__ void rotate_query(float (&q)[D * COLUMNS / 64], const RawQuery<D, COLUMNS>& raw, int lane) {
    constexpr int R = COLUMNS == 16 ? 4 : 16, T = D * COLUMNS / 64 / R;   // results of a lane in a tile, tiles
    constexpr int S = D * COLUMNS / 512, K = D / S;                  // steps, elements of a step
    constexpr uint32_t minus = 0x80008000u, one = F16 ? 0x3c003c00u : 0x3f803f80u;
    asm volatile("" : "+v"(lane));                // (in a loop over row tiles the signs are not to be kept in registers)
    const int m = lane % COLUMNS, g = lane / COLUMNS;
    // row m of tile t is element `mine` + R' t of the rotated row: what lane m / 4 (mod lanes of a column) is to hold
    constexpr int lanes = 64 / COLUMNS;
    const int mine = (m >> 2) % lanes * (D / lanes) + (COLUMNS == 16 ? 0 : (m >> 3) * 4) + (m & 3);
    const auto sign = [](int x) { return __builtin_popcount((unsigned)x) & 1 ? minus : 0u; };
    uint32_t by_step[S], by_tile[T];
#pragma unroll
    for (int s = 0; s < S; ++s) by_step[s] = sign(mine & (K * s));
#pragma unroll
    for (int t = 0; t < T; ++t) by_tile[t] = sign((mine + R * t) & (8 * g));
    const uint32_t low = one ^ (m & 1 ? 0x80000000u : 0u);
    const uint32_t high = one ^ (m & 2 ? 0x8000u : 0u) ^ (((m >> 1) ^ m) & 1 ? 0x80000000u : 0u);
    const uint32_t four = COLUMNS == 16 ? 0u : (m & 8 ? minus : 0u);
#pragma unroll
    for (int t = 0; t < T; ++t) {
        float __attribute__((ext_vector_type(R))) y = {};
#pragma unroll
        for (int s = 0; s < S; ++s) {
            uint32_t x = by_step[s] ^ by_tile[t];
            if (__builtin_popcount((unsigned)((R * t) & (K * s))) & 1) x ^= minus;
            const uint32_t other = COLUMNS == 16 ? (t & 1 ? x ^ minus : x) : x ^ four;
            const u32x4 a{low ^ x, high ^ x, low ^ other, high ^ other};
            if constexpr (COLUMNS == 16) {
                if constexpr (F16) y = __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(f16x8, a), __builtin_bit_cast(f16x8, raw.w[s]), y, 0, 0, 0);
                else y = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, raw.w[s]), y, 0, 0, 0);
            } else {
                if constexpr (F16) y = __builtin_amdgcn_mfma_f32_32x32x16_f16(__builtin_bit_cast(f16x8, a), __builtin_bit_cast(f16x8, raw.w[s]), y, 0, 0, 0);
                else y = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, raw.w[s]), y, 0, 0, 0);
            }
        }
#pragma unroll
        for (int e = 0; e < R; ++e) q[R * t + e] = y[e];
    }
}

// Rotates a row, scales it by a power of two and rounds it.
template <int D, int COLUMNS, bool F16, bool PRECISE>
__device__ __forceinline__ void take_query(Query<D, COLUMNS>& r, const KvJob& job, const RawQuery<D, COLUMNS>& raw, int lane) {
    const Kv4Attention& a = job.a;
    constexpr int E = Query<D, COLUMNS>::E;
    float q[E];
    if (a.rotate) {
        rotate_query<D, COLUMNS, F16>(q, raw, lane);
    } else {
#pragma unroll
        for (int e = 0; e < E; ++e) {
            const uint32_t u = raw.w[e / 8][e / 2 % 4];
            q[e] = F16 ? (float)__builtin_bit_cast(_Float16, (uint16_t)(e % 2 ? u >> 16 : u)) : __uint_as_float(e % 2 ? u & 0xffff0000u : u << 16);
        }
    }
    // log2(e) and the scale of the scores are in the row, so that f is a power of two and f * (s - m) exact, however large
    const float unit = a.scale * kLog2e * (a.rotate ? (D == 128 ? 0.08838834764831845f : 0.125f) : 1.0f);
    float most = 0.0f;
#pragma unroll
    for (int e = 0; e < E; ++e) {
        q[e] *= unit;
        most = fmaxf(most, fabsf(q[e]));
    }
    most = column_max<COLUMNS>(most);
    // 2^-x with most < 2^x: 1 for rows of zeros; infinite rows stay what they are
    int x2 = (int)((__float_as_uint(most) >> 23) & 255) - 126;
    x2 = most == 0.0f || x2 > 128 ? 0 : x2 < -100 ? -100 : x2;
    const float by = __uint_as_float((uint32_t)(127 - (x2 > 126 ? 126 : x2)) << 23);
    r.f = 1.0f / by;
    float even = 0.0f, odd = 0.0f;
#pragma unroll
    for (int j = 0; j < E / 8; ++j)
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            const float v = q[8 * j + e / 2 + 4 * (e % 2)] * by;
            const _Float16 hi = (_Float16)v;
            float sum = (float)hi;
            r.hi[j][e] = hi;
            if constexpr (PRECISE) {
                const _Float16 lo = (_Float16)(v - sum);
                r.lo[j][e] = lo;
                sum += (float)lo;
            }
            (e / 2 % 2 ? odd : even) += sum;
        }
    r.even = column_sum<COLUMNS>(even);
    r.odd = column_sum<COLUMNS>(odd);
}

// N consecutive results of a row.
template <int N, bool F16>
__device__ __forceinline__ void store_row(uint16_t* o, const float (&y)[N], bool wide) {
    if constexpr (N == 1) {
        o[0] = (uint16_t)pack16<F16>(y[0], 0.0f);
        return;
    } else {
        uint32_t w[N / 2];
#pragma unroll
        for (int e = 0; e < N / 2; ++e) w[e] = pack16<F16>(y[2 * e], y[2 * e + 1]);
        if (wide) {
            if constexpr (N % 8 == 0) {
#pragma unroll
                for (int e = 0; e < N / 8; ++e) reinterpret_cast<u32x4*>(o)[e] = u32x4{w[4 * e], w[4 * e + 1], w[4 * e + 2], w[4 * e + 3]};
            } else {
#pragma unroll
                for (int e = 0; e < N / 2; ++e) reinterpret_cast<uint32_t*>(o)[e] = w[e];
            }
        } else {
#pragma unroll
            for (int e = 0; e < N / 2; ++e) {
                o[2 * e] = (uint16_t)w[e];
                o[2 * e + 1] = (uint16_t)(w[e] >> 16);
            }
        }
    }
}

// Nothing moves over RQ_FENCE; RQ_NEXT: of what stands between two of them, n of a kind come next.
constexpr int kValu = 0x2, kMfma = 0x8, kLdsRead = 0x100;
#define RQ_FENCE() __builtin_amdgcn_sched_barrier(0)
#define RQ_NEXT(kind, n) __builtin_amdgcn_sched_group_barrier(kind, n, 0)

// A barrier for what lies in LDS: loads from memory stay under way.
__device__ __forceinline__ void lds_barrier() {
    __builtin_amdgcn_fence(__ATOMIC_RELEASE, "workgroup", "local");
    __builtin_amdgcn_s_barrier();
    __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "workgroup", "local");
}

__device__ __forceinline__ bool finite(float x) { return (__float_as_uint(x) & 0x7f800000u) != 0x7f800000u; }

// The pages of tiles of 64 keys, read 64 at once, so that no step waits for the table before it can ask for codes.  PAGED: pages of
// 16 or 32 tokens, the 16 keys of each quarter of a tile in a place of their own, four lanes a tile; else a tile lies in one page,
// a lane a tile.
template <bool PAGED>
constexpr int kPagesOf = PAGED ? 16 : 64;         // tiles
// The tiles that begin at k0, k0 + stride ...  Keys behind the sequence's last one are masked: whatever the table has for them is
// a page or, as numbers that are none, stands for page 0.
template <bool PAGED>
__device__ __forceinline__ int load_pages(const Kv4& c, const int32_t* table, int width, int k0, int stride, int lane) {
    const int64_t k = PAGED ? k0 + (int64_t)(lane >> 2) * stride + 16 * (lane & 3) : k0 + (int64_t)lane * stride;
    const int64_t at = k >> c.page_shift;
    const int page = table[at < width ? at : width - 1];
    return (uint32_t)page < (uint32_t)c.pages ? page : 0;
}
// The head's block of the page of quarter `quarter` of tile number n, and its first key's place in the page.  (`head_at`: of the kv
// head's block in a page)
template <bool PAGED>
__device__ __forceinline__ const uint8_t* block_of(const Kv4& c, int pages, int n, int quarter, int head_at) {
    // (a page's bytes fit 32 bits: RQ_KV4_MAX_HEADS * 256 * 136)
    return c.data + (uint64_t)(uint32_t)__builtin_amdgcn_readlane(pages, PAGED ? 4 * n + quarter : n) * (uint32_t)c.page_bytes + head_at;
}
__device__ __forceinline__ int place_of(const Kv4& c, int k0, int quarter) { return (k0 + 16 * quarter) & ((1 << c.page_shift) - 1); }

// What a key's centre adds to the sums, for the two factors it can go with: p, and p * step as it was rounded to fp16.  A centre of the
// size of the range, which the codes' share may cancel, goes with the latter, so that the rounding stays one of p; a larger one
// cannot be cancelled, and its quotient might overflow.
struct Centre {
    float with_p, with_step;
};
__device__ __forceinline__ Centre split_centre(float step, float mid) {
    const bool near = step >= 0x1p-100f && fabsf(mid) < 16.0f * step;
    // (a quotient with one correction: what cancels exactly does so here too)
    const float inv = __builtin_amdgcn_rcpf(step), x = mid * inv;
    return Centre{near ? 0.0f : mid, near ? fmaf(fmaf(-x, step, mid), inv, x) : 0.0f};
}

// with_step of a tile's keys in LDS, as two fp16 numbers each: four keys' high parts, then their low ones.  The sum with p * step then
// takes two products an instruction, at the rate of others (a product of fp16 and fp32 operands takes twice as long: a prompt's
// fp16 results 80 us and not 74).
__device__ __forceinline__ void put_centre(float* lds, int key, float x) {
    _Float16* w = reinterpret_cast<_Float16*>(lds + (key & ~3)) + (key & 3);
    const _Float16 high = (_Float16)x;
    w[0] = high;
    w[4] = (_Float16)(x - (float)high);
}
__device__ __forceinline__ f16x2 as_f16(uint32_t w) { return __builtin_bit_cast(f16x2, w); }
__device__ __forceinline__ float add_centre(uint32_t p, uint32_t with_step, float sum) { return __builtin_amdgcn_fdot2(as_f16(p), as_f16(with_step), sum, false); }

// A tile of BM rows: where they lie, and (once find_keys has been asked) the positions that they see.
struct Place {
    int b, q0, nq, base;                          // sequence, its first token, its tokens, the tile's first row
    int len;                                      // positions of the sequence
    int from, to;                                 // some row of the tile sees; `from` a multiple of kTile
};
// Row r of a tile's sequence: its token.
__device__ __forceinline__ int token_of(const KvJob& job, const Place& p, int r) { return p.nq == 1 ? 0 : r / job.group; }
// Whether a tile's sequence (or group of them) has tokens of the launch's.
__device__ __forceinline__ bool in_slice(const PrefixJob& job, const Place& p) { return p.q0 + p.nq > job.slice && p.q0 < job.slice_end; }

// Grid of `items` workgroups for each kv head, and a workgroup's number in it.
inline dim3 item_grid(int kv_heads, int64_t items) {
    const int64_t y = items < 65535 ? items : 65535;
    return dim3((unsigned)kv_heads, (unsigned)y, (unsigned)((items + y - 1) / y));
}
__device__ __forceinline__ int item_number() { return (int)(blockIdx.z * gridDim.y + blockIdx.y); }

// Row tile `tile`: a sequence's tiles begin at floor(q_start * group / BM) + its number.  False where there is none.
template <int BM>
__device__ __forceinline__ bool find_rows(const KvJob& job, int tile, Place& p) {
    const Kv4Attention& a = job.a;
    int first;
    if (a.q_start) {
        int lo = 0, hi = a.batch - 1;
        while (lo < hi) {
            const int at = (lo + hi + 1) >> 1;
            if ((int)((int64_t)a.q_start[at] * job.group / BM) + at <= tile) lo = at; else hi = at - 1;
        }
        p.b = lo;
        int q0 = a.q_start[lo], q1 = a.q_start[lo + 1];
        q0 = q0 < 0 ? 0 : q0 > a.tokens ? a.tokens : q0;
        q1 = q1 < q0 ? q0 : q1 > a.tokens ? a.tokens : q1;
        p.q0 = q0;
        p.nq = q1 - q0;
        first = (int)((int64_t)q0 * job.group / BM) + lo;
    } else {
        const int each = (job.group + BM - 1) / BM;
        p.b = p.q0 = each == 1 ? tile : tile / each;
        p.nq = 1;
        first = p.b * each;
    }
    p.base = (tile - first) * BM;
    return p.base >= 0 && p.base < p.nq * job.group;
}
// len: kv_lens of the sequence
template <int BM>
__device__ __forceinline__ void find_keys(const KvJob& job, Place& p, int len) {
    const Kv4Attention& a = job.a;
    const int rows = p.nq * job.group;
    p.len = len < 0 ? 0 : len > a.max_len ? (int)a.max_len : len;          // (max_len <= width * page size)
    const int last = (p.base + BM < rows ? p.base + BM : rows) - 1;
    const int p0 = p.len - p.nq + token_of(job, p, p.base), p1 = p.len - p.nq + token_of(job, p, last);
    const int from = a.window ? p0 - a.window + 1 : 0;
    p.from = (from < 0 ? 0 : from) & ~(kTile - 1);
    p.to = a.causal && p1 + 1 < p.len ? p1 + 1 : p.len;
}

// Tokens of the sequences of group g: the first, the one behind the last.
__device__ __forceinline__ int group_begin(const PrefixJob& job, int g) {
    int b = job.p.group_start[g];
    b = b < 0 ? 0 : b > job.a.batch ? job.a.batch : b;
    if (!job.a.q_start) return b;
    const int q = job.a.q_start[b];
    return q < 0 ? 0 : q > job.a.tokens ? job.a.tokens : q;
}
// find_rows for row tiles of groups (Place: b the group); len: of its prefix.
template <int BM>
__device__ __forceinline__ bool find_group_rows(const PrefixJob& job, int tile, Place& p) {
    int lo = 0, hi = job.p.groups - 1;
    while (lo < hi) {
        const int at = (lo + hi + 1) >> 1;
        if ((int)((int64_t)group_begin(job, at) * job.group / BM) + at <= tile) lo = at; else hi = at - 1;
    }
    const int q1 = group_begin(job, lo + 1);
    p.b = lo;
    p.q0 = group_begin(job, lo);
    p.nq = q1 > p.q0 ? q1 - p.q0 : 0;
    p.base = (tile - (int)((int64_t)p.q0 * job.group / BM) - lo) * BM;
    return p.base >= 0 && p.base < p.nq * job.group;
}
__device__ __forceinline__ int prefix_len(const PrefixJob& job, int g) {
    const int n = job.p.lens[g];
    return n < 0 ? 0 : n > job.p.max_len ? (int)job.p.max_len : n;
}
__device__ __forceinline__ int own_len(const KvJob& job, int seq) {
    const int n = job.a.kv_lens[seq];
    return n < 0 ? 0 : n > job.a.max_len ? (int)job.a.max_len : n;
}
// The group of a sequence.
__device__ __forceinline__ int group_of(const PrefixJob& job, int seq) {
    int lo = 0, hi = job.p.groups - 1;
    while (lo < hi) {
        const int at = (lo + hi + 1) >> 1;
        if (job.p.group_start[at] <= seq) lo = at; else hi = at - 1;
    }
    return lo;
}
// A token's position behind its group's prefix (below 0: in it).
__device__ __forceinline__ int own_position(const KvJob& job, int token) {
    if (!job.a.q_start) return own_len(job, token) - 1;
    int lo = 0, hi = job.a.batch - 1;
    while (lo < hi) {
        const int at = (lo + hi + 1) >> 1;
        if (job.a.q_start[at] <= token) lo = at; else hi = at - 1;
    }
    return own_len(job, lo) - job.a.q_start[lo + 1] + token;
}

}  // namespace

// Joins partial results of a row: a wave a row (job.chunks of them).
void launch_join(const KvJob& job, hipStream_t s);
// kernels_kv4_prompt.hip: many rows, 32 a wave, a workgroup of one or two groups of 4 waves or one of 8
void launch_prompt(const KvJob& job, int waves, int groups, hipStream_t s);

}  // namespace rq
