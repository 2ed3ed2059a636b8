// Attention over the 4-bit paged cache for many queries a sequence (prompts, chunks of them).  The mathematics is that of
// kernels_kv4_attention.hip, and so are rows and columns: products are taken transposed, a wave has 32 rows of its own as the
// columns of 32 x 32 products, column n the lanes n and n + 32.
//
// What is bound here is vector work: a score costs a lane seven or eight instructions' time, as long as the matrix cores take for its 512
// operations, and codes that each wave unpacked for itself would cost as much again.  So the waves of a workgroup (4 or 8)
// unpack a tile of 64 keys together, once, into LDS as fp16 operands: keys [key][element], values transposed, [element][key], keys in
// the order in which scores leave the matrix cores, so that p enters them again as it is.  The next tile is unpacked into the
// other half of LDS before the products on this one; its codes were loaded a step earlier.
//   - bf16 results: operands are the elements themselves, (code - 7.5) step + mid, times a power of two that holds the largest
//     seen so far in fp16's range (rounded to fp16 once, 2^-12: less than the result's rounding; steps and centres, bf16, are exact in fp16).  Scores need no step or centre.
//   - fp16 results (EXACT): operands are codes - 7.5, which are exact, and steps and centres are applied to the scores as in the other
//     kernel; two instructions a score and one product more.  Queries are two fp16 numbers.
// A value row that is not finite becomes zeros and its key NaN: queries that do not see it stay what they are.
#include "kv4_attention.h"

namespace rq {
namespace {

constexpr int kKeyPad = 8, kValueRow = kTile + 8;  // halfwords: rows of LDS begin 4 banks apart

template <int D, bool EXACT>
struct Tile {
    uint16_t k[kTile][D + kKeyPad];
    uint16_t v[D][kValueRow];                     // element d in row (d % 4) * D / 4 + d / 4
    float scale[EXACT ? 4 : 1][EXACT ? kTile : 4];  // EXACT: keys' steps and centres, values' steps and centres
};

// What a thread unpacks of a tile: N runs of eight bytes each of keys and of values.
template <int N>
struct Raw {
    u32x2 k[N], v[N];
    uint32_t kp, vp;                              // parameters of key `lane`
};

// Runs of a tile's keys, and as many of its values.
template <int D>
constexpr int kRuns = kTile * D / 16;

template <int D, int WAVES, int N>
__device__ __forceinline__ void load_tile(Raw<N>& t, const Kv4& c, TableRow table, int head, int k0, int end, int thread) {
    const int shift = c.page_shift, p = 1 << shift, lane = thread & 63;
    const auto block_of = [&](int key) {
        int page = table[key >> shift];
        if ((uint32_t)page >= (uint32_t)c.pages) page = 0;
        return c.data + (int64_t)page * c.page_bytes + (int64_t)(head * (p * (D + 8)));
    };
    if (shift >= 6) {                             // a tile lies in one page
        const uint8_t* block = block_of(k0);
        const int at = k0 & (p - 1);
        const uint8_t *k = block + at * (D / 2), *v = block + (p + at) * (D / 2), *w = block + p * D + at * 4;
#pragma unroll
        for (int i = 0; i < N; ++i) {
            const uint32_t run = (uint32_t)(thread + 64 * WAVES * i) * 8;
            if (kRuns<D> % (64 * WAVES) == 0 || run < kRuns<D> * 8) {
                t.k[i] = *reinterpret_cast<const u32x2*>(k + run);
                t.v[i] = *reinterpret_cast<const u32x2*>(v + run);
            }
        }
        t.kp = *reinterpret_cast<const uint32_t*>(w + (uint32_t)(lane * 4));
        t.vp = *reinterpret_cast<const uint32_t*>(w + 4 * p + (uint32_t)(lane * 4));
    } else {
        const uint8_t* of[4];                     // of each 16 keys
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            int key = k0 + 16 * i;
            if (key >= end) key = (end - 1) & ~15;                   // (those keys are masked)
            const int at = key & (p - 1);
            of[i] = block_of(key) + at * 4;       // + p * D: parameters; codes at 4 * at * (D / 8 - 1) further
            if ((lane >> 4) == i) {
                const uint8_t* w = of[i] + p * D + (lane & 15) * 4;
                t.kp = *reinterpret_cast<const uint32_t*>(w);
                t.vp = *reinterpret_cast<const uint32_t*>(w + 4 * p);
            }
            of[i] += at * (D / 2 - 4);
        }
#pragma unroll
        for (int i = 0; i < N; ++i) {
            const int run = thread + 64 * WAVES * i, q = run / (kRuns<D> / 4), in = run % (kRuns<D> / 4) * 8;
            if (run < kRuns<D>) {
                const uint8_t* x = q == 0 ? of[0] : q == 1 ? of[1] : q == 2 ? of[2] : of[3];
                t.k[i] = *reinterpret_cast<const u32x2*>(x + in);
                t.v[i] = *reinterpret_cast<const u32x2*>(x + p * (D / 2) + in);
            }
        }
    }
}

__device__ __forceinline__ f16x2 as_f16(uint32_t w) { return __builtin_bit_cast(f16x2, w); }
__device__ __forceinline__ uint32_t as_bits(f16x2 x) { return __builtin_bit_cast(uint32_t, x); }

// c - 7.5 of nibble J of both halves of a dword, exact: 64 + c less 71.5.
template <int J>
__device__ __forceinline__ f16x2 code_pair(uint32_t w) {
    const uint32_t x = J == 0 ? w << 4 : w >> (4 * J - 4);
    return as_f16(and_or(x, 0x00f000f0u, 0x54005400u)) + f16x2{(_Float16)-71.5f, (_Float16)-71.5f};
}

// The powers of two in the operands: what has been seen so far is below `limit`.
struct Range {
    float limit;
    float by;                                     // 2^UP / limit
};
// True where the range grew; `grew` is the old factor's inverse times the new one.  UP: 15 for elements, whose fp16 then has
// full precision down to 2^-29 of the largest; 7 for steps, which meet factors of up to 2^8.
template <int UP>
__device__ __forceinline__ bool widen(Range& r, float x, float& grew) {
    if (!__any(x > r.limit)) return false;
#pragma unroll
    for (int w = 1; w < 64; w *= 2) x = fmaxf(x, __shfl_xor(x, w));
    int e = (int)(__float_as_uint(x) >> 23) - 126;                   // x < 2^e
    e = e < -60 ? -60 : e > 126 ? 126 : e;
    const float limit = __uint_as_float((uint32_t)(e + 127) << 23);
    if (!(limit > r.limit)) return false;
    const float by = __uint_as_float((uint32_t)(127 + UP - e) << 23);
    grew = by / r.by;
    r.limit = limit;
    r.by = by;
    return true;
}

template <int D, bool EXACT>
struct Sums {
    float m, l, w;                                // maximum (log2), sums over the lane's keys
    typedef float f32x16 __attribute__((ext_vector_type(16)));
    f32x16 o[D / 32];
};
template <int D, bool EXACT>
__device__ __forceinline__ void scale_sums(Sums<D, EXACT>& r, float by) {
#pragma unroll
    for (int j = 0; j < D / 32; ++j)
#pragma unroll
        for (int e = 0; e < 16; ++e) r.o[j][e] *= by;
}

// Unpacks a thread's runs into LDS.  `key_range` and `value_range` widen to hold the tile.
template <int D, int WAVES, int N, bool EXACT>
__device__ __forceinline__ void unpack(Tile<D, EXACT>& to, const Raw<N>& t, int k0, int end, int thread, const Range& key_range, const Range& value_range) {
    const int lane = thread & 63;
    uint32_t kw = 0, vw = 0;                      // parameters of key `lane`, as fp16 pairs of a step and a centre
    {
        const bool there = k0 + lane < end;
        const uint32_t kp = there ? t.kp : 0u, vp = there ? t.vp : 0u;
        float ks = __uint_as_float(kp << 16), km = __uint_as_float(kp & 0xffff0000u);
        float vs = __uint_as_float(vp << 16), vm = __uint_as_float(vp & 0xffff0000u);
        if constexpr (EXACT) {
            // (a wave an array: all of them hold the parameters)
            if (thread >> 6 == 0) to.scale[0][lane] = ks;
            if (thread >> 6 == 1) to.scale[1][lane] = km;
            if (thread >> 6 == 2) to.scale[2][lane] = vs;
            if (thread >> 6 == 3) to.scale[3][lane] = vm;
        } else {
            if (!finite(vs) || !finite(vm)) {
                vs = vm = 0.0f;
                ks = __builtin_nanf("");
            }
            kw = pack_f16(ks * key_range.by, km * key_range.by);
            vw = pack_f16(vs * value_range.by, vm * value_range.by);
        }
    }
#pragma unroll
    for (int i = 0; i < N; ++i) {
        const int run = thread + 64 * WAVES * i;
        if (kRuns<D> % (64 * WAVES) != 0 && run >= kRuns<D>) break;
        {   // keys: a run is 16 elements of one key
            const int key = run / (D / 16), at = run % (D / 16) * 16;
            f16x2 step, mid;
            if constexpr (!EXACT) {
                const f16x2 sm = as_f16((uint32_t)__shfl((int)kw, key & 63));
                step = f16x2{sm[0], sm[0]};
                mid = f16x2{sm[1], sm[1]};
            }
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                f16x2 x[4] = {code_pair<0>(t.k[i][h]), code_pair<1>(t.k[i][h]), code_pair<2>(t.k[i][h]), code_pair<3>(t.k[i][h])};
                if constexpr (!EXACT)
#pragma unroll
                    for (int e = 0; e < 4; ++e) x[e] = __builtin_elementwise_fma(x[e], step, mid);
                *reinterpret_cast<u32x4*>(&to.k[key][at + 8 * h]) = u32x4{as_bits(x[0]), as_bits(x[1]), as_bits(x[2]), as_bits(x[3])};
            }
        }
        {   // values: a run is four elements of four tokens
            const int four = run / (D / 4), x4 = run % (D / 4);
            f16x2 step[2], mid[2];
            if constexpr (!EXACT)
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    const f16x2 a = as_f16((uint32_t)__shfl((int)vw, 4 * four + 2 * h)), b = as_f16((uint32_t)__shfl((int)vw, 4 * four + 2 * h + 1));
                    step[h] = f16x2{a[0], b[0]};
                    mid[h] = f16x2{a[1], b[1]};
                }
            f16x2 x[4][2];
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                x[0][h] = code_pair<0>(t.v[i][h]);
                x[1][h] = code_pair<1>(t.v[i][h]);
                x[2][h] = code_pair<2>(t.v[i][h]);
                x[3][h] = code_pair<3>(t.v[i][h]);
            }
            // keys 16 s + 4 q + 0 .. 3 go to places 16 s + 8 (q % 2) + 4 (q / 2) + 0 .. 3
            const int place = (four & ~3) * 4 + 8 * (four & 1) + 4 * (four >> 1 & 1);
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                if constexpr (!EXACT)
#pragma unroll
                    for (int h = 0; h < 2; ++h) x[e][h] = __builtin_elementwise_fma(x[e][h], step[h], mid[h]);
                *reinterpret_cast<u32x2*>(&to.v[e * (D / 4) + x4][place]) = u32x2{as_bits(x[e][0]), as_bits(x[e][1])};
            }
        }
    }
}

template <int D, bool EXACT, bool MASKED>
__device__ __forceinline__ void take_tile(Sums<D, EXACT>& r, const Query<D, 32>& q, const Tile<D, EXACT>& t, float f, float up, int k0, int lo, int hi, int lane) {
    typedef float f32x16 __attribute__((ext_vector_type(16)));
    const int n = lane & 31, h = lane >> 5;
    f32x16 s[2];
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        s[i] = f32x16{};
#pragma unroll
        for (int j = 0; j < D / 16; ++j) {
            const f16x8 a = *reinterpret_cast<const f16x8*>(&t.k[32 * i + n][h * (D / 2) + 8 * j]);
            s[i] = __builtin_amdgcn_mfma_f32_32x32x16_f16(a, q.hi[j], s[i], 0, 0, 0);
            if constexpr (EXACT) s[i] = __builtin_amdgcn_mfma_f32_32x32x16_f16(a, q.lo[j], s[i], 0, 0, 0);
        }
    }
    float mx = -INFINITY;
#pragma unroll
    for (int i = 0; i < 2; ++i)
#pragma unroll
        for (int e = 0; e < 16; e += 4) {
            const int key = 32 * i + 2 * e + 4 * h;
            f32x4 step, mid;
            if constexpr (EXACT) {
                step = *reinterpret_cast<const f32x4*>(&t.scale[0][key]);
                mid = *reinterpret_cast<const f32x4*>(&t.scale[1][key]);
            }
#pragma unroll
            for (int u = 0; u < 4; ++u) {
                float x = s[i][e + u];
                if constexpr (EXACT) x = fmaf(step[u], x, mid[u] * (q.even + q.odd));
                if constexpr (MASKED) x = k0 + key + u >= lo && k0 + key + u < hi ? x : -INFINITY;
                s[i][e + u] = x;
                mx = fmaxf(mx, x);
            }
        }
    mx = f * column_max<32>(mx);
    // p may grow to 2^8 before the sums are scaled to a new maximum
    if (__any(mx - r.m > 8.0f)) {
        const float to = fmaxf(r.m, mx), by = to == -INFINITY ? 1.0f : __builtin_amdgcn_exp2f(r.m - to);
        scale_sums(r, by);
        r.l *= by;
        r.w *= by;
        r.m = to;
    }
    const float off = (r.m == -INFINITY ? 0.0f : r.m) - up;
    uint32_t p[2][8];
#pragma unroll
    for (int i = 0; i < 2; ++i)
#pragma unroll
        for (int e = 0; e < 16; e += 4) {
            const int key = 32 * i + 2 * e + 4 * h;
            f32x4 step, mid;
            if constexpr (EXACT) {
                step = *reinterpret_cast<const f32x4*>(&t.scale[2][key]);
                mid = *reinterpret_cast<const f32x4*>(&t.scale[3][key]);
            }
            float x[4];
#pragma unroll
            for (int u = 0; u < 4; ++u) {
                const float y = __builtin_amdgcn_exp2f(fmaf(f, s[i][e + u], -off));
                r.l += y;
                x[u] = y;
                if constexpr (EXACT) {
                    if constexpr (MASKED) {       // a masked key's parameters may be infinite or NaN
                        const bool seen = s[i][e + u] != -INFINITY;
                        x[u] = seen ? y * step[u] : 0.0f;
                        r.w += seen ? y * mid[u] : 0.0f;
                    } else {
                        x[u] = y * step[u];
                        r.w = fmaf(y, mid[u], r.w);
                    }
                }
            }
            p[i][e / 2] = pack_f16(x[0], x[1]);
            p[i][e / 2 + 1] = pack_f16(x[2], x[3]);
        }
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const f16x8 b = __builtin_bit_cast(f16x8, u32x4{p[i / 2][4 * (i % 2)], p[i / 2][4 * (i % 2) + 1], p[i / 2][4 * (i % 2) + 2], p[i / 2][4 * (i % 2) + 3]});
#pragma unroll
        for (int j = 0; j < D / 32; ++j) {
            const f16x8 a = *reinterpret_cast<const f16x8*>(&t.v[32 * j + n][16 * i + 8 * h]);
            r.o[j] = __builtin_amdgcn_mfma_f32_32x32x16_f16(a, b, r.o[j], 0, 0, 0);
        }
    }
}

// A barrier for what lies in LDS: loads from memory stay under way.
__device__ __forceinline__ void lds_barrier() {
    __builtin_amdgcn_fence(__ATOMIC_RELEASE, "workgroup", "local");
    __builtin_amdgcn_s_barrier();
    __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "workgroup", "local");
}

template <int D, int WAVES, bool F16>
__global__ __launch_bounds__(64 * WAVES, 2) void k_kv4_prompt(KvJob job) {
    constexpr bool EXACT = F16;
    constexpr int BM = 32 * WAVES, N = (kRuns<D> + 64 * WAVES - 1) / (64 * WAVES);
    __shared__ __attribute__((aligned(16))) Tile<D, EXACT> tiles[2];
    const Kv4Attention& a = job.a;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int64_t item = group_index();
    const int kv = job.cache.kv_heads;
    const int64_t tc = item / kv;
    const int head = (int)(item - tc * kv);
    const int tile_no = (int)(tc / job.chunks), chunk = (int)(tc - (int64_t)tile_no * job.chunks);
    Place at;
    // the last rows of a causal prompt see most: they begin first
    if (tile_no >= job.tiles || !find_rows<BM>(job, job.tiles - 1 - tile_no, at)) return;
    const int rows = at.nq * job.group, row = at.base + 32 * wave;

    // the chunk's share of the keys that the workgroup's rows see
    const int from = at.from + chunk * job.chunk, to = at.to > from + job.chunk ? from + job.chunk : at.to;
    // what the wave's rows see: some of them, all of them
    int any_lo = 0, any_hi = 0, all_lo = 0, all_hi = 0;
    if (row < rows) {
        const int last = (row + 32 < rows ? row + 32 : rows) - 1;
        const int p0 = at.len - at.nq + token_of(job, at, row), p1 = at.len - at.nq + token_of(job, at, last);
        any_lo = a.window ? p0 - a.window + 1 : 0;
        any_hi = a.causal && p1 + 1 < to ? p1 + 1 : to;
        all_lo = a.window ? p1 - a.window + 1 : 0;
        all_hi = a.causal && p0 + 1 < to ? p0 + 1 : to;
    }
    const TableRow table = (TableRow)(uintptr_t)(a.table + (int64_t)at.b * a.width);
    const int mine = row + (lane & 31);
    const bool there = mine < rows;
    const int token = there ? token_of(job, at, mine) : 0, of = there ? mine - token * job.group : 0;
    const RawQuery<D, 32> raw_q = load_query<D, 32>(job, there, at.q0 + token, head * job.group + of, lane);
    Raw<N> raw;
    if (from < to) load_tile<D, WAVES, N>(raw, job.cache, table, head, from, to, threadIdx.x);
    Query<D, 32> q;
    take_query<D, 32, F16, F16>(q, job, raw_q, lane);
    const int pos = at.len - at.nq + token;
    const int hi = !there ? 0 : a.causal ? (pos + 1 < at.len ? pos + 1 : at.len) : at.len;
    const int lo = a.window ? (pos - a.window + 1 > 0 ? pos - a.window + 1 : 0) : 0;
    Sums<D, EXACT> r;
    r.m = -INFINITY;
    r.l = r.w = 0.0f;
#pragma unroll
    for (int j = 0; j < D / 32; ++j)
#pragma unroll
        for (int e = 0; e < 16; ++e) r.o[j][e] = 0.0f;

    Range key_range{0.0f, 1.0f}, value_range{0.0f, 1.0f};
    // EXACT: p * step; else the elements themselves
    const auto prepare = [&](int k0, int half, float& key_grew, float& value_grew) {
        const bool there_k = k0 + lane < to;
        const float ks = __uint_as_float(raw.kp << 16), km = __uint_as_float(raw.kp & 0xffff0000u);
        const float vs = __uint_as_float(raw.vp << 16), vm = __uint_as_float(raw.vp & 0xffff0000u);
        const float kx = fmaf(8.0f, ks, fabsf(km)), vx = EXACT ? vs : fmaf(8.0f, vs, fabsf(vm));
        if constexpr (!EXACT) widen<15>(key_range, there_k && kx < 0x1p126f ? kx : 0.0f, key_grew);
        widen<EXACT ? 7 : 15>(value_range, there_k && vx < 0x1p126f ? vx : 0.0f, value_grew);
        unpack<D, WAVES, N, EXACT>(tiles[half], raw, k0, to, threadIdx.x, key_range, value_range);
    };
    float key_grew = 1.0f, value_grew = 1.0f;
    int half = 0;
    if (from < to) {
        prepare(from, 0, key_grew, value_grew);
        if (from + kTile < to) load_tile<D, WAVES, N>(raw, job.cache, table, head, from + kTile, to, threadIdx.x);
    }
    lds_barrier();
    for (int k0 = from; k0 < to; k0 += kTile) {
        // (the tile's own ranges: the next one may widen them)
        const float f = EXACT ? q.f : q.f / key_range.by;
        const float up = EXACT ? (value_range.limit > 0.0f ? __builtin_amdgcn_logf(value_range.by) : 0.0f) : 0.0f;
        value_grew = 1.0f;
        if (k0 + kTile < to) {
            prepare(k0 + kTile, half ^ 1, key_grew, value_grew);
            if (k0 + 2 * kTile < to) load_tile<D, WAVES, N>(raw, job.cache, table, head, k0 + 2 * kTile, to, threadIdx.x);
        }
        if (k0 < any_hi && k0 + kTile > any_lo) {
            if (k0 >= all_lo && k0 + kTile <= all_hi) take_tile<D, EXACT, false>(r, q, tiles[half], f, up, k0, lo, hi, lane);
            else take_tile<D, EXACT, true>(r, q, tiles[half], f, up, k0, lo, hi, lane);
        }
        if (value_grew != 1.0f) {                 // sums go on in the next tile's range
            scale_sums(r, value_grew);
            if constexpr (EXACT) {
                r.l *= value_grew;
                r.w *= value_grew;
            }
        }
        half ^= 1;
        lds_barrier();
    }
    if (!there) return;                           // (both lanes of the row)
    const float l = column_sum<32>(r.l), w = EXACT ? column_sum<32>(r.w) : 0.0f;
    const float by = (l > 0.0f ? 1.0f / l : (l == 0.0f ? 0.0f : l)) * (EXACT ? 1.0f : 1.0f / value_range.by);
    float lse = l == 0.0f ? -INFINITY : r.m + __builtin_amdgcn_logf(l);
    if constexpr (EXACT) lse -= value_range.limit > 0.0f ? __builtin_amdgcn_logf(value_range.by) : 0.0f;
    const int t_row = at.q0 + token, h_row = head * job.group + of;
    const int64_t part_row = ((int64_t)chunk * a.tokens + t_row) * a.heads + h_row;
    float* part = job.part + part_row * D;
    uint16_t* out = static_cast<uint16_t*>(a.o) + (int64_t)t_row * a.o_token + (int64_t)h_row * a.o_head;
    constexpr int B = D / 4 / 2;                  // fours of elements that the lane has
#pragma unroll
    for (int i = 0; i < B; ++i) {
        const int four = i % 4 + 8 * (i / 4) + 4 * (lane >> 5);
        float y[4];
#pragma unroll
        for (int e = 0; e < 4; ++e) y[e] = ((D == 128 ? r.o[e][i] : r.o[e / 2][e % 2 * 8 + i]) + w) * by;
        if (job.chunks > 1) *reinterpret_cast<f32x4*>(part + 4 * four) = f32x4{y[0], y[1], y[2], y[3]};
        else store_row<4, F16>(out + 4 * four, y, job.wide_o);
    }
    if (lane < 32) {
        if (job.chunks > 1) job.part[(int64_t)job.chunks * a.tokens * a.heads * D + part_row] = lse;
        else if (a.lse) a.lse[(int64_t)t_row * a.heads + h_row] = lse * kLn2;
    }
}

template <int D, int WAVES>
void launch(const KvJob& job, hipStream_t s) {
    const dim3 grid = group_grid((int64_t)job.tiles * job.cache.kv_heads * job.chunks, 64 * WAVES), block(64 * WAVES);
    if (job.a.dtype == RQ_F16) launch_kernel(k_kv4_prompt<D, WAVES, true>, grid, block, 0, s, job);
    else launch_kernel(k_kv4_prompt<D, WAVES, false>, grid, block, 0, s, job);
}

}  // namespace

void launch_prompt(const KvJob& job, int waves, hipStream_t s) {
    if (job.cache.head_dim == 128) waves == 8 ? launch<128, 8>(job, s) : launch<128, 4>(job, s);
    else waves == 8 ? launch<64, 8>(job, s) : launch<64, 4>(job, s);
}

}  // namespace rq
