// Attention over the 4-bit paged cache for many queries a sequence (prompts, chunks of them).  The mathematics is that of
// kernels_kv4_attention.hip, and so are rows and columns: products are taken transposed, a wave has 32 rows of its own as the
// columns of 32 x 32 products, column n the lanes n and n + 32.
//
// What is bound here is issue: a score costs a lane seven or eight instructions' time, as long as the matrix cores take for its 512
// operations, and codes that each wave unpacked for itself would cost as much again.  So the waves of a workgroup (4 or 8)
// unpack a tile of 64 keys together, once, into LDS as fp16 operands: keys [key][element], values transposed, [element][key], keys in
// the order in which scores leave the matrix cores, so that p enters them again as it is.  The next tile is unpacked into
// another part of LDS beside the products of keys on this one; its codes were loaded two steps earlier.
//   - bf16 results: operands are the elements themselves, (code - 7.5) step + mid, times a power of two that holds the largest
//     seen so far in fp16's range (rounded to fp16 once, 2^-11: less than the result's rounding; steps and centres, bf16, are exact in fp16).  Scores need no step or centre.
//   - fp16 results (EXACT): operands are codes - 7.5, which are exact, and steps and centres are applied to the scores as in the other
//     kernel; four instructions a score and one product more.  Queries are two fp16 numbers.
// A value row that is not finite becomes zeros and its key NaN: queries that do not see it stay what they are.
//
// 8192 tokens against themselves, 32 heads to 8 of keys, 128 elements: bf16 597 .. 625 us, 880 to 920 TFLOP/s of the products that a causal
// prompt needs (a large matrix product: 1360); fp16 864 .. 868.  A step of two waves a SIMD takes 4600 cycles: vector instructions
// take 4.5 each and exponentials 9.7, some 2600 of them, the issue of 64 products 500; the rest is waiting for each other (counters: vector
// issue 51 %, matrix cores 41 %, LDS 34 %).  Operands read two groups ahead, unpacking after and not beside the products: no faster.
#include "kv4_attention.h"

namespace rq {
namespace {

constexpr int kKeyPad = 8, kValueRow = kTile + 8;  // halfwords: rows of LDS begin 4 banks apart

template <int D, bool EXACT>
struct Tile {
    uint16_t k[kTile][D + kKeyPad];
    uint16_t v[D][kValueRow];                     // element d in row (d % 4) * D / 4 + d / 4
    float scale[EXACT ? 5 : 1][EXACT ? kTile : 4];  // EXACT: keys' steps and centres, values' steps and what their centres add
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

// The tile from k0 on, number n of `pages`.
template <int D, int WAVES, int N, bool PAGED>
__device__ __forceinline__ void load_tile(Raw<N>& t, const Kv4& c, int pages, int n, int head_at, int k0, int thread) {
    const int p = 1 << c.page_shift, lane = thread & 63;
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
        w = block + (uint32_t)(p * D + 4 * (at + (lane & 15)));
    } else {
        w = block_of<PAGED>(c, pages, n, 0, head_at) + (p * D + 4 * place_of(c, k0, 0)) + (uint32_t)(lane * 4);
    }
    t.kp = *reinterpret_cast<const uint32_t*>(w);
    t.vp = *reinterpret_cast<const uint32_t*>(w + 4 * p);
#pragma unroll
    for (int i = 0; i < N; ++i) {
        const int run = thread + 64 * WAVES * i;
        if (kRuns<D> % (64 * WAVES) != 0 && run >= kRuns<D>) break;
        // (a wave's 64 runs lie in one quarter)
        const int q = PAGED ? __builtin_amdgcn_readfirstlane(run / (kRuns<D> / 4)) : 0;
        const uint8_t* x = block_of<PAGED>(c, pages, n, q, head_at) + place_of(c, k0, q) * (D / 2) + (uint32_t)((PAGED ? run % (kRuns<D> / 4) : run) * 8);
        t.k[i] = *reinterpret_cast<const u32x2*>(x);
        t.v[i] = *reinterpret_cast<const u32x2*>(x + p * (D / 2));
    }
}

__device__ __forceinline__ uint32_t as_bits(f16x2 x) { return __builtin_bit_cast(uint32_t, x); }

// c - 7.5 of nibble J of both halves of a dword, exact: 64 + c less 71.5.
template <int J>
__device__ __forceinline__ f16x2 code_pair(uint32_t w, const CodeBits& bits) {
    const uint32_t x = J == 0 ? w << 4 : w >> (4 * J - 4);
    return as_f16(bits.high(x)) + f16x2{(_Float16)-71.5f, (_Float16)-71.5f};
}

// The powers of two in the operands: what has been seen so far is below 16 * `limit`.  (Sixteenths: those of all finite elements are finite.)
struct Range {
    float limit;
    int up;                                       // log2 of the factor, 2^UP / (16 * limit)
};
// Widens to hold 16 times the wave's `x`; by how much the factor's log2 changed.  UP: 15 for elements, whose fp16 then has full precision down
// to 2^-29 of the largest; 7 for steps, which meet factors of up to 2^8.
template <int UP>
__device__ __forceinline__ int widen(Range& r, float x) {
#pragma unroll
    for (int w = 1; w < 64; w *= 2) x = fmaxf(x, __shfl_xor(x, w));
    int e = (int)(__float_as_uint(x) >> 23) - 126;                   // x < 2^e
    e = __builtin_amdgcn_readfirstlane(e < -64 ? -64 : e);
    const float limit = __uint_as_float((uint32_t)(e + 127) << 23);
    if (!(limit > r.limit)) return 0;
    const int up = UP - 4 - e, by = up - r.up;
    r.limit = limit;
    r.up = up;
    return by;
}

// log2 of the factor in the probabilities of bf16 results, which are rounded to fp16: at most 2^15 of them where one has grown to 2^8, and
// down to 2^-21 of the largest in full precision (without the factor keys 2^-25 below it, of which long sequences have many, were lost).
constexpr float kUp = 7.0f;

template <int D, bool EXACT>
struct Sums {
    float m, l, w;                                // maximum (log2), sums over the lane's keys of p and, EXACT, of what centres add
    float __attribute__((ext_vector_type(16))) o[D / 32];
};
template <int D, bool EXACT>
__device__ __forceinline__ void scale_sums(Sums<D, EXACT>& r, float by) {
#pragma unroll
    for (int j = 0; j < D / 32; ++j)
#pragma unroll
        for (int e = 0; e < 16; ++e) r.o[j][e] *= by;
}

// A tile's parameters, a key a lane: steps and centres.
struct Parameters {
    float ks, km, vs, vm;
};
// Ranges widen to hold them.
template <int D, bool EXACT>
__device__ __forceinline__ Parameters take_parameters(Tile<D, EXACT>& to, uint32_t kp, uint32_t vp, int thread, Range& keys, Range& values, int& grew, bool& far) {
    Parameters p{__uint_as_float(kp << 16), __uint_as_float(kp & 0xffff0000u), __uint_as_float(vp << 16), __uint_as_float(vp & 0xffff0000u)};
    if (!finite(p.vs) || !finite(p.vm)) {
        p.vs = p.vm = 0.0f;
        p.ks = __builtin_nanf("");
    }
    // sixteenths of the largest element that a row could have, EXACT: of the step, and 2^-64 of a centre that goes with p
    const Centre c = EXACT ? split_centre(p.vs, p.vm) : Centre{0.0f, 0.0f};
    float kx = EXACT ? 0.0f : fmaf(0.5f, p.ks, 0.0625f * fabsf(p.km));
    const float vx = EXACT ? 0.0625f * fmaxf(p.vs, 0x1p-64f * fabsf(c.with_p)) : fmaf(0.5f, p.vs, 0.0625f * fabsf(p.vm));
    kx = kx < INFINITY ? kx : 0.0f;               // (keys may be infinite or NaN)
    grew = 0;
    if (__any(kx > keys.limit || vx > values.limit)) {
        if (!EXACT) widen<15>(keys, kx);
        grew = widen<EXACT ? 7 : 15>(values, vx);
    }
    if constexpr (EXACT) {
        // (a wave an array: all of them hold the parameters)
        const int lane = thread & 63;
        if (thread >> 6 == 0) to.scale[0][lane] = p.ks;
        if (thread >> 6 == 1) to.scale[1][lane] = p.km;
        if (thread >> 6 == 2) to.scale[2][lane] = __builtin_amdgcn_ldexpf(p.vs, values.up);
        if (thread >> 6 == 3) put_centre(to.scale[3], lane, c.with_step);
        if (thread >> 6 == 0) to.scale[4][lane] = __builtin_amdgcn_ldexpf(c.with_p, values.up);
        far = __any(c.with_p != 0.0f);
    }
    return p;
}

// What a thread needs of them to unpack its runs.
template <int N>
struct Factors {
    f16x2 key[N], value[N][4];                    // step and centre
};
template <int D, int WAVES, int N, bool EXACT>
__device__ __forceinline__ Factors<N> factors_of(const Parameters& p, int thread, const Range& keys, const Range& values) {
    Factors<N> f{};
    if constexpr (!EXACT) {
        const int kw = (int)pack_f16(__builtin_amdgcn_ldexpf(p.ks, keys.up), __builtin_amdgcn_ldexpf(p.km, keys.up));
        const int vw = (int)pack_f16(__builtin_amdgcn_ldexpf(p.vs, values.up), __builtin_amdgcn_ldexpf(p.vm, values.up));
#pragma unroll
        for (int i = 0; i < N; ++i) {
            const int run = thread + 64 * WAVES * i;
            f.key[i] = as_f16((uint32_t)__builtin_amdgcn_ds_bpermute(4 * (run / (D / 16) & 63), kw));
#pragma unroll
            for (int e = 0; e < 4; ++e) f.value[i][e] = as_f16((uint32_t)__builtin_amdgcn_ds_bpermute(4 * ((4 * (run / (D / 4)) + e) & 63), vw));
        }
    }
    return f;
}

// A thread's runs on their way into LDS, in four pieces of alike length that stand beside matrix products.
template <int N>
struct Unpacked {
    f16x2 k[N][2][4], v[N][4][2];
};
template <int PIECE, int D, int WAVES, int N, bool EXACT>
__device__ __forceinline__ void unpack(Unpacked<N>& x, Tile<D, EXACT>& to, const Raw<N>& t, const Factors<N>& f, int thread, const CodeBits& bits) {
#pragma unroll
    for (int i = 0; i < N; ++i) {
        const int run = thread + 64 * WAVES * i;
        if (kRuns<D> % (64 * WAVES) != 0 && run >= kRuns<D>) break;
        const int key = run / (D / 16), at = run % (D / 16) * 16;    // keys: a run is 16 elements of one key
        const int four = run / (D / 4), x4 = run % (D / 4);          // values: four elements of four tokens
        // keys 16 s + 4 q + 0 .. 3 go to places 16 s + 8 (q % 2) + 4 (q / 2) + 0 .. 3
        const int place = (four & ~3) * 4 + 8 * (four & 1) + 4 * (four >> 1 & 1);
        if constexpr (PIECE == 0) {
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                x.k[i][h][0] = code_pair<0>(t.k[i][h], bits);
                x.k[i][h][1] = code_pair<1>(t.k[i][h], bits);
                x.k[i][h][2] = code_pair<2>(t.k[i][h], bits);
                x.k[i][h][3] = code_pair<3>(t.k[i][h], bits);
            }
        }
        if constexpr (PIECE == 1) {
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                if constexpr (!EXACT)
#pragma unroll
                    for (int e = 0; e < 4; ++e)
                        x.k[i][h][e] = __builtin_elementwise_fma(x.k[i][h][e], f16x2{f.key[i][0], f.key[i][0]}, f16x2{f.key[i][1], f.key[i][1]});
                *reinterpret_cast<u32x4*>(&to.k[key][at + 8 * h]) = u32x4{as_bits(x.k[i][h][0]), as_bits(x.k[i][h][1]), as_bits(x.k[i][h][2]), as_bits(x.k[i][h][3])};
            }
        }
        if constexpr (PIECE == 1 || PIECE == 2) {
            constexpr int h = PIECE - 1;
            x.v[i][0][h] = code_pair<0>(t.v[i][h], bits);
            x.v[i][1][h] = code_pair<1>(t.v[i][h], bits);
            x.v[i][2][h] = code_pair<2>(t.v[i][h], bits);
            x.v[i][3][h] = code_pair<3>(t.v[i][h], bits);
        }
        if constexpr (PIECE == 3) {
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                if constexpr (!EXACT)
#pragma unroll
                    for (int h = 0; h < 2; ++h)
                        x.v[i][e][h] = __builtin_elementwise_fma(x.v[i][e][h], f16x2{f.value[i][2 * h][0], f.value[i][2 * h + 1][0]},
                                                                 f16x2{f.value[i][2 * h][1], f.value[i][2 * h + 1][1]});
                *reinterpret_cast<u32x2*>(&to.v[e * (D / 4) + x4][place]) = u32x2{as_bits(x.v[i][e][0]), as_bits(x.v[i][e][1])};
            }
        }
    }
}

typedef float f32x16 __attribute__((ext_vector_type(16)));

// Operands come from LDS a group of products ahead of their use.  The compiler would rather read each right before its product, in
// few registers, and wait for LDS every time: nothing moves over RQ_FENCE, and in a group the reads come first, then products
// with vector instructions between them.
constexpr int kValu = 0x2, kMfma = 0x8, kLdsRead = 0x100;
#define RQ_FENCE() __builtin_amdgcn_sched_barrier(0)
#define RQ_NEXT(kind, n) __builtin_amdgcn_sched_group_barrier(kind, n, 0)

// Scores of a tile: products of 32 keys each with the wave's queries, before steps and centres; beside them the next tile is unpacked.
template <int D, int WAVES, int N, bool EXACT>
__device__ __forceinline__ void take_keys(f32x16 (&s)[2], const Query<D, 32>& q, const Tile<D, EXACT>& t, Tile<D, EXACT>& to, const Raw<N>& raw,
                                          const Factors<N>& f, int thread, const CodeBits& bits) {
    const int n = thread & 31, h = thread >> 5 & 1;
    constexpr int G = D / 32;                     // groups: of two steps of 16 elements, two blocks of 32 keys
    f16x8 a[2][2][2];
    Unpacked<N> x;
    const auto read = [&](int g) {
#pragma unroll
        for (int j = 0; j < 2; ++j)
#pragma unroll
            for (int i = 0; i < 2; ++i) a[g % 2][j][i] = *reinterpret_cast<const f16x8*>(&t.k[32 * i + n][h * (D / 2) + 8 * (2 * g + j)]);
    };
    read(0);
    s[0] = s[1] = f32x16{};
#pragma unroll
    for (int g = 0; g < G; ++g) {
        RQ_FENCE();
        if (g + 1 < G) read(g + 1);
        if (g == 0) {
            unpack<0, D, WAVES>(x, to, raw, f, thread, bits);
            if (G == 2) unpack<1, D, WAVES>(x, to, raw, f, thread, bits);
        } else if (g == 1) {
            unpack<G == 2 ? 2 : 1, D, WAVES>(x, to, raw, f, thread, bits);
            if (G == 2) unpack<3, D, WAVES>(x, to, raw, f, thread, bits);
        } else if (g == 2) {
            unpack<2, D, WAVES>(x, to, raw, f, thread, bits);
        } else {
            unpack<3, D, WAVES>(x, to, raw, f, thread, bits);
        }
#pragma unroll
        for (int j = 0; j < 2; ++j)
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                s[i] = __builtin_amdgcn_mfma_f32_32x32x16_f16(a[g % 2][j][i], q.hi[2 * g + j], s[i], 0, 0, 0);
                if constexpr (EXACT) s[i] = __builtin_amdgcn_mfma_f32_32x32x16_f16(a[g % 2][j][i], q.lo[2 * g + j], s[i], 0, 0, 0);
            }
        RQ_NEXT(kLdsRead, 4);
#pragma unroll
        for (int i = 0; i < (EXACT ? 8 : 4); ++i) {
            RQ_NEXT(kMfma, 1);
            RQ_NEXT(kValu, 6);
        }
    }
    RQ_FENCE();
}

// Scores to probabilities, and their products with the values.
template <int D, bool EXACT>
__device__ __forceinline__ void take_scores(Sums<D, EXACT>& r, f32x16 (&s)[2], const Query<D, 32>& q, const Tile<D, EXACT>& t, float f, bool far, int k0,
                                            bool whole, int lo, int seen, int lane) {
    const int n = lane & 31, h = lane >> 5;
    constexpr int J = D / 32;
    f16x8 a[2][J];
    const auto read = [&](int g) {                // values of 16 keys
#pragma unroll
        for (int j = 0; j < J; ++j) a[g % 2][j] = *reinterpret_cast<const f16x8*>(&t.v[32 * j + n][16 * g + 8 * h]);
    };
    read(0);
    RQ_FENCE();
    if constexpr (EXACT) {
#pragma unroll
        for (int i = 0; i < 2; ++i)
#pragma unroll
            for (int e = 0; e < 16; e += 4) {
                const int key = 32 * i + 2 * e + 4 * h;
                const f32x4 step = *reinterpret_cast<const f32x4*>(&t.scale[0][key]), mid = *reinterpret_cast<const f32x4*>(&t.scale[1][key]);
#pragma unroll
                for (int u = 0; u < 4; ++u) s[i][e + u] = fmaf(step[u], s[i][e + u], mid[u] * (q.even + q.odd));
            }
    }
    if (!whole) {
        const int from = k0 + 4 * h - lo;
#pragma unroll
        for (int i = 0; i < 2; ++i)
#pragma unroll
            for (int e = 0; e < 16; ++e) s[i][e] = (uint32_t)(from + 32 * i + 8 * (e / 4) + e % 4) < (uint32_t)seen ? s[i][e] : -INFINITY;
    }
    float mx = -INFINITY;
#pragma unroll
    for (int i = 0; i < 2; ++i)
#pragma unroll
        for (int e = 0; e < 16; e += 2) mx = fmaxf(fmaxf(mx, s[i][e]), s[i][e + 1]);
    mx = f * column_max<32>(mx);
    // p may grow to 2^8 before the sums are scaled to a new maximum
    if (__builtin_expect(__any(mx - r.m > 8.0f) || (EXACT && far), 0)) {
        const float to = fmaxf(r.m, mx), by = to == -INFINITY ? 1.0f : __builtin_amdgcn_exp2f(r.m - to);
        scale_sums(r, by);
        r.l *= by;
        r.w *= by;
        r.m = to;
        if (EXACT && far) {                       // (rare: these exponentials are taken again below)
            const float off = to == -INFINITY ? 0.0f : to;
#pragma unroll
            for (int i = 0; i < 2; ++i)
#pragma unroll
                for (int e = 0; e < 16; e += 4) {
                    const f32x4 with_p = *reinterpret_cast<const f32x4*>(&t.scale[4][32 * i + 2 * e + 4 * h]);
#pragma unroll
                    for (int u = 0; u < 4; ++u) r.w = fmaf(__builtin_amdgcn_exp2f(fmaf(f, s[i][e + u], -off)), with_p[u], r.w);
                }
        }
    }
    const float off = (r.m == -INFINITY ? 0.0f : r.m) - (EXACT ? 0.0f : kUp);
    // sixteen keys at a time, the next ones' probabilities beside the products of these
    uint32_t p[2][4];
    const auto weigh = [&](int g) {
#pragma unroll
        for (int v = 0; v < 2; ++v) {
            const int at = 8 * (g % 2) + 4 * v, key = 32 * (g / 2) + 2 * at + 4 * h;
            f32x4 step;
            u32x4 with_step;
            if constexpr (EXACT) {
                step = *reinterpret_cast<const f32x4*>(&t.scale[2][key]);
                with_step = *reinterpret_cast<const u32x4*>(&t.scale[3][key]);
            }
            float x[4];
#pragma unroll
            for (int u = 0; u < 4; ++u) {
                x[u] = __builtin_amdgcn_exp2f(fmaf(f, s[g / 2][at + u], -off));
                if constexpr (EXACT) {
                    r.l += x[u];
                    x[u] *= step[u];
                }
            }
            p[g % 2][2 * v] = pack_f16(x[0], x[1]);
            p[g % 2][2 * v + 1] = pack_f16(x[2], x[3]);
            if constexpr (EXACT)
#pragma unroll
                for (int u = 0; u < 4; ++u) r.w = add_centre(p[g % 2][2 * v + u % 2], with_step[u], r.w);
            if constexpr (!EXACT) {               // (of what the products see: two an instruction)
                const f16x2 one{(_Float16)1.0f, (_Float16)1.0f};
                r.l = __builtin_amdgcn_fdot2(as_f16(p[g % 2][2 * v]), one, r.l, false);
                r.l = __builtin_amdgcn_fdot2(as_f16(p[g % 2][2 * v + 1]), one, r.l, false);
            }
        }
    };
    weigh(0);
#pragma unroll
    for (int g = 0; g < 4; ++g) {
        RQ_FENCE();
        if (g < 3) {
            read(g + 1);
            weigh(g + 1);
        }
        const f16x8 b = __builtin_bit_cast(f16x8, u32x4{p[g % 2][0], p[g % 2][1], p[g % 2][2], p[g % 2][3]});
#pragma unroll
        for (int j = 0; j < J; ++j) r.o[j] = __builtin_amdgcn_mfma_f32_32x32x16_f16(a[g % 2][j], b, r.o[j], 0, 0, 0);
        if (g < 3) {
            RQ_NEXT(kLdsRead, EXACT ? J + 4 : J);
#pragma unroll
            for (int j = 0; j < J; ++j) {
                RQ_NEXT(kMfma, 1);
                RQ_NEXT(kValu, (EXACT ? 44 : 24) / J);
            }
        }
    }
    RQ_FENCE();
}

// A barrier for what lies in LDS: loads from memory stay under way.
__device__ __forceinline__ void lds_barrier() {
    __builtin_amdgcn_fence(__ATOMIC_RELEASE, "workgroup", "local");
    __builtin_amdgcn_s_barrier();
    __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "workgroup", "local");
}

// What a wave of the second group hands to its counterpart of the first, a lane's words side by side.
template <int D>
struct Handed {
    float o[D / 2][64], m[64], l[64], w[64];
    int up[64];
};

// GROUPS: 2 where a workgroup's rows are few: two groups of WAVES waves have the same rows and take turns at the tiles, each with tiles of
// its own in LDS, and the second hands its sums to the first at the end.
template <int D, int WAVES, int GROUPS, bool F16, bool PAGED>
__global__ __launch_bounds__(64 * WAVES * GROUPS, 2) void k_kv4_prompt(KvJob job) {
    constexpr bool EXACT = F16;
    constexpr int BM = 32 * WAVES, N = (kRuns<D> + 64 * WAVES - 1) / (64 * WAVES);
    // Eight waves are two groups, four SIMDs each, half a step apart: one has products of keys and unpacks while the other has
    // exponentials.  Three tiles then, since the one group still reads values of the last while the other unpacks the next.
    constexpr bool TWO = WAVES == 8;
    constexpr int TILES = WAVES == 8 ? 3 : 2;
    constexpr int kStride = GROUPS * kTile;       // from a group's tile to its next
    __shared__ __attribute__((aligned(16))) Tile<D, EXACT> all_tiles[GROUPS][TILES];
    const Kv4Attention& a = job.a;
    const int lane = threadIdx.x & 63, of_all = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int half = GROUPS == 1 ? 0 : of_all / WAVES, wave = of_all - half * WAVES, thread = GROUPS == 1 ? threadIdx.x : 64 * wave + lane;
    Tile<D, EXACT>* tiles = all_tiles[half];
    const int head = blockIdx.x, item = item_number();
    const int tile_no = job.chunks == 1 ? item : item / job.chunks, chunk = item - tile_no * job.chunks;
    const CodeBits bits;
    Place at;
    // the last rows of a causal prompt see most: they begin first
    if (tile_no >= job.tiles || !find_rows<BM>(job, job.tiles - 1 - tile_no, at)) return;
    find_keys<BM>(job, at, a.kv_lens[at.b]);
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
    const int32_t* table = a.table + (int64_t)at.b * a.width;
    const int mine = row + (lane & 31);
    const bool there = mine < rows;
    const int token = there ? token_of(job, at, mine) : 0, of = there ? mine - token * job.group : 0;
    const RawQuery<D, 32> raw_q = load_query<D, 32>(job, there, at.q0 + token, head * job.group + of, lane);
    const int head_at = head * ((D + 8) << job.cache.page_shift);
    int pages = 0, page_no = 0, asked = from + half * kTile;   // the tile asked for last, its number among those of `pages`
    Raw<N> raw, later;                            // the next tile, the one after it
    if (from < to) {
        pages = load_pages<PAGED>(job, table, asked, kStride, lane);
        load_tile<D, WAVES, N, PAGED>(raw, job.cache, pages, 0, head_at, asked, thread);
        if (asked + kStride < to) {
            asked += kStride;
            page_no = 1;
        }
        load_tile<D, WAVES, N, PAGED>(later, job.cache, pages, page_no, head_at, asked, thread);
    }
    Query<D, 32> q;
    take_query<D, 32, F16, F16>(q, job, raw_q, lane);
    // all that was asked for is here by now: said once, it is not waited for by name in every step (vmcnt(0); other counts stay)
    __builtin_amdgcn_s_waitcnt(0x0f70);
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

    const int seen = hi > lo ? hi - lo : 0;

    Range keys{0.0f, 0}, values{0.0f, 0};
    int at_tile = TILES - 1;                      // the tile in hand
    if (TWO && of_all >= 4) lds_barrier();
    // a step unpacks the next tile and takes this one; the first has none to take
    bool far = false;                             // EXACT: some centre of the tile in hand goes with p
    // (two steps a pass, each with registers of its own for what is under way: copies would wait for it.  A tile is asked for in
    // every step, the last one again at the end: where a load may be left out, what was loaded before it is waited for with all else.)
    const auto step = [&](int k0, Raw<N>& raw) {
        Tile<D, EXACT>& now = tiles[at_tile];
        at_tile = at_tile == TILES - 1 ? 0 : at_tile + 1;
        Tile<D, EXACT>& then = tiles[at_tile];
        const bool mine_too = k0 >= from && k0 < any_hi && k0 + kTile > any_lo;
        const int next = k0 + kStride;
        // (the tile's own ranges: the next one may widen them; neither infinite nor 0, so that a score of 0 stays 0 beside a key of 2^127
        // and one of -infinity what it is where queries and keys are tiny)
        const float f = EXACT ? q.f : __builtin_amdgcn_fmed3f(__builtin_amdgcn_ldexpf(q.f, -keys.up), 0x1p-126f, 0x1p127f);
        const bool there = next + lane < to;
        int grew;
        bool far_next = false;
        const Parameters of_next = take_parameters<D, EXACT>(then, there ? raw.kp : 0u, there ? raw.vp : 0u, thread, keys, values, grew, far_next);
        f32x16 s[2];
        if (mine_too) {
            const Factors<N> factors = factors_of<D, WAVES, N, EXACT>(of_next, thread, keys, values);
            take_keys<D, WAVES, N, EXACT>(s, q, now, then, raw, factors, thread, bits);         // (where there is no next tile, `then` is not read)
        } else {
            const Factors<N> factors = factors_of<D, WAVES, N, EXACT>(of_next, thread, keys, values);
            Unpacked<N> x;
            unpack<0, D, WAVES>(x, then, raw, factors, thread, bits);
            unpack<1, D, WAVES>(x, then, raw, factors, thread, bits);
            unpack<2, D, WAVES>(x, then, raw, factors, thread, bits);
            unpack<3, D, WAVES>(x, then, raw, factors, thread, bits);
        }
        if (asked + kStride < to) {
            asked += kStride;
            if (++page_no == kPagesOf<PAGED>) {
                pages = load_pages<PAGED>(job, table, asked, kStride, lane);
                page_no = 0;
            }
        }
        load_tile<D, WAVES, N, PAGED>(raw, job.cache, pages, page_no, head_at, asked, thread);
        if constexpr (TWO) {                      // (products of keys go first where both groups have something to issue: 1 %)
            lds_barrier();
            __builtin_amdgcn_s_setprio(0);
        }
        if (mine_too) take_scores<D, EXACT>(r, s, q, now, f, far, k0, k0 >= all_lo && k0 + kTile <= all_hi, lo, seen, lane);
        far = far_next;
        if (grew != 0) {                          // sums go on in the next tile's range
            const float by = __builtin_amdgcn_ldexpf(1.0f, grew);
            scale_sums(r, by);
            if constexpr (EXACT) r.w *= by;
        }
        lds_barrier();
        if constexpr (TWO) __builtin_amdgcn_s_setprio(1);
    };
    for (int k0 = from - kStride; from < to && k0 < to; k0 += 2 * kStride) {
        step(k0 + half * kTile, raw);
        step(k0 + half * kTile + kStride, later); // (where there is no such tile nothing is taken)
    }
    if (TWO && of_all < 4) lds_barrier();
    if constexpr (GROUPS == 2) {
        static_assert(sizeof(all_tiles) >= WAVES * sizeof(Handed<D>), "what is handed over takes the tiles' place");
        Handed<D>& h = reinterpret_cast<Handed<D>*>(all_tiles)[wave];
        if (half == 1) {
#pragma unroll
            for (int j = 0; j < D / 32; ++j)
#pragma unroll
                for (int e = 0; e < 16; ++e) h.o[16 * j + e][lane] = r.o[j][e];
            h.m[lane] = r.m;
            h.l[lane] = r.l;
            h.w[lane] = r.w;
            h.up[lane] = values.up;
        }
        lds_barrier();
        if (half == 1) return;
        // the smaller of the factors: neither side's sums overflow by it
        const int theirs = __builtin_amdgcn_readfirstlane(h.up[lane]);
        const int up = values.up < theirs ? values.up : theirs;
        const float m = fmaxf(r.m, h.m[lane]);
        const float x = m == -INFINITY ? 0.0f : __builtin_amdgcn_exp2f(r.m - m), y = m == -INFINITY ? 0.0f : __builtin_amdgcn_exp2f(h.m[lane] - m);
        const float xo = x * __builtin_amdgcn_ldexpf(1.0f, up - values.up), yo = y * __builtin_amdgcn_ldexpf(1.0f, up - theirs);
        r.l = fmaf(y, h.l[lane], x * r.l);
        r.w = fmaf(yo, h.w[lane], xo * r.w);
        r.m = m;
        values.up = up;
#pragma unroll
        for (int j = 0; j < D / 32; ++j)
#pragma unroll
            for (int e = 0; e < 16; ++e) r.o[j][e] = fmaf(yo, h.o[16 * j + e][lane], xo * r.o[j][e]);
    }
    if (!there) return;                           // (both lanes of the row)
    const float l = column_sum<32>(r.l), w = EXACT ? column_sum<32>(r.w) : 0.0f;
    const float by = __builtin_amdgcn_ldexpf(l > 0.0f ? 1.0f / l : (l == 0.0f ? 0.0f : l), -values.up);
    float lse = l == 0.0f ? -INFINITY : r.m + __builtin_amdgcn_logf(l);
    if constexpr (!EXACT) lse -= kUp;
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

template <int D, int WAVES, int GROUPS>
void launch(const KvJob& job, hipStream_t s) {
    const dim3 grid = item_grid(job.cache.kv_heads, (int64_t)job.tiles * job.chunks), block(64 * WAVES * GROUPS);
    const bool paged = job.cache.page_shift < 6;
    if constexpr (D == 64 || GROUPS == 1)
        if (job.a.dtype == RQ_F16) {
            launch_kernel(paged ? k_kv4_prompt<D, WAVES, GROUPS, true, true> : k_kv4_prompt<D, WAVES, GROUPS, true, false>, grid, block, 0, s, job);
            return;
        }
    if (paged) launch_kernel(k_kv4_prompt<D, WAVES, GROUPS, false, true>, grid, block, 0, s, job);
    else launch_kernel(k_kv4_prompt<D, WAVES, GROUPS, false, false>, grid, block, 0, s, job);
}
template <int D>
void launch(const KvJob& job, int waves, int groups, hipStream_t s) {
    if (waves == 8) launch<D, 8, 1>(job, s);
    else if (groups == 2) launch<D, 4, 2>(job, s);
    else launch<D, 4, 1>(job, s);
}

}  // namespace

void launch_prompt(const KvJob& job, int waves, int groups, hipStream_t s) {
    if (job.cache.head_dim == 128) launch<128>(job, waves, groups, s);
    else launch<64>(job, waves, groups, s);
}

}  // namespace rq
