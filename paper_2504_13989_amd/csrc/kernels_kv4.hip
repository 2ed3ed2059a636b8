// The 4-bit paged cache (kv4_layout.h): rows written, rows read back, pages copied.
//
// append: y = H x / sqrt(d) for keys (x itself for values, whose rotation sits in the weights), and per row
//   lo = clip * min(y), hi = clip * max(y), step = bf16((hi - lo) / 15), centre = bf16((hi + lo) / 2),
//   code = clamp(rne((y - centre) / step + 7.5), 0, 15);
// in fp32, every operation rounded by itself, so that a row's bytes do not depend on the call it came with.
#include "kv4_layout.h"
#include "wave_common.h"

#pragma clang fp contract(off)

namespace rq {
namespace {

constexpr int kThreads = 256;
constexpr float kFlat = 0x1p-100f;                // steps below are stored as 0: the row is its centre

// A lane holds 16 elements of a row: 8 c + 0 .. 7 and D / 2 + 8 c + 0 .. 7, c its number among the row's lanes.
constexpr int E = 16;

// Eight elements each from `at` on and `half` further.  DT: RQ_BF16, RQ_F32, RQ_F16.  ALIGNED: 16-byte loads.  (Rows are read once: past
// the caches.)
template <int DT, bool ALIGNED>
__device__ __forceinline__ void load_row(const void* X, int64_t at, int half, float (&x)[E]) {
    constexpr int W = DT == RQ_F32 ? 8 : 4, size = DT == RQ_F32 ? 4 : 2;   // dwords of eight
    uint32_t w[2][W];
#pragma unroll
    for (int h = 0; h < 2; ++h) {
        const char* p = static_cast<const char*>(X) + (at + h * half) * size;
        if constexpr (ALIGNED) {
#pragma unroll
            for (int i = 0; i < W / 4; ++i) {
                const u32x4 a = __builtin_nontemporal_load(reinterpret_cast<const u32x4*>(p) + i);
#pragma unroll
                for (int j = 0; j < 4; ++j) w[h][4 * i + j] = a[j];
            }
        } else if constexpr (DT == RQ_F32) {
#pragma unroll
            for (int i = 0; i < W; ++i) w[h][i] = reinterpret_cast<const uint32_t*>(p)[i];
        } else {
            const uint16_t* u = reinterpret_cast<const uint16_t*>(p);
#pragma unroll
            for (int i = 0; i < W; ++i) w[h][i] = (uint32_t)u[2 * i] | ((uint32_t)u[2 * i + 1] << 16);
        }
    }
#pragma unroll
    for (int h = 0; h < 2; ++h)
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            if constexpr (DT == RQ_F32) x[8 * h + i] = __uint_as_float(w[h][i]);
            else if constexpr (DT == RQ_F16) x[8 * h + i] = (float)__builtin_bit_cast(_Float16, (uint16_t)(i % 2 ? w[h][i / 2] >> 16 : w[h][i / 2]));
            else x[8 * h + i] = __uint_as_float(i % 2 ? w[h][i / 2] & 0xffff0000u : w[h][i / 2] << 16);
        }
}

__device__ __forceinline__ uint32_t bf16_bits(float x) { return (uint32_t)__builtin_bit_cast(uint16_t, (__bf16)x); }

template <int DT>
__device__ __forceinline__ void store_row(void* Y, int64_t at, int half, const float (&y)[E]) {
#pragma unroll
    for (int h = 0; h < 2; ++h) {
        const float* x = y + 8 * h;
        if constexpr (DT == RQ_F32) {             // (32 bytes a lane: left to the caches to put together)
            f32x4* p = reinterpret_cast<f32x4*>(static_cast<float*>(Y) + at + h * half);
            p[0] = f32x4{x[0], x[1], x[2], x[3]};
            p[1] = f32x4{x[4], x[5], x[6], x[7]};
        } else {
            u32x4 w;
#pragma unroll
            for (int i = 0; i < 4; ++i)
                w[i] = DT == RQ_F16 ? (uint32_t)__builtin_bit_cast(uint16_t, (_Float16)x[2 * i]) | ((uint32_t)__builtin_bit_cast(uint16_t, (_Float16)x[2 * i + 1]) << 16)
                                    : bf16_bits(x[2 * i]) | (bf16_bits(x[2 * i + 1]) << 16);
            __builtin_nontemporal_store(w, reinterpret_cast<u32x4*>(static_cast<uint16_t*>(Y) + at + h * half));
        }
    }
}

// A wave's rows lie over D / 16 lanes each: the lanes of a row are those that differ in bits 0, 1 and (D = 128) 3 of their number, which
// a DPP operand crosses in one instruction, and the tokens are numbered by the other bits.
template <int D>
constexpr int kTokens = 1024 / D;                 // of a wave
template <int D>
__device__ __forceinline__ int part_of(int lane) { return D == 128 ? (lane & 3) | (lane >> 1 & 4) : lane & 3; }
template <int D>
__device__ __forceinline__ int token_in_wave(int lane) { return D == 128 ? (lane >> 2 & 1) | (lane >> 3 & 6) : lane >> 2; }

// Butterflies across the lanes of a row: x <- x + sign * partner's x, sign = -1 on the upper lane of a pair.  The upper lane thus has
// b - a and not a - b; these signs commute with the later stages and come off with the scale.  (A DPP read needs two wait
// states after the write of its source: the s_nop before the first, seven instructions between a value's stages.)
template <int D>
__device__ __forceinline__ void cross_lanes(float (&x)[E], int at, float s0, float s1, float s2) {
#define RQ_STAGE(S, PERM)                                                                                                       \
    "v_fmac_f32_dpp %0, %0, " S " " PERM "\n\tv_fmac_f32_dpp %1, %1, " S " " PERM "\n\t"                                        \
    "v_fmac_f32_dpp %2, %2, " S " " PERM "\n\tv_fmac_f32_dpp %3, %3, " S " " PERM "\n\t"                                        \
    "v_fmac_f32_dpp %4, %4, " S " " PERM "\n\tv_fmac_f32_dpp %5, %5, " S " " PERM "\n\t"                                        \
    "v_fmac_f32_dpp %6, %6, " S " " PERM "\n\tv_fmac_f32_dpp %7, %7, " S " " PERM "\n\t"
#define RQ_EIGHT                                                                                                                \
    "+&v"(x[at]), "+&v"(x[at + 1]), "+&v"(x[at + 2]), "+&v"(x[at + 3]), "+&v"(x[at + 4]), "+&v"(x[at + 5]), "+&v"(x[at + 6]), "+&v"(x[at + 7])
    if constexpr (D == 128)
        asm("s_nop 1\n\t" RQ_STAGE("%8", "quad_perm:[1,0,3,2] row_mask:0xf bank_mask:0xf") RQ_STAGE("%9", "quad_perm:[2,3,0,1] row_mask:0xf bank_mask:0xf")
                RQ_STAGE("%10", "row_ror:8 row_mask:0xf bank_mask:0xf") "s_nop 1"
            : RQ_EIGHT
            : "v"(s0), "v"(s1), "v"(s2));
    else
        asm("s_nop 1\n\t" RQ_STAGE("%8", "quad_perm:[1,0,3,2] row_mask:0xf bank_mask:0xf") RQ_STAGE("%9", "quad_perm:[2,3,0,1] row_mask:0xf bank_mask:0xf") "s_nop 1"
            : RQ_EIGHT
            : "v"(s0), "v"(s1));
#undef RQ_STAGE
#undef RQ_EIGHT
}

// H x / sqrt(d): butterflies over strides 1, 2, 4 in the lane, 8 to d / 4 across lanes, d / 2 in the lane.  Most of the scale comes
// first, a power of two and so exact: sums do not overflow where the results are far from it.
template <int D>
__device__ __forceinline__ void rotate_row(float (&x)[E], int part) {
#pragma unroll
    for (int i = 0; i < E; i += 2) {
        const float a = x[i] * 0.125f, b = x[i + 1];
        x[i] = fmaf(b, 0.125f, a);
        x[i + 1] = fmaf(b, -0.125f, a);
    }
    const auto stage = [&](int w) {
#pragma unroll
        for (int i = 0; i < E; ++i)
            if (!(i & w)) {
                const float a = x[i], b = x[i + w];
                x[i] = a + b;
                x[i + w] = a - b;
            }
    };
    stage(2);
    stage(4);
    const float s0 = part & 1 ? -1.0f : 1.0f, s1 = part & 2 ? -1.0f : 1.0f, s2 = part & 4 ? -1.0f : 1.0f;
    cross_lanes<D>(x, 0, s0, s1, s2);
    cross_lanes<D>(x, 8, s0, s1, s2);
    stage(8);
    const float by = (D == 128 ? 8 * 0.08838834764831845f : 1.0f) * (__builtin_popcount((unsigned)part) & 1 ? -1.0f : 1.0f);
#pragma unroll
    for (int i = 0; i < E; ++i) x[i] *= by;
}

// The least and the largest of a row, NaN where it has one.
template <int D, bool MOST>
__device__ __forceinline__ float row_extreme(const float (&y)[E]) {
    const auto of = [](float a, float b) { return MOST ? __builtin_elementwise_maximum(a, b) : __builtin_elementwise_minimum(a, b); };
    float m = y[0];
#pragma unroll
    for (int i = 1; i + 1 < E; i += 2) m = of(of(m, y[i]), y[i + 1]);
    m = of(m, y[E - 1]);
    m = of(m, dpp_f<kDppXor1>(m));
    m = of(m, dpp_f<kDppXor2>(m));
    if constexpr (D == 128) m = of(m, dpp_f<kDppRor8>(m));
    return m;
}

// Codes (two dwords, element 8 h + i at bits [4 i, 4 i + 4) of dword h) and parameters of a row.
template <int D>
__device__ __forceinline__ void quantize_row(const float (&y)[E], float clip, uint32_t (&codes)[2], uint32_t& params) {
    const float lo = clip * row_extreme<D, false>(y), hi = clip * row_extreme<D, true>(y);
    // (hi - lo) / 15, correctly rounded: a quotient with one correction is, for every significand (NaN where it overflows)
    constexpr float fifteenth = 1.0f / 15.0f;
    const float range = hi - lo, q = range * fifteenth;
    const uint32_t sb = bf16_bits(fmaf(fmaf(-15.0f, q, range), fifteenth, q)), mb = bf16_bits(0.5f * (hi + lo));
    const float step = __uint_as_float(sb << 16), mid = __uint_as_float(mb << 16);
    const bool flat = step < kFlat;
    params = (flat ? 0u : sb) | (mb << 16);
    const float inv = flat ? 0.0f : 1.0f / step;
#pragma unroll
    for (int h = 0; h < 2; ++h) {
        // 2^23 + code has the code in its low bits; 2^23's own bits of the first two, shifted into the sum, are taken off beforehand
        uint32_t w = 0u - 0x4b000000u - 0xb0000000u;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const float t = (y[8 * h + i] - mid) * inv + 7.5f;
            w += __float_as_uint(__builtin_amdgcn_fmed3f(t, 0.0f, 15.0f) + 8388608.0f) << (4 * i);
        }
        codes[h] = w;
    }
}

// A workgroup's four waves take up to four heads of the same tokens, whose rows lie side by side.
struct Shape {
    int64_t items;                                // groups of a wave's tokens
    int log_heads;                                // heads of a workgroup
    dim3 grid(int kv_heads) const {
        const int64_t y = (items + (4 >> log_heads) - 1) / (4 >> log_heads), most = y < 65535 ? y : 65535;
        return dim3((unsigned)((kv_heads + (1 << log_heads) - 1) >> log_heads), (unsigned)most, (unsigned)((y + most - 1) / most));
    }
    __device__ __forceinline__ bool find(int kv_heads, int& head, int64_t& item) const {
        const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
        head = (int)(blockIdx.x << log_heads) + (wave & ((1 << log_heads) - 1));
        item = ((int64_t)blockIdx.z * gridDim.y + blockIdx.y) * (4 >> log_heads) + (wave >> log_heads);
        return head < kv_heads && item < items;
    }
};
static_assert(kThreads == 4 * 64, "four waves");

// A token's place in a page of its head.
struct Place {
    uint8_t* block;
    int token;
};
template <int D>
__device__ __forceinline__ Place place_of(const Kv4& c, int64_t slot, int head) {
    const int64_t page = slot >> c.page_shift;
    const int p = 1 << c.page_shift;
    return Place{c.data + page * c.page_bytes + (int64_t)head * (p * (D + 8)), (int)(slot & (p - 1))};
}
// Codes of a lane's elements: of keys a dword, and D / 4 bytes on another; of values halfwords 0, 8, D, D + 8 bytes on.
template <int D>
__device__ __forceinline__ uint8_t* key_codes(const Place& at, int part) { return at.block + at.token * (D / 2) + 4 * part; }
template <int D>
__device__ __forceinline__ uint8_t* value_codes(const Place& at, int p, int part) {
    return at.block + p * (D / 2) + (at.token >> 2) * (2 * D) + 16 * part + 2 * (at.token & 3);
}
template <int D>
__device__ __forceinline__ uint32_t* params(const Place& at, int p) { return reinterpret_cast<uint32_t*>(at.block + p * D) + at.token; }

// A wave takes 8 (or, short heads, 16) consecutive tokens of a head, key and value.  Value codes of two tokens make a dword: where the
// slots of an even token and the next one are such a pair, the even token's lanes write the dwords of their first eight
// elements and the odd token's those of the other; else each writes its own halfwords.
// Bound by memory, of which it reaches 4.5 TB/s (a copy: 5.0): 8192 tokens of 32 heads of 128, bf16, rotated, 170 MB: 38 us; vector issue 43 %
// (with eight elements a lane, twice the lanes and their crossings: 59).
template <int D, int DT, bool ALIGNED, bool ROTATE>
__global__ __launch_bounds__(kThreads) void k_kv4_append(Kv4 cache, Kv4Append a, Shape shape) {
    const int lane = threadIdx.x & 63, part = part_of<D>(lane);
    int head;
    int64_t many;
    if (!shape.find(cache.kv_heads, head, many)) return;
    const int64_t token = many * kTokens<D> + token_in_wave<D>(lane);
    const int64_t last = a.tokens - 1, from = token < last ? token : last;     // every lane loads: butterflies cross them
    const int64_t slot = token <= last ? a.slots[token] : -1;
    float k[E], v[E];
    load_row<DT, ALIGNED>(a.k, from * a.k_token + (int64_t)head * a.k_head + 8 * part, D / 2, k);
    load_row<DT, ALIGNED>(a.v, from * a.v_token + (int64_t)head * a.v_head + 8 * part, D / 2, v);
    if constexpr (ROTATE) rotate_row<D>(k, part);
    uint32_t kc[2], kp, vc[2], vp;
    quantize_row<D>(k, a.clip, kc, kp);
    quantize_row<D>(v, a.clip, vc, vp);
    // the other token of the pair (lane ^ 4): its slot, its codes of the elements that this lane is to write
    const auto other = [](uint32_t x) { return dpp_u<0x1B>(dpp_u<kDppHalfMirror>(x)); };             // 7 - i, then i ^ 3
    const bool odd = lane & 4;
    const int64_t pair_slot = (int64_t)(((uint64_t)other((uint32_t)((uint64_t)slot >> 32)) << 32) | other((uint32_t)slot));
    const uint32_t theirs = other(odd ? vc[0] : vc[1]);
    if (slot < 0 || slot >= cache.pages << cache.page_shift) return;
    const int p = 1 << cache.page_shift;
    const Place at = place_of<D>(cache, slot, head);
    uint32_t* kw = reinterpret_cast<uint32_t*>(key_codes<D>(at, part));
    kw[0] = kc[0];
    kw[D / 16] = kc[1];
    uint8_t* vw = value_codes<D>(at, p, part);
    if (odd ? (slot & 1) && pair_slot == slot - 1 : !(slot & 1) && pair_slot == slot + 1) {
        const uint32_t even_w = odd ? theirs : vc[0], odd_w = odd ? vc[1] : theirs;
        uint32_t* w = reinterpret_cast<uint32_t*>(odd ? vw + D - 2 : vw);
        w[0] = __builtin_amdgcn_perm(odd_w, even_w, 0x05040100u);
        w[2] = __builtin_amdgcn_perm(odd_w, even_w, 0x07060302u);
    } else {
        uint16_t* w = reinterpret_cast<uint16_t*>(vw);
        w[0] = (uint16_t)vc[0];
        w[4] = (uint16_t)(vc[0] >> 16);
        w[D / 2] = (uint16_t)vc[1];
        w[D / 2 + 4] = (uint16_t)(vc[1] >> 16);
    }
    if (part == 0) {
        uint32_t* w = params<D>(at, p);
        w[0] = kp;
        w[p] = vp;
    }
}

// Bound by the rows' stores: 65536 rows of 8 heads of 128 to fp16, 340 MB: 51.7 us, 6.6 TB/s (writing alone reaches 6.9); with eight elements a
// lane 82.
template <int D, int DT, bool ROTATE>
__global__ __launch_bounds__(kThreads) void k_kv4_read(Kv4 cache, Kv4Read a, Shape shape) {
    const int lane = threadIdx.x & 63, part = part_of<D>(lane);
    int head;
    int64_t many;
    if (!shape.find(cache.kv_heads, head, many)) return;
    const int64_t row = many * kTokens<D> + token_in_wave<D>(lane);
    const int p = 1 << cache.page_shift;
    const int64_t slot = row < a.rows ? a.slots[row] : -1;
    const bool there = slot >= 0 && slot < cache.pages << cache.page_shift;
    uint32_t kc[2] = {}, vc[2] = {}, kp = 0, vp = 0;                            // an absent row is zeros
    if (there) {
        const Place at = place_of<D>(cache, slot, head);
        const uint32_t* kw = reinterpret_cast<const uint32_t*>(key_codes<D>(at, part));
        kc[0] = kw[0];
        kc[1] = kw[D / 16];
        const uint16_t* vw = reinterpret_cast<const uint16_t*>(value_codes<D>(at, p, part));
        vc[0] = (uint32_t)vw[0] | ((uint32_t)vw[4] << 16);
        vc[1] = (uint32_t)vw[D / 2] | ((uint32_t)vw[D / 2 + 4] << 16);
        const uint32_t* q = params<D>(at, p);
        kp = q[0];
        vp = q[p];
    }
    float k[E], v[E];
#pragma unroll
    for (int i = 0; i < E; ++i) {
        k[i] = fmaf((float)((kc[i / 8] >> (4 * (i % 8))) & 15u) - 7.5f, __uint_as_float(kp << 16), __uint_as_float(kp & 0xffff0000u));
        v[i] = fmaf((float)((vc[i / 8] >> (4 * (i % 8))) & 15u) - 7.5f, __uint_as_float(vp << 16), __uint_as_float(vp & 0xffff0000u));
    }
    if constexpr (ROTATE) rotate_row<D>(k, part); // H is symmetric: the way back is the way there
    if (row >= a.rows) return;
    const int64_t at = (row * cache.kv_heads + head) * D + 8 * part;
    store_row<DT>(a.k, at, D / 2, k);
    store_row<DT>(a.v, at, D / 2, v);
}

// Pages of all layers, a workgroup for every 16 KB of one.
constexpr int kCopyLoads = 4;
template <bool STREAM>
__global__ __launch_bounds__(kThreads) void k_kv4_copy_pages(Kv4 cache, int64_t layer_bytes, const int32_t* src, const int32_t* dst,
                                                             int64_t pairs, int parts, int64_t groups) {
    const int64_t group = group_index();
    if (group >= groups) return;
    const int part = (int)(group % parts);
    const int64_t rest = group / parts, layer = rest / pairs, pair = rest - layer * pairs;
    const int64_t from = src[pair], to = dst[pair];
    if (from < 0 || from >= cache.pages || to < 0 || to >= cache.pages || from == to) return;
    const int words = (int)(cache.page_bytes / 16);
    uint8_t* base = cache.data + layer * layer_bytes;
    const u32x4* x = reinterpret_cast<const u32x4*>(base + from * cache.page_bytes);
    u32x4* y = reinterpret_cast<u32x4*>(base + to * cache.page_bytes);
    const int at = part * (kCopyLoads * kThreads) + threadIdx.x;
    u32x4 w[kCopyLoads];
#pragma unroll
    for (int i = 0; i < kCopyLoads; ++i)
        if (at + i * kThreads < words) w[i] = STREAM ? __builtin_nontemporal_load(x + at + i * kThreads) : x[at + i * kThreads];
#pragma unroll
    for (int i = 0; i < kCopyLoads; ++i)
        if (at + i * kThreads < words) {
            if constexpr (STREAM) __builtin_nontemporal_store(w[i], y + at + i * kThreads);
            else y[at + i * kThreads] = w[i];
        }
}

bool vector_rows(const void* x, int64_t token, int64_t head, int size) {
    return reinterpret_cast<uintptr_t>(x) % 16 == 0 && token * size % 16 == 0 && head * size % 16 == 0;
}

template <int D, int DT>
void launch_append(const Kv4& c, const Kv4Append& a, hipStream_t s) {
    constexpr int T = kTokens<D>, size = DT == RQ_F32 ? 4 : 2;
    const Shape shape{(a.tokens + T - 1) / T, c.kv_heads >= 4 ? 2 : c.kv_heads >= 2 ? 1 : 0};
    const dim3 grid = shape.grid(c.kv_heads), block(kThreads);
    const bool wide = vector_rows(a.k, a.k_token, a.k_head, size) && vector_rows(a.v, a.v_token, a.v_head, size);
    if (wide && a.rotate) launch_kernel(k_kv4_append<D, DT, true, true>, grid, block, 0, s, c, a, shape);
    else if (wide) launch_kernel(k_kv4_append<D, DT, true, false>, grid, block, 0, s, c, a, shape);
    else if (a.rotate) launch_kernel(k_kv4_append<D, DT, false, true>, grid, block, 0, s, c, a, shape);
    else launch_kernel(k_kv4_append<D, DT, false, false>, grid, block, 0, s, c, a, shape);
}

template <int D, int DT>
void launch_read(const Kv4& c, const Kv4Read& a, hipStream_t s) {
    constexpr int T = kTokens<D>;
    const Shape shape{(a.rows + T - 1) / T, c.kv_heads >= 4 ? 2 : c.kv_heads >= 2 ? 1 : 0};
    const dim3 grid = shape.grid(c.kv_heads), block(kThreads);
    if (a.rotate) launch_kernel(k_kv4_read<D, DT, true>, grid, block, 0, s, c, a, shape);
    else launch_kernel(k_kv4_read<D, DT, false>, grid, block, 0, s, c, a, shape);
}

}  // namespace

int kv4_append(const Kv4& c, const Kv4Append& a, hipStream_t s) {
    const bool wide = c.head_dim == 128;
    switch (a.dtype) {
        case RQ_BF16: wide ? launch_append<128, RQ_BF16>(c, a, s) : launch_append<64, RQ_BF16>(c, a, s); break;
        case RQ_F16: wide ? launch_append<128, RQ_F16>(c, a, s) : launch_append<64, RQ_F16>(c, a, s); break;
        default: wide ? launch_append<128, RQ_F32>(c, a, s) : launch_append<64, RQ_F32>(c, a, s); break;
    }
    return launch_rc();
}

int kv4_read(const Kv4& c, const Kv4Read& a, hipStream_t s) {
    const bool wide = c.head_dim == 128;
    switch (a.dtype) {
        case RQ_BF16: wide ? launch_read<128, RQ_BF16>(c, a, s) : launch_read<64, RQ_BF16>(c, a, s); break;
        case RQ_F16: wide ? launch_read<128, RQ_F16>(c, a, s) : launch_read<64, RQ_F16>(c, a, s); break;
        default: wide ? launch_read<128, RQ_F32>(c, a, s) : launch_read<64, RQ_F32>(c, a, s); break;
    }
    return launch_rc();
}

int kv4_copy_pages(const Kv4& c, int layers, int64_t layer_bytes, const int32_t* src, const int32_t* dst, int64_t pairs, hipStream_t s) {
    const int parts = (int)((c.page_bytes / 16 + kCopyLoads * kThreads - 1) / (kCopyLoads * kThreads));
    const int64_t groups = (int64_t)layers * pairs * parts;
    // Past the caches where they would not hold the pages: 143 MB of pages in 52.5 us and not 59.  Small copies, which the next
    // step reads, stay in them (9 MB: 5.5 us and not 6.7).
    const bool stream = (int64_t)layers * pairs * c.page_bytes > (32 << 20);
    const auto kernel = stream ? k_kv4_copy_pages<true> : k_kv4_copy_pages<false>;
    launch_kernel(kernel, group_grid(groups, kThreads), dim3(kThreads), 0, s, c, layer_bytes, src, dst, pairs, parts, groups);
    return launch_rc();
}

}  // namespace rq
