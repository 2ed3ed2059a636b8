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

// Eight values of a row.  DT: RQ_BF16, RQ_F32, RQ_F16.  ALIGNED: 16-byte loads.
template <int DT, bool ALIGNED>
__device__ __forceinline__ void load8(const void* X, int64_t at, float (&x)[8]) {
    if constexpr (DT == RQ_F32) {
        const float* p = static_cast<const float*>(X) + at;
        if constexpr (ALIGNED) {
            const f32x4 a = *reinterpret_cast<const f32x4*>(p), b = *reinterpret_cast<const f32x4*>(p + 4);
#pragma unroll
            for (int i = 0; i < 4; ++i) x[i] = a[i], x[4 + i] = b[i];
        } else {
#pragma unroll
            for (int i = 0; i < 8; ++i) x[i] = p[i];
        }
    } else {
        const uint16_t* p = static_cast<const uint16_t*>(X) + at;
        uint32_t w[4];
        if constexpr (ALIGNED) {
            const u32x4 a = *reinterpret_cast<const u32x4*>(p);
#pragma unroll
            for (int i = 0; i < 4; ++i) w[i] = a[i];
        } else {
#pragma unroll
            for (int i = 0; i < 4; ++i) w[i] = (uint32_t)p[2 * i] | ((uint32_t)p[2 * i + 1] << 16);
        }
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            if constexpr (DT == RQ_F16) {
                x[2 * i] = (float)__builtin_bit_cast(_Float16, (uint16_t)w[i]);
                x[2 * i + 1] = (float)__builtin_bit_cast(_Float16, (uint16_t)(w[i] >> 16));
            } else {
                x[2 * i] = __uint_as_float(w[i] << 16);
                x[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u);
            }
        }
    }
}

__device__ __forceinline__ uint32_t bf16_bits(float x) { return (uint32_t)__builtin_bit_cast(uint16_t, (__bf16)x); }

template <int DT>
__device__ __forceinline__ void store8(void* Y, int64_t at, const float (&y)[8]) {
    if constexpr (DT == RQ_F32) {
        f32x4* p = reinterpret_cast<f32x4*>(static_cast<float*>(Y) + at);
        p[0] = f32x4{y[0], y[1], y[2], y[3]};
        p[1] = f32x4{y[4], y[5], y[6], y[7]};
    } else {
        u32x4 w;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            if constexpr (DT == RQ_F16)
                w[i] = (uint32_t)__builtin_bit_cast(uint16_t, (_Float16)y[2 * i]) |
                       ((uint32_t)__builtin_bit_cast(uint16_t, (_Float16)y[2 * i + 1]) << 16);
            else
                w[i] = bf16_bits(y[2 * i]) | (bf16_bits(y[2 * i + 1]) << 16);
        }
        *reinterpret_cast<u32x4*>(static_cast<uint16_t*>(Y) + at) = w;
    }
}

// Value of the lane whose number differs in bit B of the lane's place in a DPP row.
template <int B>
__device__ __forceinline__ float lane_xor(float x) {
    if constexpr (B == 1) return dpp_f<kDppXor1>(x);
    else if constexpr (B == 2) return dpp_f<kDppXor2>(x);
    else if constexpr (B == 4) return dpp_f<0x1B>(dpp_f<kDppHalfMirror>(x));   // 7 - i, then i ^ 3
    else return dpp_f<kDppRor8>(x);
}

template <int B>
__device__ __forceinline__ void lane_butterfly(float (&x)[8], int c) {
    const uint32_t sign = (c & B) ? 0x80000000u : 0u;
#pragma unroll
    for (int i = 0; i < 8; ++i) x[i] = lane_xor<B>(x[i]) + __uint_as_float(__float_as_uint(x[i]) ^ sign);
}

// H x / sqrt(d) of a row that lies over d / 8 lanes, eight values each: strides 1, 2, 4 in the lane, the others across lanes.
// Most of the scale comes first, a power of two and so exact: sums do not overflow where the results are far from it.
template <int D>
__device__ __forceinline__ void rotate_row(float (&x)[8], int c) {
#pragma unroll
    for (int i = 0; i < 8; ++i) x[i] *= 0.125f;
#pragma unroll
    for (int w = 1; w < 8; w *= 2)
#pragma unroll
        for (int i = 0; i < 8; ++i)
            if (!(i & w)) {
                const float a = x[i], b = x[i + w];
                x[i] = a + b;
                x[i + w] = a - b;
            }
    lane_butterfly<1>(x, c);
    lane_butterfly<2>(x, c);
    lane_butterfly<4>(x, c);
    if constexpr (D == 128) {
        lane_butterfly<8>(x, c);
#pragma unroll
        for (int i = 0; i < 8; ++i) x[i] *= 8 * 0.08838834764831845f;
    }
}

// Codes (a dword, element i at bits [4i, 4i + 4)) and parameters of a row.
template <int D>
__device__ __forceinline__ void quantize_row(const float (&y)[8], float clip, uint32_t& codes, uint32_t& params) {
    float lo = y[0], hi = y[0], bad = 0.0f * y[0];
#pragma unroll
    for (int i = 1; i < 8; ++i) {
        lo = fminf(lo, y[i]);
        hi = fmaxf(hi, y[i]);
        bad += 0.0f * y[i];                       // NaN where a value is infinite or NaN, which minima pass over
    }
    lo = fminf(lo, lane_xor<1>(lo));
    hi = fmaxf(hi, lane_xor<1>(hi));
    bad += lane_xor<1>(bad);
    lo = fminf(lo, lane_xor<2>(lo));
    hi = fmaxf(hi, lane_xor<2>(hi));
    bad += lane_xor<2>(bad);
    lo = fminf(lo, lane_xor<4>(lo));
    hi = fmaxf(hi, lane_xor<4>(hi));
    bad += lane_xor<4>(bad);
    if constexpr (D == 128) {
        lo = fminf(lo, lane_xor<8>(lo));
        hi = fmaxf(hi, lane_xor<8>(hi));
        bad += lane_xor<8>(bad);
    }
    lo *= clip;
    hi *= clip;
    const uint32_t sb = bf16_bits((hi - lo) / 15.0f + bad), mb = bf16_bits(0.5f * (hi + lo));
    float step = __uint_as_float(sb << 16);
    const float mid = __uint_as_float(mb << 16);
    const bool flat = step < kFlat;
    params = (flat ? 0u : sb) | (mb << 16);
    const float inv = flat ? 0.0f : 1.0f / step;
    codes = 0;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const float t = rintf((y[i] - mid) * inv + 7.5f);
        codes |= (uint32_t)fminf(fmaxf(t, 0.0f), 15.0f) << (4 * i);
    }
}

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
template <int D>
__device__ __forceinline__ uint8_t* key_codes(const Place& at, int c) { return at.block + at.token * (D / 2) + 4 * c; }
template <int D>
__device__ __forceinline__ uint8_t* value_codes(const Place& at, int p, int c) {
    return at.block + p * (D / 2) + (at.token >> 2) * (2 * D) + 16 * c + 2 * (at.token & 3);
}
template <int D>
__device__ __forceinline__ uint32_t* params(const Place& at, int p) { return reinterpret_cast<uint32_t*>(at.block + p * D) + at.token; }

// A wave takes 512 / D consecutive tokens of a head, key and value: a row's codes are 4 bytes a lane, and the value codes
// of four tokens, which lie interleaved, leave in one go where their slots follow one another.
template <int D, int DT, bool ALIGNED, bool ROTATE>
__global__ __launch_bounds__(kThreads) void k_kv4_append(Kv4 cache, Kv4Append a, int64_t units) {
    constexpr int L = D / 8, T = 64 / L;          // lanes of a row, tokens of a wave
    const int lane = threadIdx.x & 63, c = lane % L;
    const int64_t unit = group_index() * (kThreads / 64) + (threadIdx.x >> 6);
    if (unit >= units) return;
    const int64_t four = unit / cache.kv_heads;
    const int head = (int)(unit - four * cache.kv_heads);
    const int64_t token = four * T + lane / L;
    const int64_t last = a.tokens - 1, from = token < last ? token : last;     // every lane loads: butterflies cross them
    float k[8], v[8];
    load8<DT, ALIGNED>(a.k, from * a.k_token + (int64_t)head * a.k_head + 8 * c, k);
    load8<DT, ALIGNED>(a.v, from * a.v_token + (int64_t)head * a.v_head + 8 * c, v);
    const int64_t slot = token <= last ? a.slots[token] : -1;
    if constexpr (ROTATE) rotate_row<D>(k, c);
    uint32_t kc, kp, vc, vp;
    quantize_row<D>(k, a.clip, kc, kp);
    quantize_row<D>(v, a.clip, vc, vp);
    if (slot < 0 || slot >= cache.pages << cache.page_shift) return;
    const int p = 1 << cache.page_shift;
    const Place at = place_of<D>(cache, slot, head);
    *reinterpret_cast<uint32_t*>(key_codes<D>(at, c)) = kc;
    uint16_t* vw = reinterpret_cast<uint16_t*>(value_codes<D>(at, p, c));
    vw[0] = (uint16_t)vc;
    vw[4] = (uint16_t)(vc >> 16);
    if (c == 0) {
        uint32_t* w = params<D>(at, p);
        w[0] = kp;
        w[p] = vp;
    }
}

template <int D, int DT, bool ROTATE>
__global__ __launch_bounds__(kThreads) void k_kv4_read(Kv4 cache, Kv4Read a, int64_t units) {
    constexpr int L = D / 8, T = 64 / L;
    const int lane = threadIdx.x & 63, c = lane % L;
    const int64_t unit = group_index() * (kThreads / 64) + (threadIdx.x >> 6);
    if (unit >= units) return;
    const int64_t four = unit / cache.kv_heads;
    const int head = (int)(unit - four * cache.kv_heads);
    const int64_t row = four * T + lane / L;
    const int p = 1 << cache.page_shift;
    int64_t slot = row < a.rows ? a.slots[row] : -1;
    const bool there = slot >= 0 && slot < cache.pages << cache.page_shift;
    uint32_t kc = 0, vc = 0, kp = 0, vp = 0;                                    // an absent row is zeros
    if (there) {
        const Place at = place_of<D>(cache, slot, head);
        kc = *reinterpret_cast<const uint32_t*>(key_codes<D>(at, c));
        const uint16_t* vw = reinterpret_cast<const uint16_t*>(value_codes<D>(at, p, c));
        vc = (uint32_t)vw[0] | ((uint32_t)vw[4] << 16);
        const uint32_t* w = params<D>(at, p);
        kp = w[0];
        vp = w[p];
    }
    float k[8], v[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        k[i] = fmaf((float)((kc >> (4 * i)) & 15u) - 7.5f, __uint_as_float(kp << 16), __uint_as_float(kp & 0xffff0000u));
        v[i] = fmaf((float)((vc >> (4 * i)) & 15u) - 7.5f, __uint_as_float(vp << 16), __uint_as_float(vp & 0xffff0000u));
    }
    if constexpr (ROTATE) rotate_row<D>(k, c);    // H is symmetric: the way back is the way there
    if (row >= a.rows) return;
    const int64_t at = (row * cache.kv_heads + head) * D + 8 * c;
    store8<DT>(a.k, at, k);
    store8<DT>(a.v, at, v);
}

// Pages of all layers, a workgroup for every 16 KB of one.
constexpr int kCopyLoads = 4;
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
        if (at + i * kThreads < words) w[i] = x[at + i * kThreads];
#pragma unroll
    for (int i = 0; i < kCopyLoads; ++i)
        if (at + i * kThreads < words) y[at + i * kThreads] = w[i];
}

bool vector_rows(const void* x, int64_t token, int64_t head, int size) {
    return reinterpret_cast<uintptr_t>(x) % 16 == 0 && token * size % 16 == 0 && head * size % 16 == 0;
}

template <int D, int DT>
void launch_append(const Kv4& c, const Kv4Append& a, hipStream_t s) {
    constexpr int T = 512 / D, size = DT == RQ_F32 ? 4 : 2;
    const int64_t units = (a.tokens + T - 1) / T * c.kv_heads;
    const dim3 grid = group_grid((units + kThreads / 64 - 1) / (kThreads / 64), kThreads), block(kThreads);
    const bool wide = vector_rows(a.k, a.k_token, a.k_head, size) && vector_rows(a.v, a.v_token, a.v_head, size);
    if (wide && a.rotate) launch_kernel(k_kv4_append<D, DT, true, true>, grid, block, 0, s, c, a, units);
    else if (wide) launch_kernel(k_kv4_append<D, DT, true, false>, grid, block, 0, s, c, a, units);
    else if (a.rotate) launch_kernel(k_kv4_append<D, DT, false, true>, grid, block, 0, s, c, a, units);
    else launch_kernel(k_kv4_append<D, DT, false, false>, grid, block, 0, s, c, a, units);
}

template <int D, int DT>
void launch_read(const Kv4& c, const Kv4Read& a, hipStream_t s) {
    constexpr int T = 512 / D;
    const int64_t units = (a.rows + T - 1) / T * c.kv_heads;
    const dim3 grid = group_grid((units + kThreads / 64 - 1) / (kThreads / 64), kThreads), block(kThreads);
    if (a.rotate) launch_kernel(k_kv4_read<D, DT, true>, grid, block, 0, s, c, a, units);
    else launch_kernel(k_kv4_read<D, DT, false>, grid, block, 0, s, c, a, units);
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
    launch_kernel(k_kv4_copy_pages, group_grid(groups, kThreads), dim3(kThreads), 0, s, c, layer_bytes, src, dst, pairs, parts, groups);
    return launch_rc();
}

}  // namespace rq
