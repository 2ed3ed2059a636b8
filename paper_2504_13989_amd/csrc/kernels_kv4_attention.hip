// Attention over the 4-bit paged cache (kv4_layout.h): shares and chunks of rows joined, and how a call is laid out.  The kernels are those of
// kv4_few_rows.h and kv4_many_rows.h.
#include "kv4_few_rows.h"

namespace rq {
namespace {

// Joins the shares of a row tile at a kv head, the waves take them in turn.
template <int D, int F, bool F16>
__global__ __launch_bounds__(64 * kWaves) void k_kv4_join_shares(KvJob job) {
    constexpr int C = 16 / F, per = C * D / 64;   // results of a lane
    __shared__ float lds_o[kWaves][C * D], lds_l[kWaves][C], lds_m[kWaves][C];
    const Kv4Attention& a = job.a;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, kv = job.cache.kv_heads;
    const int tile = item_number(), head = blockIdx.x;
    if (tile >= job.tiles) return;
    const int first = part_workers<D, C>(job)[2 * tile], last = part_workers<D, C>(job)[2 * tile + 1];
    Place at;
    if (first == last || !find_rows<C>(job, tile, at)) return;       // a worker had all of it
    const int mine = lane * per / D, d = lane * per % D;
    const auto slot = [&](int i) { return ((int64_t)(i + tile) * kv + head) * C; };
    // (one pass with a running maximum: sums and values come in one trip to memory)
    float top = -INFINITY, sum = 0.0f, z[per] = {};
#pragma unroll 2
    for (int i = first + wave; i <= last; i += kWaves) {
        const float l = part_sums<D, C>(job)[slot(i) + mine];
        const float* o = job.part + (slot(i) + mine) * D + d;
        const float to = fmaxf(top, l), was = top == -INFINITY ? 0.0f : __builtin_amdgcn_exp2f(top - to), by = l == -INFINITY ? 0.0f : __builtin_amdgcn_exp2f(l - to);
        top = to;
        sum = fmaf(sum, was, by);
#pragma unroll
        for (int e = 0; e < per; ++e) z[e] = fmaf(by, o[e], was * z[e]);
    }
#pragma unroll
    for (int e = 0; e < per; ++e) lds_o[wave][lane * per + e] = z[e];
    if (d == 0) {
        lds_l[wave][mine] = sum;
        lds_m[wave][mine] = top;
    }
    __syncthreads();
    const int rows = at.nq * job.group;
    const auto join = [&](int row, float (&by)[kWaves], float& most) {           // the waves' factors; the sum over them
        most = -INFINITY;
#pragma unroll
        for (int w = 0; w < kWaves; ++w) most = fmaxf(most, lds_m[w][row]);
        float all = 0.0f;
#pragma unroll
        for (int w = 0; w < kWaves; ++w) {
            by[w] = lds_m[w][row] == -INFINITY ? 0.0f : __builtin_amdgcn_exp2f(lds_m[w][row] - most);
            all = fmaf(by[w], lds_l[w][row], all);
        }
        return all;
    };
    float by[kWaves], most;
    for (int x = threadIdx.x; x < C * D; x += 64 * kWaves) {
        const int row = x / D, n = at.base + row;
        if (n >= rows) break;
        const float all = join(row, by, most);
        float y = 0.0f;
#pragma unroll
        for (int w = 0; w < kWaves; ++w) y = fmaf(by[w], lds_o[w][x], y);
        const int token = token_of(job, at, n), h = head * job.group + n - token * job.group;
        static_cast<uint16_t*>(a.o)[(int64_t)(at.q0 + token) * a.o_token + (int64_t)h * a.o_head + x % D] = (uint16_t)pack16<F16>(all == 0.0f ? 0.0f : y / all, 0.0f);
    }
    if (a.lse && wave == 0 && d == 0 && at.base + mine < rows) {
        const int n = at.base + mine, token = token_of(job, at, n), h = head * job.group + n - token * job.group;
        const float all = join(mine, by, most);
        a.lse[(int64_t)(at.q0 + token) * a.heads + h] = (most + __builtin_amdgcn_logf(all)) * kLn2;
    }
}

// Joins the chunks of a row of the kernel for many: a wave a row.  Partial results: [chunks][tokens][heads], D values each, and
// behind them log2 of the sums.
template <int D, bool F16>
__global__ __launch_bounds__(64 * kWaves) void k_kv4_join(KvJob job) {
    constexpr int per = D / 64;
    const Kv4Attention& a = job.a;
    const int lane = threadIdx.x & 63;
    const int64_t row = group_index() * kWaves + (threadIdx.x >> 6), rows = (int64_t)a.tokens * a.heads;
    if (row >= rows) return;
    const int tokens = a.q_start ? a.q_start[a.batch] - job.first_token : a.tokens;      // (rows behind the last sequence have no results)
    const float* sums = job.part + (int64_t)job.chunks * rows * D + row;
    float top = -INFINITY;
    for (int c = lane; c < job.chunks; c += 64) top = fmaxf(top, sums[c * rows]);
#pragma unroll
    for (int w = 1; w < 64; w *= 2) top = fmaxf(top, __shfl_xor(top, w));
    float all = 0.0f, y[per] = {};
#pragma unroll 16                                 // (that many chunks in one trip to memory)
    for (int c = 0; c < job.chunks; ++c) {
        const float l = sums[c * rows];
        const float by = l == -INFINITY ? 0.0f : __builtin_amdgcn_exp2f(l - top);
        const float* o = job.part + (c * rows + row) * D + lane * per;
        all += by;
#pragma unroll
        for (int e = 0; e < per; ++e) y[e] = fmaf(by, o[e], y[e]);
    }
    const int64_t token = row / a.heads;
    const int h = (int)(row - token * a.heads);
    if (token >= tokens) return;
    const float by = all == 0.0f ? 0.0f : 1.0f / all;
#pragma unroll
    for (int e = 0; e < per; ++e) y[e] *= by;
    store_row<per, F16>(static_cast<uint16_t*>(a.o) + token * a.o_token + (int64_t)h * a.o_head + lane * per, y, job.wide_o);
    if (lane == 0 && a.lse) a.lse[row] = (top + __builtin_amdgcn_logf(all)) * kLn2;
}

// How a call is launched.
struct Plan {
    int copies;                                   // of the rows among the columns; 0: the kernel for many rows
    int waves;                                    // of a workgroup; many rows: of a group of them
    int groups;                                   // many rows: groups of a workgroup, which share its keys out
    int tiles, workers, chunk, chunks;
    size_t bytes;                                 // workspace
};

Plan plan(const Kv4& c, const Kv4Attention& a, int num_cu) {
    const int group = a.heads / c.kv_heads;
    const int64_t rows = (int64_t)a.tokens * group, mean = rows / a.batch;
    const auto tiles_of = [&](int bm) { return a.q_start ? rows / bm + a.batch : (int64_t)a.batch * ((group + bm - 1) / bm); };
    // Keys of a row tile at most.  A causal tile of a window ends with its last token; another goes on to the end of the sequence, which
    // lies as many tokens behind its first one as the sequence has queries.
    const auto range_of = [&](int bm) {
        const int64_t behind = a.causal ? bm / group + 2 : a.q_start ? a.tokens : 1;
        const int64_t seen = a.window ? (int64_t)a.window + behind + kTile : a.max_len;
        return seen < a.max_len ? seen : a.max_len;
    };
    Plan p{};
    p.chunks = p.groups = 1;
    p.chunk = 1 << 30;
    // Rows of 16 in workgroups of their own fill the chip sooner and start at once; the kernel for many rows reads a key for 128 or 256 of
    // them.  By tiles of 16 rows x 64 keys, the former up to 256 a compute unit: 50 tokens against 1000, 8 heads to 4: 11 us and not 24;
    // 1000 x 1000, 8 heads: 14 and not 31; 500 x 8000 (122 a unit): 39 and 48; 1000 x 1000, 32 heads to 8 (126): 33 and 31; 2000 x 2000,
    // 32 to 8 (500): 88 and 64.
    const bool many = mean > 32 && tiles_of(16) * c.kv_heads * (range_of(16) / kTile + 1) > 256 * (int64_t)num_cu;
    p.copies = many ? 0 : mean <= 4 ? 4 : mean <= 8 ? 2 : 1;
    // Many rows.  Eight waves that share each tile unpack a key once for 256 rows: best where there are such workgroups for one and a quarter
    // rounds and more (8192 tokens against themselves, 16 heads to 4 of keys: 308 us; four waves 365; 2048 tokens, 32 to 8: 75, 67).  Below
    // that four waves; and where these alone would leave every compute unit one or two workgroups, a second four that take every other
    // tile of the same rows (4096 tokens, 8 heads of 64: 56 us and not 77; 2048 tokens, 32 heads to 8: 65 and not 67).  Fewer workgroups
    // still: keys in chunks are spread better (512 tokens against 8192, 136 workgroups: 120 us and not 153).  fp16 results of
    // 128 elements have no registers for a second four (512 x 4096: 80 us and not 42).  Where a window makes workgroups alike, a
    // second round of them costs as much as the first (276 workgroups: 54 us and not 51).
    p.waves = 4 * tiles_of(256) * c.kv_heads >= 5 * (int64_t)num_cu ? 8 : 4;
    const int64_t small = tiles_of(128) * c.kv_heads;
    p.groups = p.waves == 4 && (a.dtype != RQ_F16 || c.head_dim == 64) && 3 * small >= 2 * (int64_t)num_cu && (!a.window || small <= num_cu) ? 2 : 1;
    const int bm = p.copies ? 16 / p.copies : 32 * p.waves;
    const int64_t tiles = tiles_of(bm);
    p.tiles = (int)tiles;
    const int64_t range = range_of(bm);
    if (p.copies) {
        // Two workgroups a compute unit share the keys out (three, which registers and LDS would allow: 98.5 us and not 95).  Joining the
        // shares is a launch more, and finding them a scan: 10 us.  So where row tiles leave compute units empty, once that takes more
        // than that off the time (40 tiles of keys of 8 row tiles: 16 us either way; 79 of 96: 18 and 22; 47 of 64: 19 and 17; 66 row tiles of 256: 36 and
        // 72).  Else workgroups that end leave their place to others or their bandwidth to longer ones (16 sequences x 32 heads x 8192: 88 us, shared 92;
        // 64 x 8 x 3000, lengths all over the range: 25 and 31), but for a round and a little more (40 x 8, 64 heads, 8000: 61, shared 43) and for
        // very long ones.
        const int64_t wgs = tiles * c.kv_heads, keys = range / kTile;
        const bool few = wgs <= num_cu;
        const bool share = few ? keys * (num_cu - wgs) > 44 * (int64_t)num_cu
                               : mean <= 32 && (2 * wgs < 3 * (int64_t)num_cu ? keys > 56 : wgs < 3 * (int64_t)num_cu && keys > 256);
        if (tiles <= kMostTiles && share && tiles * (range / kTile + kLeast) < INT32_MAX) {
            p.workers = (int)((2 * num_cu + c.kv_heads - 1) / c.kv_heads);
            p.bytes = ((size_t)(p.workers + p.tiles) * c.kv_heads * (16 / p.copies) * (c.head_dim + 1) + 2 * (size_t)p.tiles) * sizeof(float);
        }
        // A row tile of its own: eight waves while the chip is not full, one where there are more row tiles than workgroups of four have
        // room and their keys are few (64 sequences x 32 heads x 200: 15 us and not 23, x 1000: 46 and 48; 700 workgroups: 13.5, 9.1).
        p.waves = p.workers ? kWaves : few ? kMostWaves : wgs > 3 * (int64_t)num_cu && range <= 1024 ? 1 : kWaves;
        return p;
    }
    // Keys in chunks where the rows alone do not fill the chip, of eight tiles at least (1500 tokens, 4 heads to one: 30 us; sixteen tiles:
    // 44; joining them is a launch more).
    const int64_t want = 2 * num_cu / (tiles * c.kv_heads), most = p.groups == 1 ? range / (8 * kTile) : 1, chunks = want < most ? want : most;
    if (chunks > 1) {
        p.chunk = (int)((range + chunks * kTile - 1) / (chunks * kTile) * kTile);
        p.chunks = (int)((range + p.chunk - 1) / p.chunk);
        p.bytes = (size_t)p.chunks * a.tokens * a.heads * (c.head_dim + 1) * sizeof(float);
    }
    return p;
}

template <int D, int F, bool F16, bool PAGED>
void launch_few(const KvJob& job, const Plan& p, hipStream_t s) {
    const dim3 grid = item_grid(job.cache.kv_heads, job.workers ? job.workers : job.tiles), block(64 * p.waves);
    if (job.workers) {
        launch_kernel(k_kv4_attention<D, F, F16, PAGED, kWaves, true>, grid, block, 0, s, job);
        launch_kernel(k_kv4_join_shares<D, F, F16>, item_grid(job.cache.kv_heads, job.tiles), dim3(64 * kWaves), 0, s, job);
    } else if (p.waves == kMostWaves) {
        launch_kernel(k_kv4_attention<D, F, F16, PAGED, kMostWaves, false>, grid, block, 0, s, job);
    } else if (p.waves == 1) {
        launch_kernel(k_kv4_attention<D, F, F16, PAGED, 1, false>, grid, block, 0, s, job);
    } else {
        launch_kernel(k_kv4_attention<D, F, F16, PAGED, kWaves, false>, grid, block, 0, s, job);
    }
}
template <int D, int F, bool F16>
void launch_few(const KvJob& job, const Plan& p, hipStream_t s) {
    if (job.cache.page_shift < 6) launch_few<D, F, F16, true>(job, p, s);
    else launch_few<D, F, F16, false>(job, p, s);
}

template <int D, bool F16>
void launch_join(const KvJob& job, hipStream_t s) {
    launch_kernel(k_kv4_join<D, F16>, group_grid(((int64_t)job.a.tokens * job.a.heads + kWaves - 1) / kWaves, 64 * kWaves), dim3(64 * kWaves), 0, s, job);
}

template <int D, bool F16>
int launch_attention(const KvJob& job, const Plan& p, hipStream_t s) {
    switch (p.copies) {
        case 4: launch_few<D, 4, F16>(job, p, s); break;
        case 2: launch_few<D, 2, F16>(job, p, s); break;
        case 1: launch_few<D, 1, F16>(job, p, s); break;
        default:
            launch_prompt(job, p.waves, p.groups, s);
            if (p.chunks > 1) launch_join<D, F16>(job, s);
    }
    return launch_rc();
}

}  // namespace

void launch_join(const KvJob& job, hipStream_t s) {
    const bool f16 = job.a.dtype == RQ_F16;
    if (job.cache.head_dim == 128) f16 ? launch_join<128, true>(job, s) : launch_join<128, false>(job, s);
    else f16 ? launch_join<64, true>(job, s) : launch_join<64, false>(job, s);
}

size_t kv4_attention_workspace(const Kv4& c, const Kv4Attention& a, int num_cu) {
    Kv4Attention x = a;                           // (the caller's size holds for results of either type, causal or not)
    size_t most = 0;
    for (const int dtype : {RQ_BF16, RQ_F16})
        for (const bool causal : {true, false}) {
            if (!causal && !a.window) continue;   // (without a window the plan is the same)
            x.dtype = dtype;
            x.causal = causal;
            const size_t bytes = plan(c, x, num_cu).bytes;
            most = bytes > most ? bytes : most;
        }
    return most;
}

rq_kv4_plan_t kv4_attention_plan(const Kv4& c, const Kv4Attention& a, int num_cu) {
    const Plan p = plan(c, a, num_cu);
    rq_kv4_plan_t r{};
    r.many = p.copies == 0;
    r.rows = p.copies ? 16 / p.copies : 32 * p.waves;
    r.waves = p.waves;
    r.groups = p.copies ? 1 : p.groups;
    r.tiles = p.tiles;
    r.workers = p.workers;
    r.chunk = p.chunk;
    r.chunks = p.chunks;
    return r;
}

int kv4_attention(const Kv4& c, const Kv4Attention& a, int num_cu, float* workspace, hipStream_t s) {
    const Plan p = plan(c, a, num_cu);
    const auto wide = [](const void* x, int64_t token, int64_t head) {
        return reinterpret_cast<uintptr_t>(x) % 16 == 0 && token % 8 == 0 && head % 8 == 0;
    };
    const KvJob job{c, a, a.heads / c.kv_heads, p.tiles, p.workers, p.chunk, p.chunks, wide(a.q, a.q_token, a.q_head), wide(a.o, a.o_token, a.o_head), workspace};
    const bool f16 = a.dtype == RQ_F16;
    if (c.head_dim == 128) return f16 ? launch_attention<128, true>(job, p, s) : launch_attention<128, false>(job, p, s);
    return f16 ? launch_attention<64, true>(job, p, s) : launch_attention<64, false>(job, p, s);
}

}  // namespace rq
