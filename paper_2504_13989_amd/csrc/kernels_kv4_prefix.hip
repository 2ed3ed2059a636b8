// Attention of sequences that share a prefix (kv4_layout.h): o = sum_j p_j v_j / sum_j p_j over the positions of a group's prefix, which all
// of its sequences see, and over a sequence's own.
//
// The rows of all sequences of a group are one set of rows against the prefix: its keys are read and unpacked once for 16 of them (kernel
// for few rows) or 128 (kernel for many).  Each sequence's own positions are a call as any other's.  Both leave partial results, a row's
// normalised sums and the logarithm of their weight for each chunk of keys, which are joined in a fixed order.  Where sharing does
// not pay for the two launches more, a sequence's rows take the prefix and its own positions one after the other.
#include "kv4_few_rows.h"
#include "kv4_prefix.h"

namespace rq {
namespace {

template <int D, int F, bool F16, bool PAGED, int W, Part PART>
__global__ __launch_bounds__(64 * W, 2) void k_kv4_prefix(PrefixJob job) {
    few_rows<D, F, F16, PAGED, W, false, PART>(job);
}

PrefixPlan plan(const Kv4& c, const Kv4Attention& a, const Kv4Prefix& x, int num_cu) {
    const int group = a.heads / c.kv_heads;
    const int64_t rows = (int64_t)a.tokens * group, shared_keys = x.max_len / kTile + 1, own_keys = a.max_len / kTile + 1;
    // (of n stretches of rows in a row, which begin where those before them end, rounded down to a tile, and one tile further each)
    const auto tiles_of = [&](int bm, int n) { return (rows + bm - 1) / bm + n - 1; };
    const auto shared_tiles = [&](int bm) { return tiles_of(bm, x.groups); };
    const auto own_tiles = [&](int bm) { return a.q_start ? tiles_of(bm, a.batch) : (int64_t)a.batch * ((group + bm - 1) / bm); };
    const auto copies_of = [](int64_t mean) { return mean <= 4 ? 4 : mean <= 8 ? 2 : 1; };
    // What a row tile of 64 keys costs, in those of the kernel for few rows: one of 128 of the other as much as three of 16.
    constexpr int kManyCost = 3;
    PrefixPlan p{};
    p.own_copies = copies_of(rows / a.batch);
    const int64_t few = own_tiles(16 / p.own_copies), own_few = few * own_keys;
    const int64_t shared_few = shared_tiles(16) * shared_keys, shared_many = kManyCost * shared_tiles(128) * shared_keys, own_many = kManyCost * own_tiles(128) * own_keys;
    p.many = shared_many < shared_few && shared_few * c.kv_heads > 16 * (int64_t)num_cu;
    p.own_many = own_many < own_few && own_few * c.kv_heads > 256 * (int64_t)num_cu;
    const int64_t together = (p.many ? shared_many : shared_few) + (p.own_many ? own_many : own_few), apart = few * shared_keys + own_few;
    p.separate = a.window != 0 || x.max_len < kTile || (apart - together) * c.kv_heads < 16 * (int64_t)num_cu;
    if (p.separate) {
        p.many = p.own_many = false;
        p.own_tiles = (int)few;
        p.waves = few * c.kv_heads <= num_cu ? 8 : 4;
        return p;
    }
    // A row tile's keys in as many chunks as cost least: rounds of workgroups that the chip holds at once, of `at_once` tiles of keys a step and
    // kStart steps besides; partial results that are written and read again (4 TB/s, steps of 1.5 us).
    constexpr int kStart = 3;
    const auto split = [&](int64_t wgs, int64_t keys, int at_once, int64_t per_cu, int& chunk, int& chunks) {
        const double join = 2.0 * a.tokens * a.heads * c.head_dim * sizeof(float) / 6e6;
        double least = 0.0;
        for (int64_t n = 1; n <= 256 && (n == 1 || n * at_once <= keys); ++n) {
            const int64_t each = (keys + n - 1) / n, real = (keys + each - 1) / each;
            const double cost = (double)((wgs * real + per_cu * num_cu - 1) / (per_cu * num_cu)) * (double)((each + at_once - 1) / at_once + kStart) + join * (double)real;
            if (n > 1 && cost >= least) continue;
            least = cost;
            chunk = (int)(each * kTile);
            chunks = (int)real;
        }
    };
    if (p.many) {
        p.shared_tiles = (int)shared_tiles(128);
        p.groups = a.dtype != RQ_F16 || c.head_dim == 64 ? 2 : 1;
        split((int64_t)p.shared_tiles * c.kv_heads, shared_keys, p.groups, p.groups == 2 ? 1 : 2, p.shared_chunk, p.shared_chunks);
    } else {
        const int64_t mean = rows / x.groups;
        p.shared_copies = copies_of(mean);
        p.shared_tiles = (int)shared_tiles(16 / p.shared_copies);
        split((int64_t)p.shared_tiles * c.kv_heads, shared_keys, 4, 2, p.shared_chunk, p.shared_chunks);
    }
    p.own_tiles = (int)(p.own_many ? own_tiles(128) : few);
    split((int64_t)p.own_tiles * c.kv_heads, own_keys, 4, 2, p.own_chunk, p.own_chunks);
    p.bytes = (size_t)(p.shared_chunks + p.own_chunks) * a.tokens * a.heads * (c.head_dim + 1) * sizeof(float);
    return p;
}

template <int D, int F, bool F16, bool PAGED>
void launch_few(const PrefixJob& job, Part part, int waves, hipStream_t s) {
    const dim3 grid = item_grid(job.cache.kv_heads, (int64_t)job.tiles * (part == Part::kSeparate ? 1 : job.chunks)), block(64 * waves);
    if (part == Part::kShared) launch_kernel(k_kv4_prefix<D, F, F16, PAGED, 4, Part::kShared>, grid, block, 0, s, job);
    else if (part == Part::kOwn) launch_kernel(k_kv4_prefix<D, F, F16, PAGED, 4, Part::kOwn>, grid, block, 0, s, job);
    else if (waves == 8) launch_kernel(k_kv4_prefix<D, F, F16, PAGED, 8, Part::kSeparate>, grid, block, 0, s, job);
    else launch_kernel(k_kv4_prefix<D, F, F16, PAGED, 4, Part::kSeparate>, grid, block, 0, s, job);
}
template <int D, int F, bool F16>
void launch_few(const PrefixJob& job, Part part, int waves, hipStream_t s) {
    if (job.cache.page_shift < 6) launch_few<D, F, F16, true>(job, part, waves, s);
    else launch_few<D, F, F16, false>(job, part, waves, s);
}
template <int D, bool F16>
void launch_few(const PrefixJob& job, Part part, int copies, int waves, hipStream_t s) {
    if (copies == 4) launch_few<D, 4, F16>(job, part, waves, s);
    else if (copies == 2) launch_few<D, 2, F16>(job, part, waves, s);
    else launch_few<D, 1, F16>(job, part, waves, s);
}
void launch_few(const PrefixJob& job, Part part, int copies, int waves, hipStream_t s) {
    const bool f16 = job.a.dtype == RQ_F16;
    if (job.cache.head_dim == 128) f16 ? launch_few<128, true>(job, part, copies, waves, s) : launch_few<128, false>(job, part, copies, waves, s);
    else f16 ? launch_few<64, true>(job, part, copies, waves, s) : launch_few<64, false>(job, part, copies, waves, s);
}

}  // namespace

size_t kv4_prefix_workspace(const Kv4& c, const Kv4Attention& a, const Kv4Prefix& p, int num_cu) {
    Kv4Attention x = a;                           // (the caller's size holds for results of either type)
    size_t most = 0;
    for (const int dtype : {RQ_BF16, RQ_F16}) {
        x.dtype = dtype;
        const size_t bytes = plan(c, x, p, num_cu).bytes;
        most = bytes > most ? bytes : most;
    }
    return most;
}

rq_kv4_prefix_plan_t kv4_prefix_plan(const Kv4& c, const Kv4Attention& a, const Kv4Prefix& x, int num_cu) {
    const PrefixPlan p = plan(c, a, x, num_cu);
    rq_kv4_prefix_plan_t r{};
    r.separate = p.separate;
    r.waves = p.separate ? p.waves : p.many ? 4 * p.groups : 4;
    r.many = p.many;
    r.own_many = p.own_many;
    r.shared_rows = p.separate ? 0 : p.many ? 128 : 16 / p.shared_copies;
    r.own_rows = p.own_many ? 128 : 16 / p.own_copies;
    r.shared_chunk = p.shared_chunk;
    r.shared_chunks = p.shared_chunks;
    r.own_chunk = p.own_chunk;
    r.own_chunks = p.own_chunks;
    return r;
}

int kv4_prefix_attention(const Kv4& c, const Kv4Attention& a, const Kv4Prefix& x, int num_cu, float* workspace, hipStream_t s) {
    const PrefixPlan p = plan(c, a, x, num_cu);
    const auto wide = [](const void* x, int64_t token, int64_t head) {
        return reinterpret_cast<uintptr_t>(x) % 16 == 0 && token % 8 == 0 && head % 8 == 0;
    };
    PrefixJob job{};
    static_cast<KvJob&>(job) = KvJob{c, a, a.heads / c.kv_heads, p.own_tiles, 0, p.own_chunk, p.own_chunks, wide(a.q, a.q_token, a.q_head),
                                     wide(a.o, a.o_token, a.o_head), workspace};
    job.p = x;
    if (p.separate) {
        launch_few(job, Part::kSeparate, p.own_copies, p.waves, s);
        return launch_rc();
    }
    job.part_chunks = p.shared_chunks + p.own_chunks;
    job.part_first = p.shared_chunks;
    if (p.own_many) launch_prefix_many(job, Part::kOwn, 1, s);
    else launch_few(job, Part::kOwn, p.own_copies, 4, s);
    PrefixJob shared = job;
    shared.tiles = p.shared_tiles;
    shared.chunk = p.shared_chunk;
    shared.chunks = p.shared_chunks;
    shared.part_first = 0;
    if (p.many) launch_prefix_many(shared, Part::kShared, p.groups, s);
    else launch_few(shared, Part::kShared, p.shared_copies, 4, s);
    job.chunks = job.part_chunks;
    launch_join(job, s);
    return launch_rc();
}

}  // namespace rq
