// Attention of sequences that share a prefix (kv4_layout.h): o = sum_j p_j v_j / sum_j p_j over the positions of a group's prefix, which all
// of its sequences see, and over a sequence's own.
//
// The rows of all sequences of a group are one set of rows against the prefix: its keys are read and unpacked once for 16 of them (kernel
// for few rows) or 128 (kernel for many).  Each sequence's own positions are a call as any other's.  Both leave partial results, a row's
// normalised sums and the logarithm of their weight for each chunk of keys, which are joined in a fixed order.  Where sharing does
// not pay for the launch more, a sequence's rows take the prefix and its own positions one after the other.
//
// One MI355X, bf16, 128 elements, 32 heads on 8: 64 queries behind 8192 positions, 300 of their own each: 33 us, 28 in the first launch, bound by
// vector issue (590 instructions for 16 rows x 64 keys), 4.6 in the join; from whole tables 70.  Four behind 1000: 10.6, latency.  fp16, 12
// sequences of 40 tokens, 64 heads on 8, 65411 positions: 1.1 ms, the many-row kernel's rate; from whole tables 1.5.
#include "kv4_few_rows.h"
#include "kv4_prefix.h"

namespace rq {
namespace {

// The kernel for few rows.  The first of a kv head's workgroups take prefixes, the others what is behind them: either fills what the other
// leaves of the chip.
struct SharedPart {
    int first_tile, tiles, chunk, chunks;
};
template <int D, int F, bool F16, bool PAGED>
__global__ __launch_bounds__(256, 2) void k_kv4_prefix(PrefixJob job, SharedPart shared) {
    __shared__ FewLds<D, 4> lds;
    int none;
    const int number = item_number(), first = (shared.tiles - shared.first_tile) * shared.chunks;
    if (number >= first) {
        few_rows<D, F, F16, PAGED, 4, false, Part::kOwn>(job, number - first, lds, none);
        return;
    }
    job.first_tile = shared.first_tile;
    job.tiles = shared.tiles;
    job.chunk = shared.chunk;
    job.chunks = shared.chunks;
    job.part_first = 0;
    few_rows<D, 1, F16, PAGED, 4, false, Part::kShared>(job, number, lds, none);
}
template <int D, int F, bool F16, bool PAGED, int W>
__global__ __launch_bounds__(64 * W, 2) void k_kv4_prefix_separate(PrefixJob job) {
    __shared__ FewLds<D, W> lds;
    int none;
    few_rows<D, F, F16, PAGED, W, false, Part::kSeparate>(job, item_number(), lds, none);
}

constexpr size_t kMostBytes = (size_t)1 << 30;    // of workspace

PrefixPlan plan(const Kv4& c, const Kv4Attention& a, const Kv4Prefix& x, int num_cu) {
    const int group = a.heads / c.kv_heads;
    const int64_t rows = (int64_t)a.tokens * group, shared_keys = x.max_len / kTile + 1, own_keys = a.max_len / kTile + 1;
    // (of n stretches of rows in a row, which begin where those before them end, rounded down to a tile, and one tile further each)
    const auto tiles_of = [&](int bm, int n) { return (rows + bm - 1) / bm + n - 1; };
    const auto shared_tiles = [&](int bm) { return tiles_of(bm, x.groups); };
    const auto own_tiles = [&](int bm) { return a.q_start ? tiles_of(bm, a.batch) : (int64_t)a.batch * ((group + bm - 1) / bm); };
    // What 64 keys cost a row tile of 128, in those of 16 rows.
    const int many_cost = a.dtype == RQ_F16 && c.head_dim == 128 ? 6 : 4;
    PrefixPlan p{};
    p.own_copies = rows / a.batch <= 4 ? 4 : rows / a.batch <= 8 ? 2 : 1;
    const int64_t few = own_tiles(16 / p.own_copies), own_few = few * own_keys;
    const int64_t shared_few = shared_tiles(16) * shared_keys, shared_many = many_cost * shared_tiles(128) * shared_keys, own_many = many_cost * own_tiles(128) * own_keys;
    // (a launch more for the rows behind the prefixes, a start and partial results of 128 rows: 30 us.  bf16, 32 heads on 8: 64 queries x 8192 few
    // 34, many 44; x 32768 98, 73; 16 x 65536 54, 63.  fp16, 64 heads on 8: 4 sequences of 40 tokens x 8192 74, 97; 12 of 20 x 32768 387, 306.)
    p.many = (shared_few - shared_many) * c.kv_heads > 90 * (int64_t)num_cu;
    p.own_many = own_many < own_few && own_few * c.kv_heads > 256 * (int64_t)num_cu;
    // Chunks of as many tiles of keys as cost least, in steps of 1.5 us.  A workgroup takes `at_once` tiles a step and kStart steps besides; the
    // chip holds per_cu * num_cu of them.  Those for many rows are all alike and take whole rounds; of those for few rows, which are of all
    // lengths, one begins when another ends, and the last ends kTail of the longest after most have.  Partial results are written and read
    // again at 4 TB/s.  (64 queries of 32 heads on 8 against 8192 keys: 33 us, in whole rounds 34.5; 90 queries of 7 tokens, 32 heads, 1000
    // keys: 64 and 84; 12 of 40 tokens x 64 heads on 8, 65411 keys, many rows: 1144 and 1095.)
    constexpr int kStart = 3;
    constexpr double kTail = 0.25;
    const double join = 2.0 * a.tokens * a.heads * c.head_dim * sizeof(float) / 6e6;
    const auto chunks_of = [](int64_t keys, int64_t each) { return (keys + each - 1) / each; };
    const auto time_of = [&](int64_t sum, int64_t longest, int64_t per_cu) {
        const double t = (double)sum / (double)(per_cu * num_cu) + kTail * (double)longest;
        return t > (double)longest ? t : (double)longest;
    };
    const auto split = [&](int64_t shared_tiles, int64_t own_tiles, int at_once, int64_t per_cu, bool many) {
        const int64_t most = shared_tiles && (shared_keys > own_keys || !own_tiles) ? shared_keys : own_keys;
        double least = 0.0;
        int64_t best = most;
        for (int64_t n = 1; n <= 256 && (n == 1 || n * at_once <= most); ++n) {
            const int64_t each = chunks_of(most, n), shared_n = shared_tiles ? chunks_of(shared_keys, each) : 0, own_n = own_tiles ? chunks_of(own_keys, each) : 0;
            const auto steps = [&](int64_t keys) { return chunks_of(each < keys ? each : keys, at_once) + kStart; };
            const int64_t sum = (shared_tiles * shared_n * steps(shared_keys) + own_tiles * own_n * steps(own_keys)) * c.kv_heads;
            const double cost = (many ? (double)(chunks_of(sum / steps(most), per_cu * num_cu) * steps(most)) : time_of(sum, steps(most), per_cu)) + join * (double)(shared_n + own_n);
            if (n > 1 && cost >= least) continue;
            least = cost;
            best = each;
        }
        if (shared_tiles) {
            p.shared_chunk = (int)(best * kTile);
            p.shared_chunks = (int)chunks_of(shared_keys, best);
        }
        if (own_tiles) {
            p.own_chunk = (int)(best * kTile);
            p.own_chunks = (int)chunks_of(own_keys, best);
        }
        return least;
    };
    p.groups = a.dtype != RQ_F16 || c.head_dim == 64 ? 2 : 1;
    p.shared_tiles = (int)shared_tiles(p.many ? 128 : 16);
    p.own_tiles = (int)(p.own_many ? own_tiles(128) : few);
    if (p.many) split(p.shared_tiles, 0, p.groups, p.groups == 2 ? 1 : 2, true);
    const double together = split(p.many ? 0 : p.shared_tiles, p.own_many ? 0 : p.own_tiles, 4, 2, false);
    if (p.own_many) split(0, p.own_tiles, 1, 2, true);
    // One launch takes every sequence by itself where the chip has that done before the prefixes' reuse pays for joining, kJoin steps.
    // (Apart and together, 25 own positions, bf16, 32 heads of 128 on 8: 2 to 16 queries x 300 10.1 and 11.4 .. 11.8, x 700 11.1 and 10.1 .. 10.6, x 1000 12.1 and
    // 10.3 .. 10.8, x 4000 23.3 and 12.7 .. 13.8; 32 x 700 11.3 and 12.5, x 2000 16.1 and 13.4.  fp16, 16 heads of 64 in 2 groups, 100 own: 4 x 500 7.6 and 11.3,
    // 16 x 1000 9.3 and 11.8, x 4000 17.9 and 13.7; 160 x 1000 37 and 27.  The rule errs by 1.3 at most for the former, by 2.5 .. 3.8 for 16 x 500, 4 x 1000 and
    // 16 x 1000 of the latter, which it takes together.)
    constexpr double kJoin = 1.7;
    const int waves = few * c.kv_heads <= num_cu ? 8 : 4;
    const int64_t each = chunks_of(shared_keys, waves) + chunks_of(own_keys, waves) + kStart;
    const double apart = time_of(few * c.kv_heads * each, each, waves == 8 ? 1 : 2);
    if (a.window != 0 || x.max_len < kTile || (!p.many && !p.own_many && apart <= together + kJoin)) {
        const int copies = p.own_copies;
        p = PrefixPlan{};
        p.separate = true;
        p.own_copies = copies;
        p.own_tiles = (int)few;
        p.waves = waves;
        return p;
    }
    // Partial results of as many tokens as kMostBytes hold (one at least), in turns of alike length: two chunks of 8 sequences of 4096 queries, 64
    // heads of 128, would take 2.2 GB.  A turn has thousands of row tiles, and the tiles of a sequence or group that two turns share at their border
    // are all that is taken twice (64 x 2048 queries of 64 heads on 8 behind 8192, bf16: 33.0 ms in 8 turns, 32.3 in one with 8.1 GB).
    const size_t token_bytes = (size_t)(p.shared_chunks + p.own_chunks) * a.heads * (c.head_dim + 1) * sizeof(float);
    const int64_t most_tokens = (int64_t)(kMostBytes / token_bytes), turns = chunks_of(a.tokens, most_tokens > 1 ? most_tokens : 1);
    p.slice = (int)chunks_of(a.tokens, turns);
    p.bytes = p.slice * token_bytes;
    return p;
}

template <int D, int F, bool F16, bool PAGED>
void launch_few(const PrefixJob& job, const SharedPart& shared, const PrefixPlan& p, hipStream_t s) {
    if (p.separate) {
        const dim3 grid = item_grid(job.cache.kv_heads, job.tiles);
        if (p.waves == 8) launch_kernel(k_kv4_prefix_separate<D, F, F16, PAGED, 8>, grid, dim3(512), 0, s, job);
        else launch_kernel(k_kv4_prefix_separate<D, F, F16, PAGED, 4>, grid, dim3(256), 0, s, job);
        return;
    }
    const int64_t items = (int64_t)(shared.tiles - shared.first_tile) * shared.chunks + (int64_t)(job.tiles - job.first_tile) * job.chunks;
    if (items) launch_kernel(k_kv4_prefix<D, F, F16, PAGED>, item_grid(job.cache.kv_heads, items), dim3(256), 0, s, job, shared);
}
template <int D, int F, bool F16>
void launch_few(const PrefixJob& job, const SharedPart& shared, const PrefixPlan& p, hipStream_t s) {
    if (job.cache.page_shift < 6) launch_few<D, F, F16, true>(job, shared, p, s);
    else launch_few<D, F, F16, false>(job, shared, p, s);
}
template <int D, bool F16>
void launch_few(const PrefixJob& job, const SharedPart& shared, const PrefixPlan& p, hipStream_t s) {
    if (p.own_copies == 4) launch_few<D, 4, F16>(job, shared, p, s);
    else if (p.own_copies == 2) launch_few<D, 2, F16>(job, shared, p, s);
    else launch_few<D, 1, F16>(job, shared, p, s);
}
// `job`: sequences by themselves, or what is behind the prefixes; `shared`: the prefixes.  Either may have no row tiles.
void launch_few(const PrefixJob& job, const SharedPart& shared, const PrefixPlan& p, hipStream_t s) {
    const bool f16 = job.a.dtype == RQ_F16;
    if (job.cache.head_dim == 128) f16 ? launch_few<128, true>(job, shared, p, s) : launch_few<128, false>(job, shared, p, s);
    else f16 ? launch_few<64, true>(job, shared, p, s) : launch_few<64, false>(job, shared, p, s);
}

// Row tiles of BM rows that have rows of tokens begin .. end - 1, where tiles begin at floor(first row / BM) + number (find_rows, find_group_rows) for
// `stretches` of rows; `tiles`: of all tokens.
struct Tiles {
    int first, end;
};
Tiles tiles_of_tokens(int bm, int group, int begin, int end, int stretches, int tiles) {
    // (a row's place is that of its stretch's first one and what it lies behind it, each rounded down)
    const int64_t first = (int64_t)begin * group / bm - 1, last = ((int64_t)end * group - 1) / bm + stretches - 1;
    return Tiles{(int)(first > 0 ? first : 0), (int)(last + 1 < tiles ? last + 1 : tiles)};
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
    r.shared_rows = p.separate ? 0 : p.many ? 128 : 16;
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
        launch_few(job, SharedPart{}, p, s);
        return launch_rc();
    }
    job.part_chunks = p.shared_chunks + p.own_chunks;
    job.part_first = p.shared_chunks;
    const int shared_bm = p.many ? 128 : 16, own_bm = p.own_many ? 128 : 16 / p.own_copies;
    const int own_each = (job.group + own_bm - 1) / own_bm;           // row tiles of a token that is a sequence
    for (job.slice = 0; job.slice < a.tokens; job.slice = job.slice_end) {
        job.slice_end = job.slice + (p.slice < a.tokens - job.slice ? p.slice : a.tokens - job.slice);
        const Tiles own = a.q_start ? tiles_of_tokens(own_bm, job.group, job.slice, job.slice_end, a.batch, p.own_tiles)
                                    : Tiles{job.slice * own_each, job.slice_end * own_each};
        const Tiles prefixes = tiles_of_tokens(shared_bm, job.group, job.slice, job.slice_end, x.groups, p.shared_tiles);
        PrefixJob part = job;
        part.first_tile = own.first;
        part.tiles = own.end;
        if (p.own_many) launch_prefix_many(part, Part::kOwn, 1, s);
        if (p.own_many) part.first_tile = part.tiles = 0;
        launch_few(part, p.many ? SharedPart{} : SharedPart{prefixes.first, prefixes.end, p.shared_chunk, p.shared_chunks}, p, s);
        if (p.many) {
            part.first_tile = prefixes.first;
            part.tiles = prefixes.end;
            part.chunk = p.shared_chunk;
            part.chunks = p.shared_chunks;
            part.part_first = 0;
            launch_prefix_many(part, Part::kShared, p.groups, s);
        }
        part.chunks = job.part_chunks;
        part.first_token = job.slice;
        part.a.tokens = job.slice_end - job.slice;
        part.a.o = static_cast<uint16_t*>(a.o) + job.slice * a.o_token;
        part.a.lse = a.lse ? a.lse + (int64_t)job.slice * a.heads : nullptr;
        launch_join(part, s);
    }
    return launch_rc();
}

}  // namespace rq
