// Attention of sequences that share a prefix: launches of the kernel for many rows, of which each leaves partial results.
#include "kv4_many_rows.h"
#include "kv4_prefix.h"

namespace rq {
namespace {

template <int D, int GROUPS, bool F16, bool PAGED, Part PART>
__global__ __launch_bounds__(256 * GROUPS, 2) void k_prefix_many(PrefixJob job) {
    many_rows<D, 4, GROUPS, F16, PAGED, PART>(job);
}

template <int D, bool F16, bool PAGED>
void launch(const PrefixJob& job, Part part, int groups, hipStream_t s) {
    const dim3 grid = item_grid(job.cache.kv_heads, (int64_t)(job.tiles - job.first_tile) * job.chunks), block(256 * groups);
    if (part == Part::kOwn) {
        launch_kernel(k_prefix_many<D, 1, F16, PAGED, Part::kOwn>, grid, block, 0, s, job);
        return;
    }
    if constexpr (D == 64 || !F16)
        if (groups == 2) {
            launch_kernel(k_prefix_many<D, 2, F16, PAGED, Part::kShared>, grid, block, 0, s, job);
            return;
        }
    launch_kernel(k_prefix_many<D, 1, F16, PAGED, Part::kShared>, grid, block, 0, s, job);
}
template <int D, bool F16>
void launch(const PrefixJob& job, Part part, int groups, hipStream_t s) {
    if (job.cache.page_shift < 6) launch<D, F16, true>(job, part, groups, s);
    else launch<D, F16, false>(job, part, groups, s);
}

}  // namespace

void launch_prefix_many(const PrefixJob& job, Part part, int groups, hipStream_t s) {
    const bool f16 = job.a.dtype == RQ_F16;
    if (job.cache.head_dim == 128) f16 ? launch<128, true>(job, part, groups, s) : launch<128, false>(job, part, groups, s);
    else f16 ? launch<64, true>(job, part, groups, s) : launch<64, false>(job, part, groups, s);
}

}  // namespace rq
