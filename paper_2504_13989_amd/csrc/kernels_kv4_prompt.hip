// Attention over the 4-bit paged cache for many queries a sequence: launches of the kernel of kv4_many_rows.h.
#include "kv4_many_rows.h"

namespace rq {
namespace {

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
