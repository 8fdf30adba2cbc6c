// kv_attend_pages: kv_attend over pages with scales of their own, or over the pages that each new token chose.
//
// Scales are kv_attend with the kernels' SCALED variants (kvx_attend_step.h, kvx_attend_tail.h).  Over chosen pages
// each new token is a sequence of its own to the step kernel, and its list, cut into parts where the rows alone do not
// fill the chip, what that goes over; nothing is shared between tokens, whose choices differ.
//
// One token over 256 of 8,193 pages of 16 (8 heads of 5 rows, bf16, D 128; 17 MB): 9.2 us, launch and four dependent
// reads, and 3.9 to join 32 parts.  48 tokens over 128 pages each (2 heads of 8 rows, 96 MB, 15 us at 6.3 TB/s): 22 us
// and 4 to join.  2,048 new tokens of 8 heads over 64 pages each take 615 us, 14 TB/s, mostly from the caches.
// Scales cost decoding nothing: 16 sequences of up to 32,768 tokens (e4m3, 4 heads of 6 rows, D 256) take 114 us and 6
// to join, 4.9 TB/s.
#include "kvx_attend_step.h"

namespace kvx {

hipError_t launch_step_scaled(const AttendArgs &a, const Shares &shares, int max_queries, hipStream_t stream) {
    const int max_rows = static_cast<int>(std::min<int64_t>(a.step_rows, static_cast<int64_t>(max_queries) * a.group));
    return a.q_type == KV_DTYPE_BF16 ? launch_rows<Bf16, true, true>(a, shares, shares.items, max_rows, stream)
                                     : launch_rows<F16, true, true>(a, shares, shares.items, max_rows, stream);
}

namespace {

template <class From>
hipError_t launch_chosen(const AttendArgs &a, const From &chosen, hipStream_t stream) {
    const int items = a.batch.num_queries * chosen.splits;
    if (a.cache_type == KV_DTYPE_E4M3)
        return a.q_type == KV_DTYPE_BF16 ? launch_rows<Bf16, true, true>(a, chosen, items, a.group, stream)
                                         : launch_rows<F16, true, true>(a, chosen, items, a.group, stream);
    return a.q_type == KV_DTYPE_BF16 ? launch_rows<Bf16, false, false>(a, chosen, items, a.group, stream)
                                     : launch_rows<F16, false, false>(a, chosen, items, a.group, stream);
}

}  // namespace

hipError_t launch_pages(const AttendArgs &a, const Chosen &chosen, hipStream_t stream) {
    return launch_chosen(a, chosen, stream);
}

hipError_t launch_pages(const AttendArgs &a, const Alone &chosen, hipStream_t stream) {
    return launch_chosen(a, chosen, stream);
}

}  // namespace kvx
