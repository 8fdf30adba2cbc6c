// kv_attend_pages: kv_attend over pages with scales of their own, or over the pages that each new token chose.
//
// Scales are kv_attend with the kernels' SCALED variants (kvx_attend_step.h, kvx_attend_tail.h).  Over chosen pages each
// new token is a sequence of its own to the step kernel, and its list, cut into parts where the rows alone do not fill the
// chip, what that goes over; nothing is shared between tokens, whose choices differ.
#include "kvx_attend_step.h"

namespace kvx {

hipError_t launch_step_scaled(const AttendArgs &a, const Shares &shares, int max_queries, hipStream_t stream) {
    const int max_rows = static_cast<int>(std::min<int64_t>(kStepRows, static_cast<int64_t>(max_queries) * a.group));
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
