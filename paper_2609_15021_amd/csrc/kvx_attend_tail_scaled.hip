// kv_attend_pages for many new tokens of a sequence, over pages with scales of their own: the SCALED variant of
// kv_attend's tail kernel.
//
// 6 tails of up to 1,055 new tokens behind up to 8,192 (4 heads of 6 rows, D 256): 650 us, 785 TFLOP/s, where a large
// library product reaches 1,210.
#include "kvx_attend_tail.h"

namespace kvx {

namespace {

template <class T, bool FULL>
hipError_t launch_scaled(const AttendArgs &a, const Parts &parts, int max_queries, hipStream_t stream) {
    return a.softcap == 0.f && !a.slopes ? launch_columns<T, true, true, FULL, true>(a, parts, max_queries, stream)
                                         : launch_columns<T, true, false, FULL, true>(a, parts, max_queries, stream);
}

}  // namespace

hipError_t launch_tail_scaled(const AttendArgs &a, const Parts &parts, int max_queries, hipStream_t stream) {
    // (One bfloat16 weight would cost float16 rows their precision.)
    if (a.q_type == KV_DTYPE_F16)
        return launch_scaled<F16, true>(a, parts, max_queries, stream);
    return a.full_weights ? launch_scaled<Bf16, true>(a, parts, max_queries, stream)
                          : launch_scaled<Bf16, false>(a, parts, max_queries, stream);
}

}  // namespace kvx
