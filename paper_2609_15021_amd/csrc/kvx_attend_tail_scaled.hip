// kv_attend_pages for many new tokens of a sequence, over pages with scales of their own: the SCALED variant of
// kv_attend's tail kernel.
//
// Weights always meet V as two numbers: one of bfloat16 would cost float16 rows their precision, and leave bfloat16
// ones off by 0.0022 of their norm instead of 0.0017, their own rounding.  6 tails of up to 1,055 new tokens behind up
// to 8,192 (4 heads of 6 rows, D 256): 768 us, 667 TFLOP/s, where a large library product reaches 1,210 (1,000 with the
// second product counted).  With 128 columns, a cap or slopes spill 7 to 13 of 256 registers.
#include "kvx_attend_tail.h"

namespace kvx {

namespace {

template <class T>
hipError_t launch_scaled(const AttendArgs &a, const Parts &parts, int max_queries, hipStream_t stream) {
    return a.softcap == 0.f && !a.slopes ? launch_columns<T, true, true, true, true>(a, parts, max_queries, stream)
                                         : launch_columns<T, true, false, true, true>(a, parts, max_queries, stream);
}

}  // namespace

hipError_t launch_tail_scaled(const AttendArgs &a, const Parts &parts, int max_queries, hipStream_t stream) {
    return a.q_type == KV_DTYPE_BF16 ? launch_scaled<Bf16>(a, parts, max_queries, stream)
                                     : launch_scaled<F16>(a, parts, max_queries, stream);
}

}  // namespace kvx
