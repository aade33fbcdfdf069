// What the experts' products (experts.hip) need of the order of the rows (route.hip).
#ifndef BT_ROUTE_H
#define BT_ROUTE_H

#include "block.h"

namespace btb {

// The numbers of a plan.
bt_status check_plan(const bt_expert_plan *p);

// out[t] = the sum of a token's rows of y, [rows, cols] in single precision; out of `dtype`.
bt_status sum_rows(const bt_expert_plan &p, const float *y, uint64_t cols, bt_dtype dtype, void *out, hipStream_t hs);

}  // namespace btb
#endif  // BT_ROUTE_H
