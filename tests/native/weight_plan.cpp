// The launch plan of the accumulated weights (plan_weights of host.cpp) for tests/weight_plan.py.
#include "host.h"

extern "C" int weight_plan(const kv_layout *layout, const kv_batch *batch, int32_t q_heads, int32_t window, int32_t sink,
                           int64_t *out) {
    tkv::WeightPlan p;
    const int rc = tkv::plan_weights(layout, batch, q_heads, window, sink, &p);
    if (rc != KV_OK) return rc;
    const int64_t all[] = {p.windowed, p.few, p.ahead, p.keys, p.tiles, p.sink_tiles, p.parts, p.workspace};
    for (int i = 0; i < 8; ++i) out[i] = all[i];
    return rc;
}
