// The gated delta rule: what lies within chunks, and the forward walks, for bf16.
#include "goom_gated_delta_walk.h"

namespace goom_layer {

template <> int launch_delta_within<bf16>(goom_ctx *ctx, const DeltaArgs &w, long long slots) { return launch_delta_within_typed<bf16>(ctx, w, slots); }

template <> int launch_delta_walk<bf16>(goom_ctx *ctx, const DeltaArgs &w, int mode, long long slots, const char *label)
{
    return launch_delta_walk_typed<bf16, FORWARD, MAPS, KEEP>(ctx, w, mode, slots, label);
}

} // namespace goom_layer
