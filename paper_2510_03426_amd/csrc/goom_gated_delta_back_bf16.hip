// The gated delta rule: the backward walks and the gradients within chunks, for bf16.
#include "goom_gated_delta_walk.h"

namespace goom_layer {

template <> int launch_delta_back<bf16>(goom_ctx *ctx, const DeltaArgs &w, int mode, long long slots, const char *label)
{
    return launch_delta_walk_typed<bf16, BACK_MAPS, BACK, BACK>(ctx, w, mode, slots, label);
}

template <> int launch_delta_gradients<bf16>(goom_ctx *ctx, const DeltaArgs &w, long long slots) { return launch_delta_gradients_typed<bf16>(ctx, w, slots); }

} // namespace goom_layer
