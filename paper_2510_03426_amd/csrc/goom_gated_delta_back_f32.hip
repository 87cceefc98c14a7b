// The gated delta rule: the backward walks and the gradients within chunks, for float.
#include "goom_gated_delta_walk.h"

namespace goom_layer {

template <> int launch_delta_back<float>(goom_ctx *ctx, const DeltaArgs &w, int mode, long long slots, const char *label)
{
    return launch_delta_walk_typed<float, BACK_MAPS, BACK, BACK>(ctx, w, mode, slots, label);
}

template <> int launch_delta_gradients<float>(goom_ctx *ctx, const DeltaArgs &w, long long slots) { return launch_delta_gradients_typed<float>(ctx, w, slots); }

} // namespace goom_layer
