// The walks of linear attention over floats.
#include "goom_linear_attention_walk.h"

namespace goom_layer {

template <> int launch_walks_of<float>(goom_ctx *ctx, const WalkArgs &w, int roles, long long slots, const char *label)
{
    return launch_walks_typed<float>(ctx, w, roles, slots, label);
}

} // namespace goom_layer
