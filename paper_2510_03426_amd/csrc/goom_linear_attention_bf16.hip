// The walks of linear attention over bfloat16.
#include "goom_linear_attention_walk.h"

namespace goom_layer {

template <> int launch_walks_of<bf16>(goom_ctx *ctx, const WalkArgs &w, int roles, long long slots, const char *label)
{
    return launch_walks_typed<bf16>(ctx, w, roles, slots, label);
}

} // namespace goom_layer
