// Rotary positions: pairs of a head's entries turned by position times frequency.
//
//     (x1, x2) -> scale (x1 cos a - x2 sin a, x1 sin a + x2 cos a),   a = position frequency
//
// Bound by the bytes of q and k, read and written once.  A thread has V pairs of a token and goes through some of its heads with the
// same sines and cosines (32,768 tokens of 16 + 16 heads of 128, bfloat16, both ways: 190 us, 5.6 TB/s).  Angles are products in two
// doubles, taken to a fraction of a turn there: positions up to 2^53 cost no accuracy (a single double's product is off by 2^-10 of a turn from 2^40 on).
#include <cmath>

#include "goom_real.h"

namespace goom_layer {

struct RotaryArgs {
    const void *q, *k;
    void *q_out, *k_out;
    const int64_t *positions;
    const float *frequencies;
    long long tokens, q_tok, q_head, k_tok, k_head;
    int heads, kv_heads, dim, pairs, blocks; // blocks: threads that share a token's heads
    int turned, copied;                      // units of V pairs, and of V entries that are copied
    int group;                               // 0, or rows of units of a workgroup
    float scale, sign;
};

constexpr double ONE_BY_2PI = 0.15915494309189535, ONE_BY_2PI_REST = -9.839338337591243e-18; // 1 / 2 pi to 107 bits

template <typename S, int V, bool INTER> __global__ __launch_bounds__(256) void rotary_kernel(RotaryArgs a)
{
    const int units = a.turned + a.copied;
    long long row;
    int u;
    if (a.group) { // rows of a workgroup, their pairs first: what a wave does is mostly one or the other
        const int x = threadIdx.x, pairs = a.group * a.turned;
        if (x >= a.group * units) return;
        const int r = x < pairs ? x / a.turned : (x - pairs) / a.copied;
        u = x < pairs ? x - r * a.turned : a.turned + (x - pairs - r * a.copied);
        row = block_of() * a.group + r;
    } else {
        const long long id = block_of() * 256 + threadIdx.x;
        row = id / units;
        u = (int)(id - row * units);
    }
    const long long token = row >> 32 ? row / a.blocks : (unsigned)row / (unsigned)a.blocks;
    const int block = (int)(row - token * a.blocks);
    if (token >= a.tokens) return;
    const int all = a.heads + a.kv_heads;
    // a head's rows, and where its results go
    auto rows = [&](int h, const S *&from, S *&to) {
        if (h < a.heads) {
            from = reinterpret_cast<const S *>(a.q) + token * a.q_tok + h * a.q_head;
            to = reinterpret_cast<S *>(a.q_out) + (token * a.heads + h) * a.dim;
        } else {
            from = reinterpret_cast<const S *>(a.k) + token * a.k_tok + (h - a.heads) * a.k_head;
            to = reinterpret_cast<S *>(a.k_out) + (token * a.kv_heads + h - a.heads) * a.dim;
        }
    };
    if (u >= a.turned) { // entries behind the pairs; the last unit ends with the head and shares entries with the one before
        const int rest = a.dim - 2 * a.pairs, n = rest < V ? rest : V, at = (u - a.turned) * V, first = 2 * a.pairs + (at + n <= rest ? at : rest - n);
        for (int h = block; h < all; h += a.blocks) {
            const S *from;
            S *to;
            rows(h, from, to);
            if (n == V) {
                float x[V];
                load_floats_unaligned<S, V>(from + first, x);
                store_floats_unaligned<S, V>(to + first, x);
            } else {
                for (int e = 0; e < n; e++) to[first + e] = from[first + e];
            }
        }
        return;
    }
    const int first = u * V + V <= a.pairs ? u * V : a.pairs - V; // (V is at most the number of pairs)
    float c[V], s[V];
    const double position = (double)a.positions[token];
#pragma unroll
    for (int e = 0; e < V; e++) {
        // turns a position in two doubles; of the product the whole turns go before anything is rounded
        const double f = a.frequencies[first + e], each = f * ONE_BY_2PI, rest = __builtin_fma(f, ONE_BY_2PI_REST, __builtin_fma(f, ONE_BY_2PI, -each));
        const double turns = __builtin_fma(position, rest, __builtin_fma(position, each, -rint(position * each)));
        sincospif(2.0f * (float)(turns - rint(turns)), &s[e], &c[e]);
        s[e] *= a.scale * a.sign;
        c[e] *= a.scale;
    }
#pragma unroll 2
    for (int h = block; h < all; h += a.blocks) {
        const S *from;
        S *to;
        rows(h, from, to);
        if (INTER) {
            float x[2 * V];
            load_floats_unaligned<S, 2 * V>(from + 2 * first, x);
#pragma unroll
            for (int e = 0; e < V; e++) {
                const float one = x[2 * e], two = x[2 * e + 1];
                x[2 * e] = one * c[e] - two * s[e];
                x[2 * e + 1] = one * s[e] + two * c[e];
            }
            store_floats_unaligned<S, 2 * V>(to + 2 * first, x);
        } else {
            float one[V], two[V];
            load_floats_unaligned<S, V>(from + first, one);
            load_floats_unaligned<S, V>(from + a.pairs + first, two);
#pragma unroll
            for (int e = 0; e < V; e++) {
                const float x = one[e], y = two[e];
                one[e] = x * c[e] - y * s[e];
                two[e] = x * s[e] + y * c[e];
            }
            store_floats_unaligned<S, V>(to + first, one);
            store_floats_unaligned<S, V>(to + a.pairs + first, two);
        }
    }
}

} // namespace goom_layer

using namespace goom_layer;
using goom::aligned;
using goom::fail;

extern "C" int goom_rotary(goom_ctx *ctx, const goom_rotary_shape *shape, const void *q, const void *k, const int64_t *positions, const float *frequencies, void *q_out,
                           void *k_out)
{
    if (!shape) return fail(ctx, GOOM_EINVAL, "null shape");
    const goom_rotary_shape &sh = *shape;
    if (!real_type(sh.type)) return fail(ctx, GOOM_EINVAL, "unknown element type %d", sh.type);
    if (sh.flags & ~(GOOM_ROTARY_INTERLEAVED | GOOM_ROTARY_BACK)) return fail(ctx, GOOM_EINVAL, "unknown flags 0x%x", (unsigned)sh.flags);
    if (sh.tokens < 0) return fail(ctx, GOOM_EINVAL, "negative number of tokens");
    if (sh.heads <= 0 || sh.kv_heads < 0) return fail(ctx, GOOM_EINVAL, "heads must be positive, kv_heads not negative");
    if (sh.dim <= 0 || sh.pairs <= 0 || sh.pairs > sh.dim / 2) return fail(ctx, GOOM_EINVAL, "pairs must be positive, and two times that at most dim");
    if (!std::isfinite((float)sh.scale)) return fail(ctx, GOOM_EINVAL, "scale must be finite, and a float");
    if (sh.heads > (1 << 20) || sh.kv_heads > (1 << 20) || sh.dim > (1 << 20) || ((int64_t)sh.heads + sh.kv_heads) * sh.dim > (1 << 30) || sh.tokens > (1ll << 40) / (((int64_t)sh.heads + sh.kv_heads) * sh.dim))
        return fail(ctx, GOOM_EUNSUPPORTED, "too many tokens, heads or entries");
    int64_t q_tok = sh.q_token, q_head = sh.q_head, k_tok = sh.k_token, k_head = sh.k_head;
    for (int64_t x : {q_tok, q_head, k_tok, k_head})
        if (x < 0 || x > (1ll << 40)) return fail(ctx, GOOM_EINVAL, "strides of tokens and heads must be 0 (both: contiguous) or at least a head's entries");
    if (((q_tok || q_head) && (q_tok < sh.dim || q_head < sh.dim)) || ((k_tok || k_head) && (k_tok < sh.dim || k_head < sh.dim)))
        return fail(ctx, GOOM_EINVAL, "strides of tokens and heads must be 0 (both: contiguous) or at least a head's entries");
    if (!q_tok) { q_tok = (int64_t)sh.heads * sh.dim; q_head = sh.dim; }
    if (!k_tok) { k_tok = (int64_t)sh.kv_heads * sh.dim; k_head = sh.dim; }
    if (sh.tokens > 0 && (!q || !q_out || !positions || !frequencies || (sh.kv_heads && (!k || !k_out)))) return fail(ctx, GOOM_EINVAL, "null data pointer");
    const size_t size = real_bytes(sh.type);
    if (!aligned(q, size) || !aligned(k, size) || !aligned(q_out, size) || !aligned(k_out, size) || !aligned(positions, 8) || !aligned(frequencies, 4))
        return fail(ctx, GOOM_EINVAL, "misaligned data pointer");
    if (int s = enter(ctx)) return s;
    if (sh.tokens == 0) return GOOM_OK;
    return with_type(sh.type, [&](auto tag) {
        typedef typename decltype(tag)::type S;
        auto run = [&](auto v) {
            constexpr int V = decltype(v)::value;
            RotaryArgs a = {q, k, q_out, k_out, positions, frequencies, sh.tokens, q_tok, q_head, k_tok, k_head, sh.heads, sh.kv_heads, sh.dim, sh.pairs};
            a.scale = (float)sh.scale;
            a.sign = sh.flags & GOOM_ROTARY_BACK ? -1.0f : 1.0f;
            a.turned = (sh.pairs + V - 1) / V;
            const int rest = sh.dim - 2 * sh.pairs;
            a.copied = (rest + V - 1) / V;
            const int all = sh.heads + sh.kv_heads;
            // a thread for each head where that leaves fewer threads than the chip holds
            const long long threads = sh.tokens * (a.turned + a.copied) * all;
            const int each = threads > (1 << 20) ? 4 : 1;
            a.blocks = (all + each - 1) / each;
            const int units = a.turned + a.copied;
            a.group = units <= 64 && rest ? 256 / units : 0; // (pairs and copies in one wave: 38 us for 36; without copies one thread after another 98 us for 100)
            const dim3 grid = a.group ? grid_of((sh.tokens * a.blocks + a.group - 1) / a.group, 256) : grid_of((sh.tokens * a.blocks * units + 255) / 256, 256);
            goom::prof_begin(ctx, "rotary positions");
            if (sh.flags & GOOM_ROTARY_INTERLEAVED) rotary_kernel<S, V, true><<<grid, 256, 0, ctx->stream>>>(a);
            else rotary_kernel<S, V, false><<<grid, 256, 0, ctx->stream>>>(a);
            goom::prof_end(ctx);
            return goom::check_hip(ctx, hipGetLastError(), "rotary positions");
        };
        // Four pairs a thread, two of neighbouring floats: a lane's access has 16 bytes at most and lies beside the next lane's.  Twice as many, us: 10,005
        // tokens of 16 heads of 77, 19 pairs of neighbouring floats 36 and 28, of 53, 26 of halves 17 and 13, of 128, pairs of floats 34 and 30; 32,768 of 32 heads
        // of 128 in bfloat16, both halves of a head 98 and 94.
        const bool two = sizeof(S) == 4 && (sh.flags & GOOM_ROTARY_INTERLEAVED);
        if (!two && sh.pairs >= 4) return run(std::integral_constant<int, 4>());
        if (sh.pairs >= 2) return run(std::integral_constant<int, 2>());
        return run(std::integral_constant<int, 1>());
    });
}
