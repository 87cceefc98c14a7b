// Norms before and after a block of a layer, with its gate and its residual stream, and their gradients.
//
//     after:  y = residual + scale (norm(x) weight + bias) act(gate)
//     before: h = residual + scale x act(gate),   y = norm(h) weight + bias
//
// Bound by the bytes of their tensors, each read and written once: a team of lanes holds one token's group in registers, 8 entries a lane
// (16 for the longest), and statistics are taken about the mean itself.  A team keeps its group from token to token, so parameters are
// loaded once and their gradients are summed in registers: one partial sum for each workgroup and channel, added up in a fixed order by a
// second launch.  32,768 tokens of 2048 channels, bfloat16, before a block, both ways: 269 us, 5.0 TB/s.
#include <cmath>

#include "goom_activation.h"

namespace goom_layer {

struct BlockNormArgs {
    const void *x, *gate, *residual, *h, *gy, *gh;
    const void *weight, *bias, *scale;
    void *y, *h_out, *gx, *ggate, *gres;
    float *mean, *rstd;      // forward: outputs (may be NULL); backward: inputs
    long long tokens;
    int channels, groups, cg; // cg: channels of a group
    int type_w, act, layer;
    float eps;
    int team, gpw, ipw;      // lanes of a team; groups and tokens that a workgroup has at once
    float *partial;          // [workgroups along x][3][channels]: gradients of weight, bias, scale
};

// Sums over a team: of up to 64 lanes by shuffles, of whole workgroups through LDS (two buffers in turn: one barrier a sum)
struct TeamSum {
    float (*meet)[2][16];
    int team, turn;
    __device__ inline void operator()(float &a, float &b)
    {
        const int within = team < 64 ? team : 64;
        for (int s = 1; s < within; s *= 2) {
            a += __shfl_xor(a, s);
            b += __shfl_xor(b, s);
        }
        if (team > 64) {
            float (*const m)[16] = meet[turn];
            turn ^= 1;
            if ((threadIdx.x & 63) == 0) {
                m[0][threadIdx.x >> 6] = a;
                m[1][threadIdx.x >> 6] = b;
            }
            __syncthreads();
            a = b = 0.0f;
            for (int w = 0; w < team / 64; w++) {
                a += m[0][w];
                b += m[1][w];
            }
        }
    }
};

// Unit u of a group: V channels from u V on, the last one V channels up to its end, whose first `skip` are the unit before's as
// well and count there.  Lane l of a team has the units l, l + team, ...  grid: (workgroups over tokens, parts of the groups)
template <typename S, int V, int J, int MOST, bool BEFORE, bool BACK> __global__ __launch_bounds__(MOST) void block_norm_kernel(BlockNormArgs a)
{
    __shared__ float meet[2][2][16];
    TeamSum sums = {meet, a.team, 0};
    const int lane = threadIdx.x % a.team, team = threadIdx.x / a.team, ti = team / a.gpw, group = blockIdx.y * a.gpw + team % a.gpw;
    const bool live = ti < a.ipw && group < a.groups;
    const int units = (a.cg + V - 1) / V;
    const float count = (float)a.cg;
    const bool gated = a.gate, scaled = a.scale;
    int chan[J], skip[J];
    // What 128 registers (1024 lanes) do not hold spills: with 16 entries a lane the parameters, read from L2 again for each token instead, and the next
    // token's entries, which are then not asked for ahead; with 8 floats the parameters on the way back.  4096 tokens of 16,384 channels, both held and
    // not, us: backwards 617 and 391 (bfloat16), 1353 and 611 (float), forwards in float 341 and 221; forwards in halves holding is faster, 110 and 125, though
    // some spills; 8192 tokens of 8192, backwards: float 578 and 439, bfloat16 181 and 201.  Scratch that is left, bytes a lane after and before a block: 16 entries
    // backwards 136 and 156 in 16 bits, 132 and 224 in floats, forwards 68 and 12 in bfloat16, 52 and 12 in halves; 8 entries of 1024 lanes, backwards, 60 and 20 in 16 bits, 0 and 72.
    constexpr bool WIDE = J * V == 16, SMALL = sizeof(S) == 2, AHEAD = !WIDE || (SMALL && !BACK), HOLD = WIDE ? SMALL && !BACK : SMALL || !(BACK && MOST == 1024);
    float w[HOLD ? J : 1][V], b[HOLD ? J : 1][V], sc[HOLD ? J : 1][V], sw[J][V], sb[J][V], ss[J][V];
    auto read_params = [&](int j, int at) {
        params<V>(a.weight, a.type_w, at, 1.0f, w[j]);
        params<V>(a.bias, a.type_w, at, 0.0f, b[j]);
        params<V>(a.scale, a.type_w, at, 1.0f, sc[j]);
    };
    auto again = [&](int j) { // the parameters' place
        if (HOLD) return j;
        int at = chan[j] >= 0 ? chan[j] : 0;
        asm volatile("" : "+v"(at)); // (read here, and kept no longer than needed)
        read_params(0, at);
        return 0;
    };
#pragma unroll
    for (int j = 0; j < J; j++) {
        const int u = lane + j * a.team;
        const bool end = u == units - 1;
        skip[j] = end ? units * V - a.cg : 0;
        chan[j] = live && u < units ? group * a.cg + (end ? a.cg - V : u * V) : -1;
        const int c = chan[j] >= 0 ? chan[j] : 0;
        if (HOLD) read_params(j, c);
#pragma unroll
        for (int e = 0; e < V; e++) sw[j][e] = sb[j][e] = ss[j][e] = 0.0f;
    }
    typedef typename Vec<S, V>::type SV;
    // what a token's entries are made of, on their way while the one before is worked on
    const bool want_x = !BACK || !BEFORE || gated || scaled;
    SV nx[J], nz[J], nr[J], nh[J], ng[J]; // x, gate, residual (backwards: the stream's gradient), h, gradient
    auto fetch = [&](long long token) {
        const long long from = (token < a.tokens ? token : 0) * a.channels;
#pragma unroll
        for (int j = 0; j < J; j++) {
            const long long at = from + (chan[j] >= 0 ? chan[j] : 0);
            if (want_x) nx[j] = load_unaligned<S, V>(reinterpret_cast<const S *>(a.x) + at);
            if (gated) nz[j] = load_unaligned<S, V>(reinterpret_cast<const S *>(a.gate) + at);
            if (!BACK && a.residual) nr[j] = load_unaligned<S, V>(reinterpret_cast<const S *>(a.residual) + at);
            if (BACK && BEFORE && a.gh) nr[j] = load_unaligned<S, V>(reinterpret_cast<const S *>(a.gh) + at);
            if (BACK && BEFORE) nh[j] = load_unaligned<S, V>(reinterpret_cast<const S *>(a.h) + at);
            if (BACK) ng[j] = load_unaligned<S, V>(reinterpret_cast<const S *>(a.gy) + at);
        }
    };
    if (AHEAD) fetch((long long)blockIdx.x * a.ipw + ti);
    for (long long token0 = (long long)blockIdx.x * a.ipw; token0 < a.tokens; token0 += (long long)gridDim.x * a.ipw) {
        const long long token = token0 + ti;
        const bool here = live && token < a.tokens; // (the same for a whole team; other lanes go along for the sums)
        const long long base = token * a.channels, stat = token * a.groups + group;
        if (!AHEAD) fetch(token);
        float x[J][V], z[J][V], r[J][V], t[J][V], g[J][V];
#pragma unroll
        for (int j = 0; j < J; j++)
#pragma unroll
            for (int e = 0; e < V; e++) {
                const bool there = here && chan[j] >= 0;
                x[j][e] = want_x && there ? (float)nx[j][e] : 0.0f;
                z[j][e] = gated && there ? (float)nz[j][e] : 0.0f;
                r[j][e] = there && ((!BACK && a.residual) || (BACK && BEFORE && a.gh)) ? (float)nr[j][e] : 0.0f;
                t[j][e] = BACK && BEFORE && there ? (float)nh[j][e] : 0.0f;
                g[j][e] = BACK && there ? (float)ng[j][e] : 0.0f;
            }
        if (AHEAD && token0 + (long long)gridDim.x * a.ipw < a.tokens) fetch(token + (long long)gridDim.x * a.ipw);
        if (!BACK) {
            // t: what is normalised.  The stream is normalised as it is stored, so that the way back finds the same
            float sum = 0.0f, none = 0.0f;
#pragma unroll
            for (int j = 0; j < J; j++) {
                if (BEFORE) {
                    const int p = again(j);
#pragma unroll
                    for (int e = 0; e < V; e++) t[j][e] = (float)(S)(r[j][e] + sc[p][e] * x[j][e] * (gated ? activate(z[j][e], a.act) : 1.0f));
                    if (a.h_out && here && chan[j] >= 0) store_floats_unaligned<S, V>(reinterpret_cast<S *>(a.h_out) + base + chan[j], t[j]);
                } else {
#pragma unroll
                    for (int e = 0; e < V; e++) t[j][e] = x[j][e];
                }
#pragma unroll
                for (int e = 0; e < V; e++) sum += chan[j] >= 0 && e >= skip[j] ? t[j][e] : 0.0f; // (a lane without channels has another one's scale, times zero)
            }
            float mean = 0.0f, square = 0.0f;
            if (a.layer) {
                sums(sum, none);
                mean = sum / count;
            }
#pragma unroll
            for (int j = 0; j < J; j++)
                if (chan[j] >= 0)
#pragma unroll
                    for (int e = 0; e < V; e++) {
                        t[j][e] -= mean;
                        square += e >= skip[j] ? t[j][e] * t[j][e] : 0.0f;
                    }
            sums(square, none);
            const float rstd = 1.0f / sqrtf(square / count + a.eps);
            if (here && lane == 0) {
                if (a.mean) a.mean[stat] = mean;
                if (a.rstd) a.rstd[stat] = rstd;
            }
#pragma unroll
            for (int j = 0; j < J; j++)
                if (here && chan[j] >= 0) {
                    const int p = again(j);
#pragma unroll
                    for (int e = 0; e < V; e++) {
                        const float n = t[j][e] * rstd * w[p][e] + b[p][e];
                        t[j][e] = BEFORE ? n : r[j][e] + sc[p][e] * n * (gated ? activate(z[j][e], a.act) : 1.0f);
                    }
                    store_floats_unaligned<S, V>(reinterpret_cast<S *>(a.y) + base + chan[j], t[j]);
                }
        } else {
            const float mean = here && a.layer ? a.mean[stat] : 0.0f, rstd = here ? a.rstd[stat] : 0.0f;
            float m1 = 0.0f, m2 = 0.0f;
#pragma unroll
            for (int j = 0; j < J; j++)
                if (here && chan[j] >= 0) {
                    float slope[V];
                    const int p = again(j);
#pragma unroll
                    for (int e = 0; e < V; e++) {
                        const float xhat = ((BEFORE ? t[j][e] : x[j][e]) - mean) * rstd;
                        float dn = g[j][e]; // the gradient of xhat weight + bias
                        if (!BEFORE) {
                            const float n = xhat * w[p][e] + b[p][e], act = gated ? activate(z[j][e], a.act) : 1.0f;
                            if (gated) slope[e] = dn * sc[p][e] * n * activate_slope(z[j][e], a.act);
                            ss[j][e] += dn * n * act;
                            dn *= sc[p][e] * act;
                        }
                        sw[j][e] += dn * xhat;
                        sb[j][e] += dn;
                        dn *= w[p][e];
                        m1 += e >= skip[j] ? dn : 0.0f;
                        m2 += e >= skip[j] ? dn * xhat : 0.0f;
                        t[j][e] = xhat;
                        g[j][e] = dn;
                    }
                    if (!BEFORE && gated) store_floats_unaligned<S, V>(reinterpret_cast<S *>(a.ggate) + base + chan[j], slope);
                }
            sums(m1, m2);
            m1 = a.layer ? m1 / count : 0.0f;
            m2 /= count;
#pragma unroll
            for (int j = 0; j < J; j++)
                if (here && chan[j] >= 0) {
#pragma unroll
                    for (int e = 0; e < V; e++) g[j][e] = rstd * (g[j][e] - m1 - t[j][e] * m2);
                    if (BEFORE) {
                        const int p = again(j);
#pragma unroll
                        for (int e = 0; e < V; e++) {
                            const float total = g[j][e] + r[j][e], act = gated ? activate(z[j][e], a.act) : 1.0f;
                            r[j][e] = total;
                            ss[j][e] += total * x[j][e] * act;
                            g[j][e] = total * sc[p][e] * act;
                            if (gated) z[j][e] = total * sc[p][e] * x[j][e] * activate_slope(z[j][e], a.act);
                        }
                        store_floats_unaligned<S, V>(reinterpret_cast<S *>(a.gres) + base + chan[j], r[j]);
                        if (gated) store_floats_unaligned<S, V>(reinterpret_cast<S *>(a.ggate) + base + chan[j], z[j]);
                    }
                    if (!BEFORE || gated || scaled) store_floats_unaligned<S, V>(reinterpret_cast<S *>(a.gx) + base + chan[j], g[j]);
                }
        }
    }
    if (BACK && a.partial) {
        float *const to = a.partial + (long long)blockIdx.x * 3 * a.channels;
        if (a.ipw == 1) { // every channel has one lane
#pragma unroll
            for (int j = 0; j < J; j++)
                if (chan[j] >= 0)
#pragma unroll
                    for (int e = 0; e < V; e++)
                        if (e >= skip[j]) {
                            to[chan[j] + e] = sw[j][e];
                            to[a.channels + chan[j] + e] = sb[j][e];
                            to[2 * a.channels + chan[j] + e] = ss[j][e];
                        }
        } else if constexpr (MOST == 512) { // its teams of a group, in order (several teams: 256 lanes)
            __shared__ float part[J * V][256];
#pragma unroll
            for (int which = 0; which < 3; which++) {
                __syncthreads();
#pragma unroll
                for (int e = 0; e < J * V; e++) part[e][threadIdx.x] = which == 0 ? sw[e / V][e % V] : which == 1 ? sb[e / V][e % V] : ss[e / V][e % V];
                __syncthreads();
                if (ti == 0)
#pragma unroll
                    for (int e = 0; e < J * V; e++)
                        if (chan[e / V] >= 0 && e % V >= skip[e / V]) {
                            float sum = 0.0f;
                            for (int k = 0; k < a.ipw; k++) sum += part[e][threadIdx.x + k * a.gpw * a.team];
                            to[which * a.channels + chan[e / V] + e % V] = sum;
                        }
            }
        }
    }
}

// parameters' gradients: partial sums [n][3][channels] added up, eight at a time side by side, in a fixed order
__global__ __launch_bounds__(256) void block_norm_sums_kernel(const float *partial, int n, int channels, void *gw, void *gb, void *gs, int type)
{
    __shared__ float part[8][32];
    const int col = blockIdx.x * 32 + (threadIdx.x & 31), row0 = threadIdx.x >> 5, all = 3 * channels;
    const int which = col / channels, c = col % channels;
    void *const to = which == 0 ? gw : which == 1 ? gb : which == 2 ? gs : nullptr;
    float sum = 0.0f;
    if (to) {
#pragma unroll 8
        for (int row = row0; row < n; row += 8) sum += partial[(long long)row * all + col];
    }
    part[row0][threadIdx.x & 31] = sum;
    __syncthreads();
    if (row0 == 0 && to) {
        for (int k = 1; k < 8; k++) sum += part[k][threadIdx.x];
        if (type == GOOM_REAL_F32) reinterpret_cast<float *>(to)[c] = sum;
        else if (type == GOOM_REAL_BF16) reinterpret_cast<bf16 *>(to)[c] = (bf16)sum;
        else reinterpret_cast<f16 *>(to)[c] = (f16)sum;
    }
}

// ---- host side

constexpr int MOST_CHANNELS = 16384; // of a group: 1024 lanes of 16

struct BlockNormPlan { int v, j, threads, team, gpw, ipw; bool many; long long blocks, parts; size_t bytes; };

static BlockNormPlan plan_norm(const goom_block_norm_shape &sh, bool back)
{
    BlockNormPlan p;
    const int cg = sh.channels / sh.groups, most = sh.type == GOOM_REAL_F32 ? 4 : 8;
    p.v = 1;
    while (p.v < most && 2 * p.v <= cg) p.v *= 2;
    const int units = (cg + p.v - 1) / p.v;
    // one unit a lane while a team is a wave at most; 8 entries a lane up to 1024 lanes, 16 beyond
    p.j = 1;
    if (units > 64) p.j = units * p.v > 8192 ? 16 / p.v : 8 / p.v;
    const int lanes = (units + p.j - 1) / p.j;
    p.team = 1;
    while (p.team < lanes && p.team < 64) p.team *= 2;
    if (lanes > 64) p.team = (lanes + 63) / 64 * 64;
    p.threads = p.team > 64 ? p.team : 256;
    // the kernel of 128 registers also where two workgroups of that one share a CU and one of the other: 16,384 tokens of 4096 channels, bfloat16,
    // before a block, backwards 202 and 163 us
    p.many = p.threads > (back && sh.type != GOOM_REAL_F32 ? 384 : 512);
    const int teams = p.threads / p.team;
    p.gpw = sh.groups < teams ? sh.groups : teams;
    p.ipw = teams / p.gpw;
    p.parts = (sh.groups + p.gpw - 1) / p.gpw;
    // Workgroups: forwards as many as the chip holds several times over.  Backwards each leaves a row of partial sums, and as many as it holds at
    // once, by the waves that the kernel's registers leave room for on a CU: 32,768 tokens of 2048 channels, bfloat16 (8 entries a lane, 12 waves): 768
    // of 256 lanes 181 us with the sums, 512 205, 1024 230, 2048 218; 6000 of 1712, float (4 entries, 16 waves): 1024 58 us, 768 65, 2048 65.
    const int entries = p.v * p.j, waves = p.many ? 16 : entries >= 8 ? 12 : entries == 4 ? 16 : 32, a_cu = waves * 64 / p.threads;
    const long long want = (sh.tokens + p.ipw - 1) / p.ipw, most_blocks = (back ? 256ll * (a_cu > 0 ? a_cu : 1) : 4096 * 256ll / p.threads) / p.parts;
    p.blocks = want < most_blocks ? want : most_blocks;
    if (p.blocks < 1) p.blocks = 1;
    p.bytes = back ? goom::align_up((size_t)p.blocks * 3 * sh.channels * 4, 256) : 0;
    return p;
}

static int check_norm(goom_ctx *ctx, const goom_block_norm_shape *sh)
{
    if (!sh) return goom::fail(ctx, GOOM_EINVAL, "null shape");
    if (!real_type(sh->type) || !real_type(sh->param_type)) return goom::fail(ctx, GOOM_EINVAL, "unknown element type %d or %d", sh->type, sh->param_type);
    if (sh->flags & ~GOOM_NORM_MEAN) return goom::fail(ctx, GOOM_EINVAL, "unknown flags 0x%x", (unsigned)sh->flags);
    if (sh->tokens < 0) return goom::fail(ctx, GOOM_EINVAL, "negative number of tokens");
    if (sh->channels <= 0) return goom::fail(ctx, GOOM_EINVAL, "channels must be positive");
    if (sh->groups <= 0 || sh->channels % sh->groups) return goom::fail(ctx, GOOM_EINVAL, "groups must be positive and divide channels");
    if (sh->activation < GOOM_ACT_NONE || sh->activation > GOOM_ACT_GELU) return goom::fail(ctx, GOOM_EINVAL, "unknown activation %d", sh->activation);
    if (!(sh->eps >= 0) || !std::isfinite((float)sh->eps) || (sh->eps > 0 && (float)sh->eps == 0)) return goom::fail(ctx, GOOM_EINVAL, "eps must be at least 0, and a float");
    if (sh->channels / sh->groups > MOST_CHANNELS) return goom::fail(ctx, GOOM_EUNSUPPORTED, "groups go up to %d channels", MOST_CHANNELS);
    if (sh->channels > (1 << 20) || sh->tokens > (1ll << 40) / sh->channels) return goom::fail(ctx, GOOM_EUNSUPPORTED, "too many tokens or channels");
    return GOOM_OK;
}

template <bool BEFORE, bool BACK> static int launch_norm(goom_ctx *ctx, const goom_block_norm_shape &sh, BlockNormArgs a, const char *label)
{
    const BlockNormPlan p = plan_norm(sh, BACK);
    a.tokens = sh.tokens;
    a.channels = sh.channels;
    a.groups = sh.groups;
    a.cg = sh.channels / sh.groups;
    a.type_w = sh.param_type;
    a.act = sh.activation;
    a.layer = (sh.flags & GOOM_NORM_MEAN) != 0;
    a.eps = (float)sh.eps;
    a.team = p.team;
    a.gpw = p.gpw;
    a.ipw = p.ipw;
    goom::prof_begin(ctx, label);
    const int rc = with_type(sh.type, [&](auto tag) {
        typedef typename decltype(tag)::type S;
        constexpr int W = sizeof(S) == 4 ? 4 : 8; // entries of a wide vector
        auto run = [&](auto v, auto j, auto most) {
            block_norm_kernel<S, decltype(v)::value, decltype(j)::value, decltype(most)::value, BEFORE, BACK><<<dim3((unsigned)p.blocks, (unsigned)p.parts), p.threads, 0, ctx->stream>>>(a);
            return goom::check_hip(ctx, hipGetLastError(), label);
        };
        typedef std::integral_constant<int, 1> One;
        typedef std::integral_constant<int, W> Wide;
        typedef std::integral_constant<int, 512> Few;
        typedef std::integral_constant<int, 1024> Many; // lanes: half the registers
        if (p.v == W) {
            if (p.j == 16 / W) return run(Wide(), std::integral_constant<int, 16 / W>(), Many());
            if (p.many) return run(Wide(), std::integral_constant<int, 8 / W>(), Many());
            if (p.j == 1) return run(Wide(), One(), Few());
            return run(Wide(), std::integral_constant<int, 8 / W>(), Few());
        }
        if constexpr (W == 8)
            if (p.v == 4) return run(std::integral_constant<int, 4>(), One(), Few());
        if (p.v == 2) return run(std::integral_constant<int, 2>(), One(), Few());
        return run(One(), One(), Few());
    });
    goom::prof_end(ctx);
    return rc;
}

static int launch_sums(goom_ctx *ctx, const goom_block_norm_shape &sh, const float *partial, void *gw, void *gb, void *gs)
{
    const BlockNormPlan p = plan_norm(sh, true);
    goom::prof_begin(ctx, "block norm: parameters' gradients");
    block_norm_sums_kernel<<<(3 * sh.channels + 31) / 32, 256, 0, ctx->stream>>>(partial, sh.tokens > 0 ? (int)p.blocks : 0, sh.channels, gw, gb, gs, sh.param_type);
    goom::prof_end(ctx);
    return goom::check_hip(ctx, hipGetLastError(), "block norm: parameters' gradients");
}

static int check_pointers(goom_ctx *ctx, const goom_block_norm_shape &sh, std::initializer_list<const void *> needed, std::initializer_list<const void *> typed,
                          std::initializer_list<const void *> params, std::initializer_list<const void *> floats)
{
    if (sh.tokens > 0)
        for (const void *p : needed)
            if (!p) return goom::fail(ctx, GOOM_EINVAL, "null data pointer");
    for (const void *p : typed)
        if (!goom::aligned(p, real_bytes(sh.type))) return goom::fail(ctx, GOOM_EINVAL, "misaligned data pointer");
    for (const void *p : params)
        if (!goom::aligned(p, real_bytes(sh.param_type))) return goom::fail(ctx, GOOM_EINVAL, "misaligned data pointer");
    for (const void *p : floats)
        if (!goom::aligned(p, 4)) return goom::fail(ctx, GOOM_EINVAL, "misaligned data pointer");
    return GOOM_OK;
}

// the backward passes' ends: the kernel, and the parameters' gradients where any is asked for
template <bool BEFORE> static int run_back(goom_ctx *ctx, const goom_block_norm_shape &sh, BlockNormArgs a, void *gw, void *gb, void *gs, void *workspace, size_t given, const char *label)
{
    const bool params = gw || gb || gs;
    if (int s = check_workspace(ctx, workspace, given, params ? plan_norm(sh, true).bytes : 0)) return s;
    if (int s = enter(ctx)) return s;
    a.partial = params ? reinterpret_cast<float *>(workspace) : nullptr;
    if (sh.tokens > 0) // (the kernel reads the first token's rows wherever it has none of its own)
        if (int s = launch_norm<BEFORE, true>(ctx, sh, a, label)) return s;
    return params ? launch_sums(ctx, sh, a.partial, gw, gb, gs) : GOOM_OK;
}

} // namespace goom_layer

using namespace goom_layer;
using goom::fail;

extern "C" {

int goom_norm_after(goom_ctx *ctx, const goom_block_norm_shape *shape, const void *x, const void *gate, const void *residual, const void *weight, const void *bias,
                    const void *scale, void *y, float *mean, float *rstd)
{
    if (int s = check_norm(ctx, shape)) return s;
    if (int s = check_pointers(ctx, *shape, {x, y}, {x, gate, residual, y}, {weight, bias, scale}, {mean, rstd})) return s;
    if (int s = enter(ctx)) return s;
    if (shape->tokens == 0) return GOOM_OK;
    BlockNormArgs a = {};
    a.x = x; a.gate = gate; a.residual = residual; a.weight = weight; a.bias = bias; a.scale = scale; a.y = y; a.mean = mean; a.rstd = rstd;
    return launch_norm<false, false>(ctx, *shape, a, "norm after a block");
}

int goom_norm_before(goom_ctx *ctx, const goom_block_norm_shape *shape, const void *x, const void *gate, const void *residual, const void *weight, const void *bias,
                     const void *scale, void *h, void *y, float *mean, float *rstd)
{
    if (int s = check_norm(ctx, shape)) return s;
    if (int s = check_pointers(ctx, *shape, {x, y}, {x, gate, residual, h, y}, {weight, bias, scale}, {mean, rstd})) return s;
    if (int s = enter(ctx)) return s;
    if (shape->tokens == 0) return GOOM_OK;
    BlockNormArgs a = {};
    a.x = x; a.gate = gate; a.residual = residual; a.weight = weight; a.bias = bias; a.scale = scale; a.h_out = h; a.y = y; a.mean = mean; a.rstd = rstd;
    return launch_norm<true, false>(ctx, *shape, a, "norm before a block");
}

size_t goom_block_norm_backward_workspace_bytes(const goom_block_norm_shape *shape) { return check_norm(nullptr, shape) ? 0 : plan_norm(*shape, true).bytes; }

int goom_norm_after_backward(goom_ctx *ctx, const goom_block_norm_shape *shape, const void *x, const void *gate, const void *grad_y, const float *mean, const float *rstd,
                             const void *weight, const void *bias, const void *scale, void *grad_x, void *grad_gate, void *grad_weight, void *grad_bias, void *grad_scale,
                             void *workspace, size_t workspace_bytes)
{
    if (int s = check_norm(ctx, shape)) return s;
    if (int s = check_pointers(ctx, *shape, {x, grad_y, rstd, grad_x, gate ? grad_gate : x, shape->flags & GOOM_NORM_MEAN ? mean : rstd}, {x, gate, grad_y, grad_x, grad_gate},
                               {weight, bias, scale, grad_weight, grad_bias, grad_scale}, {mean, rstd}))
        return s;
    BlockNormArgs a = {};
    a.x = x; a.gate = gate; a.gy = grad_y; a.weight = weight; a.bias = bias; a.scale = scale; a.gx = grad_x; a.ggate = grad_gate;
    a.mean = const_cast<float *>(mean);
    a.rstd = const_cast<float *>(rstd);
    return run_back<false>(ctx, *shape, a, grad_weight, grad_bias, grad_scale, workspace, workspace_bytes, "norm after a block: gradients");
}

int goom_norm_before_backward(goom_ctx *ctx, const goom_block_norm_shape *shape, const void *x, const void *gate, const void *h, const void *grad_y, const void *grad_h,
                              const float *mean, const float *rstd, const void *weight, const void *scale, void *grad_residual, void *grad_x, void *grad_gate,
                              void *grad_weight, void *grad_bias, void *grad_scale, void *workspace, size_t workspace_bytes)
{
    if (int s = check_norm(ctx, shape)) return s;
    const bool inner = gate || scale; // x has a gradient of its own
    if (int s = check_pointers(ctx, *shape, {h, grad_y, rstd, grad_residual, inner || grad_scale ? x : h, inner ? grad_x : h, gate ? grad_gate : h, shape->flags & GOOM_NORM_MEAN ? mean : rstd},
                               {x, gate, h, grad_y, grad_h, grad_residual, grad_x, grad_gate}, {weight, scale, grad_weight, grad_bias, grad_scale}, {mean, rstd}))
        return s;
    if (grad_scale && !inner) return fail(ctx, GOOM_EINVAL, "grad_scale without a scale or a gate");
    BlockNormArgs a = {};
    a.x = x; a.gate = gate; a.h = h; a.gy = grad_y; a.gh = grad_h; a.weight = weight; a.scale = scale; a.gres = grad_residual; a.gx = grad_x; a.ggate = grad_gate;
    a.mean = const_cast<float *>(mean);
    a.rstd = const_cast<float *>(rstd);
    return run_back<true>(ctx, *shape, a, grad_weight, grad_bias, grad_scale, workspace, workspace_bytes, "norm before a block: gradients");
}

} // extern "C"
