// Group norm with an activation, channels last, and its gradient.
//
// Bound by the bytes of its tensors.  Two ways:
//   short groups (up to 32 elements a lane of a wave): a team of 2^k lanes holds one group in registers, so that every tensor
//     is read once; statistics are taken about the mean itself.  A team keeps its group number from item to item, so weights are
//     loaded once and their gradients are summed in registers.
//   long groups (over many positions): a workgroup takes a slab of whole groups and a chunk of positions; sums first, then
//     the output in a second launch, whose reads mostly hit the last-level cache.  Sums for the mean and the variance are
//     double and taken about the group's first element: no cancellation, whatever the mean.
// Weight gradients: one partial sum per workgroup and channel, added up in a fixed order by a last launch.
// Measured: 32,768 tokens of 16 groups of 128 (bfloat16, SiLU) 60 us forward (4.5 TB/s), 109 + 7 us backward (3.7 TB/s; as many
// workgroups again, and as many partial sums, took 13 us longer); 8 x 4096 positions of 32 groups of 10 (float, GELU) 11 + 22 us
// forward, 20 + 5 + 22 + 6 us backward.
#include <cmath>

#include "goom_activation.h"

namespace goom_layer {

constexpr int TEAM_ELEMENTS = 32;    // of a group, per lane
constexpr int CHUNK_ROWS = 128;      // positions a thread of the long kernels sums at most, in floats
constexpr int SLAB_GROUPS = 512;     // groups of a slab at most: their statistics are in LDS (a multiple of every `least` below)

struct NormArgs {
    const void *x, *gy;
    const void *weight, *bias;
    void *y;                 // or grad_x
    float *mean, *rstd;      // forward: outputs (may be NULL); backward: inputs
    long long items, length;
    int channels, groups, cg; // cg: channels of a group
    int type_w, act;
    float eps;
    // short
    int team, gpw, ipw;      // lanes of a team; groups and items that a workgroup has at once
    float *partial;          // [workgroups along x][2][channels]: sums of dz xhat, of dz
    // long
    double *stats;           // [items][chunks][groups][2]
    float *sums;             // [items][chunks][2][channels]
    float *means;            // [items][groups][2]
    int gps, rows_at_once, threads;  // groups of a slab, positions at once
    long long chunks, chunk_len;
};

__device__ inline float team_sum(float v, int team)
{
    for (int s = 1; s < team; s *= 2) v += __shfl_xor(v, s);
    return v;
}

// ---- short groups.  A position's channels of a group are cu = ceil(cg / V) units of V; unit u of a group: position u / cu, unit
// u % cu of it; lane l of the team has the units l, l + team, ...  TAIL: V does not divide cg; a position's last unit ends at its last
// channel and shares its first `skip` channels with the unit before, which count there.  grid: (workgroups over items, parts of
// the groups)
template <typename S, int V, int J, bool BACK, bool TAIL> __global__ __launch_bounds__(256) void norm_team_kernel(NormArgs a)
{
    const int lane = threadIdx.x % a.team, team = threadIdx.x / a.team, ti = team / a.gpw, group = blockIdx.y * a.gpw + team % a.gpw;
    const bool live = ti < a.ipw && group < a.groups;
    const int cu = (a.cg + V - 1) / V, units = cu * (int)a.length;
    const float count = (float)a.cg * (float)a.length;
    unsigned off[J]; // of this lane's units: element offsets within the item (2^31 at most), channels
    int chan[J], skip[J];
    float w[J][V], b[J][V], sw[J][V], sb[J][V];
#pragma unroll
    for (int j = 0; j < J; j++) {
        const int u = lane + j * a.team;
        const bool end = TAIL && u % cu == cu - 1;
        skip[j] = end ? cu * V - a.cg : 0;
        chan[j] = live && u < units ? group * a.cg + (end ? a.cg - V : u % cu * V) : -1;
        off[j] = chan[j] >= 0 ? (unsigned)(u / cu) * (unsigned)a.channels + chan[j] : 0u;
        params<V>(a.weight, a.type_w, chan[j] >= 0 ? chan[j] : 0, 1.0f, w[j]);
        params<V>(a.bias, a.type_w, chan[j] >= 0 ? chan[j] : 0, 0.0f, b[j]);
#pragma unroll
        for (int e = 0; e < V; e++) sw[j][e] = sb[j][e] = 0.0f;
    }
    const long long size = a.length * a.channels;
    const S *const xs = reinterpret_cast<const S *>(a.x);
    const S *const gs = reinterpret_cast<const S *>(a.gy);
    S *const ys = reinterpret_cast<S *>(a.y);
    typedef typename Vec<S, V>::type SV;
    SV next_x[J], next_g[J]; // the next item's elements are on their way while one is worked on
    auto fetch = [&](long long item) {
        const long long from = item < a.items ? item : 0;
#pragma unroll
        for (int j = 0; j < J; j++) {
            next_x[j] = load_unaligned<S, V>(xs + from * size + off[j]);
            if (BACK) next_g[j] = load_unaligned<S, V>(gs + from * size + off[j]);
        }
    };
    fetch((long long)blockIdx.x * a.ipw + ti);
    for (long long item0 = (long long)blockIdx.x * a.ipw; item0 < a.items; item0 += (long long)gridDim.x * a.ipw) {
        const long long item = item0 + ti;
        const bool here = live && item < a.items; // (the same for a whole team; other lanes go along for the shuffles)
        float x[J][V], dz[J][V];
#pragma unroll
        for (int j = 0; j < J; j++)
#pragma unroll
            for (int e = 0; e < V; e++) {
                const bool there = here && chan[j] >= 0;
                x[j][e] = there ? (float)next_x[j][e] : 0.0f;
                dz[j][e] = BACK && there ? (float)next_g[j][e] : 0.0f;
            }
        if (item0 + (long long)gridDim.x * a.ipw < a.items) fetch(item + (long long)gridDim.x * a.ipw);
        if (!BACK) {
            float sum = 0.0f;
#pragma unroll
            for (int j = 0; j < J; j++)
#pragma unroll
                for (int e = 0; e < V; e++) sum += !TAIL || e >= skip[j] ? x[j][e] : 0.0f;
            const float mean = team_sum(sum, a.team) / count;
            float square = 0.0f;
#pragma unroll
            for (int j = 0; j < J; j++)
                if (chan[j] >= 0) {
#pragma unroll
                    for (int e = 0; e < V; e++) {
                        x[j][e] -= mean;
                        square += !TAIL || e >= skip[j] ? x[j][e] * x[j][e] : 0.0f;
                    }
                }
            const float rstd = 1.0f / sqrtf(team_sum(square, a.team) / count + a.eps);
            if (here && lane == 0) {
                if (a.mean) a.mean[item * a.groups + group] = mean;
                if (a.rstd) a.rstd[item * a.groups + group] = rstd;
            }
#pragma unroll
            for (int j = 0; j < J; j++)
                if (here && chan[j] >= 0) {
#pragma unroll
                    for (int e = 0; e < V; e++) x[j][e] = activate(x[j][e] * rstd * w[j][e] + b[j][e], a.act);
                    store_floats_unaligned<S, V>(ys + item * size + off[j], x[j]);
                }
        } else {
            const float mean = here ? a.mean[item * a.groups + group] : 0.0f, rstd = here ? a.rstd[item * a.groups + group] : 0.0f;
            float m1 = 0.0f, m2 = 0.0f;
#pragma unroll
            for (int j = 0; j < J; j++)
                if (here && chan[j] >= 0) {
#pragma unroll
                    for (int e = 0; e < V; e++) {
                        x[j][e] = (x[j][e] - mean) * rstd;
                        dz[j][e] *= activate_slope(x[j][e] * w[j][e] + b[j][e], a.act);
                        sw[j][e] += dz[j][e] * x[j][e];
                        sb[j][e] += dz[j][e];
                        dz[j][e] *= w[j][e];
                        m1 += !TAIL || e >= skip[j] ? dz[j][e] : 0.0f;
                        m2 += !TAIL || e >= skip[j] ? dz[j][e] * x[j][e] : 0.0f;
                    }
                }
            m1 = team_sum(m1, a.team) / count;
            m2 = team_sum(m2, a.team) / count;
#pragma unroll
            for (int j = 0; j < J; j++)
                if (here && chan[j] >= 0) {
#pragma unroll
                    for (int e = 0; e < V; e++) x[j][e] = rstd * (dz[j][e] - m1 - x[j][e] * m2);
                    store_floats_unaligned<S, V>(ys + item * size + off[j], x[j]);
                }
        }
    }
    if (BACK) { // the workgroup's channels: sums over its teams of a group and over positions, in order
        __shared__ float meet[256 * J * V];
        const int span = a.gpw * a.cg; // channels of this workgroup
        for (int which = 0; which < 2; which++) {
#pragma unroll
            for (int j = 0; j < J; j++)
#pragma unroll
                for (int e = 0; e < V; e++) meet[(j * V + e) * 256 + threadIdx.x] = which ? sb[j][e] : sw[j][e];
            __syncthreads();
            for (int c = threadIdx.x; c < span; c += 256) {
                const int tg = c / a.cg, cc = c % a.cg;
                if (blockIdx.y * a.gpw + tg >= a.groups) continue;
                float sum = 0.0f;
                for (int t = 0; t < a.ipw; t++)
                    for (int u = cc / V; u < units; u += cu) sum += meet[(u / a.team * V + (TAIL && cc / V == cu - 1 ? cc - (a.cg - V) : cc % V)) * 256 + (t * a.gpw + tg) * a.team + u % a.team];
                a.partial[((long long)blockIdx.x * 2 + which) * a.channels + (blockIdx.y * a.gpw) * a.cg + c] = sum;
            }
            __syncthreads();
        }
    }
}

// ---- long groups.  Thread (tx, ty): units tx, tx + columns, ... of the slab's V-element units (whatever groups their channels
// belong to), positions ty, ty + rows_at_once, ... of the chunk, DEEP of them loaded at once.  A slab of several groups has at
// most as many units as a workgroup has columns.  grid: (items chunks, slabs)
constexpr int DEEP = 4;
struct Slab { int group0, ngroups, chan0, units, columns, tx, ty; long long item, chunk, row0, row1; bool live; };

template <int V> __device__ inline Slab slab_of(const NormArgs &a)
{
    Slab s;
    s.group0 = blockIdx.y * a.gps;
    s.ngroups = a.groups - s.group0 < a.gps ? a.groups - s.group0 : a.gps;
    s.chan0 = s.group0 * a.cg;
    s.units = s.ngroups * a.cg / V;
    s.columns = a.threads / a.rows_at_once;
    s.tx = threadIdx.x % s.columns;
    s.ty = threadIdx.x / s.columns;
    s.live = s.ty < a.rows_at_once;
    s.item = blockIdx.x / a.chunks;
    s.chunk = blockIdx.x % a.chunks;
    s.row0 = s.chunk * a.chunk_len;
    s.row1 = s.row0 + a.chunk_len < a.length ? s.row0 + a.chunk_len : a.length;
    return s;
}

typedef double f64x2 __attribute__((ext_vector_type(2)));

// lanes that add up one group's sums: a power of two, at most a wave
__device__ inline int lanes_of(int ngroups)
{
    int lanes = 64;
    while (lanes > 1 && lanes * ngroups > (int)blockDim.x) lanes /= 2;
    return lanes;
}

// f(row, x, y) for the thread's rows, DEEP loads of x (and of y, unless NULL) ahead
template <typename S, int V, typename F> __device__ inline void rows_of(const NormArgs &a, const Slab &s, const S *x, const S *y, int u, F f)
{
    typedef typename Vec<S, V>::type SV;
    for (long long row0 = s.row0 + s.ty; row0 < s.row1; row0 += (long long)DEEP * a.rows_at_once) {
        SV p[DEEP], q[DEEP];
#pragma unroll
        for (int k = 0; k < DEEP; k++) {
            const long long row = row0 + k * a.rows_at_once, from = (row < s.row1 ? row : row0) * a.channels + u * V;
            p[k] = *reinterpret_cast<const SV *>(x + from);
            if (y) q[k] = *reinterpret_cast<const SV *>(y + from);
        }
#pragma unroll
        for (int k = 0; k < DEEP; k++) {
            const long long row = row0 + k * a.rows_at_once;
            if (row < s.row1) f(row, p[k], q[k]);
        }
    }
}

template <typename S, int V> __global__ __launch_bounds__(512) void norm_stats_kernel(NormArgs a)
{
    __shared__ double meet[V][512];
    const Slab s = slab_of<V>(a);
    const S *const x = reinterpret_cast<const S *>(a.x) + s.item * a.length * a.channels + s.chan0;
    double sum[V] = {}, square[V] = {}; // of the thread's channels; of all its units where the slab is one group
    for (int u = s.tx; s.live && u < s.units; u += s.columns) {
        double pivot[V];
#pragma unroll
        for (int e = 0; e < V; e++) pivot[e] = (double)(float)x[(u * V + e) / a.cg * a.cg]; // first element of the channel's group
        rows_of<S, V>(a, s, x, (const S *)nullptr, u, [&](long long, const auto &v, const auto &) {
#pragma unroll
            for (int e = 0; e < V; e++) {
                const double d = (double)(float)v[e] - pivot[e];
                sum[e] += d;
                square[e] += d * d;
            }
        });
    }
    const int lanes = lanes_of(s.ngroups), per = blockDim.x / lanes, lane = threadIdx.x % lanes;
    for (int which = 0; which < 2; which++) {
        if (which) __syncthreads();
#pragma unroll
        for (int e = 0; e < V; e++) meet[e][threadIdx.x] = which ? square[e] : sum[e];
        __syncthreads();
        for (int g0 = 0; g0 < s.ngroups; g0 += per) {
            const int g = g0 + threadIdx.x / lanes;
            const int width = s.ngroups == 1 ? s.columns * V : a.cg;
            double p = 0.0;
            if (g < s.ngroups)
                for (int k = lane; k < width; k += lanes) {
                    const int c = g * a.cg + k;
                    for (int row = 0; row < a.rows_at_once; row++) p += meet[c % V][row * s.columns + c / V];
                }
            for (int m = 1; m < lanes; m *= 2) p += __shfl_xor(p, m);
            if (g < s.ngroups && lane == 0) a.stats[((s.item * a.chunks + s.chunk) * a.groups + s.group0 + g) * 2 + which] = p;
        }
    }
}

template <typename S, int V> __global__ __launch_bounds__(512) void norm_apply_kernel(NormArgs a)
{
    __shared__ float stat[SLAB_GROUPS][2];
    const Slab s = slab_of<V>(a);
    const long long base = s.item * a.length * a.channels + s.chan0;
    const S *const x = reinterpret_cast<const S *>(a.x) + base;
    S *const y = reinterpret_cast<S *>(a.y) + base;
    const int lanes = lanes_of(s.ngroups), per = blockDim.x / lanes;
    for (int g0 = 0; g0 < s.ngroups; g0 += per) {
        const int g = g0 + threadIdx.x / lanes;
        double p = 0.0, q = 0.0;
        if (g < s.ngroups)
            for (long long k0 = threadIdx.x % lanes; k0 < a.chunks; k0 += 16ll * lanes) { // 16 chunks' sums at once
                f64x2 v[16];
#pragma unroll
                for (int k = 0; k < 16; k++) v[k] = *reinterpret_cast<const f64x2 *>(a.stats + ((s.item * a.chunks + (k0 + k * lanes < a.chunks ? k0 + k * lanes : k0)) * a.groups + s.group0 + g) * 2);
#pragma unroll
                for (int k = 0; k < 16; k++)
                    if (k0 + k * lanes < a.chunks) {
                        p += v[k][0];
                        q += v[k][1];
                    }
            }
        for (int m = 1; m < lanes; m *= 2) {
            p += __shfl_xor(p, m);
            q += __shfl_xor(q, m);
        }
        if (g >= s.ngroups || threadIdx.x % lanes) continue;
        const double n = (double)a.length * a.cg, d = p / n;
        const double var = q / n - d * d;
        stat[g][0] = (float)((double)(float)x[g * a.cg] + d);
        stat[g][1] = (float)(1.0 / sqrt((var < 0.0 ? 0.0 : var) + (double)a.eps));
        if (s.chunk == 0) {
            if (a.mean) a.mean[s.item * a.groups + s.group0 + g] = stat[g][0];
            if (a.rstd) a.rstd[s.item * a.groups + s.group0 + g] = stat[g][1];
        }
    }
    __syncthreads();
    for (int u = s.tx; s.live && u < s.units; u += s.columns) {
        float mean[V], rstd[V], w[V], b[V];
        params<V>(a.weight, a.type_w, s.chan0 + u * V, 1.0f, w);
        params<V>(a.bias, a.type_w, s.chan0 + u * V, 0.0f, b);
#pragma unroll
        for (int e = 0; e < V; e++) {
            mean[e] = stat[(u * V + e) / a.cg][0];
            rstd[e] = stat[(u * V + e) / a.cg][1];
        }
        rows_of<S, V>(a, s, x, (const S *)nullptr, u, [&](long long row, const auto &v, const auto &) {
            float z[V];
#pragma unroll
            for (int e = 0; e < V; e++) z[e] = activate(((float)v[e] - mean[e]) * rstd[e] * w[e] + b[e], a.act);
            store_floats<S, V>(y + row * a.channels + u * V, z);
        });
    }
}

// per channel: sums over the chunk's positions of dz xhat and of dz
template <typename S, int V> __global__ __launch_bounds__(512) void norm_sums_kernel(NormArgs a)
{
    __shared__ float meet[2 * V][512];
    const Slab s = slab_of<V>(a);
    const long long base = s.item * a.length * a.channels + s.chan0;
    const S *const x = reinterpret_cast<const S *>(a.x) + base;
    const S *const gy = reinterpret_cast<const S *>(a.gy) + base;
    for (int u0 = 0; u0 < s.units; u0 += s.columns) {
        const int u = u0 + s.tx;
        float sw[V] = {}, sb[V] = {};
        if (s.live && u < s.units) {
            float mean[V], rstd[V], w[V], b[V];
            params<V>(a.weight, a.type_w, s.chan0 + u * V, 1.0f, w);
            params<V>(a.bias, a.type_w, s.chan0 + u * V, 0.0f, b);
#pragma unroll
            for (int e = 0; e < V; e++) {
                const long long at = s.item * a.groups + s.group0 + (u * V + e) / a.cg;
                mean[e] = a.mean[at];
                rstd[e] = a.rstd[at];
            }
            rows_of<S, V>(a, s, x, gy, u, [&](long long, const auto &v, const auto &g) {
#pragma unroll
                for (int e = 0; e < V; e++) {
                    const float xhat = ((float)v[e] - mean[e]) * rstd[e], dz = (float)g[e] * activate_slope(xhat * w[e] + b[e], a.act);
                    sw[e] += dz * xhat;
                    sb[e] += dz;
                }
            });
        }
        __syncthreads();
#pragma unroll
        for (int e = 0; e < V; e++) {
            meet[e][threadIdx.x] = sw[e];
            meet[V + e][threadIdx.x] = sb[e];
        }
        __syncthreads();
        if (s.ty == 0 && u < s.units) {
            float *const to = a.sums + (s.item * a.chunks + s.chunk) * 2 * a.channels + s.chan0 + u * V;
#pragma unroll
            for (int e = 0; e < 2 * V; e++) {
                float sum = 0.0f;
                for (int r = 0; r < a.rows_at_once; r++) sum += meet[e][r * s.columns + s.tx];
                to[(e / V) * a.channels + e % V] = sum;
            }
        }
    }
}

// means over a group of dz w and of dz w xhat; a workgroup (of 256 or 1024 threads) a group.  grid: items groups, in one order
__global__ __launch_bounds__(1024) void norm_means_kernel(NormArgs a)
{
    __shared__ double meet[2][16];
    const long long at_group = block_of();
    if (at_group >= a.items * a.groups) return;
    const long long item = (unsigned)at_group / (unsigned)a.groups; // (2 10^9 at most)
    const int group = (unsigned)at_group % (unsigned)a.groups, wave = threadIdx.x >> 6, threads = blockDim.x;
    double m1 = 0.0, m2 = 0.0;
    // a thread has one channel (or every threads-th) and every rows-th chunk, eight chunks' sums at once
    const int cols = a.cg < threads ? a.cg : threads, rows = threads / cols, row = threadIdx.x / cols;
    for (int c = threadIdx.x % cols; row < rows && c < a.cg; c += cols) {
        const float *const from = a.sums + item * a.chunks * 2 * a.channels + group * a.cg + c;
        double p = 0.0, q = 0.0;
        for (long long k0 = row; k0 < a.chunks; k0 += 8ll * rows) {
            float x[8], y[8];
#pragma unroll
            for (int k = 0; k < 8; k++) {
                const float *const at = from + (k0 + k * rows < a.chunks ? k0 + k * rows : k0) * 2 * a.channels;
                x[k] = at[0];
                y[k] = at[a.channels];
            }
#pragma unroll
            for (int k = 0; k < 8; k++)
                if (k0 + k * rows < a.chunks) {
                    q += (double)x[k];
                    p += (double)y[k];
                }
        }
        const double w = (double)param(a.weight, a.type_w, group * a.cg + c, 1.0f);
        m1 += w * p;
        m2 += w * q;
    }
    for (int m = 1; m < 64; m *= 2) {
        m1 += __shfl_xor(m1, m);
        m2 += __shfl_xor(m2, m);
    }
    if ((threadIdx.x & 63) == 0) {
        meet[0][wave] = m1;
        meet[1][wave] = m2;
    }
    __syncthreads();
    if (threadIdx.x < 2) {
        double sum = 0.0;
        for (int k = 0; k < threads / 64; k++) sum += meet[threadIdx.x][k];
        a.means[at_group * 2 + threadIdx.x] = (float)(sum / ((double)a.length * a.cg));
    }
}

// gw[c] = sum of partial[k][0][c], gb[c] = sum of partial[k][1][c] over k < n; 32 channels a workgroup, 32 runs of k each
struct WeightArgs { const float *partial; long long n; void *gw, *gb; };
__global__ __launch_bounds__(1024) void norm_weight_kernel(NormArgs a, WeightArgs t)
{
    __shared__ double meet[32][32];
    const unsigned at = blockIdx.x;
    const int c = at / 2 * 32 + (threadIdx.x & 31), part = threadIdx.x >> 5;
    const long long len = (t.n + 31) / 32, begin = part * len, end = begin + len < t.n ? begin + len : t.n;
    double sum = 0.0;
    if (c < a.channels)
        for (long long k0 = begin; k0 < end; k0 += 32) {
            float x[32];
#pragma unroll
            for (int k = 0; k < 32; k++) x[k] = t.partial[((k0 + k < end ? k0 + k : begin) * 2 + at % 2) * a.channels + c];
#pragma unroll
            for (int k = 0; k < 32; k++) sum += k0 + k < end ? (double)x[k] : 0.0;
        }
    meet[part][threadIdx.x & 31] = sum;
    __syncthreads();
    void *out = at % 2 ? t.gb : t.gw;
    if (part == 0 && c < a.channels && out) {
#pragma unroll
        for (int k = 1; k < 32; k++) sum += meet[k][threadIdx.x];
        if (a.type_w == GOOM_REAL_F32) reinterpret_cast<float *>(out)[c] = (float)sum;
        else if (a.type_w == GOOM_REAL_BF16) reinterpret_cast<bf16 *>(out)[c] = (bf16)(float)sum;
        else reinterpret_cast<f16 *>(out)[c] = (f16)(float)sum;
    }
}

template <typename S, int V> __global__ __launch_bounds__(512) void norm_grad_kernel(NormArgs a)
{
    const Slab s = slab_of<V>(a);
    const long long base = s.item * a.length * a.channels + s.chan0;
    const S *const x = reinterpret_cast<const S *>(a.x) + base;
    const S *const gy = reinterpret_cast<const S *>(a.gy) + base;
    S *const gx = reinterpret_cast<S *>(a.y) + base;
    for (int u = s.tx; s.live && u < s.units; u += s.columns) {
        float mean[V], rstd[V], m1[V], m2[V], w[V], b[V];
        params<V>(a.weight, a.type_w, s.chan0 + u * V, 1.0f, w);
        params<V>(a.bias, a.type_w, s.chan0 + u * V, 0.0f, b);
#pragma unroll
        for (int e = 0; e < V; e++) {
            const long long at = s.item * a.groups + s.group0 + (u * V + e) / a.cg;
            mean[e] = a.mean[at];
            rstd[e] = a.rstd[at];
            m1[e] = a.means[at * 2];
            m2[e] = a.means[at * 2 + 1];
        }
        rows_of<S, V>(a, s, x, gy, u, [&](long long row, const auto &v, const auto &g) {
            float z[V];
#pragma unroll
            for (int e = 0; e < V; e++) {
                const float xhat = ((float)v[e] - mean[e]) * rstd[e], dz = (float)g[e] * activate_slope(xhat * w[e] + b[e], a.act);
                z[e] = rstd[e] * (dz * w[e] - m1[e] - xhat * m2[e]);
            }
            store_floats<S, V>(gx + row * a.channels + u * V, z);
        });
    }
}

// ---- host side

struct NormPlan {
    bool team;
    int v, j;
    long long blocks, parts;             // grid: along items (and chunks), along groups
    NormArgs a;                          // the plan's own fields
    size_t stats, sums, means, partial;  // bytes in the workspace
};

// cap: elements of an access that addresses and types allow.  Short if a group's units fit a wave with TEAM_ELEMENTS elements a lane.
static NormPlan norm_plan(const goom_norm_shape &sh, int cap, bool back)
{
    NormPlan p = {};
    NormArgs &a = p.a;
    a.items = sh.items;
    a.length = sh.length;
    a.channels = sh.channels;
    a.groups = sh.groups;
    a.cg = sh.channels / sh.groups;
    a.type_w = sh.param_type;
    a.act = sh.activation;
    a.eps = (float)sh.eps;
    int v = (int)(16 / real_bytes(sh.type)); // (whatever the addresses' alignment)
    while (v > a.cg) v /= 2;
    p.v = v;
    const long long units = (long long)sh.length * ((a.cg + v - 1) / v);
    const int most = TEAM_ELEMENTS / v < 8 ? TEAM_ELEMENTS / v : 8;
    p.team = units <= 64ll * most;
    if (p.team) {
        // as many lanes as hold the group with up to four units each: wide enough to have loads in flight
        p.j = 1;
        while (p.j < most && (p.j < 2 ? units > 16 : units > 64ll * p.j)) p.j *= 2;
        a.team = 1;
        while ((long long)a.team * p.j < units) a.team *= 2;
        const int teams = 256 / a.team;
        a.gpw = sh.groups < teams ? sh.groups : teams;
        a.ipw = teams / a.gpw;
        p.parts = (sh.groups + a.gpw - 1) / a.gpw;
        p.blocks = (sh.items + a.ipw - 1) / a.ipw;
        // Workgroups go over several items: where the weights' gradients are summed, no more partial sums than needed to fill
        // the chip
        const long long groups_at_once = back ? 1024 : 4096, cap = groups_at_once / p.parts > 0 ? groups_at_once / p.parts : 1;
        if (p.blocks > cap) p.blocks = cap;
        p.partial = back ? goom::align_up((size_t)p.blocks * 2 * sh.channels * 4, 256) : 0;
        return p;
    }
    // a slab: whole groups whose channels make whole units, 256 of these and SLAB_GROUPS groups at most (or one group)
    int least = 1;
    for (v = cap; v > 1; v /= 2) {
        for (least = 1; least * a.cg % v; least *= 2) {}
        if (sh.channels % v == 0 && (least == 1 || least * a.cg / v <= 256)) break;
        least = 1;
    }
    p.v = v;
    a.gps = (int)(256ll * v / ((long long)a.cg * least) * least);
    if (a.gps < least) a.gps = least;
    if (a.gps > SLAB_GROUPS) a.gps = SLAB_GROUPS; // (groups of one to three channels)
    if (a.gps > sh.groups) a.gps = sh.groups;
    const int columns = a.gps * a.cg / v < 256 ? a.gps * a.cg / v : 256;
    a.rows_at_once = 512 / columns > 0 ? 512 / columns : 1;
    if (columns * a.rows_at_once > 320 && a.rows_at_once > 1) { // 256 to 320 threads where that wastes fewer lanes
        const int half = a.rows_at_once / 2;
        if (columns * half >= 192) a.rows_at_once = half;
    }
    a.threads = columns * a.rows_at_once;
    p.parts = (sh.groups + a.gps - 1) / a.gps;
    // chunks: at most CHUNK_ROWS positions a thread, and enough workgroups to fill the chip
    long long chunks = (sh.length + (long long)CHUNK_ROWS * a.rows_at_once - 1) / ((long long)CHUNK_ROWS * a.rows_at_once);
    const long long want = 1024 / (sh.items * p.parts) + 1, most_chunks = (sh.length + 8ll * a.rows_at_once - 1) / (8ll * a.rows_at_once);
    if (chunks < want) chunks = want < most_chunks ? want : most_chunks > chunks ? most_chunks : chunks;
    a.chunk_len = (sh.length + chunks - 1) / chunks;
    a.chunks = (sh.length + a.chunk_len - 1) / a.chunk_len;
    p.blocks = sh.items * a.chunks;
    p.stats = back ? 0 : goom::align_up((size_t)(sh.items * a.chunks * sh.groups) * 16, 256);
    p.sums = back ? goom::align_up((size_t)(sh.items * a.chunks) * 2 * sh.channels * 4, 256) : 0;
    p.means = back ? goom::align_up((size_t)(sh.items * sh.groups) * 8, 256) : 0;
    return p;
}

// bytes that hold for every access width (the workspace is asked for before the addresses are known)
static size_t norm_bytes(const goom_norm_shape &sh, bool back)
{
    size_t most = 0;
    for (int cap = 1; cap * real_bytes(sh.type) <= 16; cap *= 2) {
        const NormPlan p = norm_plan(sh, cap, back);
        const size_t need = p.stats + p.sums + p.means + p.partial;
        if (need > most) most = need;
    }
    return most;
}

static int norm_cap(const goom_norm_shape &sh, const void *a, const void *b, const void *c)
{
    const size_t size = real_bytes(sh.type);
    int v = (int)(16 / size);
    while (v > 1 && (sh.channels % v || !goom::aligned(a, v * size) || !goom::aligned(b, v * size) || !goom::aligned(c, v * size))) v /= 2;
    return v;
}

static int check_norm(goom_ctx *ctx, const goom_norm_shape *sh)
{
    if (!sh) return goom::fail(ctx, GOOM_EINVAL, "null shape");
    if (!real_type(sh->type) || !real_type(sh->param_type)) return goom::fail(ctx, GOOM_EINVAL, "unknown element type %d", real_type(sh->type) ? sh->param_type : sh->type);
    if (sh->flags) return goom::fail(ctx, GOOM_EINVAL, "unknown flags 0x%x", (unsigned)sh->flags);
    if (sh->items < 0 || sh->length <= 0 || sh->channels <= 0) return goom::fail(ctx, GOOM_EINVAL, "items must not be negative, length and channels positive");
    if (sh->groups <= 0 || sh->channels % sh->groups) return goom::fail(ctx, GOOM_EINVAL, "groups must be positive and divide channels");
    if (sh->activation < GOOM_ACT_NONE || sh->activation > GOOM_ACT_GELU) return goom::fail(ctx, GOOM_EINVAL, "unknown activation %d", sh->activation);
    if (!(sh->eps >= 0.0) || !std::isfinite((float)sh->eps) || (sh->eps > 0.0 && (float)sh->eps == 0.0f)) return goom::fail(ctx, GOOM_EINVAL, "eps must be finite and not negative, and a float");
    if (sh->items > (1ll << 31) || sh->length > (1ll << 31) || sh->channels > (1 << 20) || (double)sh->items * sh->length * sh->channels > 1e15 || (double)sh->items * sh->groups > 2e9)
        return goom::fail(ctx, GOOM_EUNSUPPORTED, "too many items, positions or channels");
    return GOOM_OK;
}

static int threads_of(const NormPlan &p) { return p.team ? 256 : (p.a.threads + 63) / 64 * 64; }

// (a grid has fewer than 2^32 threads along its first axis)
static int check_grid(goom_ctx *ctx, const NormPlan &p)
{
    if (p.blocks > 0xffffffffll / threads_of(p) || p.parts > 65535) return goom::fail(ctx, GOOM_EUNSUPPORTED, "too many items or groups");
    return GOOM_OK;
}

// f(vector width, units a lane, whether cg leaves a rest)
template <typename S, typename F> static int with_team(int v, int j, int cg, F f)
{
    auto units = [&](auto vec) {
        constexpr int V = decltype(vec)::value;
        if constexpr (V * sizeof(S) <= 16) {
            auto lanes = [&](auto tail) {
                if constexpr (V <= 4)
                    if (j == 8) return f(vec, std::integral_constant<int, 8>(), tail);
                if (j == 4) return f(vec, std::integral_constant<int, 4>(), tail);
                if (j == 2) return f(vec, std::integral_constant<int, 2>(), tail);
                return f(vec, std::integral_constant<int, 1>(), tail);
            };
            if constexpr (V > 1)
                if (cg % V) return lanes(std::true_type());
            return lanes(std::false_type());
        }
        return 0;
    };
    return v == 8 ? units(std::integral_constant<int, 8>()) : v == 4 ? units(std::integral_constant<int, 4>()) : v == 2 ? units(std::integral_constant<int, 2>()) : units(std::integral_constant<int, 1>());
}

template <typename S, typename F> static int with_width(int v, F f)
{
    if constexpr (sizeof(S) == 2)
        if (v == 8) return f(std::integral_constant<int, 8>());
    return v == 4 ? f(std::integral_constant<int, 4>()) : v == 2 ? f(std::integral_constant<int, 2>()) : f(std::integral_constant<int, 1>());
}

} // namespace goom_layer

using namespace goom_layer;
using goom::aligned;
using goom::fail;

extern "C" {

size_t goom_group_norm_workspace_bytes(const goom_norm_shape *shape) { return check_norm(nullptr, shape) || shape->items == 0 ? 0 : norm_bytes(*shape, false); }

size_t goom_group_norm_backward_workspace_bytes(const goom_norm_shape *shape) { return check_norm(nullptr, shape) || shape->items == 0 ? 0 : norm_bytes(*shape, true); }

int goom_group_norm(goom_ctx *ctx, const goom_norm_shape *shape, const void *x, const void *weight, const void *bias, void *y, float *mean, float *rstd, void *workspace,
                    size_t workspace_bytes)
{
    if (int s = check_norm(ctx, shape)) return s;
    if (shape->items == 0) return ctx ? GOOM_OK : fail(nullptr, GOOM_EINVAL, "null context");
    if (!x || !y) return fail(ctx, GOOM_EINVAL, "null data pointer");
    const size_t size = real_bytes(shape->type), wsize = real_bytes(shape->param_type);
    if (!aligned(x, size) || !aligned(y, size) || !aligned(weight, wsize) || !aligned(bias, wsize) || !aligned(mean, 4) || !aligned(rstd, 4))
        return fail(ctx, GOOM_EINVAL, "misaligned data pointer");
    NormPlan p = norm_plan(*shape, norm_cap(*shape, x, y, nullptr), false);
    if (int s = check_grid(ctx, p)) return s;
    if (int s = check_workspace(ctx, workspace, workspace_bytes, norm_bytes(*shape, false))) return s;
    if (int s = enter(ctx)) return s;
    NormArgs &a = p.a;
    a.x = x;
    a.weight = weight;
    a.bias = bias;
    a.y = y;
    a.mean = mean;
    a.rstd = rstd;
    a.stats = reinterpret_cast<double *>(workspace);
    return with_type(shape->type, [&](auto tag) {
        typedef typename decltype(tag)::type S;
        const dim3 grid((unsigned)p.blocks, (unsigned)p.parts);
        if (p.team) {
            goom::prof_begin(ctx, "group norm");
            with_team<S>(p.v, p.j, a.cg, [&](auto vec, auto units, auto tail) {
                norm_team_kernel<S, decltype(vec)::value, decltype(units)::value, false, decltype(tail)::value><<<grid, 256, 0, ctx->stream>>>(a);
                return 0;
            });
            goom::prof_end(ctx);
        } else {
            const int threads = threads_of(p);
            goom::prof_begin(ctx, "group norm: sums");
            with_width<S>(p.v, [&](auto vec) {
                norm_stats_kernel<S, decltype(vec)::value><<<grid, threads, 0, ctx->stream>>>(a);
                return 0;
            });
            goom::prof_end(ctx);
            goom::prof_begin(ctx, "group norm: output");
            with_width<S>(p.v, [&](auto vec) {
                norm_apply_kernel<S, decltype(vec)::value><<<grid, threads, 0, ctx->stream>>>(a);
                return 0;
            });
            goom::prof_end(ctx);
        }
        return goom::check_hip(ctx, hipGetLastError(), "group norm");
    });
}

int goom_group_norm_backward(goom_ctx *ctx, const goom_norm_shape *shape, const void *x, const void *grad_y, const float *mean, const float *rstd, const void *weight, const void *bias,
                             void *grad_x, void *grad_weight, void *grad_bias, void *workspace, size_t workspace_bytes)
{
    if (int s = check_norm(ctx, shape)) return s;
    const size_t size = real_bytes(shape->type), wsize = real_bytes(shape->param_type);
    if (shape->items > 0 && (!x || !grad_y || !mean || !rstd || !grad_x)) return fail(ctx, GOOM_EINVAL, "null data pointer");
    const void *const typed[] = {x, grad_y, grad_x}, *const params[] = {weight, bias, grad_weight, grad_bias};
    for (const void *q : typed)
        if (!aligned(q, size)) return fail(ctx, GOOM_EINVAL, "misaligned data pointer");
    for (const void *q : params)
        if (!aligned(q, wsize)) return fail(ctx, GOOM_EINVAL, "misaligned data pointer");
    if (!aligned(mean, 4) || !aligned(rstd, 4)) return fail(ctx, GOOM_EINVAL, "misaligned data pointer");
    NormPlan p = {};
    if (shape->items > 0) {
        p = norm_plan(*shape, norm_cap(*shape, x, grad_y, grad_x), true);
        if (int s = check_grid(ctx, p)) return s;
    } else { // sums over nothing
        p.team = true;
        p.a.channels = shape->channels;
        p.a.type_w = shape->param_type;
    }
    if (int s = check_workspace(ctx, workspace, workspace_bytes, shape->items ? norm_bytes(*shape, true) : 0)) return s;
    if (int s = enter(ctx)) return s;
    NormArgs &a = p.a;
    a.x = x;
    a.gy = grad_y;
    a.weight = weight;
    a.bias = bias;
    a.y = grad_x;
    a.mean = const_cast<float *>(mean);
    a.rstd = const_cast<float *>(rstd);
    a.partial = a.sums = reinterpret_cast<float *>(workspace);
    a.means = reinterpret_cast<float *>(reinterpret_cast<unsigned char *>(workspace) + p.sums);
    // p.blocks: workgroups along the items, or items chunks: [blocks][2][channels] partial sums either way
    const WeightArgs weights = {a.sums, p.blocks, grad_weight, grad_bias};
    const unsigned wants_weights = grad_weight || grad_bias ? (unsigned)((shape->channels + 31) / 32 * 2) : 0;
    return with_type(shape->type, [&](auto tag) {
        typedef typename decltype(tag)::type S;
        const dim3 grid((unsigned)p.blocks, (unsigned)p.parts);
        if (p.team) {
            if (shape->items > 0) {
                goom::prof_begin(ctx, "group norm gradient");
                with_team<S>(p.v, p.j, a.cg, [&](auto vec, auto units, auto tail) {
                    norm_team_kernel<S, decltype(vec)::value, decltype(units)::value, true, decltype(tail)::value><<<grid, 256, 0, ctx->stream>>>(a);
                    return 0;
                });
                goom::prof_end(ctx);
            }
            if (wants_weights) {
                goom::prof_begin(ctx, "group norm gradient: weights");
                norm_weight_kernel<<<wants_weights, 1024, 0, ctx->stream>>>(a, weights);
                goom::prof_end(ctx);
            }
        } else {
            const int threads = threads_of(p);
            const int means_threads = a.chunks * a.cg <= 4096 ? 256 : 1024;
            goom::prof_begin(ctx, "group norm gradient: sums");
            with_width<S>(p.v, [&](auto vec) {
                norm_sums_kernel<S, decltype(vec)::value><<<grid, threads, 0, ctx->stream>>>(a);
                return 0;
            });
            norm_means_kernel<<<grid_of(a.items * a.groups, means_threads), means_threads, 0, ctx->stream>>>(a);
            goom::prof_end(ctx);
            goom::prof_begin(ctx, "group norm gradient");
            with_width<S>(p.v, [&](auto vec) {
                norm_grad_kernel<S, decltype(vec)::value><<<grid, threads, 0, ctx->stream>>>(a);
                return 0;
            });
            goom::prof_end(ctx);
            if (wants_weights) {
                goom::prof_begin(ctx, "group norm gradient: weights");
                norm_weight_kernel<<<wants_weights, 1024, 0, ctx->stream>>>(a, weights);
                goom::prof_end(ctx);
            }
        }
        return goom::check_hip(ctx, hipGetLastError(), "group norm gradient");
    });
}

} // extern "C"
