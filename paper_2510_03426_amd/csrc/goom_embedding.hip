// Token embeddings and their gradient.
//
// Forward: one pass, bound by the rows read and written.
// Gradient: a sum over the positions of each token, in a fixed order.  The positions are sorted by token (a stable radix
// sort, up to 9 bits a pass), so that a token's gradients are a run of sorted positions; the waves of a table row, each with its
// columns, add the run up and write the row, zeros where the run is empty, so that the table is written once and never read.  Tokens of text are far
// from equally frequent: blocks of 32 sorted positions that lie inside one run are summed beforehand, side by side, and the
// row's waves take their sums.
#include <cmath>

#include "goom_real.h"

namespace goom_layer {

constexpr int RUN = 32;       // sorted positions of a block that is summed beforehand
constexpr int MAX_BINS = 512; // digits of a sorting pass

template <typename S, int V> __global__ __launch_bounds__(256) void embedding_kernel(const S *table, const int64_t *tokens, S *rows, long long n, long long vocab, int width, float scale)
{
    const int units = width / V;
    for (long long u = blockIdx.x * 256ll + threadIdx.x; u < n * units; u += gridDim.x * 256ll) {
        const long long row = u / units;
        const int col = (int)(u - row * units) * V;
        const long long t = tokens[row];
        float x[V];
        if (t >= 0 && t < vocab) {
            load_floats<S, V>(table + t * width + col, x);
#pragma unroll
            for (int e = 0; e < V; e++) x[e] *= scale;
        } else {
#pragma unroll
            for (int e = 0; e < V; e++) x[e] = 0.0f;
        }
        store_floats<S, V>(rows + row * width + col, x);
    }
}

// ---- sorting: keys are tokens, `vocab` for those outside; values are positions
struct SortPass {
    const int64_t *tokens; // first pass: keys come from here, positions are the indices
    const unsigned *keys, *values;
    unsigned *out_keys, *out_values, *counts; // counts: [tiles][bins]
    unsigned n, vocab, tile;
    int shift, bits;
};

__device__ inline unsigned sort_key(const SortPass &p, unsigned i)
{
    if (!p.tokens) return p.keys[i];
    const long long t = p.tokens[i];
    return t >= 0 && t < p.vocab ? (unsigned)t : p.vocab;
}

__global__ __launch_bounds__(256) void sort_count_kernel(SortPass p)
{
    __shared__ unsigned count[MAX_BINS];
    const int bins = 1 << p.bits;
    for (int d = threadIdx.x; d < bins; d += 256) count[d] = 0;
    __syncthreads();
    const unsigned begin = blockIdx.x * p.tile, end = p.n - begin < p.tile ? p.n : begin + p.tile;
    for (unsigned i = begin + threadIdx.x; i < end; i += 256) atomicAdd(&count[sort_key(p, i) >> p.shift & (bins - 1)], 1u);
    __syncthreads();
    for (int d = threadIdx.x; d < bins; d += 256) p.counts[blockIdx.x * (unsigned)bins + d] = count[d];
}

// Each wave has a quarter of the tile and goes through it 64 entries at a time; entries of equal digit keep their order.
__global__ __launch_bounds__(256) void sort_scatter_kernel(SortPass p)
{
    __shared__ unsigned at[4][MAX_BINS]; // counts of the waves' quarters, then where each wave's next entry of a digit goes
    __shared__ unsigned sums[256];
    const int bins = 1 << p.bits, lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    for (int d = threadIdx.x; d < 4 * MAX_BINS; d += 256) at[d / MAX_BINS][d % MAX_BINS] = 0;
    __syncthreads();
    const unsigned begin = blockIdx.x * p.tile + wave * (p.tile / 4), limit = (p.n < (blockIdx.x + 1u) * p.tile ? p.n : (blockIdx.x + 1u) * p.tile);
    const unsigned end = begin + p.tile / 4 < limit ? begin + p.tile / 4 : limit;
    for (unsigned i = begin + lane; i < end; i += 64) atomicAdd(&at[wave][sort_key(p, i) >> p.shift & (bins - 1)], 1u);
    // entries of each digit in all tiles, and in the tiles before this one; a thread has two neighbouring digits
    unsigned total[2] = {0, 0}, before[2] = {0, 0};
#pragma unroll
    for (int k = 0; k < 2; k++) {
        const int d = threadIdx.x * 2 + k;
        if (d < bins)
            for (unsigned t0 = 0; t0 < gridDim.x; t0 += 16) {
                unsigned c[16];
#pragma unroll
                for (int t = 0; t < 16; t++) c[t] = t0 + t < gridDim.x ? p.counts[(t0 + t) * (unsigned)bins + d] : 0;
#pragma unroll
                for (int t = 0; t < 16; t++) {
                    total[k] += c[t];
                    before[k] += t0 + t < blockIdx.x ? c[t] : 0;
                }
            }
    }
    sums[threadIdx.x] = total[0] + total[1];
    __syncthreads();
    for (int s = 1; s < 256; s *= 2) { // running sums over the digits
        const unsigned x = (int)threadIdx.x >= s ? sums[threadIdx.x - s] : 0;
        __syncthreads();
        sums[threadIdx.x] += x;
        __syncthreads();
    }
    unsigned base = sums[threadIdx.x] - total[0] - total[1];
#pragma unroll
    for (int k = 0; k < 2; k++) {
        const int d = threadIdx.x * 2 + k;
        unsigned next = base + before[k];
        if (d < bins)
            for (int v = 0; v < 4; v++) {
                const unsigned c = at[v][d];
                at[v][d] = next;
                next += c;
            }
        base += total[k];
    }
    __syncthreads();
    for (unsigned i0 = begin; i0 < end; i0 += 64) {
        const unsigned i = i0 + lane;
        const bool live = i < end;
        const unsigned key = live ? sort_key(p, i) : 0, digit = key >> p.shift & (bins - 1);
        unsigned long long same = __ballot(live);
        for (int b = 0; b < p.bits; b++) {
            const unsigned long long m = __ballot(digit >> b & 1);
            same &= digit >> b & 1 ? m : ~m;
        }
        const unsigned rank = __popcll(same & ((1ull << lane) - 1));
        unsigned to = 0;
        if (live) to = at[wave][digit] + rank;
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront"); // all lanes have read before a digit's first lane moves it on
        if (live) {
            if (rank == 0) at[wave][digit] += __popcll(same);
            p.out_keys[to] = key;
            p.out_values[to] = p.tokens ? i : p.values[i];
        }
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    }
}

// start[t] = first sorted position whose token is at least t, t = 0 .. vocab.  A thread writes the tokens from its left
// neighbour's on up to its own; gaps of more than 64 (few positions, many tokens) are written by the whole workgroup.
__global__ __launch_bounds__(256) void run_start_kernel(const unsigned *keys, unsigned *start, unsigned n, unsigned vocab)
{
    __shared__ unsigned gaps[256][2];
    __shared__ int count;
    if (threadIdx.x == 0) count = 0;
    __syncthreads();
    const unsigned i = blockIdx.x * 256 + threadIdx.x;
    if (i <= n) {
        const unsigned from = i == 0 ? 0 : keys[i - 1] + 1, to = i == n ? vocab : keys[i];
        if (from <= to && to - from > 64) {
            const int at = atomicAdd(&count, 1);
            gaps[at][0] = i;
            gaps[at][1] = from;
        } else {
            for (unsigned t = from; t <= to; t++) start[t] = i;
        }
    }
    __syncthreads();
    for (int k = 0; k < count; k++) {
        const unsigned at = gaps[k][0], to = at == n ? vocab : keys[at];
        for (unsigned t = gaps[k][1] + threadIdx.x; t <= to; t += 256) start[t] = at;
    }
}

// x += rows of grad at sorted positions [i, end), in order
template <typename S, int V> __device__ inline void add_rows(float (&x)[V], const S *grad, const unsigned *values, unsigned i, unsigned end, int width, int col)
{
    for (; i + 8 <= end; i += 8) { // eight rows in flight
        float y[8][V];
#pragma unroll
        for (int k = 0; k < 8; k++) load_floats<S, V>(grad + (long long)values[i + k] * width + col, y[k]);
#pragma unroll
        for (int k = 0; k < 8; k++)
#pragma unroll
            for (int e = 0; e < V; e++) x[e] += y[k][e];
    }
    for (; i < end; i++) {
        float y[V];
        load_floats<S, V>(grad + (long long)values[i] * width + col, y);
#pragma unroll
        for (int e = 0; e < V; e++) x[e] += y[e];
    }
}

// sums of the blocks of RUN sorted positions that belong to one token; grid: (blocks, parts of 64 V columns)
template <typename S, int V> __global__ __launch_bounds__(64) void run_block_kernel(const S *grad, const unsigned *keys, const unsigned *values, float *sums, unsigned vocab, int width)
{
    const unsigned i = blockIdx.x * RUN;
    const unsigned key = keys[i];
    if (key != keys[i + RUN - 1] || key >= vocab) return;
    const int col = (blockIdx.y * 64 + threadIdx.x) * V;
    if (col >= width) return;
    float x[V] = {};
    add_rows<S, V>(x, grad, values, i, i + RUN, width, col);
    store_floats<float, V>(sums + (long long)blockIdx.x * width + col, x);
}

// 64 V columns of a table row a wave: the run's head, its whole blocks, its tail.  grid: vocab parts / 4
template <typename S, typename W, int V> __global__ __launch_bounds__(256) void table_row_kernel(const S *grad, const unsigned *values, const unsigned *start, const float *sums, W *table, long long vocab, int width, int parts, float scale)
{
    const long long task = blockIdx.x * 4ll + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), row = task / parts;
    const int col = ((int)(task - row * parts) * 64 + (threadIdx.x & 63)) * V;
    if (row >= vocab) return;
    const unsigned begin = start[row], end = start[row + 1];
    const unsigned first = (begin + RUN - 1) / RUN, last = end / RUN; // whole blocks: first .. last - 1
    if (col >= width) return;
    float x[V] = {};
    if (first < last) {
        add_rows<S, V>(x, grad, values, begin, first * RUN, width, col);
        unsigned b = first;
        for (; b + 8 <= last; b += 8) {
            float y[8][V];
#pragma unroll
            for (int k = 0; k < 8; k++) load_floats<float, V>(sums + (long long)(b + k) * width + col, y[k]);
#pragma unroll
            for (int k = 0; k < 8; k++)
#pragma unroll
                for (int e = 0; e < V; e++) x[e] += y[k][e];
        }
        for (; b < last; b++) {
            float y[V];
            load_floats<float, V>(sums + (long long)b * width + col, y);
#pragma unroll
            for (int e = 0; e < V; e++) x[e] += y[e];
        }
        add_rows<S, V>(x, grad, values, last * RUN, end, width, col);
    } else {
        add_rows<S, V>(x, grad, values, begin, end, width, col);
    }
#pragma unroll
    for (int e = 0; e < V; e++) x[e] *= scale;
    store_floats<W, V>(table + row * width + col, x);
}

struct EmbeddingPlan {
    int passes, bits;
    unsigned tile, tiles;
    size_t counts, list, start, sums, bytes; // bytes of each part: counts, one list of n (four of them), run starts, block sums
};

static EmbeddingPlan embedding_plan(long long n, long long vocab, int width)
{
    EmbeddingPlan p;
    int total = 1;
    while ((1ll << total) <= vocab) total++; // keys 0 .. vocab
    p.passes = (total + 8) / 9;
    p.bits = (total + p.passes - 1) / p.passes;
    // Tiles of 1024 up to 65,536 positions: every tile adds up the counts of all tiles, which must stay few
    p.tile = n <= 65536 ? 1024 : n <= (1 << 20) ? 8192 : 65536;
    p.tiles = (unsigned)((n + p.tile - 1) / p.tile);
    auto up = [](size_t b) { return goom::align_up(b, 256); };
    p.counts = up((size_t)p.tiles * (1u << p.bits) * 4);
    p.list = up((size_t)n * 4);
    p.start = up((size_t)(vocab + 1) * 4);
    p.sums = up((size_t)(n / RUN) * width * 4);
    p.bytes = p.counts + 4 * p.list + p.start + p.sums;
    return p;
}

static int check_embedding(goom_ctx *ctx, long long n, long long vocab, int width)
{
    if (n < 0 || vocab <= 0 || width <= 0) return goom::fail(ctx, GOOM_EINVAL, "n must not be negative, vocab and width positive");
    if (n >= (1ll << 31) || vocab >= (1ll << 31) || (double)vocab * width > 1e12) return goom::fail(ctx, GOOM_EUNSUPPORTED, "up to 2^31 - 1 tokens and table rows, and 10^12 entries");
    return GOOM_OK;
}

// elements of a vector access that widths and addresses allow, up to 16 bytes of the larger type
static int vector_of(int width, std::initializer_list<std::pair<const void *, size_t>> arrays)
{
    int v = 8;
    for (auto &a : arrays)
        while (v > 1 && (width % v || v * a.second > 16 || !goom::aligned(a.first, v * a.second))) v /= 2;
    return v;
}

template <typename F> static int with_vector(int v, F f)
{
    switch (v) {
    case 8: return f(std::integral_constant<int, 8>());
    case 4: return f(std::integral_constant<int, 4>());
    case 2: return f(std::integral_constant<int, 2>());
    default: return f(std::integral_constant<int, 1>());
    }
}

} // namespace goom_layer

using namespace goom_layer;
using goom::aligned;
using goom::fail;

extern "C" {

int goom_embedding(goom_ctx *ctx, const void *table, const int64_t *tokens, void *rows, int64_t n, int64_t vocab, int width, int type, double scale)
{
    if (!real_type(type)) return fail(ctx, GOOM_EINVAL, "unknown element type %d", type);
    if (int s = check_embedding(ctx, n, vocab, width)) return s;
    if (!std::isfinite(scale)) return fail(ctx, GOOM_EINVAL, "scale must be finite");
    if (n == 0) return ctx ? GOOM_OK : fail(nullptr, GOOM_EINVAL, "null context");
    if (!table || !tokens || !rows) return fail(ctx, GOOM_EINVAL, "null data pointer");
    const size_t size = real_bytes(type);
    if (!aligned(table, size) || !aligned(rows, size) || !aligned(tokens, 8)) return fail(ctx, GOOM_EINVAL, "misaligned data pointer");
    if (int s = enter(ctx)) return s;
    const int v = vector_of(width, {{table, size}, {rows, size}});
    const long long blocks = (n * (width / v) + 255) / 256;
    goom::prof_begin(ctx, "embedding");
    const int rc = with_type(type, [&](auto tag) {
        typedef typename decltype(tag)::type S;
        return with_vector(v, [&](auto vec) {
            constexpr int V = decltype(vec)::value;
            if constexpr (V * sizeof(S) <= 16)
                embedding_kernel<S, V><<<(unsigned)(blocks < (1 << 20) ? blocks : 1 << 20), 256, 0, ctx->stream>>>(reinterpret_cast<const S *>(table), tokens, reinterpret_cast<S *>(rows), n,
                                                                                                             vocab, width, (float)scale);
            return goom::check_hip(ctx, hipGetLastError(), "embedding");
        });
    });
    goom::prof_end(ctx);
    return rc;
}

size_t goom_embedding_backward_workspace_bytes(int64_t n, int64_t vocab, int width)
{
    if (check_embedding(nullptr, n, vocab, width)) return 0;
    return embedding_plan(n, vocab, width).bytes;
}

int goom_embedding_backward(goom_ctx *ctx, const int64_t *tokens, const void *grad, void *grad_table, int64_t n, int64_t vocab, int width, int type, int table_type, double scale,
                            void *workspace, size_t workspace_bytes)
{
    if (!real_type(type) || !real_type(table_type)) return fail(ctx, GOOM_EINVAL, "unknown element type %d", real_type(type) ? table_type : type);
    if (int s = check_embedding(ctx, n, vocab, width)) return s;
    if (!std::isfinite(scale)) return fail(ctx, GOOM_EINVAL, "scale must be finite");
    if (!grad_table || (n > 0 && (!tokens || !grad))) return fail(ctx, GOOM_EINVAL, "null data pointer");
    const size_t size = real_bytes(type), wsize = real_bytes(table_type);
    if (!aligned(grad, size) || !aligned(grad_table, wsize) || !aligned(tokens, 8)) return fail(ctx, GOOM_EINVAL, "misaligned data pointer");
    const EmbeddingPlan plan = embedding_plan(n, vocab, width);
    if (int s = check_workspace(ctx, workspace, workspace_bytes, plan.bytes)) return s;
    if (int s = enter(ctx)) return s;
    unsigned char *ws = reinterpret_cast<unsigned char *>(workspace);
    auto take = [&](size_t bytes) {
        unsigned char *p = ws;
        ws += bytes;
        return p;
    };
    unsigned *const counts = reinterpret_cast<unsigned *>(take(plan.counts));
    unsigned *lists[2][2];
    for (auto &pair : lists)
        for (auto &l : pair) l = reinterpret_cast<unsigned *>(take(plan.list));
    unsigned *const start = reinterpret_cast<unsigned *>(take(plan.start));
    float *const sums = reinterpret_cast<float *>(take(plan.sums));

    const unsigned *keys = lists[0][0], *values = lists[0][1];
    goom::prof_begin(ctx, "embedding gradient: sort");
    for (int k = 0; n > 0 && k < plan.passes; k++) {
        SortPass p = {k == 0 ? tokens : nullptr, keys, values, lists[k & 1][0], lists[k & 1][1], counts, (unsigned)n, (unsigned)vocab, plan.tile, k * plan.bits, plan.bits};
        sort_count_kernel<<<plan.tiles, 256, 0, ctx->stream>>>(p);
        sort_scatter_kernel<<<plan.tiles, 256, 0, ctx->stream>>>(p);
        keys = p.out_keys;
        values = p.out_values;
    }
    run_start_kernel<<<(unsigned)(n / 256 + 1), 256, 0, ctx->stream>>>(keys, start, (unsigned)n, (unsigned)vocab);
    goom::prof_end(ctx);
    const int v = vector_of(width, {{grad, size}, {grad_table, wsize}, {sums, 4}});
    const int rc = with_type(type, [&](auto tag) {
        typedef typename decltype(tag)::type S;
        return with_vector(v, [&](auto vec) {
            constexpr int V = decltype(vec)::value;
            if constexpr (V <= 4) {
                const S *const gr = reinterpret_cast<const S *>(grad);
                if (n >= RUN) {
                    goom::prof_begin(ctx, "embedding gradient: frequent tokens");
                    run_block_kernel<S, V><<<dim3((unsigned)(n / RUN), (width + 64 * V - 1) / (64 * V)), 64, 0, ctx->stream>>>(gr, keys, values, sums, (unsigned)vocab, width);
                    goom::prof_end(ctx);
                }
                goom::prof_begin(ctx, "embedding gradient: rows");
                with_type(table_type, [&](auto wtag) {
                    typedef typename decltype(wtag)::type W;
                    const int parts = (width + 64 * V - 1) / (64 * V);
                    table_row_kernel<S, W, V><<<(unsigned)((vocab * parts + 3) / 4), 256, 0, ctx->stream>>>(gr, values, start, sums, reinterpret_cast<W *>(grad_table), vocab, width, parts, (float)scale);
                    return 0;
                });
                goom::prof_end(ctx);
            }
            return goom::check_hip(ctx, hipGetLastError(), "embedding gradient");
        });
    });
    return rc;
}

} // extern "C"
