// Token embeddings and their gradient.
//
// Forward: one pass, bound by the rows read and written.
// Gradient: a sum over the positions of each token, in a fixed order.  The positions are sorted by token (a stable radix
// sort, up to 9 bits a pass), so that a token's gradients are a run of sorted positions; the waves of a table row, each with its
// columns, add the run up and write the row, zeros where the run is empty, so that the table is written once and never read.  Tokens of text are far
// from equally frequent: blocks of 32 sorted positions that lie inside one run are summed beforehand, side by side, and the
// row's waves take their sums.
// Measured: 32,768 tokens of 50,257, width 1024, bfloat16: forward 21 us (6.3 TB/s), gradient 28 us of sorting, 8 of runs, 35 of table
// rows (4.9 TB/s).
#include <cmath>

#include "goom_real.h"

namespace goom_layer {

constexpr int RUN = 32;       // sorted positions of a block that is summed beforehand
constexpr int MAX_BINS = 512; // digits of a sorting pass

// Rows are taken in units of V columns, whatever the width: the last unit ends at the row's end and overlaps the one before it (both
// write the same values).
__device__ inline int column(int col, int width, int v) { return col + v <= width ? col : width - v; }

template <typename S, int V> __global__ __launch_bounds__(256) void embedding_kernel(const S *table, const int64_t *tokens, S *rows, long long n, long long vocab, int width, float scale)
{
    const int units = (width + V - 1) / V;
    for (long long u = blockIdx.x * 256ll + threadIdx.x; u < n * units; u += gridDim.x * 256ll) {
        const long long row = u / units;
        const int col = column((int)(u - row * units) * V, width, V);
        const long long t = tokens[row];
        float x[V];
        if (t >= 0 && t < vocab) {
            load_floats_unaligned<S, V>(table + t * width + col, x);
#pragma unroll
            for (int e = 0; e < V; e++) x[e] *= scale;
        } else {
#pragma unroll
            for (int e = 0; e < V; e++) x[e] = 0.0f;
        }
        store_floats_unaligned<S, V>(rows + row * width + col, x);
    }
}

// ---- sorting: keys are tokens, `vocab` for those outside; values are positions
struct SortPass {
    const int64_t *tokens; // first pass: keys come from here, positions are the indices
    const unsigned *keys, *values;
    unsigned *out_keys, *out_values;
    unsigned *counts; // [tiles][bins]
    unsigned n, vocab, tile;
    int shift, bits;
};

__device__ inline unsigned token_key(long long t, unsigned vocab) { return t >= 0 && t < vocab ? (unsigned)t : vocab; }

// keys of the lane's entries i, i + 64, ..., all loads at once; entries from `end` on have none
template <int N> __device__ inline void load_keys(const SortPass &p, unsigned i, unsigned end, unsigned (&key)[N])
{
    if (p.tokens) {
        long long t[N];
#pragma unroll
        for (int k = 0; k < N; k++) t[k] = p.tokens[i + k * 64 < end ? i + k * 64 : 0];
#pragma unroll
        for (int k = 0; k < N; k++) key[k] = token_key(t[k], p.vocab);
    } else {
#pragma unroll
        for (int k = 0; k < N; k++) key[k] = p.keys[i + k * 64 < end ? i + k * 64 : 0];
    }
}

// lanes whose digit equals this lane's, among those that are live
__device__ inline unsigned long long same_digit(unsigned digit, int bits, bool live)
{
    unsigned long long same = __ballot(live);
    for (int b = 0; b < bits; b++) {
        const unsigned long long m = __ballot(digit >> b & 1);
        same &= digit >> b & 1 ? m : ~m;
    }
    return same;
}

// one addition a wave and digit: frequent tokens' digits would have the lanes wait for each other
__device__ inline unsigned long long add_count(unsigned *count, unsigned digit, int bits, bool live)
{
    const unsigned long long same = same_digit(digit, bits, live);
    if (live && !(same & ((1ull << (threadIdx.x & 63)) - 1))) atomicAdd(&count[digit], (unsigned)__popcll(same));
    return same;
}

constexpr int ROUNDS = 4; // entries of a lane that are loaded at once

// counts of the digits by tiles (counted by the scattering pass before, with atomics in memory, frequent tokens' counts made it
// twice as long: 16 us for 8)
__global__ __launch_bounds__(256) void sort_count_kernel(SortPass p)
{
    __shared__ unsigned count[MAX_BINS];
    const int bins = 1 << p.bits;
    for (int d = threadIdx.x; d < bins; d += 256) count[d] = 0;
    __syncthreads();
    const unsigned begin = blockIdx.x * p.tile, end = p.n - begin < p.tile ? p.n : begin + p.tile;
    for (unsigned i = begin + (threadIdx.x >> 6) * 64 * ROUNDS + (threadIdx.x & 63); i < end; i += 256 * ROUNDS) {
        unsigned key[ROUNDS];
        load_keys<ROUNDS>(p, i, end, key);
#pragma unroll
        for (int k = 0; k < ROUNDS; k++) add_count(count, key[k] >> p.shift & (bins - 1), p.bits, i + k * 64 < end);
    }
    __syncthreads();
    for (int d = threadIdx.x; d < bins; d += 256) p.counts[blockIdx.x * (unsigned)bins + d] = count[d];
}

// Each wave has a quarter of the tile and goes through it 64 entries at a time; entries of equal digit keep their order.
__global__ __launch_bounds__(256) void sort_scatter_kernel(SortPass p)
{
    __shared__ unsigned at[4][MAX_BINS]; // counts of the waves' quarters, then where each wave's next entry of a digit goes
    __shared__ unsigned waves[4];
    const int bins = 1 << p.bits, lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const unsigned begin = blockIdx.x * p.tile + wave * (p.tile / 4), limit = (p.n < (blockIdx.x + 1u) * p.tile ? p.n : (blockIdx.x + 1u) * p.tile);
    const unsigned end = begin + p.tile / 4 < limit ? begin + p.tile / 4 : limit;
    unsigned key[ROUNDS]; // the first entries; they stay here in tiles of 1024
    if (begin < end) load_keys<ROUNDS>(p, begin + lane, end, key);
    for (int d = threadIdx.x; d < 4 * MAX_BINS; d += 256) at[d / MAX_BINS][d % MAX_BINS] = 0;
    // entries of each digit in all tiles, and in the tiles before this one; a thread has two neighbouring digits
    unsigned total[2] = {0, 0}, before[2] = {0, 0};
    if ((int)threadIdx.x * 2 < bins)
        for (unsigned t0 = 0; t0 < gridDim.x; t0 += 32) {
            unsigned long long c[32];
#pragma unroll
            for (int t = 0; t < 32; t++) c[t] = t0 + t < gridDim.x ? *reinterpret_cast<const unsigned long long *>(p.counts + (t0 + t) * (unsigned)bins + threadIdx.x * 2) : 0;
#pragma unroll
            for (int t = 0; t < 32; t++) {
                total[0] += (unsigned)c[t];
                total[1] += (unsigned)(c[t] >> 32);
                if (t0 + t < blockIdx.x) {
                    before[0] += (unsigned)c[t];
                    before[1] += (unsigned)(c[t] >> 32);
                }
            }
        }
    unsigned sum = total[0] + total[1]; // running sums over the digits: of the wave, then of the waves
    for (int s = 1; s < 64; s *= 2) {
        const unsigned x = __shfl_up(sum, s);
        sum += lane >= s ? x : 0;
    }
    if (lane == 63) waves[wave] = sum;
    __syncthreads();
    unsigned long long same[ROUNDS]; // of the first entries, too
    for (unsigned i0 = begin; i0 < end; i0 += 64 * ROUNDS) {
        unsigned more[ROUNDS];
        if (i0 != begin) load_keys<ROUNDS>(p, i0 + lane, end, more);
#pragma unroll
        for (int k = 0; k < ROUNDS; k++) {
            const unsigned digit = (i0 != begin ? more[k] : key[k]) >> p.shift & (bins - 1);
            const unsigned long long m = add_count(at[wave], digit, p.bits, i0 + lane + k * 64 < end);
            if (i0 == begin) same[k] = m;
        }
    }
    __syncthreads();
    unsigned base = sum - total[0] - total[1];
    for (int v = 0; v < wave; v++) base += waves[v];
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
    for (unsigned i0 = begin; i0 < end; i0 += 64 * ROUNDS) {
        if (i0 != begin) load_keys<ROUNDS>(p, i0 + lane, end, key);
        unsigned value[ROUNDS];
#pragma unroll
        for (int k = 0; k < ROUNDS; k++) {
            const unsigned i = i0 + k * 64 + lane;
            value[k] = p.tokens ? i : p.values[i < end ? i : 0];
        }
#pragma unroll
        for (int k = 0; k < ROUNDS; k++) {
            if (i0 + k * 64 >= end) break;
            const bool live = i0 + k * 64 + lane < end;
            const unsigned digit = key[k] >> p.shift & (bins - 1);
            const unsigned long long mine = i0 == begin ? same[k] : same_digit(digit, p.bits, live);
            const unsigned rank = __popcll(mine & ((1ull << lane) - 1));
            unsigned to = 0;
            if (live) to = at[wave][digit] + rank;
            __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront"); // all lanes have read before a digit's first lane moves it on
            if (live) {
                if (rank == 0) at[wave][digit] += __popcll(mine);
                p.out_keys[to] = key[k];
                p.out_values[to] = value[k];
            }
            __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
        }
    }
}

// The whole sort of up to SMALL positions by one workgroup, in LDS: five launches fewer, and as fast up to here.
constexpr int SMALL = 4096;
__global__ __launch_bounds__(1024) void sort_small_kernel(const int64_t *tokens, unsigned *out_keys, unsigned *out_values, unsigned n, unsigned vocab, int passes, int bits)
{
    __shared__ unsigned keys[SMALL];
    __shared__ unsigned short values[SMALL];
    __shared__ unsigned at[16][MAX_BINS];
    __shared__ unsigned waves[16];
    constexpr int N = SMALL / 1024;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, bins = 1 << bits;
    const unsigned begin = wave * 64 * N + lane; // a wave has 64 N entries in order, a lane every 64th of them
    unsigned key[N], value[N];
    long long t[N];
#pragma unroll
    for (int k = 0; k < N; k++) t[k] = tokens[begin + k * 64 < n ? begin + k * 64 : 0];
#pragma unroll
    for (int k = 0; k < N; k++) {
        key[k] = token_key(t[k], vocab);
        value[k] = begin + k * 64;
    }
    for (int pass = 0; pass < passes; pass++) {
        const int shift = pass * bits;
        for (int d = threadIdx.x; d < 16 * MAX_BINS; d += 1024) at[d / MAX_BINS][d % MAX_BINS] = 0;
        __syncthreads();
        unsigned long long same[N];
#pragma unroll
        for (int k = 0; k < N; k++) same[k] = add_count(at[wave], key[k] >> shift & (bins - 1), bits, begin + k * 64 < n);
        __syncthreads();
        unsigned total = 0;
        const int d = threadIdx.x;
        if (d < bins)
#pragma unroll
            for (int v = 0; v < 16; v++) total += at[v][d];
        unsigned sum = total;
        for (int s = 1; s < 64; s *= 2) {
            const unsigned x = __shfl_up(sum, s);
            sum += lane >= s ? x : 0;
        }
        if (lane == 63) waves[wave] = sum;
        __syncthreads();
        if (d < bins) {
            unsigned next = sum - total;
            for (int v = 0; v < wave; v++) next += waves[v];
#pragma unroll
            for (int v = 0; v < 16; v++) {
                const unsigned c = at[v][d];
                at[v][d] = next;
                next += c;
            }
        }
        __syncthreads();
#pragma unroll
        for (int k = 0; k < N; k++) {
            const bool live = begin + k * 64 < n;
            const unsigned digit = key[k] >> shift & (bins - 1);
            const unsigned rank = __popcll(same[k] & ((1ull << lane) - 1));
            unsigned to = 0;
            if (live) to = at[wave][digit] + rank;
            __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
            if (live) {
                if (rank == 0) at[wave][digit] += __popcll(same[k]);
                keys[to] = key[k];
                values[to] = (unsigned short)value[k];
            }
            __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
        }
        __syncthreads();
#pragma unroll
        for (int k = 0; k < N; k++) {
            key[k] = keys[begin + k * 64];
            value[k] = values[begin + k * 64];
        }
    }
#pragma unroll
    for (int k = 0; k < N; k++)
        if (begin + k * 64 < n) {
            out_keys[begin + k * 64] = key[k];
            out_values[begin + k * 64] = value[k];
        }
}

// x += rows of grad at sorted positions [i, end), in order
template <typename S, int V> __device__ inline void add_rows(float (&x)[V], const S *grad, const unsigned *values, unsigned i, unsigned end, int width, int col)
{
    for (; i + 8 <= end; i += 8) { // eight rows in flight
        float y[8][V];
#pragma unroll
        for (int k = 0; k < 8; k++) load_floats_unaligned<S, V>(grad + (long long)values[i + k] * width + col, y[k]);
#pragma unroll
        for (int k = 0; k < 8; k++)
#pragma unroll
            for (int e = 0; e < V; e++) x[e] += y[k][e];
    }
    for (; i < end; i++) {
        float y[V];
        load_floats_unaligned<S, V>(grad + (long long)values[i] * width + col, y);
#pragma unroll
        for (int e = 0; e < V; e++) x[e] += y[e];
    }
}

// start[t] = first sorted position whose token is at least t, t = 0 .. vocab.  A thread writes the tokens from its left
// neighbour's on up to its own; gaps of more than 64 (few positions, many tokens) are written by the whole workgroup.
__device__ inline void run_starts(const unsigned *keys, unsigned *start, unsigned n, unsigned vocab, unsigned block)
{
    __shared__ unsigned gaps[256][3];
    __shared__ int count;
    if (threadIdx.x == 0) count = 0;
    __syncthreads();
    const unsigned i = block * 256 + threadIdx.x;
    if (i <= n) {
        const unsigned from = i == 0 ? 0 : keys[i - 1] + 1, to = i == n ? vocab : keys[i];
        if (from <= to && to - from > 64) {
            const int at = atomicAdd(&count, 1);
            gaps[at][0] = i;
            gaps[at][1] = from;
            gaps[at][2] = to;
        } else {
            for (unsigned t = from; t <= to; t++) start[t] = i;
        }
    }
    __syncthreads();
    for (int k = 0; k < count; k++) {
        const unsigned at = gaps[k][0], to = gaps[k][2];
        for (unsigned t = gaps[k][1] + threadIdx.x; t <= to; t += 256) start[t] = at;
    }
}

// The first n / 256 + 1 workgroups: run starts.  The others: sums of the blocks of RUN sorted positions that belong to one token, a
// wave each 64 V columns of a block.
template <typename S, int V> __global__ __launch_bounds__(256) void runs_kernel(const S *grad, const unsigned *keys, const unsigned *values, unsigned *start, float *sums, unsigned n, unsigned vocab, int width, int parts)
{
    const long long at = block_of();
    if (at <= n / 256) {
        run_starts(keys, start, n, vocab, (unsigned)at);
        return;
    }
    const unsigned task = (unsigned)(at - n / 256 - 1) * 4 + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), block = task / parts; // (below 2^29)
    const unsigned i = block * RUN;
    if (block >= n / RUN) return;
    const unsigned key = keys[i];
    if (key != keys[i + RUN - 1] || key >= vocab) return;
    int col = ((int)(task - block * parts) * 64 + (threadIdx.x & 63)) * V;
    if (col >= width) return;
    col = column(col, width, V);
    float x[V] = {};
    add_rows<S, V>(x, grad, values, i, i + RUN, width, col);
    store_floats_unaligned<float, V>(sums + (long long)block * width + col, x);
}

// 64 V columns of a table row a wave: the run's head, its whole blocks, its tail.  grid: vocab parts / 4, in one order
template <typename S, typename W, int V> __global__ __launch_bounds__(256) void table_row_kernel(const S *grad, const unsigned *values, const unsigned *start, const float *sums, W *table, long long vocab, int width, int parts, float scale)
{
    const long long task = block_of() * 4 + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), row = task / parts;
    int col = ((int)(task - row * parts) * 64 + (threadIdx.x & 63)) * V;
    if (row >= vocab) return;
    const unsigned begin = start[row], end = start[row + 1];
    const unsigned first = (begin + RUN - 1) / RUN, last = end / RUN; // whole blocks: first .. last - 1
    if (col >= width) return;
    col = column(col, width, V);
    float x[V] = {};
    if (first < last) {
        add_rows<S, V>(x, grad, values, begin, first * RUN, width, col);
        unsigned b = first;
        for (; b + 8 <= last; b += 8) {
            float y[8][V];
#pragma unroll
            for (int k = 0; k < 8; k++) load_floats_unaligned<float, V>(sums + (long long)(b + k) * width + col, y[k]);
#pragma unroll
            for (int k = 0; k < 8; k++)
#pragma unroll
                for (int e = 0; e < V; e++) x[e] += y[k][e];
        }
        for (; b < last; b++) {
            float y[V];
            load_floats_unaligned<float, V>(sums + (long long)b * width + col, y);
#pragma unroll
            for (int e = 0; e < V; e++) x[e] += y[e];
        }
        add_rows<S, V>(x, grad, values, last * RUN, end, width, col);
    } else {
        add_rows<S, V>(x, grad, values, begin, end, width, col);
    }
#pragma unroll
    for (int e = 0; e < V; e++) x[e] *= scale;
    store_floats_unaligned<W, V>(table + row * width + col, x);
}

// Up to FEW positions need no sorting: every row's waves look at all tokens themselves.  One launch.
constexpr int FEW = 256;
template <typename S, typename W, int V> __global__ __launch_bounds__(256) void few_rows_kernel(const S *grad, const int64_t *tokens, W *table, unsigned n, long long vocab, int width, int parts, float scale)
{
    const long long task = block_of() * 4 + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), row = task / parts;
    const int lane = threadIdx.x & 63;
    int col = ((int)(task - row * parts) * 64 + lane) * V;
    if (row >= vocab) return;
    unsigned long long mine[FEW / 64]; // positions of this row's token
#pragma unroll
    for (int k = 0; k < FEW / 64; k++) mine[k] = __ballot(k * 64 + lane < (int)n && tokens[k * 64 + lane < (int)n ? k * 64 + lane : 0] == row);
    if (col >= width) return;
    col = column(col, width, V);
    float x[V] = {};
#pragma unroll
    for (int k = 0; k < FEW / 64; k++)
        while (mine[k]) {
            const int i = k * 64 + __builtin_ctzll(mine[k]);
            mine[k] &= mine[k] - 1;
            float y[V];
            load_floats_unaligned<S, V>(grad + (long long)i * width + col, y);
#pragma unroll
            for (int e = 0; e < V; e++) x[e] += y[e];
        }
#pragma unroll
    for (int e = 0; e < V; e++) x[e] *= scale;
    store_floats_unaligned<W, V>(table + row * width + col, x);
}

struct EmbeddingPlan {
    int passes, bits;
    bool small;
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
    p.small = n <= SMALL;
    p.counts = p.small ? 0 : up((size_t)p.tiles * (1u << p.bits) * 4);
    p.list = up((size_t)n * 4);
    p.start = up((size_t)(vocab + 1) * 4);
    p.sums = up((size_t)(n / RUN) * width * 4);
    p.bytes = p.counts + 4 * p.list + p.start + p.sums;
    return p;
}

static int check_embedding(goom_ctx *ctx, long long n, long long vocab, int width)
{
    if (n < 0 || vocab <= 0 || width <= 0) return goom::fail(ctx, GOOM_EINVAL, "n must not be negative, vocab and width positive");
    if (n >= (1ll << 31) || vocab >= (1ll << 31) || (double)vocab * width > 1e11 || (double)n * width > 1e12)
        return goom::fail(ctx, GOOM_EUNSUPPORTED, "up to 2^31 - 1 tokens and table rows, 10^11 entries of the table and 10^12 of the rows");
    return GOOM_OK;
}

// columns of a unit: 16 bytes of the larger type, no more than a row has
static int vector_of(int width, size_t size)
{
    int v = (int)(16 / size);
    while (v > width) v /= 2;
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
    if (!std::isfinite((float)scale)) return fail(ctx, GOOM_EINVAL, "scale must be finite, and a float");
    if (n == 0) return ctx ? GOOM_OK : fail(nullptr, GOOM_EINVAL, "null context");
    if (!table || !tokens || !rows) return fail(ctx, GOOM_EINVAL, "null data pointer");
    const size_t size = real_bytes(type);
    if (!aligned(table, size) || !aligned(rows, size) || !aligned(tokens, 8)) return fail(ctx, GOOM_EINVAL, "misaligned data pointer");
    if (int s = enter(ctx)) return s;
    const int v = vector_of(width, size);
    const long long blocks = (n * ((width + v - 1) / v) + 255) / 256;
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
    if (!std::isfinite((float)scale)) return fail(ctx, GOOM_EINVAL, "scale must be finite, and a float");
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
    if (n > FEW) goom::prof_begin(ctx, "embedding gradient: sort");
    if (n <= FEW) {
        // no sorting
    } else if (plan.small) {
        sort_small_kernel<<<1, 1024, 0, ctx->stream>>>(tokens, lists[0][0], lists[0][1], (unsigned)n, (unsigned)vocab, plan.passes, plan.bits);
    } else {
        for (int k = 0; k < plan.passes; k++) {
            SortPass p = {k == 0 ? tokens : nullptr, keys, values, lists[k & 1][0], lists[k & 1][1], counts, (unsigned)n, (unsigned)vocab, plan.tile, k * plan.bits, plan.bits};
            sort_count_kernel<<<plan.tiles, 256, 0, ctx->stream>>>(p);
            sort_scatter_kernel<<<plan.tiles, 256, 0, ctx->stream>>>(p);
            keys = p.out_keys;
            values = p.out_values;
        }
    }
    if (n > FEW) goom::prof_end(ctx);
    const int v = vector_of(width, 4); // (block sums are floats)
    const int rc = with_type(type, [&](auto tag) {
        typedef typename decltype(tag)::type S;
        return with_vector(v, [&](auto vec) {
            constexpr int V = decltype(vec)::value;
            if constexpr (V <= 4) {
                const S *const gr = reinterpret_cast<const S *>(grad);
                const int parts = (width + 64 * V - 1) / (64 * V);
                const dim3 row_groups = grid_of((vocab * parts + 3) / 4, 256);
                if (n > FEW) {
                    goom::prof_begin(ctx, "embedding gradient: runs");
                    runs_kernel<S, V><<<grid_of(n / 256 + 1 + (n / RUN * parts + 3) / 4, 256), 256, 0, ctx->stream>>>(gr, keys, values, start, sums, (unsigned)n, (unsigned)vocab, width, parts);
                    goom::prof_end(ctx);
                }
                goom::prof_begin(ctx, "embedding gradient: rows");
                with_type(table_type, [&](auto wtag) {
                    typedef typename decltype(wtag)::type W;
                    W *const out = reinterpret_cast<W *>(grad_table);
                    if (n > FEW) table_row_kernel<S, W, V><<<row_groups, 256, 0, ctx->stream>>>(gr, values, start, sums, out, vocab, width, parts, (float)scale);
                    else few_rows_kernel<S, W, V><<<row_groups, 256, 0, ctx->stream>>>(gr, tokens, out, (unsigned)n, vocab, width, parts, (float)scale);
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
