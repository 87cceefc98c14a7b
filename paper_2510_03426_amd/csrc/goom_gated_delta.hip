// The gated delta rule: single tokens, and the C ABI.  The kernels for many tokens are in goom_gated_delta_walk.h.
#include <cmath>

#include "goom_gated_delta_walk.h"

namespace goom_layer {

// ---- single tokens.  With x = S^T k and z = S^T q of the state before, both sums over its rows in the one pass that reads it,
//     u = beta (v - a x),   S' = a S + k u^T,   o = scale (a z + (k . q) u).
// Bound by the states' bytes.  A workgroup has 32 columns of a head's state (eight groups of four) and its threads every 32nd row,
// which stay in registers until u is known; sums meet in LDS in a fixed order.  256 tokens of 16 heads of 128 x 128: 115 us, 4.7 TB/s (64
// columns a workgroup the same, 128 a tenth more); one token of 16 heads of 64: 5 us, a launch and two waits.
template <typename S> __global__ __launch_bounds__(256) void delta_step_kernel(goom_delta_shape sh, const S *q, const S *k, const S *v, const float *log_decay,
                                                                               const float *beta, const float *state, S *o, float *next)
{
    const int h = blockIdx.x % sh.heads, col = blockIdx.y * 32 + (threadIdx.x & 7) * 4, row0 = threadIdx.x >> 3;
    const long long s = blockIdx.x / sh.heads;
    const int kh = h / (sh.heads / sh.qk_heads);
    const float decay = power2(log2_of(log_decay[s * sh.heads + h])), be = beta[s * sh.heads + h];
    const S *const qh = q + s * sh.q_token + kh * sh.q_head, *const kv = k + s * sh.k_token + kh * sh.k_head, *const vh = v + s * sh.v_token + h * sh.v_head;
    const long long base = (s * sh.heads + h) * (long long)sh.dk * sh.dv;
    constexpr int ROWS = GOOM_MAX_DIM / 32;
    float st[ROWS][4], kr[ROWS], sum[9] = {}; // k . S and q . S of four columns, k . q
#pragma unroll
    for (int u = 0; u < ROWS; u++) {
        const int row = row0 + u * 32;
        kr[u] = 0.0f;
#pragma unroll
        for (int e = 0; e < 4; e++) st[u][e] = 0.0f;
        if (row < sh.dk) {
            kr[u] = (float)kv[row];
            const float *p = state ? state + base + (long long)row * sh.dv + col : nullptr;
            if (p && col + 4 <= sh.dv) {
                const f32x4 four = load_unaligned<float, 4>(p);
#pragma unroll
                for (int e = 0; e < 4; e++) st[u][e] = four[e];
            } else if (p) {
#pragma unroll
                for (int e = 0; e < 4; e++)
                    if (col + e < sh.dv) st[u][e] = p[e];
            }
            const float qr = (float)qh[row];
            sum[8] += kr[u] * qr;
#pragma unroll
            for (int e = 0; e < 4; e++) {
                sum[e] += kr[u] * st[u][e];
                sum[4 + e] += qr * st[u][e];
            }
        }
    }
    __shared__ float part[4][8][9];
#pragma unroll
    for (int e = 0; e < 9; e++) { // the wave's eight rows, then the four waves
        sum[e] += __shfl_xor(sum[e], 8);
        sum[e] += __shfl_xor(sum[e], 16);
        sum[e] += __shfl_xor(sum[e], 32);
        if ((threadIdx.x & 63) < 8) part[threadIdx.x >> 6][threadIdx.x & 7][e] = sum[e];
    }
    __syncthreads();
#pragma unroll
    for (int e = 0; e < 9; e++) {
        const int c = threadIdx.x & 7;
        sum[e] = (part[0][c][e] + part[1][c][e]) + (part[2][c][e] + part[3][c][e]);
    }
    float u4[4];
#pragma unroll
    for (int e = 0; e < 4; e++) u4[e] = col + e < sh.dv ? be * ((float)vh[col + e] - decay * sum[e]) : 0.0f;
#pragma unroll
    for (int u = 0; u < ROWS; u++) {
        const int row = row0 + u * 32;
        if (row < sh.dk) {
#pragma unroll
            for (int e = 0; e < 4; e++) st[u][e] = decay * st[u][e] + kr[u] * u4[e];
            float *p = next + base + (long long)row * sh.dv + col;
            if (col + 4 <= sh.dv) {
                store_floats_unaligned<float, 4>(p, st[u]);
            } else {
#pragma unroll
                for (int e = 0; e < 4; e++)
                    if (col + e < sh.dv) p[e] = st[u][e];
            }
        }
    }
    if (threadIdx.x < 8)
#pragma unroll
        for (int e = 0; e < 4; e++)
            if (col + e < sh.dv) o[(s * sh.heads + h) * (long long)sh.dv + col + e] = (S)((float)sh.scale * (decay * sum[4 + e] + sum[8] * u4[e]));
}

// ---- host side

static int chunk_len(int type) { return type == GOOM_REAL_BF16 ? chunk_of<bf16>() : chunk_of<float>(); }
static_assert(chunk_of<f16>() == chunk_of<float>(), "one chunk for halves and floats");

// fills in the strides that 0 stands for; GOOM_OK or an error
static int check_shape(goom_ctx *ctx, const goom_delta_shape *given, goom_delta_shape &sh, bool packed, bool step)
{
    if (!given) return goom::fail(ctx, GOOM_EINVAL, "null shape");
    sh = *given;
    if (!real_type(sh.type)) return goom::fail(ctx, GOOM_EINVAL, "unknown element type %d", sh.type);
    if (sh.flags) return goom::fail(ctx, GOOM_EINVAL, "unknown flags 0x%x", (unsigned)sh.flags);
    if (sh.seqs < 0 || sh.tokens < 0) return goom::fail(ctx, GOOM_EINVAL, "negative number of sequences or tokens");
    if (sh.heads <= 0 || sh.qk_heads <= 0 || sh.heads % sh.qk_heads) return goom::fail(ctx, GOOM_EINVAL, "qk_heads must be positive and divide heads");
    if (sh.dk <= 0 || sh.dv <= 0) return goom::fail(ctx, GOOM_EINVAL, "dk and dv must be positive");
    if (sh.dk > GOOM_MAX_DIM || sh.dv > GOOM_MAX_DIM) return goom::fail(ctx, GOOM_EUNSUPPORTED, "dk and dv go up to %d", GOOM_MAX_DIM);
    if (!std::isfinite((float)sh.scale)) return goom::fail(ctx, GOOM_EINVAL, "scale must be finite, and a float");
    if (sh.seqs == 0 && sh.tokens > 0) return goom::fail(ctx, GOOM_EINVAL, "tokens without a sequence");
    if (!packed && sh.seqs > 0 && sh.tokens % sh.seqs) return goom::fail(ctx, GOOM_EINVAL, "without offsets the sequences have tokens / seqs tokens each");
    if (step && sh.seqs != sh.tokens) return goom::fail(ctx, GOOM_EINVAL, "one token a sequence");
    // sequences, and chunks, times heads and the parts of each must stay below 2^31
    if (sh.seqs > (1 << 24) / sh.heads || sh.tokens > (1ll << 40) || sh.tokens / chunk_len(sh.type) > (1 << 24) / sh.heads)
        return goom::fail(ctx, GOOM_EUNSUPPORTED, "too many sequences, heads or tokens");
    if (step && sh.seqs * sh.heads > 0xffffffffll / 256) return goom::fail(ctx, GOOM_EUNSUPPORTED, "too many sequences or heads"); // threads of a grid's first axis
    const int64_t rows[3][3] = {{sh.q_token, sh.q_head, sh.dk}, {sh.k_token, sh.k_head, sh.dk}, {sh.v_token, sh.v_head, sh.dv}};
    for (auto &x : rows)
        if (x[0] < 0 || x[1] < 0 || ((x[0] || x[1]) && (x[0] < x[2] || x[1] < x[2])) || x[0] > (1ll << 40) || x[1] > (1ll << 40))
            return goom::fail(ctx, GOOM_EINVAL, "strides of tokens and heads must be 0 (both: contiguous) or at least a head's entries");
    if (!sh.q_token) { sh.q_token = (int64_t)sh.qk_heads * sh.dk; sh.q_head = sh.dk; }
    if (!sh.k_token) { sh.k_token = (int64_t)sh.qk_heads * sh.dk; sh.k_head = sh.dk; }
    if (!sh.v_token) { sh.v_token = (int64_t)sh.heads * sh.dv; sh.v_head = sh.dv; }
    if (!step && (sh.q_token > (1 << 22) || sh.k_token > (1 << 22) || sh.v_token > (1 << 22) || (int64_t)sh.heads * sh.dv > (1 << 22))) // 32-bit offsets within a chunk
        return goom::fail(ctx, GOOM_EUNSUPPORTED, "more than 2^22 elements from token to token");
    return GOOM_OK;
}

struct Pieces { long long len, slots, per_seq; }; // sequences in pieces of len tokens

static Pieces pieces_of(const goom_delta_shape &sh, bool packed, long long len)
{
    const long long each = sh.seqs > 0 ? sh.tokens / sh.seqs : 0;
    if (packed) return {len, sh.tokens / len + sh.seqs, 0};
    const long long per = each > 0 ? (each + len - 1) / len : 1;
    return {len, sh.seqs * per, per};
}

// what a call needs room for, by parts
struct DeltaPlan {
    Pieces chunk, seg;
    bool maps;      // sequences are cut into segments
    int dk, cols, pitch, parts, map_parts, ch;
    size_t m, vecs, totals, map, order, state, rows, sum, bytes; // state, rows, sum: two each
};

static DeltaPlan plan_of(const goom_delta_shape &sh, bool packed, bool backward)
{
    DeltaPlan p = {};
    p.ch = chunk_len(sh.type);
    p.dk = delta_rows(sh.dk);
    p.cols = delta_columns(sh.dv);
    p.parts = (sh.dv + p.cols - 1) / p.cols;
    p.map_parts = (p.dk + p.cols - 1) / p.cols; // (zeros past dk)
    p.pitch = p.parts * p.cols;
    p.chunk = pieces_of(sh, packed, p.ch);
    // Segments where the walks are fewer than the chip has CUs: as many as make two a CU.  A cut costs a walk without outputs over the columns of A and B:
    // with 256 walks of 64 chunks (8 x 4096 tokens, 16 heads of 128, bfloat16) both directions took 2120 us uncut, 2450 us in two segments each.
    const long long walks = sh.seqs * sh.heads * p.parts, mean = sh.seqs > 0 ? (sh.tokens + sh.seqs - 1) / sh.seqs : 0, least = 4 * p.ch;
    long long want = walks > 0 && walks < 256 ? 512 / walks : 1;
    if (want > mean / least) want = mean / least;
    p.maps = want > 1;
    const long long len = p.maps ? ((mean + want - 1) / want + p.ch - 1) / p.ch * p.ch : (sh.tokens / p.ch + 1) * p.ch; // (no sequence is longer)
    p.seg = pieces_of(sh, packed, len);
    if (!p.maps) p.seg = {len, sh.seqs, 1};
    // Without tokens one walk passes the states on, and nothing is kept: what is in the workspace then is written by kernels that are not launched
    if (sh.tokens == 0) return p;
    const size_t records = (size_t)p.chunk.slots * sh.heads, cuts = (size_t)p.seg.slots * sh.heads;
    p.m = goom::align_up(records * m_floats(p.ch) * sizeof(float), 256);
    p.vecs = goom::align_up(records * (p.ch == 64 ? sizeof(ChunkVec<64>) : sizeof(ChunkVec<32>)), 256);
    p.totals = p.maps ? goom::align_up(cuts * p.dk * p.pitch * 4, 256) : 0;
    p.map = p.maps ? goom::align_up(cuts * p.dk * p.dk * 4, 256) : 0;
    // Packed sequences, whole, of more walks than CUs: the longest first (us, in any order and so: 37 sequences of up to 2198 tokens, 888 walks, floats
    // 347 and 260, 444 walks 267 and 250; 30 of up to 3914, 960 walks, bfloat16 587 and 489; the ordering itself, beside the chunks' matrices, up to 6).  Of
    // very many none is long beside all the others.
    p.order = packed && !p.maps && sh.seqs > 1 && sh.seqs <= 4096 && walks > 256 ? goom::align_up((size_t)sh.seqs * sizeof(int), 256) : 0;
    p.state = backward ? goom::align_up(records * p.dk * p.pitch * 4, 256) : 0;
    p.rows = backward ? goom::align_up(records * p.ch * p.pitch * 4, 256) : 0;
    p.sum = backward && sh.heads != sh.qk_heads ? goom::align_up((size_t)sh.tokens * sh.heads * sh.dk * 4, 256) : 0;
    p.bytes = p.m + p.vecs + p.totals + p.map + p.order + 2 * (p.state + p.rows + p.sum);
    return p;
}

static Cut cut_of(const goom_delta_shape &sh, const int64_t *offsets, const Pieces &p)
{
    return {offsets, sh.tokens, sh.seqs, sh.seqs > 0 ? sh.tokens / sh.seqs : 0, p.len, p.per_seq ? p.per_seq : 1};
}

static DeltaArgs delta_args(const goom_delta_shape &sh, const DeltaPlan &p, const int64_t *offsets, const void *q, const void *k, const void *v, const float *log_decay,
                            const float *beta)
{
    DeltaArgs w = {};
    w.chunk = cut_of(sh, offsets, p.chunk);
    w.seg = cut_of(sh, offsets, p.seg);
    w.q = q; w.q_tok = sh.q_token; w.q_head = sh.q_head;
    w.k = k; w.k_tok = sh.k_token; w.k_head = sh.k_head;
    w.v = v; w.v_tok = sh.v_token; w.v_head = sh.v_head;
    w.o_tok = (long long)sh.heads * sh.dv;
    w.log_decay = log_decay;
    w.beta = beta;
    w.heads = sh.heads;
    w.share = sh.heads / sh.qk_heads;
    w.dk = sh.dk;
    w.dv = sh.dv;
    w.scale = (float)sh.scale;
    w.pitch = p.pitch;
    w.parts = p.parts;
    w.map_parts = p.map_parts;
    return w;
}

static int launch_carry(goom_ctx *ctx, const goom_delta_shape &sh, const DeltaArgs &w, bool back)
{
    return with_delta(sh.dk, sh.dv, [&](auto rows, auto cols) {
        constexpr int DK = decltype(rows)::value, DV = decltype(cols)::value;
        constexpr size_t bytes = carry_bytes<DK>();
        static std::atomic<unsigned long long> done{0}, done_back{0};
        auto *kernel = back ? delta_carry_kernel<DK, DV, true> : delta_carry_kernel<DK, DV, false>;
        if (int st = allow_lds(ctx, reinterpret_cast<const void *>(kernel), bytes, back ? done_back : done)) return st;
        goom::prof_begin(ctx, "gated delta rule: carries");
        kernel<<<grid_of(sh.seqs * sh.heads * w.parts, DV * 4), DV * 4, bytes, ctx->stream>>>(w);
        goom::prof_end(ctx);
        return goom::check_hip(ctx, hipGetLastError(), "gated delta rule: carries");
    });
}

template <typename S> static int run_forward(goom_ctx *ctx, const goom_delta_shape &sh, const DeltaPlan &p, const DeltaArgs &w)
{
    if (sh.tokens > 0) {
        if (int s = launch_delta_within<S>(ctx, w, p.chunk.slots)) return s;
        if (p.maps) {
            if (int s = launch_delta_walk<S>(ctx, w, MAPS, p.seg.slots, "gated delta rule: segments' maps")) return s;
            if (int s = launch_carry(ctx, sh, w, false)) return s;
        }
    }
    return launch_delta_walk<S>(ctx, w, FORWARD, p.seg.slots, "gated delta rule");
}

struct BackPointers { const void *go; const float *state, *grad_final; float *grad_state; void *gq, *gk, *gv; float *g_log_decay, *g_beta; };

template <typename S> static int run_backward(goom_ctx *ctx, const goom_delta_shape &sh, const DeltaPlan &p, DeltaArgs w, const BackPointers &b, float *kept_s, float *kept_d,
                                              float *rows_e, float *rows_w, float *sum_q, float *sum_k)
{
    if (sh.tokens > 0) {
        if (int s = launch_delta_within<S>(ctx, w, p.chunk.slots)) return s;
        w.init = b.state;
        if (p.maps) {
            if (int s = launch_delta_walk<S>(ctx, w, MAPS, p.seg.slots, "gated delta rule: segments' maps")) return s;
            if (int s = launch_carry(ctx, sh, w, false)) return s;
        }
        w.kept = kept_s;
        w.rows = rows_e;
        if (int s = launch_delta_walk<S>(ctx, w, KEEP, p.seg.slots, "gated delta rule: states")) return s;
    }
    w.init = b.grad_final;
    w.fin = b.grad_state;
    w.go = b.go;
    w.gv = b.gv;
    w.kept = kept_d;
    w.rows = rows_w;
    if (p.maps && sh.tokens > 0) {
        if (int s = launch_delta_back<S>(ctx, w, BACK_MAPS, p.seg.slots, "gated delta rule: segments' adjoints")) return s;
        if (int s = launch_carry(ctx, sh, w, true)) return s;
    }
    if (int s = launch_delta_back<S>(ctx, w, BACK, p.seg.slots, "gated delta rule: adjoints")) return s;
    if (sh.tokens == 0) return GOOM_OK;
    w.kept_s = kept_s;
    w.kept_d = kept_d;
    w.rows_e = rows_e;
    w.rows_w = rows_w;
    w.gq = sum_q ? (void *)sum_q : b.gq;
    w.gk = sum_k ? (void *)sum_k : b.gk;
    w.grad_float = sum_q != nullptr;
    w.g_log_decay = b.g_log_decay;
    w.g_beta = b.g_beta;
    return launch_delta_gradients<S>(ctx, w, p.chunk.slots);
}

} // namespace goom_layer

using namespace goom_layer;
using goom::aligned;
using goom::fail;

extern "C" {

size_t goom_gated_delta_workspace_bytes(const goom_delta_shape *shape, int packed)
{
    goom_delta_shape sh;
    if (check_shape(nullptr, shape, sh, packed != 0, false) || sh.seqs == 0) return 0;
    return plan_of(sh, packed != 0, false).bytes;
}

int goom_gated_delta(goom_ctx *ctx, const goom_delta_shape *shape, const void *q, const void *k, const void *v, const float *log_decay, const float *beta,
                     const int64_t *offsets, const float *state, void *o, float *final_state, void *workspace, size_t workspace_bytes)
{
    goom_delta_shape sh;
    if (int s = check_shape(ctx, shape, sh, offsets != nullptr, false)) return s;
    if (sh.seqs == 0) return ctx ? GOOM_OK : fail(nullptr, GOOM_EINVAL, "null context");
    const size_t size = real_bytes(sh.type);
    if (sh.tokens > 0 && (!q || !k || !v || !log_decay || !beta || !o)) return fail(ctx, GOOM_EINVAL, "null data pointer");
    for (const void *p : {q, k, v, (const void *)o})
        if (!aligned(p, size)) return fail(ctx, GOOM_EINVAL, "misaligned data pointer");
    for (const float *p : {log_decay, beta, state, (const float *)final_state})
        if (!aligned(p, 4)) return fail(ctx, GOOM_EINVAL, "misaligned data pointer");
    if (!aligned(offsets, 8)) return fail(ctx, GOOM_EINVAL, "misaligned data pointer");
    const DeltaPlan p = plan_of(sh, offsets != nullptr, false);
    if (int s = check_workspace(ctx, workspace, workspace_bytes, p.bytes)) return s;
    if (int s = enter(ctx)) return s;
    DeltaArgs w = delta_args(sh, p, offsets, q, k, v, log_decay, beta);
    unsigned char *ws = reinterpret_cast<unsigned char *>(workspace);
    w.m = reinterpret_cast<float *>(ws);
    w.vecs = ws + p.m;
    w.totals = p.maps ? reinterpret_cast<float *>(ws + p.m + p.vecs) : nullptr;
    w.maps = reinterpret_cast<float *>(ws + p.m + p.vecs + p.totals);
    w.order = p.order ? reinterpret_cast<int *>(ws + p.m + p.vecs + p.totals + p.map) : nullptr;
    w.init = state;
    w.fin = final_state;
    w.o = o;
    return with_type(sh.type, [&](auto tag) { return run_forward<typename decltype(tag)::type>(ctx, sh, p, w); });
}

int goom_gated_delta_step(goom_ctx *ctx, const goom_delta_shape *shape, const void *q, const void *k, const void *v, const float *log_decay, const float *beta,
                          const float *state, void *o, float *next_state)
{
    goom_delta_shape sh;
    if (int s = check_shape(ctx, shape, sh, false, true)) return s;
    if (sh.seqs == 0) return ctx ? GOOM_OK : fail(nullptr, GOOM_EINVAL, "null context");
    const size_t size = real_bytes(sh.type);
    if (!q || !k || !v || !log_decay || !beta || !o || !next_state) return fail(ctx, GOOM_EINVAL, "null data pointer");
    for (const void *p : {q, k, v, (const void *)o})
        if (!aligned(p, size)) return fail(ctx, GOOM_EINVAL, "misaligned data pointer");
    for (const float *p : {log_decay, beta, state, (const float *)next_state})
        if (!aligned(p, 4)) return fail(ctx, GOOM_EINVAL, "misaligned data pointer");
    if (int s = enter(ctx)) return s;
    const dim3 grid((unsigned)(sh.seqs * sh.heads), (sh.dv + 31) / 32);
    goom::prof_begin(ctx, "gated delta rule: one token");
    const int rc = with_type(sh.type, [&](auto tag) {
        typedef typename decltype(tag)::type S;
        delta_step_kernel<S><<<grid, 256, 0, ctx->stream>>>(sh, reinterpret_cast<const S *>(q), reinterpret_cast<const S *>(k), reinterpret_cast<const S *>(v), log_decay, beta,
                                                            state, reinterpret_cast<S *>(o), next_state);
        return goom::check_hip(ctx, hipGetLastError(), "gated delta rule: one token");
    });
    goom::prof_end(ctx);
    return rc;
}

size_t goom_gated_delta_backward_workspace_bytes(const goom_delta_shape *shape, int packed)
{
    goom_delta_shape sh;
    if (check_shape(nullptr, shape, sh, packed != 0, false) || sh.seqs == 0) return 0;
    return plan_of(sh, packed != 0, true).bytes;
}

int goom_gated_delta_backward(goom_ctx *ctx, const goom_delta_shape *shape, const void *q, const void *k, const void *v, const float *log_decay, const float *beta,
                              const int64_t *offsets, const float *state, const void *grad_o, const float *grad_final, void *grad_q, void *grad_k, void *grad_v,
                              float *grad_log_decay, float *grad_beta, float *grad_state, void *workspace, size_t workspace_bytes)
{
    goom_delta_shape sh;
    if (int s = check_shape(ctx, shape, sh, offsets != nullptr, false)) return s;
    if (sh.seqs == 0) return ctx ? GOOM_OK : fail(nullptr, GOOM_EINVAL, "null context");
    const size_t size = real_bytes(sh.type);
    if (sh.tokens > 0 && (!q || !k || !v || !log_decay || !beta || !grad_o || !grad_q || !grad_k || !grad_v || !grad_log_decay || !grad_beta))
        return fail(ctx, GOOM_EINVAL, "null data pointer");
    for (const void *p : {q, k, v, grad_o, (const void *)grad_q, (const void *)grad_k, (const void *)grad_v})
        if (!aligned(p, size)) return fail(ctx, GOOM_EINVAL, "misaligned data pointer");
    for (const float *p : {log_decay, beta, state, grad_final, (const float *)grad_log_decay, (const float *)grad_beta, (const float *)grad_state})
        if (!aligned(p, 4)) return fail(ctx, GOOM_EINVAL, "misaligned data pointer");
    if (!aligned(offsets, 8)) return fail(ctx, GOOM_EINVAL, "misaligned data pointer");
    const DeltaPlan p = plan_of(sh, offsets != nullptr, true);
    if (int s = check_workspace(ctx, workspace, workspace_bytes, p.bytes)) return s;
    if (int s = enter(ctx)) return s;
    DeltaArgs w = delta_args(sh, p, offsets, q, k, v, log_decay, beta);
    unsigned char *ws = reinterpret_cast<unsigned char *>(workspace);
    auto take = [&](size_t bytes) {
        unsigned char *const at = bytes ? ws : nullptr;
        ws += bytes;
        return reinterpret_cast<float *>(at);
    };
    w.m = take(p.m);
    w.vecs = take(p.vecs);
    w.totals = take(p.totals);
    w.maps = take(p.map);
    w.order = reinterpret_cast<int *>(take(p.order));
    float *const kept_s = take(p.state), *const kept_d = take(p.state), *const rows_e = take(p.rows), *const rows_w = take(p.rows);
    float *const sum_q = take(p.sum), *const sum_k = take(p.sum);
    w.back = 1;
    const BackPointers b = {grad_o, state, grad_final, grad_state, grad_q, grad_k, grad_v, grad_log_decay, grad_beta};
    if (int s = with_type(sh.type, [&](auto tag) { return run_backward<typename decltype(tag)::type>(ctx, sh, p, w, b, kept_s, kept_d, rows_e, rows_w, sum_q, sum_k); })) return s;
    if (p.sum && sh.tokens > 0)
        return launch_shared_sums(ctx, sh.type, sum_q, grad_q, sh.dk, sum_k, grad_k, sh.dk, sh.tokens, sh.qk_heads, sh.heads / sh.qk_heads, offsets, sh.seqs,
                                  "gated delta rule: shared heads");
    return GOOM_OK;
}

} // extern "C"
