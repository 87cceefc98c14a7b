// Linear attention with a decay for each head: single tokens, and the C ABI.  The walks over many tokens are in
// goom_linear_attention_walk.h.
#include <cmath>

#include "goom_linear_attention_walk.h"

namespace goom_layer {

// sums over heads that share keys and values: y[token][kv head][.] = sum over the group of x[token][head][.], floats.  Two such
// arrays in one launch, blockIdx.y apart.  Tokens before the first sequence and after the last one have no sums, and none are written.
struct SharedSum { const float *x; void *y; long long n; int d; }; // n: units of V entries
template <typename S, int V>
__global__ __launch_bounds__(256) void shared_sum_kernel(SharedSum k, SharedSum v, int group, int kv_heads, const int64_t *offsets, long long seqs, long long tokens)
{
    const SharedSum &t = blockIdx.y ? v : k;
    const int units = t.d / V;
    long long begin = 0, end = t.n;
    if (offsets) {
        auto cut = [&](long long at) { return at < 0 ? 0 : at > tokens ? tokens : at; };
        const long long first = cut(offsets[0]), start = cut(offsets[seqs - 1]), last = cut(offsets[seqs]);
        begin = first * kv_heads * units;
        end = (last > start ? last : start) * kv_heads * units; // (the last sequence has no tokens if its end is before its start)
    }
    for (long long u = begin + blockIdx.x * 256ll + threadIdx.x; u < end; u += gridDim.x * 256ll) {
        const long long row = t.n < (1ll << 31) ? (unsigned)u / (unsigned)units : u / units;
        const float *const p = t.x + row * group * t.d + (u - row * units) * V;
        float sum[V] = {};
        for (int h = 0; h < group; h++) {
            float x[V];
            load_floats<float, V>(p + (long long)h * t.d, x);
#pragma unroll
            for (int e = 0; e < V; e++) sum[e] += x[e];
        }
        store_floats<S, V>(reinterpret_cast<S *>(t.y) + u * V, sum);
    }
}

// ---- single tokens: S <- g S + k v^T, o = scale q^T S.  One pass over the state, bound by its bytes.  A workgroup has 32
// columns of a head's state (eight groups of four) and its threads every 32nd row; their sums meet in LDS in a fixed order.
// 256 sequences of 16 heads of 128 x 128: 109 us, 5.0 TB/s.
template <typename S> __global__ __launch_bounds__(256) void step_kernel(goom_attention_shape sh, const S *q, const S *k, const S *v, const float *log_decay,
                                                                                  const float *state, S *o, float *next)
{
    const int h = blockIdx.x % sh.heads, col = blockIdx.y * 32 + (threadIdx.x & 7) * 4, row0 = threadIdx.x >> 3;
    const long long s = blockIdx.x / sh.heads;
    const int kv = h / (sh.heads / sh.kv_heads);
    const float decay = decay_power(log2_decay(log_decay[h]), 1);
    const S *const qh = q + s * sh.q_token + h * sh.q_head, *const kh = k + s * sh.k_token + kv * sh.k_head, *const vh = v + s * sh.v_token + kv * sh.v_head;
    const long long base = (s * sh.heads + h) * (long long)sh.dk * sh.dv;
    float x[4], y[4] = {0, 0, 0, 0};
    constexpr int ROWS = GOOM_MAX_DIM / 32;
    float st[ROWS][4], kr[ROWS], qr[ROWS];
#pragma unroll
    for (int e = 0; e < 4; e++) x[e] = col + e < sh.dv ? (float)vh[col + e] : 0.0f;
#pragma unroll
    for (int u = 0; u < ROWS; u++) {
        const int row = row0 + u * 32;
        kr[u] = qr[u] = 0.0f;
#pragma unroll
        for (int e = 0; e < 4; e++) st[u][e] = 0.0f;
        if (row < sh.dk) {
            kr[u] = (float)kh[row];
            qr[u] = (float)qh[row];
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
        }
    }
#pragma unroll
    for (int u = 0; u < ROWS; u++) {
        const int row = row0 + u * 32;
        if (row < sh.dk) {
#pragma unroll
            for (int e = 0; e < 4; e++) {
                st[u][e] = decay * st[u][e] + kr[u] * x[e];
                y[e] += qr[u] * st[u][e];
            }
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
    __shared__ float part[4][32];
#pragma unroll
    for (int e = 0; e < 4; e++) { // the wave's eight rows, then the four waves
        y[e] += __shfl_xor(y[e], 8);
        y[e] += __shfl_xor(y[e], 16);
        y[e] += __shfl_xor(y[e], 32);
        if ((threadIdx.x & 63) < 8) part[threadIdx.x >> 6][(threadIdx.x & 7) * 4 + e] = y[e];
    }
    __syncthreads();
    const int c = blockIdx.y * 32 + threadIdx.x;
    if (threadIdx.x < 32 && c < sh.dv)
        o[(s * sh.heads + h) * (long long)sh.dv + c] =
            (S)((float)sh.scale * ((part[0][threadIdx.x] + part[1][threadIdx.x]) + (part[2][threadIdx.x] + part[3][threadIdx.x])));
}

// ---- host side

static int padded_head(int d) { return d <= 32 ? 32 : d <= 64 ? 64 : 128; } // as with_walk() pads

static int launch_walks(goom_ctx *ctx, int type, const WalkArgs &w, int roles, long long slots, const char *label)
{
    return with_type(type, [&](auto tag) { return launch_walks_of<typename decltype(tag)::type>(ctx, w, roles, slots, label); });
}

// Segments: how long, and how many slots there are in all.
struct Segments { long long len, slots, per_seq; };

static Segments choose_segments(const goom_attention_shape &sh, int roles, bool packed)
{
    // As many walks as the chip holds at once: more would start a second round, fewer leave CUs idle
    const long long resident = with_type(sh.type, [&](auto tag) {
        typedef typename decltype(tag)::type S;
        return with_walk<S>(sh.dk, sh.dv, [](auto rows, auto cols, auto waves) { return WalkLds<S, decltype(rows)::value, decltype(cols)::value, decltype(waves)::value, true>::resident; });
    });
    // (sequences of different lengths: two rounds of shorter ones, which even out.  Two, three, four and six rounds: 7 sequences of 9000
    // tokens in all, 8 heads of 128, bfloat16, both directions 237, 272, 282 and 280 us; 20 of 30,000, 16 heads of 64 437, 396, 412 and 435;
    // 37 of 30,011, 12 float heads of 50 and 72, forward 278, 279, 273 and 275.  Places are counted for (dk, dv) also where walks of different
    // sizes go together, padded to the larger.)
    const long long walks = sh.seqs * sh.heads * roles, round = 256 * resident * (packed ? 2 : 1), mean = sh.seqs > 0 ? (sh.tokens + sh.seqs - 1) / sh.seqs : 0;
    long long want = walks > 0 ? round / walks : 1; // segments a sequence of mean length
    // Not below two chunks each (one, where lengths differ): measured at 8 x 1000 float tokens of 8 heads of 32 and 64, forward and
    // backward, 141, 132 and 132 us with four, two and one chunks; at 5 ragged sequences of 1500 tokens in all, 86, 73 and 70 us
    const long long least = packed ? CHUNK : 2 * CHUNK, most = (mean + least - 1) / least;
    if (want > most) want = most;
    if (want < 1) want = 1;
    long long len = (mean + want - 1) / want;
    len = (len + CHUNK - 1) / CHUNK * CHUNK;
    if (len < CHUNK) len = CHUNK;
    Segments g;
    if (packed) {
        if (want == 1) len = (sh.tokens / CHUNK + 1) * CHUNK; // no sequence is longer
        g = {len, want == 1 ? sh.seqs : sh.tokens / len + sh.seqs, want == 1 ? 1 : 0};
    } else {
        g = {len, 0, mean > 0 ? (mean + len - 1) / len : 1};
        g.slots = sh.seqs * g.per_seq;
    }
    return g;
}

// floats of the segments' states for walks over (ka, nc)
static size_t totals_bytes(const goom_attention_shape &sh, const Segments &g, int ka, int nc)
{
    if (g.per_seq == 1) return 0;
    return goom::align_up((size_t)(g.slots * sh.heads) * padded_head(ka) * padded_head(nc) * 4, 256);
}

static WalkArgs walk_args(const goom_attention_shape &sh, const float *log_decay, const int64_t *offsets, const Segments &g)
{
    WalkArgs w = {};
    w.log_decay = log_decay;
    w.offsets = offsets;
    w.tokens = sh.tokens;
    w.seqs = sh.seqs;
    w.seq_len = sh.seqs > 0 ? sh.tokens / sh.seqs : 0;
    w.seg_len = g.len;
    w.segs = g.per_seq;
    w.heads = sh.heads;
    return w;
}

struct Rows { const void *p; long long tok, head; int group, d; }; // one of q, k, v, grad_o

static WalkRole role(const Rows &a, const Rows &b, const Rows &c, void *y, int y_float, int heads, int reverse)
{
    WalkRole r = {};
    r.a = a.p; r.a_tok = a.tok; r.a_head = a.head; r.a_group = a.group;
    r.b = b.p; r.b_tok = b.tok; r.b_head = b.head; r.b_group = b.group;
    r.c = c.p; r.c_tok = c.tok; r.c_head = c.head; r.c_group = c.group;
    r.ka = a.d;
    r.nc = c.d;
    r.y = y;
    r.y_float = y_float;
    r.y_head = c.d;
    r.y_tok = (long long)heads * c.d;
    r.reverse = reverse;
    r.p_scale = r.w_scale = r.u_scale = 1.0f;
    r.state_row = c.d;
    r.state_col = 1;
    return r;
}

// fills in the strides that 0 stands for; GOOM_OK or an error
static int check_shape(goom_ctx *ctx, const goom_attention_shape *given, goom_attention_shape &sh, bool packed, bool need_equal)
{
    if (!given) return goom::fail(ctx, GOOM_EINVAL, "null shape");
    sh = *given;
    if (!real_type(sh.type)) return goom::fail(ctx, GOOM_EINVAL, "unknown element type %d", sh.type);
    if (sh.flags) return goom::fail(ctx, GOOM_EINVAL, "unknown flags 0x%x", (unsigned)sh.flags);
    if (sh.seqs < 0 || sh.tokens < 0) return goom::fail(ctx, GOOM_EINVAL, "negative number of sequences or tokens");
    if (sh.heads <= 0 || sh.kv_heads <= 0 || sh.heads % sh.kv_heads) return goom::fail(ctx, GOOM_EINVAL, "kv_heads must be positive and divide heads");
    if (sh.dk <= 0 || sh.dv <= 0) return goom::fail(ctx, GOOM_EINVAL, "dk and dv must be positive");
    if (sh.dk > GOOM_MAX_DIM || sh.dv > GOOM_MAX_DIM) return goom::fail(ctx, GOOM_EUNSUPPORTED, "dk and dv go up to %d", GOOM_MAX_DIM);
    if (!std::isfinite((float)sh.scale)) return goom::fail(ctx, GOOM_EINVAL, "scale must be finite, and a float");
    if (sh.seqs == 0 && sh.tokens > 0) return goom::fail(ctx, GOOM_EINVAL, "tokens without a sequence");
    if (!packed && sh.seqs > 0 && sh.tokens % sh.seqs) return goom::fail(ctx, GOOM_EINVAL, "without offsets the sequences have tokens / seqs tokens each");
    if (need_equal && sh.seqs != sh.tokens) return goom::fail(ctx, GOOM_EINVAL, "one token a sequence");
    if (sh.seqs > (1 << 24) / sh.heads || sh.tokens > (1ll << 40) || sh.tokens / CHUNK > (1 << 24) / sh.heads) return goom::fail(ctx, GOOM_EUNSUPPORTED, "too many sequences, heads or tokens");
    if (need_equal && sh.seqs * sh.heads > 0xffffffffll / 256) return goom::fail(ctx, GOOM_EUNSUPPORTED, "too many sequences or heads"); // threads of a grid's first axis
    const int64_t rows[3][3] = {{sh.q_token, sh.q_head, sh.dk}, {sh.k_token, sh.k_head, sh.dk}, {sh.v_token, sh.v_head, sh.dv}};
    for (auto &x : rows)
        if (x[0] < 0 || x[1] < 0 || ((x[0] || x[1]) && (x[0] < x[2] || x[1] < x[2])) || x[0] > (1ll << 40) || x[1] > (1ll << 40))
            return goom::fail(ctx, GOOM_EINVAL, "strides of tokens and heads must be 0 (both: contiguous) or at least a head's entries");
    if (!sh.q_token) { sh.q_token = (int64_t)sh.heads * sh.dk; sh.q_head = sh.dk; }
    if (!sh.k_token) { sh.k_token = (int64_t)sh.kv_heads * sh.dk; sh.k_head = sh.dk; }
    if (!sh.v_token) { sh.v_token = (int64_t)sh.kv_heads * sh.dv; sh.v_head = sh.dv; }
    if (!need_equal && (sh.q_token > (1 << 22) || sh.k_token > (1 << 22) || sh.v_token > (1 << 22) || (int64_t)sh.heads * sh.dv > (1 << 22))) // 32-bit offsets within a chunk
        return goom::fail(ctx, GOOM_EUNSUPPORTED, "more than 2^22 elements from token to token");
    return GOOM_OK;
}

int enter(goom_ctx *ctx)
{
    if (!ctx) return goom::fail(nullptr, GOOM_EINVAL, "null context");
    if (!ctx->prof_keep) goom::prof_reset(ctx);
    return goom::check_hip(ctx, hipSetDevice(ctx->device), "hipSetDevice");
}

int check_workspace(goom_ctx *ctx, const void *ws, size_t given, size_t need)
{
    if (!need) return GOOM_OK;
    if (!ws || given < need) return goom::fail(ctx, GOOM_EWORKSPACE, "workspace of %zu bytes needed, %zu given", need, ws ? given : (size_t)0);
    if (!goom::aligned(ws, 256)) return goom::fail(ctx, GOOM_EINVAL, "workspace must be 256-byte aligned");
    return GOOM_OK;
}

// bytes of the backward pass's workspace by parts: states of the three walks, floats of shared heads' gradients
struct BackwardPlan {
    Segments seg;
    bool together; // the three walks in one launch
    size_t totals_q, totals_k, totals_v, sum_k, sum_v, bytes;
};

static BackwardPlan backward_plan(const goom_attention_shape &sh, bool packed)
{
    BackwardPlan p;
    p.seg = choose_segments(sh, 3, packed);
    // Walks of different sizes go together, padded to the larger, where they are, before they are cut into segments, no more than the
    // chip has CUs: a small pass is bound by its launches.  (Both directions, together and apart: one sequence of 6000 tokens, 32 bfloat16 heads
    // of 110 and 25, 401 and 459 us, of 128 and 64, 330 and 377; two of 600 142 and 161.  Floats pay six products for the padding: 8295 tokens, 4 heads of
    // 110 and 25, packed from 7 sequences 243 and 202 us, from 15 236 and 189, 15 equal ones 219 and 235; of 50 and 100, 15 packed, 234 and
    // 208; of 64 and 30, 15 equal, 101 and 126.  So only up to 64.)
    const int most = sh.dk > sh.dv ? sh.dk : sh.dv, least = sh.dk > sh.dv ? sh.dv : sh.dk;
    p.together = padded_head(least) == padded_head(most) || (sh.seqs * sh.heads * 3 <= 256 && (sh.type != GOOM_REAL_F32 || padded_head(most) <= 64));
    const int dk = p.together ? most : sh.dk, dv = p.together ? most : sh.dv;
    p.totals_q = totals_bytes(sh, p.seg, dv, dk);
    p.totals_k = totals_bytes(sh, p.seg, dv, dk);
    p.totals_v = totals_bytes(sh, p.seg, dk, dv);
    const bool shared = sh.heads != sh.kv_heads;
    p.sum_k = shared ? goom::align_up((size_t)sh.tokens * sh.heads * sh.dk * 4, 256) : 0;
    p.sum_v = shared ? goom::align_up((size_t)sh.tokens * sh.heads * sh.dv * 4, 256) : 0;
    p.bytes = p.totals_q + p.totals_k + p.totals_v + p.sum_k + p.sum_v;
    return p;
}

} // namespace goom_layer

using namespace goom_layer;
using goom::aligned;
using goom::fail;

extern "C" {

size_t goom_linear_attention_workspace_bytes(const goom_attention_shape *shape, int packed)
{
    goom_attention_shape sh;
    if (check_shape(nullptr, shape, sh, packed != 0, false)) return 0;
    return totals_bytes(sh, choose_segments(sh, 1, packed != 0), sh.dk, sh.dv);
}

int goom_linear_attention(goom_ctx *ctx, const goom_attention_shape *shape, const void *q, const void *k, const void *v, const float *log_decay,
                          const int64_t *offsets, const float *state, void *o, float *final_state, void *workspace, size_t workspace_bytes)
{
    goom_attention_shape sh;
    if (int s = check_shape(ctx, shape, sh, offsets != nullptr, false)) return s;
    if (sh.seqs == 0) return ctx ? GOOM_OK : fail(nullptr, GOOM_EINVAL, "null context");
    const size_t size = real_bytes(sh.type);
    if (!log_decay || (sh.tokens > 0 && (!q || !k || !v || !o))) return fail(ctx, GOOM_EINVAL, "null data pointer");
    if (!aligned(q, size) || !aligned(k, size) || !aligned(v, size) || !aligned(o, size) || !aligned(log_decay, 4) || !aligned(state, 4) || !aligned(final_state, 4) ||
        !aligned(offsets, 8))
        return fail(ctx, GOOM_EINVAL, "misaligned data pointer");
    const Segments g = choose_segments(sh, 1, offsets != nullptr);
    const size_t need = totals_bytes(sh, g, sh.dk, sh.dv);
    if (int s = check_workspace(ctx, workspace, workspace_bytes, need)) return s;
    if (int s = enter(ctx)) return s;
    WalkArgs w = walk_args(sh, log_decay, offsets, g);
    const int group = sh.heads / sh.kv_heads;
    const Rows rq = {q, sh.q_token, sh.q_head, 1, sh.dk}, rk = {k, sh.k_token, sh.k_head, group, sh.dk}, rv = {v, sh.v_token, sh.v_head, group, sh.dv};
    WalkRole &r = w.role[0];
    r = role(rq, rk, rv, o, 0, sh.heads, 0);
    r.p_scale = r.w_scale = (float)sh.scale;
    r.init = state;
    r.fin = final_state;
    r.totals = need ? reinterpret_cast<float *>(workspace) : nullptr;
    return launch_walks(ctx, sh.type, w, 1, g.slots, "linear attention");
}

int goom_linear_attention_step(goom_ctx *ctx, const goom_attention_shape *shape, const void *q, const void *k, const void *v, const float *log_decay, const float *state,
                               void *o, float *next_state)
{
    goom_attention_shape sh;
    if (int s = check_shape(ctx, shape, sh, false, true)) return s;
    if (sh.seqs == 0) return ctx ? GOOM_OK : fail(nullptr, GOOM_EINVAL, "null context");
    const size_t size = real_bytes(sh.type);
    if (!q || !k || !v || !log_decay || !o || !next_state) return fail(ctx, GOOM_EINVAL, "null data pointer");
    if (!aligned(q, size) || !aligned(k, size) || !aligned(v, size) || !aligned(o, size) || !aligned(log_decay, 4) || !aligned(state, 4) || !aligned(next_state, 4))
        return fail(ctx, GOOM_EINVAL, "misaligned data pointer");
    if (int s = enter(ctx)) return s;
    const dim3 grid((unsigned)(sh.seqs * sh.heads), (sh.dv + 31) / 32);
    goom::prof_begin(ctx, "linear attention: one token");
    const int rc = with_type(sh.type, [&](auto tag) {
        typedef typename decltype(tag)::type S;
        step_kernel<S><<<grid, 256, 0, ctx->stream>>>(sh, reinterpret_cast<const S *>(q), reinterpret_cast<const S *>(k), reinterpret_cast<const S *>(v), log_decay, state,
                                              reinterpret_cast<S *>(o), next_state);
        return goom::check_hip(ctx, hipGetLastError(), "linear attention step");
    });
    goom::prof_end(ctx);
    return rc;
}

size_t goom_linear_attention_backward_workspace_bytes(const goom_attention_shape *shape, int packed)
{
    goom_attention_shape sh;
    if (check_shape(nullptr, shape, sh, packed != 0, false)) return 0;
    return backward_plan(sh, packed != 0).bytes;
}

int goom_linear_attention_backward(goom_ctx *ctx, const goom_attention_shape *shape, const void *q, const void *k, const void *v, const float *log_decay,
                                   const int64_t *offsets, const float *state, const void *grad_o, const float *grad_final, void *grad_q, void *grad_k, void *grad_v,
                                   float *grad_state, void *workspace, size_t workspace_bytes)
{
    goom_attention_shape sh;
    if (int s = check_shape(ctx, shape, sh, offsets != nullptr, false)) return s;
    if (sh.seqs == 0) return ctx ? GOOM_OK : fail(nullptr, GOOM_EINVAL, "null context");
    const size_t size = real_bytes(sh.type);
    if (!log_decay || (sh.tokens > 0 && (!q || !k || !v || !grad_o || !grad_q || !grad_k || !grad_v))) return fail(ctx, GOOM_EINVAL, "null data pointer");
    const void *const typed[] = {q, k, v, grad_o, grad_q, grad_k, grad_v}, *const floats[] = {log_decay, state, grad_final, grad_state};
    for (const void *p : typed)
        if (!aligned(p, size)) return fail(ctx, GOOM_EINVAL, "misaligned data pointer");
    for (const void *p : floats)
        if (!aligned(p, 4)) return fail(ctx, GOOM_EINVAL, "misaligned data pointer");
    if (!aligned(offsets, 8)) return fail(ctx, GOOM_EINVAL, "misaligned data pointer");
    const BackwardPlan plan = backward_plan(sh, offsets != nullptr);
    if (int s = check_workspace(ctx, workspace, workspace_bytes, plan.bytes)) return s;
    if (int s = enter(ctx)) return s;

    unsigned char *ws = reinterpret_cast<unsigned char *>(workspace);
    auto take = [&](size_t bytes) {
        void *p = bytes ? ws : nullptr;
        ws += bytes;
        return reinterpret_cast<float *>(p);
    };
    float *const totals_q = take(plan.totals_q), *const totals_k = take(plan.totals_k), *const totals_v = take(plan.totals_v);
    float *const sum_k = take(plan.sum_k), *const sum_v = take(plan.sum_v);
    const int group = sh.heads / sh.kv_heads, shared = group > 1;
    const Rows rq = {q, sh.q_token, sh.q_head, 1, sh.dk}, rk = {k, sh.k_token, sh.k_head, group, sh.dk}, rv = {v, sh.v_token, sh.v_head, group, sh.dv},
               rg = {grad_o, (long long)sh.heads * sh.dv, sh.dv, 1, sh.dv};
    const float scale = (float)sh.scale;
    WalkRole gq = role(rg, rv, rk, grad_q, 0, sh.heads, 0);
    gq.p_scale = gq.w_scale = scale;
    gq.init = state;
    gq.state_row = 1;
    gq.state_col = sh.dv;
    gq.totals = totals_q;
    WalkRole gk = role(rv, rg, rq, shared ? (void *)sum_k : grad_k, shared, sh.heads, 1);
    gk.p_scale = gk.u_scale = scale;
    gk.init = grad_final;
    gk.state_row = 1;
    gk.state_col = sh.dv;
    gk.totals = totals_k;
    WalkRole gv = role(rk, rq, rg, shared ? (void *)sum_v : grad_v, shared, sh.heads, 1);
    gv.p_scale = gv.u_scale = scale;
    gv.init = grad_final;
    gv.fin = grad_state;
    gv.totals = totals_v;

    WalkArgs w = walk_args(sh, log_decay, offsets, plan.seg);
    w.role[0] = gq;
    w.role[1] = gk;
    w.role[2] = gv;
    if (plan.together) {
        if (int s = launch_walks(ctx, sh.type, w, 3, plan.seg.slots, "linear attention: gradients")) return s;
    } else {
        if (int s = launch_walks(ctx, sh.type, w, 2, plan.seg.slots, "linear attention: gradients of q and k")) return s;
        w.role[0] = gv;
        if (int s = launch_walks(ctx, sh.type, w, 1, plan.seg.slots, "linear attention: gradient of v")) return s;
    }
    if (shared && sh.tokens > 0) {
        const long long rows = sh.tokens * sh.kv_heads;
        return with_type(sh.type, [&](auto tag) {
            typedef typename decltype(tag)::type S;
            const bool vec = sh.dk % 4 == 0 && sh.dv % 4 == 0 && aligned(grad_k, 4 * size) && aligned(grad_v, 4 * size);
            const int V = vec ? 4 : 1;
            const long long most = rows * (sh.dk > sh.dv ? sh.dk : sh.dv) / V, blocks = (most + 255) / 256;
            const SharedSum ks = {sum_k, grad_k, rows * sh.dk / V, sh.dk}, vs = {sum_v, grad_v, rows * sh.dv / V, sh.dv};
            auto *kernel = vec ? shared_sum_kernel<S, 4> : shared_sum_kernel<S, 1>;
            goom::prof_begin(ctx, "linear attention: shared heads");
            kernel<<<dim3((unsigned)(blocks < 16384 ? blocks : 16384), 2), 256, 0, ctx->stream>>>(ks, vs, group, sh.kv_heads, offsets, sh.seqs, sh.tokens);
            goom::prof_end(ctx);
            return goom::check_hip(ctx, hipGetLastError(), "linear attention: shared heads");
        });
    }
    return GOOM_OK;
}

} // extern "C"
