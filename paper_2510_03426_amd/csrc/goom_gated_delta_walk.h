#pragma once

// The gated delta rule, many tokens at once: forward and backward.
//
//     S_t = a_t (S_{t-1} - beta_t k_t (k_t^T S_{t-1})) + beta_t k_t v_t^T,    o_t = scale S_t^T q_t,    a_t = exp(log_decay_t)
//
// A chunk's tokens i, with b_i = log a_1 + .. + log a_i from the chunk's start, G_ij = e^(b_i - b_j) (k_i . k_j) below the diagonal,
// P_ij = scale e^(b_i - b_j) (q_i . k_j) on and below it, S the state before the chunk and S' the one after it:
//     Y = V - e^b K S,   E = (I + G beta)^-1 Y = Y - M (beta Y),   U = beta E,   O = scale e^b Q S + P U,   S' = e^(b_C) S + (e^(b_C - b) K)^T U
// with M = (I + G beta)^-1 G, strictly lower triangular.  The state's adjoint D' goes the other way:
//     dU = P^T dO + e^(b_C - b) K D',   W = dU - M^T (beta dU),   dV = beta W,   D = e^(b_C) D' + scale (e^b Q)^T dO - (e^b K)^T dV
// and with both states and U, W at hand every chunk's other gradients are its own:
//     dQ = scale e^b dO S^T + dP K,   dK = e^(b_C - b) U D'^T - e^b dV S^T + dP^T Q - (dG + dG^T) K,   dP = scale e^(b_i - b_j) dO_i . U_j,
//     dG = e^(b_i - b_j) dV_i . U_j,   dbeta = W . E,   dlog_a_t = sum over s >= t in the chunk of (q_s . dq_s - v_s . dv_s) + <D', S'>.
// Nothing is divided by a decay or by beta, so both may be zero.
//
// Kernels: what lies within chunks (M, P, sums of logarithms), all chunks at once; the walk along each sequence, whose waves own
// columns of the state in registers; the gradients, all chunks at once.  Where there are fewer walks than the chip holds, sequences
// are cut into segments: a segment is an affine map of the state, S -> A S + B, whose A and B are one walk from (I, 0) without
// outputs; the maps are chained, then all segments walked at once.  Operands and their parts are those of the linear attention.
#include "goom_linear_attention_walk.h"

namespace goom_layer {

struct Cut { const int64_t *offsets; long long tokens, seqs, seq_len, seg_len, segs; }; // sequences in pieces of seg_len tokens

// tokens of a chunk
template <typename S> constexpr int chunk_of() { return Parts<S>::IN > 1 ? 32 : 64; }
constexpr int pair_blocks(int ch) { return ch == 64 ? 6 : 2; }
constexpr int pair_frags(int ch) { return pair_blocks(ch) * COMPUTED * 64; }
// M of a chunk, floats in memory: rows of 32 entries, behind the first 32 rows of 64; eight of them a unit
constexpr int m_floats(int ch) { return ch == 64 ? 32 * 32 + 32 * 64 : 32 * 32; }
constexpr int m_units(int ch) { return m_floats(ch) / 8; }
// in LDS in parts, planes of rows of pitches of their own
constexpr int M_LOW = 32 + PITCH_PAD, M_HIGH = 64 + PITCH_PAD;
constexpr int m_plane(int ch) { return 32 * M_LOW + (ch == 64 ? 32 * M_HIGH : 0); }

// of a chunk and head: powers and betas, zeros past the end of the sequence
template <int CH> struct ChunkVec {
    double b2[CH];                        // sums of log2 of the decays
    float up[CH], down[CH], beta[CH];     // e^b, e^(b_C - b)
    float whole, pad[15];                 // e^(b_C)
};

struct DeltaArgs {
    Cut chunk, seg;
    const void *q, *k, *v, *go;
    long long q_tok, q_head, k_tok, k_head, v_tok, v_head, o_tok; // elements
    const float *log_decay, *beta;
    float *m;                // M, [chunk slots][heads][m_floats]
    void *vecs;              // ChunkVec [chunk slots][heads]
    const float *init;       // NULL or [seqs][heads][dk][dv]: the state before the first token, or (backwards) its adjoint after the last
    float *fin;              // NULL or the same: the last state, or the first one's adjoint
    void *o;
    float *totals;           // NULL: one segment a sequence; [slots][heads][parts][state registers]: B, then the incoming states
    float *maps;             // A, [slots][heads][DK][DK]
    float *kept, *rows;      // KEEP: states before, BACK: adjoints after each chunk [chunk slots][heads][DK][pitch]; E or W [chunk slots][heads][CH][pitch]
    void *gv;
    // gradients
    const float *kept_s, *kept_d, *rows_e, *rows_w;
    void *gq, *gk;           // [tokens][heads][dk], floats where heads share q and k
    float *g_log_decay, *g_beta;
    int heads, share, dk, dv, pitch;
    int parts, map_parts;    // workgroups' column parts of the state, and of A
    unsigned slots;
    int back, grad_float;    // back: of a backward pass
    float scale;
    int *order;              // NULL, or the sequences in the order in which their walks start
};

// log2 of a decay; below 2^-160, which is zero as a float whatever it is divided by, finite (a NaN stays one)
__device__ inline double log2_of(float log_decay)
{
    const double x = (double)log_decay * 1.4426950408889634;
    return x < -160.0 ? -160.0 : x;
}
// 2^x, to a unit of the last place: only a fraction is rounded, for the hardware's exponential, and the whole part scales.  (With x rounded to a float
// the power is off by |x| of its units: e^-20 by eleven.)  Beyond 2000 either way the fraction is what is left: infinity, zero, or a NaN's.
__device__ inline float power2(double x)
{
    const float whole = rintf(__builtin_amdgcn_fmed3f((float)x, -2000.0f, 2000.0f));
    return ldexpf(__builtin_amdgcn_exp2f((float)(x - (double)whole)), (int)whole);
}
// The same with the exponent rounded, for the weights of pairs in G and P and their gradients, 2^x with x <= 0 unless states grow: |x| 2^x stays below 0.54, so
// a weight is off by less than half a unit of the largest, a token's own, that the same sums have.  With power2 throughout, us: 8 x 4096 tokens of 16 heads of 128,
// both directions, 1827 for 1801; 65,536 of 16 heads of 64 597 for 587.
__device__ inline float weight2(double x) { return __builtin_amdgcn_exp2f((float)x); }

__device__ inline int wave_of() { return __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6); } // (in a scalar register)
// a value the compiler knows nothing about: what is computed from it stays where it is, and out of registers everywhere else
__device__ inline int opaque(int x)
{
    asm volatile("" : "+v"(x));
    return x;
}

// rows of a tile of 16 in the order in which a lane's accumulator entries of two tiles are eight consecutive ones
__device__ inline int turned_row(int t, int i) { return t / 2 * 32 + (i >> 2) * 8 + t % 2 * 4 + (i & 3); }

// ---- what lies within a chunk

template <typename S, int DK> struct WithinLds {
    static constexpr int CH = chunk_of<S>(), PK = DK + PITCH_PAD, TILE = CH * PK * Parts<S>::IN, PM = CH + 4;
    static constexpr size_t tile = TILE * sizeof(bf16), square = CH * PM * sizeof(float); // first the rows of k, then the matrix
    static constexpr size_t bytes = (tile > square ? tile : square) + CH * (sizeof(double) + sizeof(float));
    static constexpr int fit = (int)((160 << 10) / bytes), resident = fit > 5 ? 5 : fit;
};

// M21 = (I - M22 beta2) G21 (I - beta1 M11) for the pairs of diagonal blocks of SIZE, by tiles of 16 x 16, a wave each; what comes of the
// first product waits at the pair's place above the diagonal
template <int SIZE, int CH> __device__ inline void join_blocks(float *m, const float *beta)
{
    constexpr int PM = CH + 4, TILES = (SIZE / 16) * (SIZE / 16), ALL = CH / (2 * SIZE) * TILES;
    const int lane = threadIdx.x & 63, wave = wave_of(), i = lane & 15, g = lane >> 4;
    const bool mine = wave < ALL;
    const int r0 = wave / TILES * 2 * SIZE, tr = wave % TILES / (SIZE / 16) * 16, tc = wave % TILES % (SIZE / 16) * 16;
    float *const below = m + (r0 + SIZE) * PM + r0, *const above = m + r0 * PM + r0 + SIZE;
    const float *const m11 = m + r0 * PM + r0, *const m22 = m + (r0 + SIZE) * PM + r0 + SIZE, *const b1 = beta + r0, *const b2 = b1 + SIZE;
    if (mine) { // G21 - (G21 beta1) M11
        f32x4 c = {0, 0, 0, 0};
#pragma unroll
        for (int k = g; k < SIZE; k += 4) c = __builtin_amdgcn_mfma_f32_16x16x4f32(below[(tr + i) * PM + k] * b1[k], m11[k * PM + tc + i], c, 0, 0, 0);
#pragma unroll
        for (int e = 0; e < 4; e++) above[(tr + g * 4 + e) * PM + tc + i] = below[(tr + g * 4 + e) * PM + tc + i] - c[e];
    }
    if (TILES > 1) {
        __syncthreads();
    } else { // one tile, of the wave's own: its lanes read what others of them wrote, in that order
        __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
        __builtin_amdgcn_wave_barrier();
        __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
    }
    if (mine) { // and that less M22 (beta2 that)
        f32x4 c = {0, 0, 0, 0};
#pragma unroll
        for (int k = g; k < SIZE; k += 4) c = __builtin_amdgcn_mfma_f32_16x16x4f32(m22[(tr + i) * PM + k] * b2[k], above[k * PM + tc + i], c, 0, 0, 0);
#pragma unroll
        for (int e = 0; e < 4; e++) below[(tr + g * 4 + e) * PM + tc + i] = above[(tr + g * 4 + e) * PM + tc + i] - c[e];
    }
    __syncthreads();
    if (SIZE == 16) { // rows of 32 are written whole, and read whole by the next join: what waited above the diagonal is zero again
        if (mine)
#pragma unroll
            for (int e = 0; e < 4; e++) above[(g * 4 + e) * PM + i] = 0.0f;
        __syncthreads();
    }
}

// The sequences, longest first: walks take as long as their sequences, and a long one that starts last is waited for.  One workgroup, by counting
// chunks (1023 and more are one number); among equals the order is any, which changes nothing but when a walk starts.
__device__ inline void order_sequences(const DeltaArgs &w, unsigned *count)
{
    constexpr int MOST = 1024;
    __shared__ unsigned wave_sum[4];
    auto place = [&](long long s) {
        long long start, len;
        span(w.seg, s, start, len);
        const long long chunks = (len + w.chunk.seg_len - 1) / w.chunk.seg_len;
        return MOST - 1 - (int)(chunks < MOST - 1 ? chunks : MOST - 1);
    };
    for (int x = threadIdx.x; x < MOST; x += 256) count[x] = 0;
    __syncthreads();
    for (long long s = threadIdx.x; s < w.seg.seqs; s += 256) atomicAdd(&count[place(s)], 1u);
    __syncthreads();
    unsigned own[4], sum = 0; // four neighbouring counts, then sums of all before
#pragma unroll
    for (int x = 0; x < 4; x++) {
        own[x] = sum;
        sum += count[threadIdx.x * 4 + x];
    }
    unsigned before = sum;
    for (int x = 1; x < 64; x *= 2) {
        const unsigned y = __shfl_up(before, x);
        if ((int)(threadIdx.x & 63) >= x) before += y;
    }
    if ((threadIdx.x & 63) == 63) wave_sum[threadIdx.x >> 6] = before;
    __syncthreads();
    before -= sum;
    for (int x = 0; x < (int)(threadIdx.x >> 6); x++) before += wave_sum[x];
#pragma unroll
    for (int x = 0; x < 4; x++) count[threadIdx.x * 4 + x] = before + own[x];
    __syncthreads();
    for (long long s = threadIdx.x; s < w.seg.seqs; s += 256) w.order[atomicAdd(&count[place(s)], 1u)] = (int)s;
}

// Bound by its waits (barriers, and the rows of a block of 16 one after another), of five workgroups a CU (two: 96 us): 8 x 4096 tokens of 16
// heads of 128, bfloat16: 68 us for 245 MB, 3.6 TB/s.  M goes to memory in floats, once: with M and P in parts, as operands, it was 150 us.
template <typename S, int DK> __global__ __launch_bounds__(256, (WithinLds<S, DK>::resident)) void within_kernel(DeltaArgs w)
{
    typedef WithinLds<S, DK> Lds;
    constexpr int CH = Lds::CH, PK = Lds::PK, PM = Lds::PM, IP = Parts<S>::IN, KP = CH * PK;
    extern __shared__ __align__(16) unsigned char lds[];
    bf16 *const k_lds = reinterpret_cast<bf16 *>(lds);
    float *const m = reinterpret_cast<float *>(lds);
    double *const b2 = reinterpret_cast<double *>(lds + (Lds::tile > Lds::square ? Lds::tile : Lds::square));
    float *const beta = reinterpret_cast<float *>(b2 + CH);
    const int qk_heads = w.heads / w.share;
    const long long block = block_of();
    const int kh = block % qk_heads;
    const long long slot = block / qk_heads;
    if (slot >= w.slots) { // the last workgroup's
        if (w.order && block == (long long)w.slots * qk_heads) order_sequences(w, reinterpret_cast<unsigned *>(lds));
        return;
    }
    const Place at = find_place(w.chunk, slot);
    if (at.seg < 0 || at.seg >= at.nseg || at.len == 0) return;
    const long long t0 = at.seg * CH, tok = at.start + t0;
    const int n = at.len - t0 < CH ? (int)(at.len - t0) : CH;
    const int lane = threadIdx.x & 63, wave = wave_of(), i = lane & 15, g = lane >> 4;
    float ld = 0.0f, be = 0.0f; // of wave 0: the head's, a head ahead
    auto fetch = [&](int h) {
        if (wave == 0 && lane < n) {
            const long long from = (tok + lane) * w.heads + h;
            ld = w.log_decay[from];
            be = w.beta[from];
        }
    };
    fetch(kh * w.share);
    {
        TileRows<S, DK, 256, CH> kx;
        kx.fetch(reinterpret_cast<const S *>(w.k) + tok * w.k_tok + kh * w.k_head, w.k_tok, n, w.dk);
        kx.template put_any<PK>(k_lds, n, w.dk);
    }
    __syncthreads();

    // k_i . k_j, by tiles on and below the diagonal
    constexpr int SIDE = CH / 16, TILES = SIDE * (SIDE + 1) / 2, TURNS = (TILES + 3) / 4;
    f32x4 square[TURNS];
    auto tile_of = [&](int u, int &r, int &c) {
        c = wave + u * 4;
        r = 0;
        while (c > r) c -= ++r;
    };
#pragma unroll
    for (int u = 0; u < TURNS; u++) {
        square[u] = f32x4{0, 0, 0, 0};
        if (wave + u * 4 >= TILES) continue;
        int r, c;
        tile_of(u, r, c);
#pragma unroll
        for (int x = 0; x < DK / 32; x++) {
            Frag a[IP], b[IP];
            row_frag(a, k_lds + (r * 16 + i) * PK + x * 32 + g * 8, KP);
            row_frag(b, k_lds + (c * 16 + i) * PK + x * 32 + g * 8, KP);
            square[u] = product(a, b, square[u]);
        }
    }

    for (int s = 0; s < w.share; s++) {
        const int h = kh * w.share + s;
        const long long record = slot * w.heads + h;
        if (wave == 0) {
            double sum = lane < n ? log2_of(ld) : 0.0;
#pragma unroll
            for (int step = 1; step < CH; step *= 2) {
                const double x = __shfl_up(sum, step);
                if (lane >= step) sum += x;
            }
            const double end = __shfl(sum, CH - 1);
            if (lane < CH) {
                const float mine = lane < n ? be : 0.0f;
                ChunkVec<CH> &vec = reinterpret_cast<ChunkVec<CH> *>(w.vecs)[record];
                b2[lane] = sum;
                beta[lane] = mine;
                vec.b2[lane] = sum;
                vec.beta[lane] = mine;
                vec.up[lane] = lane < n ? power2(sum) : 0.0f;
                vec.down[lane] = lane < n ? power2(end - sum) : 0.0f;
                if (lane == 0) vec.whole = power2(end);
            }
            if (s + 1 < w.share) fetch(h + 1);
        }
        __syncthreads(); // (and the rows of k, or the last head's M, are read)
#pragma unroll
        for (int u = 0; u < TURNS; u++) {
            if (wave + u * 4 >= TILES) continue;
            int r, c;
            tile_of(u, r, c);
            const int col = c * 16 + i;
#pragma unroll
            for (int e = 0; e < 4; e++) {
                const int row = r * 16 + g * 4 + e;
                m[row * PM + col] = col < row ? square[u][e] * weight2(b2[row] - b2[col]) : 0.0f;
            }
        }
        __syncthreads();
        // rows of M one after another, in blocks of 16: M_i = G_i - sum_j G_ij beta_j M_j; a lane has a column of one block
        if (wave == 0 && lane < CH) {
            float x[16];
            float *const d = m + g * 16 * PM + g * 16;
            const float *const of = beta + g * 16;
#pragma unroll
            for (int r = 0; r < 16; r++) {
                float y = d[r * PM + i];
#pragma unroll
                for (int c = 0; c < r; c++) y -= d[r * PM + c] * (of[c] * x[c]);
                x[r] = y;
            }
#pragma unroll
            for (int r = 0; r < 16; r++) d[r * PM + i] = x[r]; // (after all reads: the lanes of a wave go together)
        }
        __syncthreads();
        join_blocks<16, CH>(m, beta);
        if constexpr (CH == 64) join_blocks<32, CH>(m, beta);
        float *const to = w.m + record * m_floats(CH);
        for (int u = threadIdx.x; u < m_units(CH); u += 256) {
            const int row = u < 128 ? u / 4 : 32 + (u - 128) / 8, col = (u < 128 ? u % 4 : u % 8) * 8;
            const f32x4 *const from = reinterpret_cast<const f32x4 *>(m + row * PM + col);
            reinterpret_cast<f32x4 *>(to + u * 8)[0] = from[0];
            reinterpret_cast<f32x4 *>(to + u * 8)[1] = from[1];
        }
    }
}

// ---- the walks

enum DeltaMode {
    FORWARD,      // outputs
    MAPS,         // segments' A and B
    KEEP,         // states before the chunks, and E
    BACK_MAPS,    // the adjoint's B
    BACK          // adjoints after the chunks, W, the gradient of v
};

// Waves that load for the others: they fetch the next chunk's rows and M, form P of this chunk, and put what was fetched into LDS, while
// the walking waves do nothing but multiply.  (With every wave at both, one chunk after another, a chunk of 64 tokens and heads of 128 took
// 17,500 cycles, half of them waits.)
constexpr int LOADERS = 4;

template <typename S, int DK, int DV, int MODE> struct DeltaLds {
    static constexpr int CH = chunk_of<S>(), PK = DK + PITCH_PAD, PV = DV + PITCH_PAD, NW = DV / 16, WAVES = NW + LOADERS;
    static constexpr bool REV = MODE == BACK_MAPS || MODE == BACK, OUT = MODE == FORWARD, P = OUT || REV;
    static constexpr int K_TILE = CH * PK * Parts<S>::IN, V_TILE = CH * PV * Parts<S>::IN, M_TILE = m_plane(CH) * COMPUTED; // elements
    // Two buffers in turn for what is read until a chunk's end; one for what is read before the barrier in the middle of it, behind which the
    // next chunk's comes (forwards Q, V and M)
    static constexpr int Q_BUFFERS = OUT ? 1 : REV ? 2 : 0, OTHERS = OUT ? 1 : 2;
    static constexpr int FRAGS = P ? pair_frags(CH) : 0, VEC = 3 * CH + 4; // up, down, beta, whole
    static constexpr size_t bytes = FRAGS * sizeof(Frag) + (K_TILE * (2 + Q_BUFFERS) + (V_TILE + M_TILE) * OTHERS) * sizeof(bf16) + (P ? CH * sizeof(double) : 0) + 2 * VEC * sizeof(float);
    static constexpr int fit = (int)((160 << 10) / bytes), resident = fit > 2 ? 2 : fit;
    static constexpr int per_simd = (resident * WAVES + 3) / 4;
};

struct WalkPlace { long long start, len, seg0, seg1, chunk0; int h, kh, col_part, nc, nchunks; bool map, last; long long state0; };

// the loading waves
template <typename S, int DK, int DV, int MODE> __device__ inline void delta_load(const DeltaArgs &w, const WalkPlace at, unsigned char *lds)
{
    typedef DeltaLds<S, DK, DV, MODE> Lds;
    constexpr int THREADS = LOADERS * 64, KS = DK / 32, IP = Parts<S>::IN, CH = Lds::CH, KP = CH * Lds::PK;
    constexpr bool REV = Lds::REV, EARLY = Lds::OUT && IP > 1;
    Frag *const p_lds = reinterpret_cast<Frag *>(lds);
    bf16 *const k_lds = reinterpret_cast<bf16 *>(p_lds + Lds::FRAGS), *const q_lds = k_lds + 2 * Lds::K_TILE, *const v_lds = q_lds + Lds::Q_BUFFERS * Lds::K_TILE,
               *const m_lds = v_lds + Lds::OTHERS * Lds::V_TILE;
    double *const b2_lds = reinterpret_cast<double *>(m_lds + Lds::OTHERS * Lds::M_TILE);
    float *const vec_lds = reinterpret_cast<float *>(b2_lds + (Lds::P ? CH : 0));
    const int lane = threadIdx.x & 63, wave = wave_of(), i = lane & 15, g = lane >> 4;

    const S *const k = reinterpret_cast<const S *>(w.k) + at.start * w.k_tok + at.kh * w.k_head;
    const S *const q = reinterpret_cast<const S *>(w.q) + at.start * w.q_tok + at.kh * w.q_head;
    const S *const v = REV ? reinterpret_cast<const S *>(w.go) + at.start * w.o_tok + at.h * (long long)w.dv + at.col_part
                           : reinterpret_cast<const S *>(w.v) + at.start * w.v_tok + at.h * w.v_head + at.col_part;
    const long long v_tok = REV ? w.o_tok : w.v_tok;
    TileRows<S, DK, THREADS, CH> kx, qx;
    TileRows<S, DV, THREADS, CH> vx;
    constexpr int UNITS = m_units(CH), MU = (UNITS + THREADS - 1) / THREADS;
    f32x8 mx[MU];
    double b2 = 0;
    float vec[3], whole = 0;
    auto chunk_at = [&](int step) { return REV ? at.nchunks - 1 - step : step; };
    auto rows_at = [&](int c) {
        const long long t0 = at.seg0 + (long long)c * CH;
        return at.seg1 - t0 < CH ? (int)(at.seg1 - t0) : CH;
    };
    auto fetch = [&](int step) {
        const int c = chunk_at(step), n = rows_at(c);
        const long long t0 = at.seg0 + (long long)c * CH, record = (at.chunk0 + c) * w.heads + at.h;
        kx.fetch(k + t0 * w.k_tok, w.k_tok, n, w.dk);
        if (!at.map) vx.fetch(v + t0 * v_tok, v_tok, n, at.nc);
        const float *const from = w.m + record * m_floats(CH);
#pragma unroll
        for (int u = 0; u < MU; u++) {
            const int x = u * THREADS + threadIdx.x < UNITS ? u * THREADS + threadIdx.x : UNITS - 1;
            mx[u] = *reinterpret_cast<const f32x8 *>(from + x * 8);
        }
        const ChunkVec<CH> &cv = reinterpret_cast<const ChunkVec<CH> *>(w.vecs)[record];
        const int x = threadIdx.x & (CH - 1);
        if (Lds::P) b2 = cv.b2[x];
        vec[0] = cv.up[x];
        vec[1] = cv.down[x];
        vec[2] = cv.beta[x];
        whole = cv.whole;
        if (Lds::Q_BUFFERS) qx.fetch(q + t0 * w.q_tok, w.q_tok, n, w.dk);
    };
    // Rows of two or three parts cost the loading waves most: those of k, which have two buffers, are put beside P, which two of the four
    // waves form (30,011 packed tokens of 12 heads of 50 x 72, floats: 361 -> 345 us; in bfloat16, whose P takes all four, 362 -> 373 us)
    auto put_k = [&](int step) { kx.template put_any<Lds::PK>(k_lds + (step & 1) * Lds::K_TILE, rows_at(chunk_at(step)), w.dk); };
    auto put = [&](int step) {
        const int n = rows_at(chunk_at(step)), two = step & 1, other = Lds::OTHERS == 2 ? two : 0;
        if (!EARLY) put_k(step);
        if (!at.map) vx.template put_any<Lds::PV>(v_lds + other * Lds::V_TILE, n, at.nc);
#pragma unroll
        for (int u = 0; u < MU; u++) {
            const int x = u * THREADS + threadIdx.x;
            if (UNITS % THREADS && x >= UNITS) continue;
            Frag parts[COMPUTED];
            split(mx[u], parts);
            bf16 *const to = m_lds + other * Lds::M_TILE + (x < 128 ? x / 4 * M_LOW + x % 4 * 8 : 32 * M_LOW + (x - 128) / 8 * M_HIGH + x % 8 * 8);
#pragma unroll
            for (int p = 0; p < COMPUTED; p++) *reinterpret_cast<Frag *>(to + p * m_plane(CH)) = parts[p];
        }
        if (threadIdx.x < CH) {
            float *const to = vec_lds + two * Lds::VEC;
#pragma unroll
            for (int x = 0; x < 3; x++) to[x * CH + threadIdx.x] = vec[x];
            if (threadIdx.x == 0) to[3 * CH] = whole;
            if (Lds::P) b2_lds[threadIdx.x] = b2;
        }
        if (Lds::Q_BUFFERS) qx.template put_any<Lds::PK>(q_lds + (Lds::Q_BUFFERS == 2 ? two : 0) * Lds::K_TILE, n, w.dk);
    };
    fetch(0);
    if (EARLY) put_k(0);
    put(0);
    if (Lds::P && at.nchunks > 1) fetch(1);
    __syncthreads();
    for (int step = 0; step < at.nchunks; step++) {
        if (Lds::P) {
            // P: a lane has eight consecutive j of row i, or (backwards) eight consecutive i of row j
            const bf16 *const kt = k_lds + (step & 1) * Lds::K_TILE, *const qt = q_lds + (Lds::Q_BUFFERS == 2 ? step & 1 : 0) * Lds::K_TILE;
            for (int block = wave; block < pair_blocks(CH); block += LOADERS) {
                int t, ks;
                p_place<REV>(block, CH, t, ks);
                const int row = REV ? turned_row(t, i) : t * 16 + i, col = ks * 32 + g * 8;
                const bf16 *const one = (REV ? kt : qt) + row * Lds::PK + g * 8, *const other = (REV ? qt : kt) + turned_row(2 * ks, i) * Lds::PK + g * 8;
                f32x4 p0 = {0, 0, 0, 0}, p1 = {0, 0, 0, 0};
#pragma unroll
                for (int kk = 0; kk < KS; kk++) {
                    Frag a[IP], b0[IP], b1[IP];
                    row_frag(a, one + kk * 32, KP);
                    row_frag(b0, other + kk * 32, KP);
                    row_frag(b1, other + 4 * Lds::PK + kk * 32, KP);
                    p0 = product(b0, a, p0);
                    p1 = product(b1, a, p1);
                }
                f32x8 p8 = __builtin_shufflevector(p0, p1, 0, 1, 2, 3, 4, 5, 6, 7);
                const double mine = b2_lds[row];
#pragma unroll
                for (int e = 0; e < 8; e++) {
                    const double age = REV ? b2_lds[col + e] - mine : mine - b2_lds[col + e];
                    p8[e] = (REV ? row <= col + e : col + e <= row) ? w.scale * p8[e] * weight2(age) : 0.0f;
                }
                Frag parts[COMPUTED];
                split(p8, parts);
#pragma unroll
                for (int p = 0; p < COMPUTED; p++) p_lds[(block * COMPUTED + p) * 64 + lane] = parts[p];
            }
            if (EARLY && step + 1 < at.nchunks) put_k(step + 1);
            __syncthreads();
        }
        // With P to form, a chunk's rows have been on their way since the chunk before; without, they are fetched and put within one (measured: the other
        // way round the walks that keep states take 15 % longer, the adjoints' 16 %)
        if (!Lds::P && step + 1 < at.nchunks) fetch(step + 1);
        if (step + 1 < at.nchunks) put(step + 1);
        if (Lds::P && step + 2 < at.nchunks) fetch(step + 2);
        __syncthreads();
    }
}

// the walking waves: each has 16 of the DV columns of the state
template <typename S, int DK, int DV, int MODE> __device__ inline void delta_walk(const DeltaArgs &w, const WalkPlace at, float *total, unsigned char *lds)
{
    typedef DeltaLds<S, DK, DV, MODE> Lds;
    constexpr int KS = DK / 32, TT = Lds::CH / 16, IP = Parts<S>::IN, CH = Lds::CH, KP = CH * Lds::PK, VP = CH * Lds::PV, HALVES = CH / 32;
    constexpr bool REV = Lds::REV, OUT = Lds::OUT, TOTAL = MODE == MAPS || MODE == BACK_MAPS;
    const Frag *const p_lds = reinterpret_cast<const Frag *>(lds);
    const bf16 *const k_lds = reinterpret_cast<const bf16 *>(p_lds + Lds::FRAGS), *const q_lds = k_lds + 2 * Lds::K_TILE, *const v_lds = q_lds + Lds::Q_BUFFERS * Lds::K_TILE,
                     *const m_lds = v_lds + Lds::OTHERS * Lds::V_TILE;
    const float *const vec_lds = reinterpret_cast<const float *>(reinterpret_cast<const double *>(m_lds + Lds::OTHERS * Lds::M_TILE) + (Lds::P ? CH : 0));
    const int lane = threadIdx.x & 63, wave = wave_of() - LOADERS, i = lane & 15, g = lane >> 4, col0 = wave * 16, col = col0 + i;
    auto row_of = [&](int t, int e) { return t / 2 * 32 + g * 8 + t % 2 * 4 + e; };
    const bool here = col < at.nc;
    const unsigned own = (unsigned)(g * 8 * w.pitch + col); // the lane's place in what is kept of a chunk

    // ---- the incoming state
    f32x4 R[DK / 16];
    if (total) total += (long long)wave * (DK / 16) * 256 + lane * 4;
#pragma unroll
    for (int t = 0; t < DK / 16; t++) {
        f32x4 x = {0, 0, 0, 0};
        if (TOTAL) {
            if (at.map)
#pragma unroll
                for (int e = 0; e < 4; e++) x[e] = row_of(t, e) == at.col_part + col && here ? 1.0f : 0.0f;
        } else if (total && at.len) {
            x = *reinterpret_cast<const f32x4 *>(total + t * 256);
        } else if (w.init) {
#pragma unroll
            for (int e = 0; e < 4; e++)
                if (row_of(t, e) < w.dk && here) x[e] = w.init[at.state0 + (long long)row_of(t, e) * w.dv + col];
        }
        R[t] = x;
    }
    if (at.nchunks > 0) __syncthreads();
    for (int step = 0; step < at.nchunks; step++) {
        const int c = REV ? at.nchunks - 1 - step : step, two = step & 1, other = Lds::OTHERS == 2 ? two : 0;
        const long long t0 = at.seg0 + (long long)c * CH, record = (at.chunk0 + c) * w.heads + at.h;
        const int n = at.seg1 - t0 < CH ? (int)(at.seg1 - t0) : CH;
        const bf16 *const kt = k_lds + two * Lds::K_TILE, *const qt = q_lds + (Lds::Q_BUFFERS == 2 ? two : 0) * Lds::K_TILE, *const vt = v_lds + other * Lds::V_TILE,
                         *const mt = m_lds + other * Lds::M_TILE;
        const float *const vec = vec_lds + two * Lds::VEC;
        auto eight = [&](int which, int half) { return *reinterpret_cast<const f32x8 *>(vec + which * CH + half * 32 + g * 8); };

        if (MODE == KEEP || MODE == BACK) {
            float *const to = w.kept + record * (DK * (long long)w.pitch) + at.col_part;
#pragma unroll
            for (int t = 0; t < DK / 16; t++)
#pragma unroll
                for (int e = 0; e < 4; e++) (to + (t / 2 * 32 + t % 2 * 4 + e) * w.pitch)[own] = R[t][e];
        }

        // ---- K against the state, a lane with eight consecutive tokens of a column; Q with consecutive columns of a token
        f32x4 x[TT], y[OUT ? TT : 1];
#pragma unroll
        for (int t = 0; t < TT; t++) {
            x[t] = f32x4{0, 0, 0, 0};
            if (OUT) y[t] = f32x4{0, 0, 0, 0};
        }
#pragma unroll
        for (int kk = 0; kk < KS; kk++) {
            Frag rf[COMPUTED];
            split(__builtin_shufflevector(R[2 * kk], R[2 * kk + 1], 0, 1, 2, 3, 4, 5, 6, 7), rf);
#pragma unroll
            for (int t = 0; t < TT; t++) {
                Frag kf[IP];
                row_frag(kf, kt + turned_row(t, i) * Lds::PK + kk * 32 + g * 8, KP);
                x[t] = product(kf, rf, x[t]);
                if (OUT) {
                    Frag qf[IP];
                    row_frag(qf, qt + (t * 16 + i) * Lds::PK + kk * 32 + g * 8, KP);
                    y[t] = product(rf, qf, y[t]);
                }
            }
        }
        auto get = [&](int half) { return f32x8(__builtin_shufflevector(x[2 * half], x[2 * half + 1], 0, 1, 2, 3, 4, 5, 6, 7)); };
        auto set = [&](int half, const f32x8 &y8) {
            x[2 * half] = __builtin_shufflevector(y8, y8, 0, 1, 2, 3);
            x[2 * half + 1] = __builtin_shufflevector(y8, y8, 4, 5, 6, 7);
        };
        if (REV) __syncthreads(); // P is there
        // ---- Y (or dU), and with M the rows E (or W)
        f32x8 go8[REV ? HALVES : 1];
#pragma unroll
        for (int half = 0; half < HALVES; half++) {
            if (REV) {
                set(half, eight(1, half) * get(half));
            } else {
                f32x8 in = {0, 0, 0, 0, 0, 0, 0, 0};
                if (!at.map) {
                    Frag vf[IP];
                    col_frag<Lds::PV>(vf, vt, VP, half * 32, col0, 4, lane);
                    in = widen(vf);
                }
                set(half, in - eight(0, half) * get(half));
            }
        }
        if (REV) {
#pragma unroll
            for (int half = 0; half < HALVES; half++) {
                Frag gf[IP];
                col_frag<Lds::PV>(gf, vt, VP, half * 32, col0, 4, lane);
                go8[half] = widen(gf);
#pragma unroll
                for (int t = 0; t < TT; t++) {
                    if (!p_has<true>(t, half)) continue;
                    Frag pf[COMPUTED];
#pragma unroll
                    for (int u = 0; u < COMPUTED; u++) pf[u] = p_lds[(p_block<true>(t, half, CH) * COMPUTED + u) * 64 + lane];
                    x[t] = product(pf, gf, x[t]);
                }
            }
        }
        {
            Frag bf[HALVES][COMPUTED];
#pragma unroll
            for (int half = 0; half < HALVES; half++) split(-(eight(2, half) * get(half)), bf[half]);
#pragma unroll
            for (int half = 0; half < HALVES; half++)
#pragma unroll
                for (int t = 0; t < TT; t++) {
                    if (!p_has<REV>(t, half)) continue;
                    Frag mf[COMPUTED];
                    if (REV && half == 0) col_frag<M_LOW>(mf, mt, m_plane(CH), 0, t % 2 * 4, 8, lane);
                    else if (REV) col_frag<M_HIGH>(mf, mt + 32 * M_LOW, m_plane(CH), 0, t / 2 * 32 + t % 2 * 4, 8, lane);
                    else if (t < 2) row_frag(mf, mt + turned_row(t, i) * M_LOW + g * 8, m_plane(CH));
                    else row_frag(mf, mt + 32 * M_LOW + (turned_row(t, i) - 32) * M_HIGH + half * 32 + g * 8, m_plane(CH));
                    x[t] = product(mf, bf[half], x[t]);
                }
        }
        if (OUT) __syncthreads(); // P is there, and Q, V and M are read
        if (MODE == KEEP || MODE == BACK) {
            float *const to = w.rows + record * (CH * (long long)w.pitch) + at.col_part;
#pragma unroll
            for (int half = 0; half < HALVES; half++)
#pragma unroll
                for (int e = 0; e < 8; e++) (to + (half * 32 + e) * w.pitch)[own] = get(half)[e];
        }
        // ---- U (or dV)
#pragma unroll
        for (int half = 0; half < HALVES; half++) set(half, get(half) * eight(2, half));
        if (MODE == BACK && here) {
            S *const to = reinterpret_cast<S *>(w.gv) + (at.start + t0) * w.o_tok + at.h * (long long)w.dv + at.col_part + col;
#pragma unroll
            for (int half = 0; half < HALVES; half++)
#pragma unroll
                for (int e = 0; e < 8; e++) {
                    const int row = half * 32 + g * 8 + e;
                    if (row < n) to[row * w.o_tok] = (S)get(half)[e];
                }
        }
        if (OUT) {
            Frag uf[HALVES][COMPUTED];
#pragma unroll
            for (int half = 0; half < HALVES; half++) split(get(half), uf[half]);
#pragma unroll
            for (int t = 0; t < TT; t++) {
                y[t] *= w.scale * vec[t * 16 + i];
#pragma unroll
                for (int half = 0; half < HALVES; half++) {
                    if (!p_has<false>(t, half)) continue;
                    Frag pf[COMPUTED];
#pragma unroll
                    for (int u = 0; u < COMPUTED; u++) pf[u] = p_lds[(p_block<false>(t, half, CH) * COMPUTED + u) * 64 + lane];
                    y[t] = product(uf[half], pf, y[t]);
                }
            }
#pragma unroll
            for (int t = 0; t < TT; t++) {
                const int row = t * 16 + i, first = col0 + g * 4;
                if (row < n) {
                    S *const to = reinterpret_cast<S *>(w.o) + (at.start + t0 + row) * w.o_tok + at.h * (long long)w.dv + at.col_part + first;
                    float out[4] = {y[t][0], y[t][1], y[t][2], y[t][3]};
                    if (first + 4 <= at.nc) store_floats_unaligned<S, 4>(to, out);
                    else
#pragma unroll
                        for (int e = 0; e < 4; e++)
                            if (first + e < at.nc) to[e] = (S)out[e];
                }
            }
        }
        // ---- the next state, unless nobody needs it
        if (TOTAL || step + 1 < at.nchunks || (at.last && w.fin)) {
            const float decay = vec[3 * CH];
#pragma unroll
            for (int t = 0; t < DK / 16; t++) R[t] *= decay;
#pragma unroll
            for (int half = 0; half < HALVES; half++) {
                Frag uf[COMPUTED], gf[COMPUTED];
                if (REV) {
                    split(-(eight(0, half) * get(half)), uf);
                    split(w.scale * (eight(0, half) * go8[half]), gf);
                } else {
                    split(eight(1, half) * get(half), uf);
                }
#pragma unroll
                for (int t = 0; t < DK / 16; t++) {
                    Frag kf[IP];
                    col_frag<Lds::PK>(kf, kt, KP, half * 32, t / 2 * 32 + t % 2 * 4, 8, lane);
                    R[t] = product(kf, uf, R[t]);
                    if (REV) {
                        Frag qf[IP];
                        col_frag<Lds::PK>(qf, qt, KP, half * 32, t / 2 * 32 + t % 2 * 4, 8, lane);
                        R[t] = product(qf, gf, R[t]);
                    }
                }
            }
        }
        __syncthreads();
    }

#pragma unroll
    for (int t = 0; t < DK / 16; t++) {
        if (TOTAL && at.map) {
#pragma unroll
            for (int e = 0; e < 4; e++)
                if (at.col_part + col < DK) w.maps[(long long)(row_of(t, e)) * DK + at.col_part + col + at.state0] = R[t][e];
        } else if (TOTAL) {
            *reinterpret_cast<f32x4 *>(total + t * 256) = R[t];
        } else if (at.last && w.fin) {
#pragma unroll
            for (int e = 0; e < 4; e++)
                if (row_of(t, e) < w.dk && here) w.fin[at.state0 + (long long)row_of(t, e) * w.dv + col] = R[t][e];
        }
    }
}

// Bound by a chunk's chain of products, K S, M (beta Y), P U and the state's, each of which waits for the one before and for a barrier or two: the
// first four waves fetch the next chunk and form its P meanwhile, the others own 16 columns of the state each.  8 x 4096 tokens of 16 heads of
// 128, bfloat16, us: forward 356 (1.8 TB/s; with P formed by the waves that multiply 497, with two loading waves 454), the states before
// every chunk again 266, the adjoints 483.  65,536 tokens of 16 heads of 64 in 32 segments a head: maps 251, walk 259.  A kernel whose
// registers spill is 1.6 to 2.5 times as slow: scratch loads wait behind the chunk that is on its way.  (One still does: segments' adjoints of floats with
// heads of up to 32 and values of more, 7 registers at its bound of 128.)
// grid: slots heads parts, in one order; the parts of a head and segment run on one XCD (of 8, dealt round robin), whose L2 has what they share
template <typename S, int DK, int DV, int MODE>
__global__ __launch_bounds__((DeltaLds<S, DK, DV, MODE>::WAVES * 64), (DeltaLds<S, DK, DV, MODE>::per_simd)) void delta_walk_kernel(const DeltaArgs w)
{
    typedef DeltaLds<S, DK, DV, MODE> Lds;
    extern __shared__ __align__(16) unsigned char lds[];
    const int parts = w.parts + (MODE == MAPS ? w.map_parts : 0);
    const long long block = block_of(), group = block / (8 * parts);
    const int in = (int)(block % (8 * parts)), part = in / 8;
    const long long item = group * 8 + in % 8;
    if (item >= (long long)w.slots * w.heads) return;
    long long slot = item / w.heads;
    if (w.order) slot = w.order[slot];
    const Place place = find_place(w.seg, slot);
    if (place.seg < 0 || place.seg >= place.nseg) return; // a slot that no sequence has
    WalkPlace at;
    at.h = (int)(item % w.heads);
    at.kh = at.h / w.share;
    at.last = Lds::REV ? place.seg == 0 : place.seg == place.nseg - 1; // in walking order
    at.map = MODE == MAPS && part >= w.parts;                          // columns of A
    if ((MODE == MAPS || MODE == BACK_MAPS) && at.last && !(at.map && w.back)) return; // (the way back goes through the last segment's A as well)
    at.start = place.start;
    at.len = place.len;
    at.col_part = (at.map ? part - w.parts : part) * DV;
    const int columns = at.map ? w.dk : w.dv;
    at.nc = columns - at.col_part < DV ? columns - at.col_part : DV;
    at.seg0 = place.seg * w.seg.seg_len;
    at.seg1 = at.seg0 + w.seg.seg_len < at.len ? at.seg0 + w.seg.seg_len : at.len;
    at.nchunks = (int)((at.seg1 - at.seg0 + Lds::CH - 1) / Lds::CH);
    at.chunk0 = at.len ? first_slot(w.chunk, place.seq) + at.seg0 / Lds::CH : 0;
    at.state0 = at.map ? item * (DK * DK) : (place.seq * w.heads + at.h) * (long long)w.dk * w.dv + at.col_part;
    float *const total = w.totals && !at.map ? w.totals + (item * w.parts + part) * (long long)(DK * DV) : nullptr;
    if (threadIdx.x >= LOADERS * 64) delta_walk<S, DK, DV, MODE>(w, at, total, lds);
    else if (at.nchunks > 0) delta_load<S, DK, DV, MODE>(w, at, lds);
}

// Segments' maps -> incoming states, in walking order: S <- A S + B (REV: A^T D + B).  A workgroup has DV columns of one head's state, 16 a
// wave; the next A and B are on their way while these are multiplied, A in parts in LDS.  grid: seqs heads parts
template <int DK, int DV, bool REV> __global__ __launch_bounds__(DV * 4) void delta_carry_kernel(DeltaArgs w)
{
    constexpr int KS = DK / 32, THREADS = DV * 4, PA = DK + PITCH_PAD, PLANE = DK * PA, UNITS = DK * DK / 8, PER = (UNITS + THREADS - 1) / THREADS;
    extern __shared__ __align__(16) unsigned char lds[];
    bf16 *const a_lds = reinterpret_cast<bf16 *>(lds);
    const long long block = block_of();
    const int part = (int)(block % w.parts), h = (int)(block / w.parts % w.heads);
    const long long s = block / w.parts / w.heads;
    if (s >= w.seg.seqs) return;
    long long start, len;
    span(w.seg, s, start, len);
    const long long nseg = len > 0 ? (len + w.seg.seg_len - 1) / w.seg.seg_len : 0, slot0 = first_slot(w.seg, s);
    const int lane = threadIdx.x & 63, wave = wave_of(), i = lane & 15, g = lane >> 4, col = part * DV + wave * 16 + i;
    f32x4 R[DK / 16], B[DK / 16];
    f32x8 A[PER];
    auto total = [&](long long c) {
        const long long slot = slot0 + (REV ? nseg - 1 - c : c);
        return reinterpret_cast<f32x4 *>(w.totals + ((slot * w.heads + h) * w.parts + part) * (long long)(DK * DV) + (long long)wave * (DK / 16) * 256 + lane * 4);
    };
    auto fetch = [&](long long c) {
        const long long slot = slot0 + (REV ? nseg - 1 - c : c);
        const float *const from = w.maps + (slot * w.heads + h) * (long long)(DK * DK);
#pragma unroll
        for (int u = 0; u < PER; u++)
            if (UNITS % THREADS == 0 || u * THREADS + threadIdx.x < UNITS) A[u] = *reinterpret_cast<const f32x8 *>(from + (u * THREADS + threadIdx.x) * 8);
        const f32x4 *const b = total(c);
#pragma unroll
        for (int t = 0; t < DK / 16; t++) B[t] = b[t * 64];
    };
#pragma unroll
    for (int t = 0; t < DK / 16; t++) {
        f32x4 x = {0, 0, 0, 0};
        if (w.init)
#pragma unroll
            for (int e = 0; e < 4; e++) {
                const int row = t / 2 * 32 + g * 8 + t % 2 * 4 + e;
                if (row < w.dk && col < w.dv) x[e] = w.init[((s * w.heads + h) * (long long)w.dk + row) * w.dv + col];
            }
        R[t] = x;
    }
    if (nseg > 1) fetch(0);
    for (long long c = 0; c < nseg; c++) {
        f32x4 *const to = total(c);
#pragma unroll
        for (int t = 0; t < DK / 16; t++) to[t * 64] = R[t]; // (B is in registers)
        if (c + 1 == nseg) break;
        __syncthreads();
#pragma unroll
        for (int u = 0; u < PER; u++) {
            const int at = (u * THREADS + threadIdx.x) * 8, row = at / DK, x = at % DK;
            if (UNITS % THREADS && at >= UNITS * 8) continue;
            Frag parts[COMPUTED];
            split(A[u], parts);
#pragma unroll
            for (int p = 0; p < COMPUTED; p++) *reinterpret_cast<Frag *>(a_lds + p * PLANE + row * PA + x) = parts[p];
        }
        f32x4 X[DK / 16];
#pragma unroll
        for (int t = 0; t < DK / 16; t++) X[t] = B[t];
        __syncthreads();
        if (c + 2 < nseg) fetch(c + 1);
#pragma unroll
        for (int kk = 0; kk < KS; kk++) {
            Frag rf[COMPUTED];
            split(__builtin_shufflevector(R[2 * kk], R[2 * kk + 1], 0, 1, 2, 3, 4, 5, 6, 7), rf);
#pragma unroll
            for (int t = 0; t < DK / 16; t++) {
                Frag af[COMPUTED];
                if (REV) col_frag<PA>(af, a_lds, PLANE, kk * 32, t / 2 * 32 + t % 2 * 4, 8, lane);
                else row_frag(af, a_lds + turned_row(t, i) * PA + kk * 32 + g * 8, PLANE);
                X[t] = product(af, rf, X[t]);
            }
        }
#pragma unroll
        for (int t = 0; t < DK / 16; t++) R[t] = X[t];
    }
}
template <int DK> constexpr size_t carry_bytes() { return COMPUTED * DK * (DK + PITCH_PAD) * sizeof(bf16); }

// ---- the gradients of q, k, the decays and beta, a chunk and head a workgroup: four waves, each with 16 or 32 columns of q and k (of fewer than
// 64, and some of the chunk's rows), two workgroups a CU.  Bound by the bytes of what is kept of the walks: 8 x 4096 tokens of 16 heads of 128,
// bfloat16: 612 us for 2.4 GB, 3.9 TB/s, the states and adjoints 1.1 of them.  (With row addresses kept from slab to slab, 27 registers spilled and 0.2 GB
// more, 720; eight waves of a tile each 782; persistent, with waves that load, 778; two workgroups of eight waves a CU, whose registers spill, 1360.)

template <typename S, int DK, int DV> struct GradLds {
    static constexpr int CH = chunk_of<S>(), IP = Parts<S>::IN, PK = DK + PITCH_PAD, SLAB = DV, PV = SLAB + PITCH_PAD, PP = CH + PITCH_PAD;
    static constexpr int NW = 4, THREADS = NW * 64, NT = DK == 128 ? 2 : 1, TILES = DK / 16 / NT;
    static constexpr int TT = CH / 16, GROUPS = NW / TILES < TT ? NW / TILES : TT, EACH = TT / GROUPS; // waves of a tile share the chunk's rows, EACH 16
    static constexpr int K_TILE = CH * PK * IP, V_PLANE = CH * PV, PAIRS = CH * PP;
    // first the rows of U, dV (in parts) and dO, a slab at a time, then those of k and q and the pairs
    static constexpr size_t row_bytes = V_PLANE * (2 * COMPUTED + IP) * sizeof(bf16), pair_bytes = (COMPUTED * PAIRS + 2 * K_TILE) * sizeof(bf16);
    static constexpr size_t shared_bytes = row_bytes > pair_bytes ? row_bytes : pair_bytes;
    // .. and b, e^b, e^(b_C - b), v . dv, q . dq by tiles, single sums
    static constexpr size_t bytes = shared_bytes + CH * sizeof(double) + (3 * CH + TILES * CH + 2 * NW) * sizeof(float);
    static constexpr int resident = 2 * bytes <= (160 << 10) ? 2 : 1;
};

template <typename S, int DK, int DV> __global__ __launch_bounds__(256, (GradLds<S, DK, DV>::resident)) void delta_grad_kernel(const DeltaArgs w)
{
    typedef GradLds<S, DK, DV> Lds;
    constexpr int CH = Lds::CH, IP = Lds::IP, PK = Lds::PK, PV = Lds::PV, PP = Lds::PP, SLAB = Lds::SLAB, NW = Lds::NW, THREADS = Lds::THREADS, KP = CH * PK, VP = Lds::V_PLANE;
    constexpr int TT = Lds::TT, EACH = Lds::EACH, HALVES = CH / 32, BLOCKS = pair_blocks(CH), TILES = Lds::TILES, NT = Lds::NT, CS = NT == 2 ? 8 : 4;
    extern __shared__ __align__(16) unsigned char lds[];
    bf16 *const u_lds = reinterpret_cast<bf16 *>(lds), *const dv_lds = u_lds + COMPUTED * VP, *const do_lds = dv_lds + COMPUTED * VP;
    bf16 *const pairs = reinterpret_cast<bf16 *>(lds), *const k_lds = pairs + COMPUTED * Lds::PAIRS, *const q_lds = k_lds + Lds::K_TILE;
    double *const b2 = reinterpret_cast<double *>(lds + Lds::shared_bytes);
    float *const up = reinterpret_cast<float *>(b2 + CH), *const down = up + CH, *const vdv_lds = down + CH, *const qdq = vdv_lds + CH, *const sums = qdq + TILES * CH;

    const long long block = block_of(), slot = block / w.heads;
    if (slot >= w.slots) return;
    const int h = (int)(block - slot * w.heads), kh = h / w.share;
    const Place at = find_place(w.chunk, slot);
    if (at.seg < 0 || at.seg >= at.nseg || at.len == 0) return;
    const long long t0 = at.seg * CH, tok = at.start + t0, record = block;
    const int n = at.len - t0 < CH ? (int)(at.len - t0) : CH;
    const int lane = threadIdx.x & 63, wave = wave_of();
    const int tile = wave % TILES, first = wave / TILES * EACH, col0 = tile * NT * 16; // the wave's columns of q and k, col0 + (i / 4) CS + 4 nt + i % 4 of lane i of 16, and its rows: tiles of 16 from `first` on
    const bool columns = wave / TILES < Lds::GROUPS;
    const ChunkVec<CH> &vec = reinterpret_cast<const ChunkVec<CH> *>(w.vecs)[record];

    // a slab's rows: a thread has eight entries of each of PER
    typedef TileRows<S, SLAB, THREADS, CH> Rows;
    constexpr int PER = Rows::N;
    Rows gx, vx;
    f32x8 s8[NT], d8[NT];
    auto fetch_states = [&](int col) {
        if (columns)
#pragma unroll
            for (int nt = 0; nt < NT; nt++) {
                const long long from = (record * DK + col0 + 4 * nt) * (long long)w.pitch + col;
                const int l = opaque(threadIdx.x);
                const unsigned mine = ((unsigned)(((l >> 2 & 3) * CS + (l & 3)) * w.pitch + (l >> 4 & 3) * 8)) * 4; // bytes
                d8[nt] = *reinterpret_cast<const f32x8 *>(reinterpret_cast<const char *>(w.kept_d + from) + mine);
                s8[nt] = *reinterpret_cast<const f32x8 *>(reinterpret_cast<const char *>(w.kept_s + from) + mine);
            }
    };
    if (threadIdx.x < CH) {
        b2[threadIdx.x] = vec.b2[threadIdx.x];
        up[threadIdx.x] = vec.up[threadIdx.x];
        down[threadIdx.x] = vec.down[threadIdx.x];
    }

    f32x4 dq[EACH][NT], k_last[EACH][NT], k_row[EACH][NT];
#pragma unroll
    for (int t = 0; t < EACH; t++)
#pragma unroll
        for (int nt = 0; nt < NT; nt++) dq[t][nt] = k_last[t][nt] = k_row[t][nt] = f32x4{0, 0, 0, 0};
    // The pairs' sums, blocks of 16 rows by 32: dO_i . U_j for those on and below the diagonal; dV_r . U_s and U_r . dV_s for a block on it, and one of the
    // two for the block beside that
    struct Dots { f32x4 a, b; };
    const Dots zero = {{0, 0, 0, 0}, {0, 0, 0, 0}};
    Dots p_dots[2] = {zero, zero}, low = zero, high = zero, off = zero;
    const bool z_mine = wave < TT, o_mine = CH == 64;
    int p_t[2], p_ks[2];
    bool p_mine[2];
#pragma unroll
    for (int u = 0; u < 2; u++) {
        const int b = CH == 64 ? wave + 4 * u : wave - 2;
        p_mine[u] = b >= 0 && b < BLOCKS && (CH == 64 || u == 0);
        p_place<false>(p_mine[u] ? b : 0, CH, p_t[u], p_ks[u]);
    }
    float ds = 0, gbeta[PER], vdv[PER];
#pragma unroll
    for (int x = 0; x < PER; x++) gbeta[x] = vdv[x] = 0.0f;
    for (int slab = 0; slab < w.dv; slab += SLAB) {
        const int nc = w.dv - slab < SLAB ? w.dv - slab : SLAB;
        long long go_tok = w.o_tok, v_tok = w.v_tok; // formed anew for each slab, with the rows' places: kept from slab to slab they were spilled
        int rows = n;
        asm volatile("" : "+s"(go_tok), "+s"(v_tok), "+s"(rows));
        const int me = opaque(threadIdx.x), my_row = me / (SLAB / 8), my_col = me % (SLAB / 8) * 8;
        const bool mine = my_row < CH; // (of fewer rows than threads)
        gx.fetch(reinterpret_cast<const S *>(w.go) + tok * w.o_tok + h * (long long)w.dv + slab, go_tok, rows, nc);
        vx.fetch(reinterpret_cast<const S *>(w.v) + tok * w.v_tok + h * w.v_head + slab, v_tok, rows, nc);
        f32x8 e8[PER], w8[PER];
        float be[PER];
#pragma unroll
        for (int x = 0; x < PER; x++) {
            const int row = mine ? my_row + x * Rows::STEP : 0;
            const long long from = record * (CH * (long long)w.pitch) + slab;
            const unsigned here = (unsigned)(row * w.pitch + my_col) * 4; // bytes
            e8[x] = *reinterpret_cast<const f32x8 *>(reinterpret_cast<const char *>(w.rows_e + from) + here);
            w8[x] = *reinterpret_cast<const f32x8 *>(reinterpret_cast<const char *>(w.rows_w + from) + here);
            be[x] = vec.beta[row];
        }
        if (slab) __syncthreads();
        gx.template put_any<PV>(do_lds, rows, nc);
        if (mine)
#pragma unroll
            for (int x = 0; x < PER; x++) {
                bf16 *const to = u_lds + (my_row + x * Rows::STEP) * PV + my_col;
                Frag parts[COMPUTED], vf[IP];
                split(be[x] * e8[x], parts);
#pragma unroll
                for (int p = 0; p < COMPUTED; p++) *reinterpret_cast<Frag *>(to + p * VP) = parts[p];
                const f32x8 dv8 = be[x] * w8[x];
                split(dv8, parts);
#pragma unroll
                for (int p = 0; p < COMPUTED; p++) *reinterpret_cast<Frag *>(to + (COMPUTED + p) * VP) = parts[p];
                split_in(vx.unit(x, rows, nc), vf);
                const f32x8 v8 = widen(vf);
#pragma unroll
                for (int e = 0; e < 8; e++) {
                    gbeta[x] += e8[x][e] * w8[x][e];
                    vdv[x] += v8[e] * dv8[e];
                }
            }
        __builtin_amdgcn_sched_barrier(0);
        fetch_states(slab); // (not earlier: registers)
        __syncthreads();
        const int l = opaque(threadIdx.x & 63), own = (l & 15) * PV + (l >> 4) * 8, turned = turned_row(0, l & 15) * PV + (l >> 4) * 8;
        if (columns)
#pragma unroll
            for (int kk = 0; kk < SLAB / 32; kk++) {
                Frag f[NT][COMPUTED];
#pragma unroll
                for (int nt = 0; nt < NT; nt++) {
                    if (first == 0)
#pragma unroll
                        for (int e = 0; e < 8; e++) ds += s8[nt][e] * d8[nt][e];
                    split(d8[nt], f[nt]);
                }
#pragma unroll
                for (int t = 0; t < EACH; t++) {
                    Frag uf[COMPUTED];
                    row_frag(uf, u_lds + (first + t) * 16 * PV + kk * 32 + own, VP);
#pragma unroll
                    for (int nt = 0; nt < NT; nt++) k_last[t][nt] = product(f[nt], uf, k_last[t][nt]);
                    if (t % 2) __builtin_amdgcn_sched_barrier(0); // (registers: no more rows read ahead)
                }
                __builtin_amdgcn_sched_barrier(0);
#pragma unroll
                for (int nt = 0; nt < NT; nt++) split(s8[nt], f[nt]);
                if (kk + 1 < SLAB / 32) fetch_states(slab + kk * 32 + 32);
#pragma unroll
                for (int t = 0; t < EACH; t++) {
                    Frag gf[IP], vf[COMPUTED];
                    row_frag(gf, do_lds + (first + t) * 16 * PV + kk * 32 + own, VP);
                    row_frag(vf, dv_lds + (first + t) * 16 * PV + kk * 32 + own, VP);
#pragma unroll
                    for (int nt = 0; nt < NT; nt++) {
                        dq[t][nt] = product(f[nt], gf, dq[t][nt]);
                        k_row[t][nt] = product(f[nt], vf, k_row[t][nt]);
                    }
                    if (t % 2) __builtin_amdgcn_sched_barrier(0);
                }
                __builtin_amdgcn_sched_barrier(0);
            }
        auto dots = [&](auto lane_parts, const bf16 *lane_rows, auto other_parts, const bf16 *others, int t, int ks, Dots &to) {
#pragma unroll
            for (int kk = 0; kk < SLAB / 32; kk++) {
                Frag a[decltype(lane_parts)::value], b0[decltype(other_parts)::value], b1[decltype(other_parts)::value];
                const bf16 *const other = others + ks * 32 * PV + kk * 32 + turned;
                row_frag(a, lane_rows + t * 16 * PV + kk * 32 + own, VP);
                row_frag(b0, other, VP);
                row_frag(b1, other + 4 * PV, VP);
                to.a = product(b0, a, to.a);
                to.b = product(b1, a, to.b);
                __builtin_amdgcn_sched_barrier(0);
            }
        };
        typedef std::integral_constant<int, IP> In;
        typedef std::integral_constant<int, COMPUTED> Three;
#pragma unroll
        for (int u = 0; u < 2; u++)
            if (p_mine[u]) dots(In(), do_lds, Three(), u_lds, p_t[u], p_ks[u], p_dots[u]);
        if (z_mine) {
            dots(Three(), dv_lds, Three(), u_lds, wave, wave / 2, low);
            dots(Three(), u_lds, Three(), dv_lds, wave, wave / 2, high);
        }
        if (o_mine) {
            if (wave >= 2) dots(Three(), dv_lds, Three(), u_lds, wave, 0, off);
            else dots(Three(), u_lds, Three(), dv_lds, wave, 1, off);
        }
    }
#pragma unroll
    for (int x = 0; x < PER; x++) { // the rows' sums over all slabs
        const int me = opaque(threadIdx.x), my_row = me / (SLAB / 8);
#pragma unroll
        for (int y = 1; y < SLAB / 8; y *= 2) {
            gbeta[x] += __shfl_xor(gbeta[x], y);
            vdv[x] += __shfl_xor(vdv[x], y);
        }
        const int row = my_row + x * Rows::STEP;
        if (my_row < CH && me % (SLAB / 8) == 0) {
            vdv_lds[row] = vdv[x];
            if (row < n) w.g_beta[(tok + row) * w.heads + h] = gbeta[x];
        }
    }

    // ---- the pairs, row by row: dP, then - (dG + dG^T)
    {
        TileRows<S, DK, THREADS, CH> kx, qx;
        kx.fetch(reinterpret_cast<const S *>(w.k) + tok * w.k_tok + kh * w.k_head, w.k_tok, n, w.dk);
        qx.fetch(reinterpret_cast<const S *>(w.q) + tok * w.q_tok + kh * w.q_head, w.q_tok, n, w.dk);
        __syncthreads();
        kx.template put_any<PK>(k_lds, n, w.dk);
        qx.template put_any<PK>(q_lds, n, w.dk);
    }
    {
        const int lane = opaque(threadIdx.x & 63), i = lane & 15, g = lane >> 4, own = i * PP + g * 8, in = i * PK + g * CS; // own, in: places in a tile of pairs, and of k and q
        auto eight = [&](const Dots &d) { return f32x8(__builtin_shufflevector(d.a, d.b, 0, 1, 2, 3, 4, 5, 6, 7)); };
        auto write = [&](int t, int ks, const f32x8 &x) {
            Frag parts[COMPUTED];
            split(x, parts);
#pragma unroll
            for (int p = 0; p < COMPUTED; p++) *reinterpret_cast<Frag *>(pairs + p * Lds::PAIRS + t * 16 * PP + ks * 32 + own) = parts[p];
        };
#pragma unroll
        for (int u = 0; u < 2; u++)
            if (p_mine[u]) {
                const int row = p_t[u] * 16 + i, col = p_ks[u] * 32 + g * 8;
                f32x8 x = eight(p_dots[u]);
#pragma unroll
                for (int e = 0; e < 8; e++) x[e] = row >= col + e ? w.scale * x[e] * weight2(b2[row] - b2[col + e]) : 0.0f;
                write(p_t[u], p_ks[u], x);
            }
        __syncthreads();
        float kdk = 0;
        auto entries = [&](const bf16 *from, int t, int nt) { // the lane's four entries of a row
            f32x4 x = {0, 0, 0, 0};
            const bf16 *const p = from + (first + t) * 16 * PK + col0 + 4 * nt + in;
#pragma unroll
            for (int u = IP - 1; u >= 0; u--) x += __builtin_convertvector(*reinterpret_cast<const bf16x4 *>(p + u * KP), f32x4);
            return x;
        };
        auto dot = [](const f32x4 &a, const f32x4 &b) { return a[0] * b[0] + a[1] * b[1] + a[2] * b[2] + a[3] * b[3]; };
        if (columns) {
#pragma unroll
            for (int t = 0; t < EACH; t++)
#pragma unroll
                for (int nt = 0; nt < NT; nt++) {
                    const int row = (first + t) * 16 + i;
                    dq[t][nt] *= w.scale * up[row];
                    k_last[t][nt] *= down[row];
                    kdk += dot(entries(k_lds, t, nt), k_last[t][nt]);
                    k_row[t][nt] = k_last[t][nt] - up[row] * k_row[t][nt];
                }
#pragma unroll
            for (int half = 0; half < HALVES; half++) {
                Frag kf[NT][IP], qf[NT][IP];
#pragma unroll
                for (int nt = 0; nt < NT; nt++) {
                    col_frag<PK>(kf[nt], k_lds, KP, half * 32, col0 + 4 * nt, CS, lane);
                    col_frag<PK>(qf[nt], q_lds, KP, half * 32, col0 + 4 * nt, CS, lane);
                }
#pragma unroll
                for (int t = 0; t < EACH; t++) {
                    Frag x[COMPUTED];
                    if (half <= (first + t) / 2) {
                        row_frag(x, pairs + (first + t) * 16 * PP + half * 32 + own, Lds::PAIRS);
#pragma unroll
                        for (int nt = 0; nt < NT; nt++) dq[t][nt] = product(kf[nt], x, dq[t][nt]);
                    }
                    if (half >= (first + t) / 2) {
                        col_frag<PP>(x, pairs, Lds::PAIRS, half * 32, (first + t) * 16, 4, lane);
#pragma unroll
                        for (int nt = 0; nt < NT; nt++) k_row[t][nt] = product(qf[nt], x, k_row[t][nt]);
                    }
                    __builtin_amdgcn_sched_barrier(0);
                }
            }
        }
#pragma unroll
        for (int x = 1; x < 64; x *= 2) {
            kdk += __shfl_xor(kdk, x);
            ds += __shfl_xor(ds, x);
        }
        if (lane == 0) {
            sums[wave] = kdk;
            sums[NW + wave] = ds;
        }
        __syncthreads();
        if (z_mine) {
            const int row = wave * 16 + i, col = wave / 2 * 32 + g * 8;
            const f32x8 a = eight(low), b = eight(high);
            f32x8 x;
#pragma unroll
            for (int e = 0; e < 8; e++) {
                const int c = col + e;
                x[e] = c < row ? -a[e] * weight2(b2[row] - b2[c]) : c > row ? -b[e] * weight2(b2[c] - b2[row]) : 0.0f;
            }
            write(wave, wave / 2, x);
        }
        if (o_mine) {
            const int row = wave * 16 + i, col = (1 - wave / 2) * 32 + g * 8;
            f32x8 x = eight(off);
#pragma unroll
            for (int e = 0; e < 8; e++) x[e] *= -weight2(wave >= 2 ? b2[row] - b2[col + e] : b2[col + e] - b2[row]);
            write(wave, 1 - wave / 2, x);
        }
        __syncthreads();
        if (columns) {
#pragma unroll
            for (int half = 0; half < HALVES; half++) {
                Frag kf[NT][IP];
#pragma unroll
                for (int nt = 0; nt < NT; nt++) col_frag<PK>(kf[nt], k_lds, KP, half * 32, col0 + 4 * nt, CS, lane);
#pragma unroll
                for (int t = 0; t < EACH; t++) {
                    Frag x[COMPUTED];
                    row_frag(x, pairs + (first + t) * 16 * PP + half * 32 + own, Lds::PAIRS);
#pragma unroll
                    for (int nt = 0; nt < NT; nt++) k_row[t][nt] = product(kf[nt], x, k_row[t][nt]);
                    if (t % 2) __builtin_amdgcn_sched_barrier(0);
                }
            }
#pragma unroll
            for (int t = 0; t < EACH; t++) {
                const int row = (first + t) * 16 + i, col = col0 + g * CS;
                float a = 0;
#pragma unroll
                for (int nt = 0; nt < NT; nt++) a += dot(entries(q_lds, t, nt), dq[t][nt]);
                a += __shfl_xor(a, 16);
                a += __shfl_xor(a, 32);
                if (g == 0) qdq[tile * CH + row] = a;
                if (row < n) {
                    const long long to = ((tok + row) * w.heads + h) * (long long)w.dk + col;
                    auto store = [&](void *out, const f32x4 (&x)[NT]) {
                        float y[NT * 4];
#pragma unroll
                        for (int e = 0; e < NT * 4; e++) y[e] = x[e / 4][e % 4];
                        if (col + NT * 4 <= w.dk) {
                            if (w.grad_float) store_floats_unaligned<float, NT * 4>(reinterpret_cast<float *>(out) + to, y);
                            else store_floats_unaligned<S, NT * 4>(reinterpret_cast<S *>(out) + to, y);
                        } else {
#pragma unroll
                            for (int e = 0; e < NT * 4; e++)
                                if (col + e < w.dk) {
                                    if (w.grad_float) reinterpret_cast<float *>(out)[to + e] = y[e];
                                    else reinterpret_cast<S *>(out)[to + e] = (S)y[e];
                                }
                        }
                    };
                    store(w.gq, dq[t]);
                    store(w.gk, k_row[t]);
                }
            }
        }
    }
    __syncthreads();
    if (wave == 0) { // sums towards the chunk's end; a token's decay has what all later ones and the next state make of it
        double s = 0;
        if (lane < CH) {
            s = -(double)vdv_lds[lane];
            for (int x = 0; x < TILES; x++) s += qdq[x * CH + lane];
        }
        if (lane == n - 1) {
            double end = 0, d = 0;
            for (int x = 0; x < NW; x++) {
                end += sums[x];
                d += sums[NW + x];
            }
            s += end + vec.whole * d;
        }
        if (lane >= n) s = 0;
#pragma unroll
        for (int x = 1; x < 64; x *= 2) {
            const double y = __shfl_down(s, x);
            if (lane + x < 64) s += y;
        }
        if (lane < n) {
            const long long to = (tok + lane) * w.heads + h;
            w.g_log_decay[to] = power2(log2_of(w.log_decay[to])) == 0.0f ? 0.0f : (float)s; // what is forgotten whole has no slope
        }
    }
}

// ---- launches

template <typename S, int DK, int DV, int MODE> static int launch_delta_walk_sized(goom_ctx *ctx, DeltaArgs w, long long slots, const char *label)
{
    w.slots = (unsigned)slots;
    const int parts = w.parts + (MODE == MAPS ? w.map_parts : 0);
    typedef DeltaLds<S, DK, DV, MODE> Lds;
    auto *kernel = delta_walk_kernel<S, DK, DV, MODE>;
    constexpr size_t bytes = Lds::bytes;
    static_assert(bytes <= (160 << 10), "LDS of a CU");
    static std::atomic<unsigned long long> done{0};
    if (int st = allow_lds(ctx, reinterpret_cast<const void *>(kernel), bytes, done)) return st;
    goom::prof_begin(ctx, label);
    kernel<<<grid_of((slots * w.heads + 7) / 8 * 8 * parts, Lds::WAVES * 64), Lds::WAVES * 64, bytes, ctx->stream>>>(w);
    goom::prof_end(ctx);
    return goom::check_hip(ctx, hipGetLastError(), label);
}

// columns of a workgroup
constexpr int delta_columns(int dv) { return dv <= 32 ? 32 : 64; }
constexpr int delta_rows(int dk) { return dk <= 32 ? 32 : dk <= 64 ? 64 : 128; }

template <typename F> static int with_delta(int dk, int dv, F f)
{
    auto columns = [&](auto rows) {
        if (dv <= 32) return f(rows, std::integral_constant<int, 32>());
        return f(rows, std::integral_constant<int, 64>());
    };
    return dk <= 32 ? columns(std::integral_constant<int, 32>()) : dk <= 64 ? columns(std::integral_constant<int, 64>()) : columns(std::integral_constant<int, 128>());
}

// slots: of segments in the walks and carries, of chunks in the others
template <typename S> int launch_delta_within(goom_ctx *ctx, const DeltaArgs &w, long long slots);
template <typename S> int launch_delta_walk(goom_ctx *ctx, const DeltaArgs &w, int mode, long long slots, const char *label);
template <typename S> int launch_delta_back(goom_ctx *ctx, const DeltaArgs &w, int mode, long long slots, const char *label);
template <typename S> int launch_delta_gradients(goom_ctx *ctx, const DeltaArgs &w, long long slots);

template <typename S> int launch_delta_within_typed(goom_ctx *ctx, DeltaArgs w, long long slots)
{
    w.slots = (unsigned)slots;
    return with_delta(w.dk, 64, [&](auto rows, auto) {
        constexpr int DK = decltype(rows)::value;
        auto *kernel = within_kernel<S, DK>;
        static std::atomic<unsigned long long> done{0};
        if (int st = allow_lds(ctx, reinterpret_cast<const void *>(kernel), WithinLds<S, DK>::bytes, done)) return st;
        goom::prof_begin(ctx, "gated delta rule: within chunks");
        kernel<<<grid_of(slots * (w.heads / w.share) + (w.order ? 1 : 0), 256), 256, WithinLds<S, DK>::bytes, ctx->stream>>>(w);
        goom::prof_end(ctx);
        return goom::check_hip(ctx, hipGetLastError(), "gated delta rule: within chunks");
    });
}

template <typename S, int FIRST, int SECOND, int THIRD> int launch_delta_walk_typed(goom_ctx *ctx, const DeltaArgs &w, int mode, long long slots, const char *label)
{
    return with_delta(w.dk, w.dv, [&](auto rows, auto cols) {
        constexpr int DK = decltype(rows)::value, DV = decltype(cols)::value;
        if (mode == FIRST) return launch_delta_walk_sized<S, DK, DV, FIRST>(ctx, w, slots, label);
        if (mode == SECOND) return launch_delta_walk_sized<S, DK, DV, SECOND>(ctx, w, slots, label);
        return launch_delta_walk_sized<S, DK, DV, THIRD>(ctx, w, slots, label);
    });
}

template <typename S> int launch_delta_gradients_typed(goom_ctx *ctx, DeltaArgs w, long long slots)
{
    w.slots = (unsigned)slots;
    return with_delta(w.dk, w.dv, [&](auto rows, auto cols) {
        constexpr int DK = decltype(rows)::value, DV = decltype(cols)::value;
        typedef GradLds<S, DK, DV> Lds;
        static_assert(Lds::bytes <= (160 << 10), "LDS of a CU");
        auto *kernel = delta_grad_kernel<S, DK, DV>;
        static std::atomic<unsigned long long> done{0};
        if (int st = allow_lds(ctx, reinterpret_cast<const void *>(kernel), Lds::bytes, done)) return st;
        goom::prof_begin(ctx, "gated delta rule: gradients within chunks");
        kernel<<<grid_of(slots * w.heads, Lds::THREADS), Lds::THREADS, Lds::bytes, ctx->stream>>>(w);
        goom::prof_end(ctx);
        return goom::check_hip(ctx, hipGetLastError(), "gated delta rule: gradients");
    });
}

} // namespace goom_layer
