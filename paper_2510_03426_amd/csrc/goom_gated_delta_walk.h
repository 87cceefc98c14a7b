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
constexpr int kind_frags(int ch) { return pair_blocks(ch) * COMPUTED * 64; }

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
    int heads, share, dk, dv;
    float scale;
    Frag *frags;             // [chunk slots][heads][kinds][blocks][parts][64]
    void *vecs;              // ChunkVec [chunk slots][heads]
    int kinds, m, mt, p, pt; // which kind of fragments is which; -1: none
    const float *init;       // NULL or [seqs][heads][dk][dv]: the state before the first token, or (backwards) its adjoint after the last
    float *fin;              // NULL or the same: the last state, or the first one's adjoint
    void *o;
    float *totals;           // NULL: one segment a sequence; [slots][heads][parts][state registers]: B, then the incoming states
    float *maps;             // A, [slots][heads][DK][DK]
    float *kept, *rows;      // KEEP: states before, BACK: adjoints after each chunk [chunk slots][heads][DK][pitch]; E or W [chunk slots][heads][CH][pitch]
    int pitch;
    void *gv;
    int parts, map_parts;    // workgroups' column parts of the state, and of A
    unsigned slots;
    // gradients
    const float *kept_s, *kept_d, *rows_e, *rows_w;
    void *gq, *gk;           // [tokens][heads][dk], floats where heads share q and k
    int grad_float;
    float *g_log_decay, *g_beta;
};

// log2 of a decay; below 2^-160, which is zero as a float whatever it is divided by, finite (a NaN stays one)
__device__ inline double log2_of(float log_decay)
{
    const double x = (double)log_decay * 1.4426950408889634;
    return x < -160.0 ? -160.0 : x;
}
__device__ inline float power2(double x) { return __builtin_amdgcn_exp2f((float)x); }

// rows of a tile of 16 in the order in which a lane's accumulator entries of two tiles are eight consecutive ones
__device__ inline int turned_row(int t, int i) { return t / 2 * 32 + (i >> 2) * 8 + t % 2 * 4 + (i & 3); }

// ---- what lies within a chunk

template <typename S, int DK> struct WithinLds {
    static constexpr int CH = chunk_of<S>(), PK = DK + PITCH_PAD, TILE = CH * PK * Parts<S>::IN, PM = CH + 4;
    static constexpr size_t bytes = 2 * TILE * sizeof(bf16) + 2 * CH * PM * sizeof(float) + CH * (sizeof(double) + sizeof(float));
};

// M21 = (I - M22 beta2) G21 (I - beta1 M11) for the pairs of diagonal blocks of SIZE: every wave has tiles of 16 x 16
template <int SIZE, int CH> __device__ inline void join_blocks(float *m, const float *beta)
{
    constexpr int PM = CH + 4, TILES = (SIZE / 16) * (SIZE / 16), ALL = CH / (2 * SIZE) * TILES;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, i = lane & 15, g = lane >> 4;
    const bool mine = wave < ALL;
    const int r0 = wave / TILES * 2 * SIZE, tr = r0 + SIZE + wave % TILES / (SIZE / 16) * 16, tc = r0 + wave % TILES % (SIZE / 16) * 16;
#pragma unroll
    for (int pass = 0; pass < 2; pass++) { // G21 - (G21 beta1) M11, then that less M22 (beta2 that)
        f32x4 c = {0, 0, 0, 0};
        if (mine) {
#pragma unroll
            for (int k = 0; k < SIZE; k += 4) {
                const int x = pass == 0 ? r0 + k + g : r0 + SIZE + k + g;
                c = __builtin_amdgcn_mfma_f32_16x16x4f32(m[(tr + i) * PM + x] * beta[x], m[x * PM + tc + i], c, 0, 0, 0);
            }
#pragma unroll
            for (int e = 0; e < 4; e++) c[e] = m[(tr + g * 4 + e) * PM + tc + i] - c[e];
        }
        __syncthreads();
        if (mine)
#pragma unroll
            for (int e = 0; e < 4; e++) m[(tr + g * 4 + e) * PM + tc + i] = c[e];
        __syncthreads();
    }
}

template <typename S, int DK> __global__ __launch_bounds__(256) void within_kernel(DeltaArgs w)
{
    typedef WithinLds<S, DK> Lds;
    constexpr int CH = Lds::CH, PK = Lds::PK, PM = Lds::PM, IP = Parts<S>::IN, KP = CH * PK, BLOCKS = pair_blocks(CH);
    extern __shared__ __align__(16) unsigned char lds[];
    bf16 *const k_lds = reinterpret_cast<bf16 *>(lds), *const q_lds = k_lds + Lds::TILE;
    float *const kk = reinterpret_cast<float *>(q_lds + Lds::TILE), *const m = kk + CH * PM;
    double *const b2 = reinterpret_cast<double *>(m + CH * PM);
    float *const beta = reinterpret_cast<float *>(b2 + CH);
    const int qk_heads = w.heads / w.share;
    const long long block = block_of();
    const int kh = block % qk_heads;
    const long long slot = block / qk_heads;
    if (slot >= w.slots) return;
    const Place at = find_place(w.chunk, slot);
    if (at.seg < 0 || at.seg >= at.nseg || at.len == 0) return;
    const long long t0 = at.seg * CH, tok = at.start + t0;
    const int n = at.len - t0 < CH ? (int)(at.len - t0) : CH;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, i = lane & 15, g = lane >> 4;
    const bool pairs = w.p >= 0 || w.pt >= 0;

    TileRows<S, DK, 256, CH> kx, qx;
    kx.fetch(reinterpret_cast<const S *>(w.k) + tok * w.k_tok + kh * w.k_head, w.k_tok, n, w.dk);
    if (pairs) qx.fetch(reinterpret_cast<const S *>(w.q) + tok * w.q_tok + kh * w.q_head, w.q_tok, n, w.dk);
    kx.template put<PK>(k_lds, n, w.dk);
    if (pairs) qx.template put<PK>(q_lds, n, w.dk);
    __syncthreads();

    // k_i . k_j, by tiles on and below the diagonal; q_i . k_j by fragments, which their waves keep
    constexpr int SIDE = CH / 16;
    for (int tile = wave; tile < SIDE * (SIDE + 1) / 2; tile += 4) {
        int r = 0, c = tile;
        while (c > r) c -= ++r;
        f32x4 acc = {0, 0, 0, 0};
#pragma unroll
        for (int x = 0; x < DK / 32; x++) {
            Frag a[IP], b[IP];
            row_frag(a, k_lds + (r * 16 + i) * PK + x * 32 + g * 8, KP);
            row_frag(b, k_lds + (c * 16 + i) * PK + x * 32 + g * 8, KP);
            acc = product(a, b, acc);
        }
#pragma unroll
        for (int e = 0; e < 4; e++) kk[(r * 16 + g * 4 + e) * PM + c * 16 + i] = acc[e];
    }
    constexpr int MINE = (BLOCKS + 3) / 4;
    f32x8 dots[MINE], dots_t[MINE];
    auto rows_dot = [&](const bf16 *lane_row, const bf16 *turned, int ks) { // the lane's row against eight consecutive ones from ks 32 + g 8 on
        f32x4 p0 = {0, 0, 0, 0}, p1 = {0, 0, 0, 0};
        const bf16 *const other = turned + turned_row(2 * ks, i) * PK + g * 8;
#pragma unroll
        for (int x = 0; x < DK / 32; x++) {
            Frag a[IP], b0[IP], b1[IP];
            row_frag(a, lane_row + g * 8 + x * 32, KP);
            row_frag(b0, other + x * 32, KP);
            row_frag(b1, other + 4 * PK + x * 32, KP);
            p0 = product(b0, a, p0);
            p1 = product(b1, a, p1);
        }
        return f32x8(__builtin_shufflevector(p0, p1, 0, 1, 2, 3, 4, 5, 6, 7));
    };
#pragma unroll
    for (int u = 0; u < MINE; u++) {
        const int block = wave + u * 4;
        int t, ks;
        if (block < BLOCKS) {
            if (w.p >= 0) {
                p_place<false>(block, CH, t, ks);
                dots[u] = rows_dot(q_lds + (t * 16 + i) * PK, k_lds, ks);
            }
            if (w.pt >= 0) {
                p_place<true>(block, CH, t, ks);
                dots_t[u] = rows_dot(k_lds + turned_row(t, i) * PK, q_lds, ks);
            }
        }
    }

    for (int s = 0; s < w.share; s++) {
        const int h = kh * w.share + s;
        const long long record = slot * w.heads + h;
        ChunkVec<CH> &vec = reinterpret_cast<ChunkVec<CH> *>(w.vecs)[record];
        __syncthreads();
        if (wave == 0) {
            const long long to = (tok + lane) * w.heads + h;
            double sum = lane < n ? log2_of(w.log_decay[to]) : 0.0;
            const float be = lane < n ? w.beta[to] : 0.0f;
#pragma unroll
            for (int step = 1; step < CH; step *= 2) {
                const double x = __shfl_up(sum, step);
                if (lane >= step) sum += x;
            }
            const double end = __shfl(sum, CH - 1);
            if (lane < CH) {
                b2[lane] = sum;
                beta[lane] = be;
                vec.b2[lane] = sum;
                vec.beta[lane] = be;
                vec.up[lane] = lane < n ? power2(sum) : 0.0f;
                vec.down[lane] = lane < n ? power2(end - sum) : 0.0f;
                if (lane == 0) vec.whole = power2(end);
            }
        }
        __syncthreads();
        for (int u = threadIdx.x; u < CH * CH; u += 256) {
            const int r = u / CH, c = u % CH;
            m[r * PM + c] = c < r ? kk[r * PM + c] * power2(b2[r] - b2[c]) : 0.0f;
        }
        __syncthreads();
        // rows of M one after another, in blocks of 16: M_i = G_i - sum_j G_ij beta_j M_j; a lane has a column of one block
        if (wave == 0 && lane < CH) {
            float x[16];
            float *const d = m + g * 16 * PM + g * 16;
            const float *const be = beta + g * 16;
#pragma unroll
            for (int r = 0; r < 16; r++) {
                float y = d[r * PM + i];
#pragma unroll
                for (int c = 0; c < r; c++) y -= d[r * PM + c] * be[c] * x[c];
                x[r] = y;
            }
#pragma unroll
            for (int r = 0; r < 16; r++) d[r * PM + i] = x[r]; // (after all reads: the lanes of a wave go together)
        }
        __syncthreads();
        join_blocks<16, CH>(m, beta);
        if constexpr (CH == 64) join_blocks<32, CH>(m, beta);

        auto put = [&](int kind, int block, const f32x8 &x) {
            Frag parts[COMPUTED];
            split(x, parts);
            Frag *const to = w.frags + ((record * w.kinds + kind) * BLOCKS + block) * (COMPUTED * 64) + lane;
#pragma unroll
            for (int q = 0; q < COMPUTED; q++) to[q * 64] = parts[q];
        };
#pragma unroll
        for (int u = 0; u < MINE; u++) {
            const int block = wave + u * 4;
            if (block >= BLOCKS) continue;
            int t, ks;
            f32x8 x;
            p_place<false>(block, CH, t, ks);
            if (w.m >= 0) {
                const int row = turned_row(t, i), col = ks * 32 + g * 8;
                const f32x4 *const from = reinterpret_cast<const f32x4 *>(m + row * PM + col);
                x = __builtin_shufflevector(from[0], from[1], 0, 1, 2, 3, 4, 5, 6, 7);
                put(w.m, block, x);
            }
            if (w.p >= 0) {
                const int row = t * 16 + i, col = ks * 32 + g * 8;
#pragma unroll
                for (int e = 0; e < 8; e++) x[e] = col + e <= row ? w.scale * dots[u][e] * power2(b2[row] - b2[col + e]) : 0.0f;
                put(w.p, block, x);
            }
            p_place<true>(block, CH, t, ks);
            if (w.mt >= 0) {
                const int row = turned_row(t, i), col = ks * 32 + g * 8;
#pragma unroll
                for (int e = 0; e < 8; e++) x[e] = m[(col + e) * PM + row];
                put(w.mt, block, x);
            }
            if (w.pt >= 0) {
                const int row = turned_row(t, i), col = ks * 32 + g * 8;
#pragma unroll
                for (int e = 0; e < 8; e++) x[e] = row <= col + e ? w.scale * dots_t[u][e] * power2(b2[col + e] - b2[row]) : 0.0f;
                put(w.pt, block, x);
            }
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

template <typename S, int DK, int DV, int NW, int MODE> struct DeltaLds {
    static constexpr int CH = chunk_of<S>(), PK = DK + PITCH_PAD, PV = DV + PITCH_PAD;
    static constexpr bool REV = MODE == BACK_MAPS || MODE == BACK, OUT = MODE == FORWARD, Q = OUT || REV, P = OUT || REV;
    static constexpr int K_TILE = CH * PK * Parts<S>::IN, V_TILE = CH * PV * Parts<S>::IN; // elements
    static constexpr int FRAGS = kind_frags(CH) * (P ? 2 : 1);
    static constexpr size_t bytes = FRAGS * sizeof(Frag) + (K_TILE * (Q ? 2 : 1) + V_TILE) * sizeof(bf16) + 4 * CH * sizeof(float);
    static constexpr int fit = (int)((160 << 10) / bytes), most = 8 / NW;
    static constexpr int resident = fit < 1 ? 1 : fit > most ? most : fit;
    static constexpr int per_simd = (resident * NW + 3) / 4;
};

// DK: dk, padded; NW waves of one or two tiles of 16 of the DV columns
template <typename S, int DK, int DV, int NW, int MODE>
__device__ inline void delta_walk(const DeltaArgs &w, const Place &at, long long slot, int h, int part, unsigned char *lds)
{
    typedef DeltaLds<S, DK, DV, NW, MODE> Lds;
    constexpr int THREADS = NW * 64, NT = DV / 16 / NW, KS = DK / 32, CS = NT == 2 ? 8 : 4, TT = Lds::CH / 16;
    constexpr int IP = Parts<S>::IN, CH = Lds::CH, KP = CH * Lds::PK, VP = CH * Lds::PV, HALVES = CH / 32;
    constexpr bool REV = Lds::REV, OUT = Lds::OUT, TOTAL = MODE == MAPS || MODE == BACK_MAPS;
    static_assert(NT == 1 || NT == 2, "a wave has one or two column tiles");
    Frag *const m_lds = reinterpret_cast<Frag *>(lds), *const p_lds = m_lds + kind_frags(CH);
    bf16 *const k_lds = reinterpret_cast<bf16 *>(m_lds + Lds::FRAGS), *const v_lds = k_lds + Lds::K_TILE, *const q_lds = v_lds + Lds::V_TILE;
    float *const vec_lds = reinterpret_cast<float *>(q_lds + (Lds::Q ? Lds::K_TILE : 0)); // up, down, beta

    const bool last = REV ? at.seg == 0 : at.seg == at.nseg - 1; // in walking order
    const bool map = MODE == MAPS && part >= w.parts; // columns of A
    if (TOTAL && last && !(map && w.mt >= 0)) return; // (the way back goes through the last segment's A as well)
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, i = lane & 15, g = lane >> 4;
    const int col0 = wave * NT * 16; // the wave's columns: col0 + (i / 4) CS + 4 nt + i % 4
    const int col_part = (map ? part - w.parts : part) * DV, nc_all = map ? w.dk : w.dv, nc = nc_all - col_part < DV ? nc_all - col_part : DV;
    const int kh = h / w.share;
    const bool empty = at.len == 0;
    auto row_of = [&](int t, int e) { return t / 2 * 32 + g * 8 + t % 2 * 4 + e; };
    auto col_of = [&](int nt) { return col0 + (i >> 2) * CS + 4 * nt + (i & 3); };

    // ---- the incoming state
    f32x4 R[DK / 16][NT];
    float *const total = w.totals && !map ? w.totals + ((slot * w.heads + h) * w.parts + part) * (long long)(DK * DV) + (long long)wave * NT * (DK / 16) * 256 + lane * 4 : nullptr;
    const long long state0 = (at.seq * w.heads + h) * (long long)w.dk * w.dv + col_part;
#pragma unroll
    for (int t = 0; t < DK / 16; t++)
#pragma unroll
        for (int nt = 0; nt < NT; nt++) {
            f32x4 x = {0, 0, 0, 0};
            const int col = col_of(nt);
            if (TOTAL) {
                if (map)
#pragma unroll
                    for (int e = 0; e < 4; e++) x[e] = row_of(t, e) == col_part + col && col < nc ? 1.0f : 0.0f;
            } else if (total && !empty) {
                x = *reinterpret_cast<const f32x4 *>(total + (nt * (DK / 16) + t) * 256);
            } else if (w.init) {
#pragma unroll
                for (int e = 0; e < 4; e++) {
                    const int row = row_of(t, e);
                    if (row < w.dk && col < nc) x[e] = w.init[state0 + (long long)row * w.dv + col];
                }
            }
            R[t][nt] = x;
        }

    const S *const k = reinterpret_cast<const S *>(w.k) + at.start * w.k_tok + kh * w.k_head;
    const S *const q = reinterpret_cast<const S *>(w.q) + at.start * w.q_tok + kh * w.q_head;
    const S *const v = REV ? reinterpret_cast<const S *>(w.go) + at.start * w.o_tok + h * (long long)w.dv + col_part
                           : reinterpret_cast<const S *>(w.v) + at.start * w.v_tok + h * w.v_head + col_part;
    const long long v_tok = REV ? w.o_tok : w.v_tok;
    const long long seg0 = at.seg * w.seg.seg_len, seg1 = seg0 + w.seg.seg_len < at.len ? seg0 + w.seg.seg_len : at.len;
    const int nchunks = (int)((seg1 - seg0 + CH - 1) / CH);
    const long long chunk0 = empty ? 0 : (first_slot(w.chunk, at.seq) + seg0 / CH);
    TileRows<S, DK, THREADS, CH> kx, qx;
    TileRows<S, DV, THREADS, CH> vx;
    constexpr int KIND = kind_frags(CH), MF = (KIND + THREADS - 1) / THREADS;
    Frag mx[MF], px[MF];
    float vec[3];
    float whole = 0;
    auto chunk_at = [&](int step) { return REV ? nchunks - 1 - step : step; };
    auto fetch = [&](int step) {
        const int c = chunk_at(step);
        const long long t0 = seg0 + (long long)c * CH, record = (chunk0 + c) * w.heads + h;
        const int n = seg1 - t0 < CH ? (int)(seg1 - t0) : CH;
        kx.fetch(k + t0 * w.k_tok, w.k_tok, n, w.dk);
        if (Lds::Q) qx.fetch(q + t0 * w.q_tok, w.q_tok, n, w.dk);
        if (!map) vx.fetch(v + t0 * v_tok, v_tok, n, nc);
        const Frag *const frags = w.frags + record * w.kinds * KIND;
#pragma unroll
        for (int u = 0; u < MF; u++) {
            const int at = u * THREADS + threadIdx.x < KIND ? u * THREADS + threadIdx.x : KIND - 1;
            mx[u] = frags[(REV ? w.mt : w.m) * KIND + at];
            if (Lds::P) px[u] = frags[(REV ? w.pt : w.p) * KIND + at];
        }
        const ChunkVec<CH> &cv = reinterpret_cast<const ChunkVec<CH> *>(w.vecs)[record];
        if (threadIdx.x < CH) {
            vec[0] = cv.up[threadIdx.x];
            vec[1] = cv.down[threadIdx.x];
            vec[2] = cv.beta[threadIdx.x];
        }
        whole = cv.whole;
    };
    if (nchunks > 0) fetch(0);
    for (int step = 0; step < nchunks; step++) {
        const int c = chunk_at(step);
        const long long t0 = seg0 + (long long)c * CH, record = (chunk0 + c) * w.heads + h;
        const int n = seg1 - t0 < CH ? (int)(seg1 - t0) : CH;
        const float decay = whole;
        __syncthreads();
        kx.template put<Lds::PK>(k_lds, n, w.dk);
        if (Lds::Q) qx.template put<Lds::PK>(q_lds, n, w.dk);
        if (!map) vx.template put<Lds::PV>(v_lds, n, nc);
#pragma unroll
        for (int u = 0; u < MF; u++)
            if (u * THREADS + threadIdx.x < KIND) {
                m_lds[u * THREADS + threadIdx.x] = mx[u];
                if (Lds::P) p_lds[u * THREADS + threadIdx.x] = px[u];
            }
        if (threadIdx.x < CH)
#pragma unroll
            for (int x = 0; x < 3; x++) vec_lds[x * CH + threadIdx.x] = vec[x];
        __syncthreads();
        if (step + 1 < nchunks) fetch(step + 1); // while this chunk is worked on

        if (MODE == KEEP || MODE == BACK) {
            float *const to = w.kept + record * (DK * (long long)w.pitch) + col_part;
#pragma unroll
            for (int t = 0; t < DK / 16; t++)
#pragma unroll
                for (int nt = 0; nt < NT; nt++)
#pragma unroll
                    for (int e = 0; e < 4; e++) to[row_of(t, e) * w.pitch + col_of(nt)] = R[t][nt][e];
        }

        // ---- K against the state, a lane with eight consecutive tokens of a column; Q with consecutive columns of a token
        f32x4 x[TT][NT], y[OUT ? TT : 1][NT];
#pragma unroll
        for (int t = 0; t < TT; t++)
#pragma unroll
            for (int nt = 0; nt < NT; nt++) {
                x[t][nt] = f32x4{0, 0, 0, 0};
                if (OUT) y[t][nt] = f32x4{0, 0, 0, 0};
            }
#pragma unroll
        for (int kk = 0; kk < KS; kk++) {
            Frag rf[NT][COMPUTED];
#pragma unroll
            for (int nt = 0; nt < NT; nt++) split(__builtin_shufflevector(R[2 * kk][nt], R[2 * kk + 1][nt], 0, 1, 2, 3, 4, 5, 6, 7), rf[nt]);
#pragma unroll
            for (int t = 0; t < TT; t++) {
                Frag kf[IP];
                row_frag(kf, k_lds + turned_row(t, i) * Lds::PK + kk * 32 + g * 8, KP);
#pragma unroll
                for (int nt = 0; nt < NT; nt++) x[t][nt] = product(kf, rf[nt], x[t][nt]);
                if (OUT) {
                    Frag qf[IP];
                    row_frag(qf, q_lds + (t * 16 + i) * Lds::PK + kk * 32 + g * 8, KP);
#pragma unroll
                    for (int nt = 0; nt < NT; nt++) y[t][nt] = product(rf[nt], qf, y[t][nt]);
                }
            }
        }
        auto eight = [&](int which, int half) { return *reinterpret_cast<const f32x8 *>(vec_lds + which * CH + half * 32 + g * 8); };
        auto pair = [&](const f32x4 &a, const f32x4 &b) { return f32x8(__builtin_shufflevector(a, b, 0, 1, 2, 3, 4, 5, 6, 7)); };
        // ---- Y (or dU), and with M the rows E (or W)
        f32x8 r8[HALVES][NT], go8[REV ? HALVES : 1][NT];
        if (REV) {
            f32x4 local[TT][NT];
#pragma unroll
            for (int t = 0; t < TT; t++)
#pragma unroll
                for (int nt = 0; nt < NT; nt++) local[t][nt] = f32x4{0, 0, 0, 0};
#pragma unroll
            for (int half = 0; half < HALVES; half++)
#pragma unroll
                for (int nt = 0; nt < NT; nt++) {
                    Frag gf[IP];
                    col_frag<Lds::PV>(gf, v_lds, VP, half * 32, col0 + 4 * nt, CS, lane);
                    go8[half][nt] = widen(gf);
#pragma unroll
                    for (int t = 0; t < TT; t++) {
                        if (!p_has<true>(t, half)) continue;
                        Frag pf[COMPUTED];
#pragma unroll
                        for (int u = 0; u < COMPUTED; u++) pf[u] = p_lds[(p_block<true>(t, half, CH) * COMPUTED + u) * 64 + lane];
                        local[t][nt] = product(pf, gf, local[t][nt]);
                    }
                }
#pragma unroll
            for (int half = 0; half < HALVES; half++)
#pragma unroll
                for (int nt = 0; nt < NT; nt++)
                    r8[half][nt] = pair(local[2 * half][nt], local[2 * half + 1][nt]) + eight(1, half) * pair(x[2 * half][nt], x[2 * half + 1][nt]);
        } else {
#pragma unroll
            for (int half = 0; half < HALVES; half++)
#pragma unroll
                for (int nt = 0; nt < NT; nt++) {
                    f32x8 in = {0, 0, 0, 0, 0, 0, 0, 0};
                    if (!map) {
                        Frag vf[IP];
                        col_frag<Lds::PV>(vf, v_lds, VP, half * 32, col0 + 4 * nt, CS, lane);
                        in = widen(vf);
                    }
                    r8[half][nt] = in - eight(0, half) * pair(x[2 * half][nt], x[2 * half + 1][nt]);
                }
        }
        {
            f32x4 acc[TT][NT];
#pragma unroll
            for (int t = 0; t < TT; t++)
#pragma unroll
                for (int nt = 0; nt < NT; nt++) acc[t][nt] = f32x4{0, 0, 0, 0};
#pragma unroll
            for (int half = 0; half < HALVES; half++) {
                Frag bf[NT][COMPUTED];
#pragma unroll
                for (int nt = 0; nt < NT; nt++) split(eight(2, half) * r8[half][nt], bf[nt]);
#pragma unroll
                for (int t = 0; t < TT; t++) {
                    if (!p_has<REV>(t, half)) continue;
                    Frag mf[COMPUTED];
#pragma unroll
                    for (int u = 0; u < COMPUTED; u++) mf[u] = m_lds[(p_block<REV>(t, half, CH) * COMPUTED + u) * 64 + lane];
#pragma unroll
                    for (int nt = 0; nt < NT; nt++) acc[t][nt] = product(mf, bf[nt], acc[t][nt]);
                }
            }
#pragma unroll
            for (int half = 0; half < HALVES; half++)
#pragma unroll
                for (int nt = 0; nt < NT; nt++) r8[half][nt] -= pair(acc[2 * half][nt], acc[2 * half + 1][nt]);
        }
        if (MODE == KEEP || MODE == BACK) {
            float *const to = w.rows + record * (CH * (long long)w.pitch) + col_part;
#pragma unroll
            for (int half = 0; half < HALVES; half++)
#pragma unroll
                for (int nt = 0; nt < NT; nt++)
#pragma unroll
                    for (int e = 0; e < 8; e++) to[(half * 32 + g * 8 + e) * w.pitch + col_of(nt)] = r8[half][nt][e];
        }
        // ---- U (or dV)
#pragma unroll
        for (int half = 0; half < HALVES; half++)
#pragma unroll
            for (int nt = 0; nt < NT; nt++) r8[half][nt] *= eight(2, half);
        if (MODE == BACK) {
#pragma unroll
            for (int half = 0; half < HALVES; half++)
#pragma unroll
                for (int nt = 0; nt < NT; nt++)
#pragma unroll
                    for (int e = 0; e < 8; e++) {
                        const int row = half * 32 + g * 8 + e;
                        if (row < n && col_of(nt) < nc)
                            reinterpret_cast<S *>(w.gv)[(at.start + t0 + row) * w.o_tok + h * (long long)w.dv + col_part + col_of(nt)] = (S)r8[half][nt][e];
                    }
        }
        if (OUT) {
#pragma unroll
            for (int half = 0; half < HALVES; half++) {
                Frag uf[NT][COMPUTED];
#pragma unroll
                for (int nt = 0; nt < NT; nt++) split(r8[half][nt], uf[nt]);
#pragma unroll
                for (int t = 0; t < TT; t++) {
                    if (half == 0) {
                        const float scale = w.scale * vec_lds[t * 16 + i];
#pragma unroll
                        for (int nt = 0; nt < NT; nt++) y[t][nt] *= scale;
                    }
                    if (!p_has<false>(t, half)) continue;
                    Frag pf[COMPUTED];
#pragma unroll
                    for (int u = 0; u < COMPUTED; u++) pf[u] = p_lds[(p_block<false>(t, half, CH) * COMPUTED + u) * 64 + lane];
#pragma unroll
                    for (int nt = 0; nt < NT; nt++) y[t][nt] = product(uf[nt], pf, y[t][nt]);
                }
            }
#pragma unroll
            for (int t = 0; t < TT; t++) {
                const int row = t * 16 + i, col = col0 + g * CS;
                if (row < n) {
                    S *const to = reinterpret_cast<S *>(w.o) + (at.start + t0 + row) * w.o_tok + h * (long long)w.dv + col_part + col;
                    float out[NT * 4];
#pragma unroll
                    for (int e = 0; e < NT * 4; e++) out[e] = y[t][e / 4][e % 4];
                    if (col + NT * 4 <= nc) store_floats_unaligned<S, NT * 4>(to, out);
                    else
#pragma unroll
                        for (int e = 0; e < NT * 4; e++)
                            if (col + e < nc) to[e] = (S)out[e];
                }
            }
        }
        if (!TOTAL && step == nchunks - 1 && !(last && w.fin)) break; // nobody needs the next state
        // ---- the next state
#pragma unroll
        for (int t = 0; t < DK / 16; t++)
#pragma unroll
            for (int nt = 0; nt < NT; nt++) R[t][nt] *= decay;
#pragma unroll
        for (int half = 0; half < HALVES; half++) {
            Frag uf[NT][COMPUTED], gf[REV ? NT : 1][COMPUTED];
#pragma unroll
            for (int nt = 0; nt < NT; nt++) {
                if (REV) {
                    split(-(eight(0, half) * r8[half][nt]), uf[nt]);
                    split(w.scale * (eight(0, half) * go8[half][nt]), gf[nt]);
                } else {
                    split(eight(1, half) * r8[half][nt], uf[nt]);
                }
            }
#pragma unroll
            for (int t = 0; t < DK / 16; t++) {
                Frag kf[IP];
                col_frag<Lds::PK>(kf, k_lds, KP, half * 32, t / 2 * 32 + t % 2 * 4, 8, lane);
#pragma unroll
                for (int nt = 0; nt < NT; nt++) R[t][nt] = product(kf, uf[nt], R[t][nt]);
                if (REV) {
                    Frag qf[IP];
                    col_frag<Lds::PK>(qf, q_lds, KP, half * 32, t / 2 * 32 + t % 2 * 4, 8, lane);
#pragma unroll
                    for (int nt = 0; nt < NT; nt++) R[t][nt] = product(qf, gf[nt], R[t][nt]);
                }
            }
        }
    }

#pragma unroll
    for (int t = 0; t < DK / 16; t++)
#pragma unroll
        for (int nt = 0; nt < NT; nt++) {
            const int col = col_of(nt);
            if (TOTAL && map) {
#pragma unroll
                for (int e = 0; e < 4; e++)
                    if (col_part + col < DK) w.maps[((slot * w.heads + h) * DK + row_of(t, e)) * (long long)DK + col_part + col] = R[t][nt][e];
            } else if (TOTAL) {
                *reinterpret_cast<f32x4 *>(total + (nt * (DK / 16) + t) * 256) = R[t][nt];
            } else if (last && w.fin) {
#pragma unroll
                for (int e = 0; e < 4; e++)
                    if (row_of(t, e) < w.dk && col < nc) w.fin[state0 + (long long)row_of(t, e) * w.dv + col] = R[t][nt][e];
            }
        }
}

// grid: slots heads parts, in one order; the parts of a head and segment run on one XCD (of 8, dealt round robin), whose L2 has what they share
template <typename S, int DK, int DV, int NW, int MODE>
__global__ __launch_bounds__(NW * 64, (DeltaLds<S, DK, DV, NW, MODE>::per_simd)) void delta_walk_kernel(DeltaArgs w)
{
    extern __shared__ __align__(16) unsigned char lds[];
    const int parts = w.parts + (MODE == MAPS ? w.map_parts : 0);
    const long long block = block_of(), group = block / (8 * parts);
    const int in = (int)(block % (8 * parts));
    const long long item = group * 8 + in % 8;
    if (item >= (long long)w.slots * w.heads) return;
    const int h = (int)(item % w.heads);
    const long long slot = item / w.heads;
    const Place at = find_place(w.seg, slot);
    if (at.seg < 0 || at.seg >= at.nseg) return; // a slot that no sequence has
    delta_walk<S, DK, DV, NW, MODE>(w, at, slot, h, in / 8, lds);
}

// Segments' maps -> incoming states, in walking order: S <- A S + B (REV: A^T D + B).  A workgroup has 16 NW columns of one head's state.
// grid: seqs heads (dv / 16 NW)
template <int DK, int DV, int NW, int NT, bool REV> __global__ __launch_bounds__(NW * 64) void delta_carry_kernel(DeltaArgs w)
{
    constexpr int CS = NT == 2 ? 8 : 4, KS = DK / 32;
    const long long block = block_of();
    const int part = (int)(block % w.parts), h = (int)(block / w.parts % w.heads);
    const long long s = block / w.parts / w.heads;
    if (s >= w.seg.seqs) return;
    long long start, len;
    span(w.seg, s, start, len);
    const long long nseg = len > 0 ? (len + w.seg.seg_len - 1) / w.seg.seg_len : 0, slot0 = first_slot(w.seg, s);
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, i = lane & 15, g = lane >> 4;
    f32x4 R[DK / 16][NT];
#pragma unroll
    for (int t = 0; t < DK / 16; t++)
#pragma unroll
        for (int nt = 0; nt < NT; nt++) {
            f32x4 x = {0, 0, 0, 0};
            const int col = part * DV + wave * NT * 16 + (i >> 2) * CS + 4 * nt + (i & 3);
            if (w.init)
#pragma unroll
                for (int e = 0; e < 4; e++) {
                    const int row = t / 2 * 32 + g * 8 + t % 2 * 4 + e;
                    if (row < w.dk && col < w.dv) x[e] = w.init[((s * w.heads + h) * (long long)w.dk + row) * w.dv + col];
                }
            R[t][nt] = x;
        }
    for (long long c = 0; c < nseg; c++) {
        const long long slot = slot0 + (REV ? nseg - 1 - c : c);
        float *const total = w.totals + ((slot * w.heads + h) * w.parts + part) * (long long)(DK * DV) + (long long)wave * NT * (DK / 16) * 256 + lane * 4;
        f32x4 B[DK / 16][NT];
        const bool more = c + 1 < nseg;
#pragma unroll
        for (int t = 0; t < DK / 16; t++)
#pragma unroll
            for (int nt = 0; nt < NT; nt++) {
                f32x4 *const at = reinterpret_cast<f32x4 *>(total + (nt * (DK / 16) + t) * 256);
                if (more) B[t][nt] = *at;
                *at = R[t][nt];
            }
        if (!more) break;
        const float *const A = w.maps + (slot * w.heads + h) * (long long)(DK * DK);
#pragma unroll
        for (int kk = 0; kk < KS; kk++) {
            Frag rf[NT][COMPUTED];
#pragma unroll
            for (int nt = 0; nt < NT; nt++) split(__builtin_shufflevector(R[2 * kk][nt], R[2 * kk + 1][nt], 0, 1, 2, 3, 4, 5, 6, 7), rf[nt]);
#pragma unroll
            for (int t = 0; t < DK / 16; t++) {
                f32x8 a;
                if (REV) {
#pragma unroll
                    for (int e = 0; e < 8; e++) a[e] = A[(kk * 32 + g * 8 + e) * DK + turned_row(t, i)];
                } else {
                    a = *reinterpret_cast<const f32x8 *>(A + turned_row(t, i) * DK + kk * 32 + g * 8);
                }
                Frag af[COMPUTED];
                split(a, af);
#pragma unroll
                for (int nt = 0; nt < NT; nt++) B[t][nt] = product(af, rf[nt], B[t][nt]);
            }
        }
#pragma unroll
        for (int t = 0; t < DK / 16; t++)
#pragma unroll
            for (int nt = 0; nt < NT; nt++) R[t][nt] = B[t][nt];
    }
}

// ---- the gradients of q, k, the decays and beta, a chunk and head a workgroup

template <typename S, int DK, int DV> struct GradLds {
    static constexpr int CH = chunk_of<S>(), IP = Parts<S>::IN, PK = DK + PITCH_PAD, SLAB = DV < 64 ? DV : 64, PV = SLAB + PITCH_PAD;
    static constexpr int NW = DK / 16 < 4 ? 4 : DK / 16;
    static constexpr int K_TILE = CH * PK * IP, V_PLANE = CH * PV, ROWS = V_PLANE * (2 * COMPUTED + 2 * IP); // U, dV in parts, dO, V
    static constexpr int JOBS = 4 * pair_blocks(CH);
    static constexpr size_t frag_bytes = JOBS * COMPUTED * 64 * sizeof(Frag), row_bytes = ROWS * sizeof(bf16);
    static constexpr size_t shared_bytes = frag_bytes > row_bytes ? frag_bytes : row_bytes;
    // + sums of q . dq by waves, betas' gradients, v . dv, and single sums
    static constexpr size_t bytes = shared_bytes + 2 * K_TILE * sizeof(bf16) + CH * sizeof(double) + (3 * CH + NW * CH + 2 * CH + 2 * NW) * sizeof(float);
};

template <typename S, int DK, int DV> __global__ __launch_bounds__((GradLds<S, DK, DV>::NW * 64)) void delta_grad_kernel(DeltaArgs w)
{
    typedef GradLds<S, DK, DV> Lds;
    constexpr int CH = Lds::CH, IP = Lds::IP, PK = Lds::PK, PV = Lds::PV, SLAB = Lds::SLAB, NW = Lds::NW, THREADS = NW * 64, KP = CH * PK, VP = CH * PV;
    constexpr int TT = CH / 16, HALVES = CH / 32, BLOCKS = pair_blocks(CH), MINE = (Lds::JOBS + NW - 1) / NW, UNITS = CH * SLAB / 8;
    extern __shared__ __align__(16) unsigned char lds[];
    Frag *const frags = reinterpret_cast<Frag *>(lds);
    bf16 *const u_lds = reinterpret_cast<bf16 *>(lds), *const dv_lds = u_lds + COMPUTED * VP, *const do_lds = dv_lds + COMPUTED * VP, *const v_lds = do_lds + IP * VP;
    bf16 *const k_lds = reinterpret_cast<bf16 *>(lds + Lds::shared_bytes), *const q_lds = k_lds + Lds::K_TILE;
    double *const b2 = reinterpret_cast<double *>(q_lds + Lds::K_TILE);
    float *const up = reinterpret_cast<float *>(b2 + CH), *const down = up + CH, *const beta = down + CH, *const qdq = beta + CH, *const gbeta = qdq + NW * CH,
                 *const vdv = gbeta + CH, *const sums = vdv + CH;

    const long long block = block_of();
    const int h = (int)(block % w.heads), kh = h / w.share;
    const long long slot = block / w.heads;
    if (slot >= w.slots) return;
    const Place at = find_place(w.chunk, slot);
    if (at.seg < 0 || at.seg >= at.nseg || at.len == 0) return;
    const long long t0 = at.seg * CH, tok = at.start + t0, record = slot * w.heads + h;
    const int n = at.len - t0 < CH ? (int)(at.len - t0) : CH;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, i = lane & 15, g = lane >> 4;
    const bool columns = wave < DK / 16; // the wave's columns of q and k: 16 wave + 0 .. 15
    const ChunkVec<CH> &vec = reinterpret_cast<const ChunkVec<CH> *>(w.vecs)[record];
    const S *const go = reinterpret_cast<const S *>(w.go) + tok * w.o_tok + h * (long long)w.dv;
    const S *const v = reinterpret_cast<const S *>(w.v) + tok * w.v_tok + h * w.v_head;
    {
        TileRows<S, DK, THREADS, CH> kx, qx;
        kx.fetch(reinterpret_cast<const S *>(w.k) + tok * w.k_tok + kh * w.k_head, w.k_tok, n, w.dk);
        qx.fetch(reinterpret_cast<const S *>(w.q) + tok * w.q_tok + kh * w.q_head, w.q_tok, n, w.dk);
        kx.template put<PK>(k_lds, n, w.dk);
        qx.template put<PK>(q_lds, n, w.dk);
    }
    if (threadIdx.x < CH) {
        b2[threadIdx.x] = vec.b2[threadIdx.x];
        up[threadIdx.x] = vec.up[threadIdx.x];
        down[threadIdx.x] = vec.down[threadIdx.x];
        beta[threadIdx.x] = vec.beta[threadIdx.x];
        gbeta[threadIdx.x] = vdv[threadIdx.x] = 0.0f;
    }

    f32x4 dq[TT], k_last[TT], k_row[TT];
#pragma unroll
    for (int t = 0; t < TT; t++) dq[t] = k_last[t] = k_row[t] = f32x4{0, 0, 0, 0};
    f32x4 job0[MINE], job1[MINE];
#pragma unroll
    for (int u = 0; u < MINE; u++) job0[u] = job1[u] = f32x4{0, 0, 0, 0};
    float ds = 0;
    // the pairs' jobs: dO . U and dV . U, each with the lane's row first (later token) and second
    auto place = [&](int job, int &kind, int &t, int &ks) {
        kind = job / BLOCKS;
        if (kind & 1) p_place<true>(job % BLOCKS, CH, t, ks);
        else p_place<false>(job % BLOCKS, CH, t, ks);
    };
    for (int slab = 0; slab < w.dv; slab += SLAB) {
        const int nc = w.dv - slab < SLAB ? w.dv - slab : SLAB;
        TileRows<S, SLAB, THREADS, CH> gx, vx;
        gx.fetch(go + slab, w.o_tok, n, nc);
        vx.fetch(v + slab, w.v_tok, n, nc);
        __syncthreads();
        gx.template put<PV>(do_lds, n, nc);
        vx.template put<PV>(v_lds, n, nc);
        __syncthreads();
        for (int u = threadIdx.x; u < (UNITS + 63) / 64 * 64; u += THREADS) { // (whole waves, for the sums over rows' lanes)
            const int row = u / (SLAB / 8), col = u % (SLAB / 8) * 8;
            const bool there = u < UNITS;
            const long long from = record * (CH * (long long)w.pitch) + (there ? row : 0) * (long long)w.pitch + slab + col;
            const f32x8 e8 = *reinterpret_cast<const f32x8 *>(w.rows_e + from), w8 = *reinterpret_cast<const f32x8 *>(w.rows_w + from);
            const float be = beta[there ? row : 0];
            Frag parts[COMPUTED], vf[IP];
            split(be * e8, parts);
#pragma unroll
            for (int p = 0; p < COMPUTED; p++)
                if (there) *reinterpret_cast<Frag *>(u_lds + p * VP + row * PV + col) = parts[p];
            const f32x8 dv8 = be * w8;
            split(dv8, parts);
#pragma unroll
            for (int p = 0; p < COMPUTED; p++)
                if (there) *reinterpret_cast<Frag *>(dv_lds + p * VP + row * PV + col) = parts[p];
            row_frag(vf, v_lds + (there ? row : 0) * PV + col, VP);
            const f32x8 v8 = widen(vf);
            float a = 0, b = 0;
#pragma unroll
            for (int e = 0; e < 8; e++) {
                a += e8[e] * w8[e];
                b += v8[e] * dv8[e];
            }
#pragma unroll
            for (int x = 1; x < SLAB / 8; x *= 2) {
                a += __shfl_xor(a, x);
                b += __shfl_xor(b, x);
            }
            if (there && col == 0) {
                gbeta[row] += a;
                vdv[row] += b;
            }
        }
        __syncthreads();
        if (columns) {
            const float *const s0 = w.kept_s + record * (DK * (long long)w.pitch) + (wave * 16 + i) * (long long)w.pitch + slab + g * 8;
            const float *const d0 = w.kept_d + record * (DK * (long long)w.pitch) + (wave * 16 + i) * (long long)w.pitch + slab + g * 8;
#pragma unroll
            for (int kk = 0; kk < SLAB / 32; kk++) {
                const f32x8 s8 = *reinterpret_cast<const f32x8 *>(s0 + kk * 32), d8 = *reinterpret_cast<const f32x8 *>(d0 + kk * 32);
#pragma unroll
                for (int e = 0; e < 8; e++) ds += s8[e] * d8[e];
                Frag sf[COMPUTED], df[COMPUTED];
                split(s8, sf);
                split(d8, df);
#pragma unroll
                for (int t = 0; t < TT; t++) {
                    const int from = (t * 16 + i) * PV + kk * 32 + g * 8;
                    Frag gf[IP], uf[COMPUTED], vf[COMPUTED];
                    row_frag(gf, do_lds + from, VP);
                    row_frag(uf, u_lds + from, VP);
                    row_frag(vf, dv_lds + from, VP);
                    dq[t] = product(sf, gf, dq[t]);
                    k_last[t] = product(df, uf, k_last[t]);
                    k_row[t] = product(sf, vf, k_row[t]);
                }
            }
        }
#pragma unroll
        for (int u = 0; u < MINE; u++) {
            const int job = wave + u * NW;
            if (job >= Lds::JOBS) continue;
            int kind, t, ks;
            place(job, kind, t, ks);
            const int mine = (t * 16 + i) * PV + g * 8, other = turned_row(2 * ks, i) * PV + g * 8;
            auto dots = [&](auto lane_parts, const bf16 *lane_rows, auto other_parts, const bf16 *others) {
#pragma unroll
                for (int kk = 0; kk < SLAB / 32; kk++) {
                    Frag a[decltype(lane_parts)::value], b0[decltype(other_parts)::value], b1[decltype(other_parts)::value];
                    row_frag(a, lane_rows + mine + kk * 32, VP);
                    row_frag(b0, others + other + kk * 32, VP);
                    row_frag(b1, others + other + 4 * PV + kk * 32, VP);
                    job0[u] = product(b0, a, job0[u]);
                    job1[u] = product(b1, a, job1[u]);
                }
            };
            typedef std::integral_constant<int, IP> In;
            typedef std::integral_constant<int, COMPUTED> Three;
            if (kind == 0) dots(In(), do_lds, Three(), u_lds);
            else if (kind == 1) dots(Three(), u_lds, In(), do_lds);
            else if (kind == 2) dots(Three(), dv_lds, Three(), u_lds);
            else dots(Three(), u_lds, Three(), dv_lds);
        }
    }
    __syncthreads();
#pragma unroll
    for (int u = 0; u < MINE; u++) {
        const int job = wave + u * NW;
        if (job >= Lds::JOBS) continue;
        int kind, t, ks;
        place(job, kind, t, ks);
        const int row = t * 16 + i, col = ks * 32 + g * 8;
        f32x8 x = __builtin_shufflevector(job0[u], job1[u], 0, 1, 2, 3, 4, 5, 6, 7);
#pragma unroll
        for (int e = 0; e < 8; e++) {
            const int c = col + e, later = kind & 1 ? c : row, earlier = kind & 1 ? row : c;
            const bool there = kind < 2 ? later >= earlier : later > earlier;
            x[e] = there ? (kind < 2 ? w.scale : -1.0f) * x[e] * power2(b2[later] - b2[earlier]) : 0.0f;
        }
        Frag parts[COMPUTED];
        split(x, parts);
#pragma unroll
        for (int p = 0; p < COMPUTED; p++) frags[(job * COMPUTED + p) * 64 + lane] = parts[p];
    }
    const int col0 = wave * 16;
    float kdk = 0;
    auto four = [&](const bf16 *tile, int t) { // the lane's four entries of a row
        f32x4 x = {0, 0, 0, 0};
        const bf16 *const p = tile + (t * 16 + i) * PK + col0 + g * 4;
#pragma unroll
        for (int u = IP - 1; u >= 0; u--) x += __builtin_convertvector(*reinterpret_cast<const bf16x4 *>(p + u * KP), f32x4);
        return x;
    };
    if (columns)
#pragma unroll
        for (int t = 0; t < TT; t++) {
            const int row = t * 16 + i;
            dq[t] *= w.scale * up[row];
            k_last[t] *= down[row];
            const f32x4 k4 = four(k_lds, t);
            kdk += k4[0] * k_last[t][0] + k4[1] * k_last[t][1] + k4[2] * k_last[t][2] + k4[3] * k_last[t][3];
            k_row[t] = k_last[t] - up[row] * k_row[t];
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
    if (columns) {
#pragma unroll
        for (int half = 0; half < HALVES; half++) {
            Frag kf[IP], qf[IP];
            col_frag<PK>(kf, k_lds, KP, half * 32, col0, 4, lane);
            col_frag<PK>(qf, q_lds, KP, half * 32, col0, 4, lane);
#pragma unroll
            for (int t = 0; t < TT; t++) {
                auto frag = [&](int kind, int at, Frag (&x)[COMPUTED]) {
#pragma unroll
                    for (int p = 0; p < COMPUTED; p++) x[p] = frags[((kind * BLOCKS + at) * COMPUTED + p) * 64 + lane];
                };
                Frag x[COMPUTED];
                if (p_has<false>(t, half)) {
                    frag(0, p_block<false>(t, half, CH), x);
                    dq[t] = product(kf, x, dq[t]);
                    frag(2, p_block<false>(t, half, CH), x);
                    k_row[t] = product(kf, x, k_row[t]);
                }
                if (p_has<true>(t, half)) {
                    frag(1, p_block<true>(t, half, CH), x);
                    k_row[t] = product(qf, x, k_row[t]);
                    frag(3, p_block<true>(t, half, CH), x);
                    k_row[t] = product(kf, x, k_row[t]);
                }
            }
        }
#pragma unroll
        for (int t = 0; t < TT; t++) {
            const int row = t * 16 + i, col = col0 + g * 4;
            const f32x4 q4 = four(q_lds, t);
            float a = q4[0] * dq[t][0] + q4[1] * dq[t][1] + q4[2] * dq[t][2] + q4[3] * dq[t][3];
            a += __shfl_xor(a, 16);
            a += __shfl_xor(a, 32);
            if (g == 0) qdq[wave * CH + row] = a;
            if (row < n) {
                const long long to = ((tok + row) * w.heads + h) * (long long)w.dk + col;
                auto store = [&](void *out, const f32x4 &x) {
                    float y[4] = {x[0], x[1], x[2], x[3]};
                    if (col + 4 <= w.dk) {
                        if (w.grad_float) store_floats_unaligned<float, 4>(reinterpret_cast<float *>(out) + to, y);
                        else store_floats_unaligned<S, 4>(reinterpret_cast<S *>(out) + to, y);
                    } else {
#pragma unroll
                        for (int e = 0; e < 4; e++)
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
    __syncthreads();
    if (wave == 0) { // sums towards the chunk's end; a token's decay has what all later ones and the next state make of it
        double s = 0;
        if (lane < CH) {
            s = -(double)vdv[lane];
            for (int x = 0; x < DK / 16; x++) s += qdq[x * CH + lane];
        }
        if (lane == n - 1) {
            double end = 0, d = 0;
            for (int x = 0; x < DK / 16; x++) {
                end += sums[x];
                d += sums[NW + x];
            }
            s += end + vec.whole * d;
        }
        if (lane >= n) s = 0;
#pragma unroll
        for (int step = 1; step < 64; step *= 2) {
            const double x = __shfl_down(s, step);
            if (lane + step < 64) s += x;
        }
        if (lane < n) {
            const long long to = (tok + lane) * w.heads + h;
            w.g_beta[to] = gbeta[lane];
            w.g_log_decay[to] = power2(log2_of(w.log_decay[to])) == 0.0f ? 0.0f : (float)s; // what is forgotten whole has no slope
        }
    }
}

// ---- launches

template <typename S, int DK, int DV, int NW, int MODE> static int launch_delta_walk_sized(goom_ctx *ctx, DeltaArgs w, long long slots, const char *label)
{
    w.slots = (unsigned)slots;
    const int parts = w.parts + (MODE == MAPS ? w.map_parts : 0);
    auto *kernel = delta_walk_kernel<S, DK, DV, NW, MODE>;
    constexpr size_t bytes = DeltaLds<S, DK, DV, NW, MODE>::bytes;
    static_assert(bytes <= (160 << 10), "LDS of a CU");
    static std::atomic<unsigned long long> done{0};
    if (int st = allow_lds(ctx, reinterpret_cast<const void *>(kernel), bytes, done)) return st;
    goom::prof_begin(ctx, label);
    kernel<<<grid_of((slots * w.heads + 7) / 8 * 8 * parts, NW * 64), NW * 64, bytes, ctx->stream>>>(w);
    goom::prof_end(ctx);
    return goom::check_hip(ctx, hipGetLastError(), label);
}

// columns of a workgroup, and its waves
constexpr int delta_columns(int dv) { return dv <= 32 ? 32 : 64; }
constexpr int delta_rows(int dk) { return dk <= 32 ? 32 : dk <= 64 ? 64 : 128; }

template <typename F> static int with_delta(int dk, int dv, F f)
{
    auto columns = [&](auto rows) {
        if (dv <= 32) return f(rows, std::integral_constant<int, 32>(), std::integral_constant<int, 2>());
        return f(rows, std::integral_constant<int, 64>(), std::integral_constant<int, 4>());
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
    return with_delta(w.dk, 64, [&](auto rows, auto, auto) {
        constexpr int DK = decltype(rows)::value;
        auto *kernel = within_kernel<S, DK>;
        static std::atomic<unsigned long long> done{0};
        if (int st = allow_lds(ctx, reinterpret_cast<const void *>(kernel), WithinLds<S, DK>::bytes, done)) return st;
        goom::prof_begin(ctx, "gated delta rule: within chunks");
        kernel<<<grid_of(slots * (w.heads / w.share), 256), 256, WithinLds<S, DK>::bytes, ctx->stream>>>(w);
        goom::prof_end(ctx);
        return goom::check_hip(ctx, hipGetLastError(), "gated delta rule: within chunks");
    });
}

template <typename S, int FIRST, int SECOND, int THIRD> int launch_delta_walk_typed(goom_ctx *ctx, const DeltaArgs &w, int mode, long long slots, const char *label)
{
    return with_delta(w.dk, w.dv, [&](auto rows, auto cols, auto waves) {
        constexpr int DK = decltype(rows)::value, DV = decltype(cols)::value, NW = decltype(waves)::value;
        if (mode == FIRST) return launch_delta_walk_sized<S, DK, DV, NW, FIRST>(ctx, w, slots, label);
        if (mode == SECOND) return launch_delta_walk_sized<S, DK, DV, NW, SECOND>(ctx, w, slots, label);
        return launch_delta_walk_sized<S, DK, DV, NW, THIRD>(ctx, w, slots, label);
    });
}

template <typename S> int launch_delta_gradients_typed(goom_ctx *ctx, DeltaArgs w, long long slots)
{
    w.slots = (unsigned)slots;
    auto run = [&](auto rows, auto cols) {
        constexpr int DK = decltype(rows)::value, DV = decltype(cols)::value;
        typedef GradLds<S, DK, DV> Lds;
        static_assert(Lds::bytes <= (160 << 10), "LDS of a CU");
        auto *kernel = delta_grad_kernel<S, DK, DV>;
        static std::atomic<unsigned long long> done{0};
        if (int st = allow_lds(ctx, reinterpret_cast<const void *>(kernel), Lds::bytes, done)) return st;
        goom::prof_begin(ctx, "gated delta rule: gradients within chunks");
        kernel<<<grid_of(slots * w.heads, Lds::NW * 64), Lds::NW * 64, Lds::bytes, ctx->stream>>>(w);
        goom::prof_end(ctx);
        return goom::check_hip(ctx, hipGetLastError(), "gated delta rule: gradients");
    };
    return with_delta(w.dk, w.dv, [&](auto rows, auto cols, auto) { return run(rows, cols); });
}

} // namespace goom_layer
