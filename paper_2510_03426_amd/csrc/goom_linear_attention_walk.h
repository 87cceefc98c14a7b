#pragma once

// Linear attention with a decay for each head: forward, single tokens, backward.
//
// One kernel, the walk, computes for rows a_i, b_j (of ka entries) and c_j (of nc entries), a head's decay g and a state R
//     y_i = p sum_{j <= i} g^(i-j) (a_i . b_j) c_j + w g^i' a_i R
// 64 tokens (a chunk) at a time: with the pairs inside a chunk as a masked 64 x 64 matrix P, what precedes the chunk as the
// state R (already decayed to the chunk's first token, i' = 0), and
//     R <- g^n R + u sum_j g^(n-j') b_j c_j^T
// for the next.  The forward pass is one walk (a, b, c = q, k, v); the backward pass is three of the same kind:
//     grad_q: grad_o, v, k forwards;     grad_k: v, grad_o, q and grad_v: k, q, grad_o backwards in time,
// where j' counts from the end and R starts as the final state's gradient.  Nothing but inputs, outputs and a few states
// touches memory.  Where there are fewer walks than the chip holds at once, every sequence is cut into segments: segment totals
// (the walk without outputs), carries, then all segments at once.
//
// Measured (bfloat16; a copy reaches 5.09 TB/s): 65,536 tokens of 16 heads of 64: totals 71 us (3.8 TB/s), carries 10, walk 141
// (3.8 TB/s); 8 x 4096 tokens of 16 heads of 128: 69 + 11 + 177 us, the three walks of the backward pass 592.  What bounds it: no one
// unit.  Of a wave's 19,100 cycles a chunk (950 other vector and 236 matrix instructions, two waves a SIMD) 25 % issue vector
// instructions, in 31 % it is ready and waits to issue, in 34 % it waits for LDS, memory and barriers; the matrix unit is busy for 39 %.
//
// A workgroup walks one head of one segment.  Each wave owns nc / NW columns of the state, which stay in its registers as
// accumulators of the matrix instruction for the whole walk; the rows of the tiles are numbered such that a lane's
// accumulator entries are eight consecutive ones of the contraction (rows or tokens), so that the state and P turn into
// operands of the next product without moving between lanes.  P is shared out over the waves by rows and passed through LDS.
#include <atomic>

#include "goom_real.h"

namespace goom_layer {

constexpr int CHUNK = 64; // tokens; the pairs of a chunk cost 64 (ka + nc) multiplications a token, the state 2 ka nc

struct WalkRole {
    const void *a, *b, *c;
    void *y;                 // NULL in walks without outputs
    long long a_tok, a_head, b_tok, b_head, c_tok, c_head, y_tok, y_head; // elements
    int a_group, b_group, c_group; // heads that share a row set: 1, or heads / kv_heads
    int ka, nc;
    int reverse;
    int y_float;             // y holds floats, whatever the type
    float p_scale, w_scale, u_scale;
    const float *init;       // NULL or states [seqs][heads][.][.]
    float *fin;              // NULL or states, written after the last token
    int state_row, state_col; // elements between entries of init and fin along ka and along nc
    float *totals;           // [slots][heads][state registers]; NULL: one segment a sequence
};

struct WalkArgs {
    WalkRole role[3];
    const float *log_decay;
    const int64_t *offsets;
    long long tokens, seqs, seq_len, seg_len, segs; // without offsets: seq_len tokens and segs segments a sequence
    int heads, roles, parts; // parts: column parts of DV columns
    unsigned slots;
};

// ---- the sequence and segment of a workgroup.  With offsets, sequence s has the slots from floor(start / seg_len) + s on:
// at least one, and as many as it has segments, without a pass over the lengths.
struct Place { long long seq, seg, nseg, start, len; };

template <typename W> __device__ inline void span(const W &w, long long s, long long &start, long long &len)
{
    if (w.offsets) {
        long long b = w.offsets[s], e = w.offsets[s + 1];
        b = b < 0 ? 0 : b > w.tokens ? w.tokens : b;
        e = e < b ? b : e > w.tokens ? w.tokens : e;
        start = b;
        len = e - b;
    } else {
        start = s * w.seq_len;
        len = w.seq_len;
    }
}

template <typename W> __device__ inline long long first_slot(const W &w, long long s)
{
    if (!w.offsets) return s * w.segs;
    long long start, len;
    span(w, s, start, len);
    return start / w.seg_len + s;
}

template <typename W> __device__ inline Place find_place(const W &w, long long slot)
{
    Place p;
    if (!w.offsets) {
        p.seq = slot / w.segs;
        p.seg = slot - p.seq * w.segs;
    } else { // the last sequence whose first slot is at most `slot`: 64 probes at a time
        long long lo = 0, hi = w.seqs;
        const int lane = threadIdx.x & 63;
        while (hi - lo > 1) {
            const long long step = (hi - lo + 63) / 64, at = lo + lane * step;
            const unsigned long long m = __ballot(at < hi && first_slot(w, at < hi ? at : lo) <= slot);
            const int k = __popcll(m);
            lo += (k > 0 ? k - 1 : 0) * step;
            hi = lo + step < hi ? lo + step : hi;
        }
        p.seq = lo;
        p.seg = slot - first_slot(w, lo);
    }
    span(w, p.seq, p.start, p.len);
    p.nseg = (p.len + w.seg_len - 1) / w.seg_len;
    if (p.nseg < 1) p.nseg = 1;
    return p;
}

// log2 of a decay.  2^-200 is zero as a float already: finite, so that g^0 = 1 for a decay of zero too (a NaN stays one)
__device__ inline float log2_decay(float log_decay)
{
    const float g2 = log_decay * 1.44269504088896341f;
    return g2 < -200.0f ? -200.0f : g2;
}
// g^x for whole x >= 0
__device__ inline float decay_power(float g2, int x) { return __builtin_amdgcn_exp2f(g2 * (float)x); }

// ---- operands: eight consecutive entries of the contraction per lane (lane / 16 picks which eight of 32), as sums of bf16
// parts, each 8 bits further down.  Inputs are held exactly: one part for bfloat16, two for halves (11 bits, and products and
// states of halves may leave their range), three for floats.  Computed operands (P, the state where outputs are formed from it, the
// decayed rows that enter it) are floats, held in three parts whatever the type: 24 bits, so that outputs are off by no more than sums of
// floats are.  (Two parts, 16 bits: 0.22 % of the bfloat16 outputs of 8 x 4096 tokens of heads of 128 were a neighbour of the
// rounded exact value, for 0.015 % and for 0.018 % of an evaluation in floats; both directions took 12 % less time.)  Of a product of
// parts i and j those with i + j up to two matter.  (On floats' own matrix instruction a product takes eight instructions of
// 32 cycles; six of 16 cycles here.)
typedef bf16x8 Frag;
template <typename S> struct Parts;
template <> struct Parts<bf16> { static constexpr int IN = 1; };
template <> struct Parts<f16> { static constexpr int IN = 2; };
template <> struct Parts<float> { static constexpr int IN = 3; };
constexpr int COMPUTED = 3;
constexpr int PITCH_PAD = 8;

template <int NA, int NB> __device__ inline f32x4 product(const Frag (&a)[NA], const Frag (&b)[NB], f32x4 c)
{
#pragma unroll
    for (int i = 0; i < NA; i++)
#pragma unroll
        for (int j = 0; j < NB; j++)
            if (i + j < 3) c = __builtin_amdgcn_mfma_f32_16x16x32_bf16(a[i], b[j], c, 0, 0, 0);
    return c;
}

// Pairs share a word: the hardware converts two floats at once, and each half widens in one instruction.
__device__ inline unsigned pack2(float a, float b) { return __builtin_bit_cast(unsigned, __builtin_convertvector((f32x2){a, b}, bf16x2)); }
__device__ inline float low_half(unsigned u) { return __builtin_bit_cast(float, u << 16); }
__device__ inline float high_half(unsigned u) { return __builtin_bit_cast(float, u & 0xffff0000u); }

template <int N> __device__ inline void split(f32x8 x, bf16x8 (&p)[N])
{
    typedef unsigned u32x4 __attribute__((ext_vector_type(4)));
#pragma unroll
    for (int i = 0; i < N; i++) {
        u32x4 w;
#pragma unroll
        for (int e = 0; e < 4; e++) {
            w[e] = pack2(x[2 * e], x[2 * e + 1]);
            if (i + 1 < N) {
                x[2 * e] -= low_half(w[e]);
                x[2 * e + 1] -= high_half(w[e]);
            }
        }
        p[i] = __builtin_bit_cast(bf16x8, w);
    }
}

__device__ inline f32x8 widen(bf16x8 x)
{
    typedef unsigned u32x4 __attribute__((ext_vector_type(4)));
    const u32x4 w = __builtin_bit_cast(u32x4, x);
    return f32x8{low_half(w[0]), high_half(w[0]), low_half(w[1]), high_half(w[1]), low_half(w[2]), high_half(w[2]), low_half(w[3]), high_half(w[3])};
}
template <int N> __device__ inline f32x8 widen(const Frag (&p)[N])
{
    f32x8 x = widen(p[N - 1]);
#pragma unroll
    for (int i = N - 2; i >= 0; i--) x += widen(p[i]);
    return x;
}

// eight entries of one row; `plane` elements between the parts
template <int N> __device__ inline void row_frag(Frag (&x)[N], const bf16 *p, int plane)
{
#pragma unroll
    for (int k = 0; k < N; k++) x[k] = *reinterpret_cast<const Frag *>(p + k * plane);
}

// rows t0 + 8 (lane / 16) + 0 .. 7 of one column: column c0 + (i / 4) cs + i % 4 for i = lane % 16
template <int PITCH, int N> __device__ inline void col_frag(Frag (&x)[N], const bf16 *tile, int plane, int t0, int c0, int cs, int lane)
{
    // the transposing read: of each 16 lanes, lane s gives the address of four columns of row s / 4, and lane i gets
    // the four rows of column i
    const int s = lane & 15, row = t0 + (lane >> 4) * 8 + (s >> 2), col = c0 + (s & 3) * cs;
    typedef __attribute__((address_space(3))) s16x4 *lds;
#pragma unroll
    for (int k = 0; k < N; k++) {
        const bf16 *const p = tile + k * plane + row * PITCH + col;
        const s16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds)p), hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds)(p + 4 * PITCH));
        x[k] = __builtin_bit_cast(Frag, __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7));
    }
}

// eight elements of a type into parts
__device__ inline void split_in(bf16x8 v, Frag (&p)[1]) { p[0] = v; }
__device__ inline void split_in(f16x8 v, Frag (&p)[2]) { split(__builtin_convertvector(v, f32x8), p); }
__device__ inline void split_in(f32x8 v, Frag (&p)[3]) { split(v, p); }

// Rows 0 .. n-1 of `d` entries, on their way from memory into a tile of CH rows of D entries with zeros elsewhere: fetched into
// registers, all loads in flight at once (rows and columns that are not there are read from ones that are), and put into LDS
// where the walk gets to them.  A thread's units of eight entries lie in one column, STEP rows apart.
template <typename S, int D, int THREADS, int CH> struct TileRows {
    typedef typename Vec<S, 8>::type SV;
    static constexpr int UNITS = CH * D / 8, N = (UNITS + THREADS - 1) / THREADS, STEP = THREADS / (D / 8);
    static_assert(THREADS % (D / 8) == 0, "units of a thread in one column");
    SV x[N];

    __device__ static inline int row0() { return threadIdx.x / (D / 8); }
    __device__ static inline int col0() { return threadIdx.x % (D / 8) * 8; }

    // Units are read whole, whatever their alignment; the last one of a row whose entries make no whole units from eight entries
    // before the row's end, and put() moves it into place.  Rows of fewer than eight entries: element by element.
    __device__ static inline int shift(int d) { return -d & 7; }
    __device__ inline void fetch(const S *src, long long stride, int n, int d)
    {
        // byte offsets within the chunk, 32 bits (checked by the host)
        const unsigned bytes = (unsigned)stride * sizeof(S), first = col0() + 8 <= d ? col0() : col0() < d && d >= 8 ? d - 8 : 0, col = first * sizeof(S);
        const char *const p = reinterpret_cast<const char *>(src);
        if (d >= 8) {
            if (n == CH) {
                const unsigned at = row0() * bytes + col, step = STEP * bytes;
#pragma unroll
                for (int k = 0; k < N; k++) {
                    x[k] = SV{}; // (of threads without a row: what is split must be some number)
                    if (UNITS % THREADS == 0 || row0() + k * STEP < CH) x[k] = load_unaligned<S, 8>(reinterpret_cast<const S *>(p + (at + k * step)));
                }
            } else {
#pragma unroll
                for (int k = 0; k < N; k++) {
                    const int row = row0() + k * STEP;
                    x[k] = load_unaligned<S, 8>(reinterpret_cast<const S *>(p + ((row < n ? row : n - 1) * bytes + col)));
                }
            }
        } else {
#pragma unroll
            for (int k = 0; k < N; k++) {
                const int row = row0() + k * STEP;
                const S *const q = reinterpret_cast<const S *>(p + (row < n ? row : n - 1) * bytes);
#pragma unroll
                for (int c = 0; c < 8; c++) x[k][c] = c < d ? q[c < d ? c : 0] : (S)0.0f;
            }
        }
    }
    template <int PITCH> __device__ inline void put(bf16 *tile, int n, int d) const
    {
        if (n == CH && d == D) put_units<PITCH, false, false>(tile, n, d);
        else if (d < 8 || !shift(d)) put_units<PITCH, true, false>(tile, n, d);
        else put_units<PITCH, true, true>(tile, n, d);
    }
    // unit k as it belongs into the tile, in one way for all sizes
    __device__ inline SV unit(int k, int n, int d) const
    {
        const int col = col0(), move = d >= 8 && col + 8 > d ? shift(d) : 0;
        SV v = x[k];
        if (d & 7) { // some lanes move
            const SV z = {};
            if (move & 4) v = __builtin_shufflevector(v, z, 4, 5, 6, 7, 8, 9, 10, 11);
            if (move & 2) v = __builtin_shufflevector(v, z, 2, 3, 4, 5, 6, 7, 8, 9);
            if (move & 1) v = __builtin_shufflevector(v, z, 1, 2, 3, 4, 5, 6, 7, 8);
        }
        if (col >= d || row0() + k * STEP >= n) v = SV{};
        return v;
    }
    // put() without its three ways, where the choice would be all but free: a kernel of the gated delta rule has up to nine of these
    template <int PITCH> __device__ inline void put_any(bf16 *tile, int n, int d) const
    {
#pragma unroll
        for (int k = 0; k < N; k++) {
            const int row = row0() + k * STEP;
            Frag p[Parts<S>::IN];
            split_in(unit(k, n, d), p);
            if (UNITS % THREADS == 0 || row < CH)
#pragma unroll
                for (int q = 0; q < Parts<S>::IN; q++) *reinterpret_cast<Frag *>(tile + (q * CH + row) * PITCH + col0()) = p[q];
        }
    }
    // CUT: rows or columns may be missing; MOVE: the rows' last units are to be moved
    template <int PITCH, bool CUT, bool MOVE> __device__ inline void put_units(bf16 *tile, int n, int d) const
    {
        const bool there = col0() < d;
        bf16 *const to0 = tile + row0() * PITCH + col0();
#pragma unroll
        for (int k = 0; k < N; k++) {
            SV v = x[k];
            if (MOVE) {
                const SV z = {};
                SV w = v;
                if (shift(d) & 4) w = __builtin_shufflevector(w, z, 4, 5, 6, 7, 8, 9, 10, 11);
                if (shift(d) & 2) w = __builtin_shufflevector(w, z, 2, 3, 4, 5, 6, 7, 8, 9);
                if (shift(d) & 1) w = __builtin_shufflevector(w, z, 1, 2, 3, 4, 5, 6, 7, 8);
                if (col0() + 8 > d) v = w;
            }
            if (CUT && (!there || row0() + k * STEP >= n)) v = SV{};
            Frag p[Parts<S>::IN];
            split_in(v, p);
#pragma unroll
            for (int q = 0; q < Parts<S>::IN; q++)
                if (UNITS % THREADS == 0 || row0() + k * STEP < CH) *reinterpret_cast<Frag *>(to0 + (q * CH + k * STEP) * PITCH) = p[q];
        }
    }
};

// Powers of the decay in LDS, written once a walk: formed in every chunk anew they were a quarter of its instructions.  PAIRS: the
// weights of eight neighbouring j (zeros where there is no pair) for each i - j of the first of them
constexpr int PAIRS = 96;

template <typename S, int DK, int DV, int NW, bool OUT> struct WalkLds {
    // Tokens of a step.  Inputs of two and three parts: half, so that two workgroups share a CU (20,700 cycles a chunk of 64 with one).
    // Where only the state is wanted, twice as many: more loads in flight for each barrier.
    static constexpr int CH = (Parts<S>::IN > 1 ? CHUNK / 2 : CHUNK) * (OUT ? 1 : 2);
    static constexpr int P_BLOCKS = CH == CHUNK ? 6 : 2; // 16 x 32 blocks of P that have pairs in them
    static constexpr int PK = DK + PITCH_PAD, PV = DV + PITCH_PAD;
    static constexpr int K_TILE = CH * PK * Parts<S>::IN, V_TILE = CH * PV * Parts<S>::IN; // elements
    static constexpr int P_FRAGS = OUT ? P_BLOCKS * COMPUTED * 64 : 0;
    static constexpr int WEIGHTS = CH + (OUT ? CH + 8 * PAIRS : 0); // floats
    static constexpr size_t bytes = (K_TILE * (OUT ? 2 : 1) + V_TILE) * sizeof(bf16) + P_FRAGS * sizeof(Frag) + WEIGHTS * sizeof(float);
    // workgroups of a CU: as many as its LDS holds, and no more than leave their waves the registers for the state (DK DV / 64 NW
    // a lane), the outputs and the rows on their way: three waves a SIMD with 168 each, or two with 256
    static constexpr int waves = DK * DV / (64 * NW) > 16 ? 2 : 3;
    static constexpr int fit = (int)((160 << 10) / bytes), most = waves * 4 / NW;
    static constexpr int resident = fit < 1 ? 1 : fit > most ? most : fit;
    static constexpr int per_simd = (resident * NW + 3) / 4;
};

// the blocks of P with pairs in them: of rows 16 it on and columns 32 ks on, in order; and back
template <bool REV> __device__ constexpr bool p_has(int it, int ks) { return REV ? ks >= it / 2 : ks <= it / 2; }
template <bool REV> __device__ constexpr int p_block(int it, int ks, int ch)
{
    return ch == 32 ? it : REV ? (it < 2 ? it * 2 + ks : it + 2) : (it < 2 ? it : it * 2 - 2 + ks);
}
template <bool REV> __device__ inline void p_place(int block, int ch, int &it, int &ks)
{
    if (ch == 32) { it = block; ks = 0; }
    else if (REV) { it = block < 4 ? block / 2 : block - 2; ks = block < 4 ? block % 2 : 1; }
    else { it = block < 2 ? block : block / 2 + 1; ks = block < 2 ? 0 : block % 2; }
}

// DK, DV: ka and nc (of one of `parts` column parts), padded; NW waves of NT tiles of 16 columns each
template <typename S, int DK, int DV, int NW, bool OUT, bool REV>
__device__ inline void walk(const WalkArgs &w, const WalkRole &r, const Place &at, long long slot, int h, int part, unsigned char *lds)
{
    typedef WalkLds<S, DK, DV, NW, OUT> Lds;
    constexpr int THREADS = NW * 64, NT = DV / 16 / NW, KS = DK / 32, CS = NT == 2 ? 8 : 4;
    constexpr int IP = Parts<S>::IN, OP = COMPUTED;
    constexpr int CH = Lds::CH, KP = CH * Lds::PK, VP = CH * Lds::PV; // tokens of a step, elements from part to part
    static_assert(NT == 1 || NT == 2, "a wave has one or two column tiles");
    f32x8 *const pair_weights = reinterpret_cast<f32x8 *>(lds);                      // (OUT)
    float *const row_weights = reinterpret_cast<float *>(lds) + (OUT ? 8 * PAIRS : 0); // (OUT) w g^x
    float *const state_weights = row_weights + (OUT ? CH : 0);                         // u g^(CH - j')
    Frag *const p_lds = reinterpret_cast<Frag *>(reinterpret_cast<float *>(lds) + Lds::WEIGHTS);
    bf16 *const b_lds = reinterpret_cast<bf16 *>(p_lds + Lds::P_FRAGS);
    bf16 *const c_lds = b_lds + Lds::K_TILE;
    bf16 *const a_lds = c_lds + Lds::V_TILE;

    const bool last = REV ? at.seg == 0 : at.seg == at.nseg - 1; // in walking order
    if (!OUT && last) return;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, i = lane & 15, g = lane >> 4;
    const float g2 = log2_decay(w.log_decay[h]);
    const int col0 = wave * NT * 16; // the wave's columns: col0 + (i / 4) CS + 4 nt + i % 4

    // ---- the incoming state
    f32x4 R[DK / 16][NT];
    float *const total = r.totals ? r.totals + ((slot * w.heads + h) * w.parts + part) * (long long)(DK * DV) + (long long)wave * NT * (DK / 16) * 256 + lane * 4 : nullptr;
    const int nc = r.nc - part * DV < DV ? r.nc - part * DV : DV;
    const long long state0 = (at.seq * w.heads + h) * (long long)r.ka * r.nc + (long long)part * DV * r.state_col;
    const bool empty = at.len == 0;
#pragma unroll
    for (int t = 0; t < DK / 16; t++)
#pragma unroll
        for (int nt = 0; nt < NT; nt++) {
            f32x4 x = {0, 0, 0, 0};
            if (OUT && total && !empty) {
                x = *reinterpret_cast<const f32x4 *>(total + (nt * (DK / 16) + t) * 256);
            } else if (OUT && r.init) {
                const float scale = REV || empty ? 1.0f : decay_power(g2, 1);
                const int col = col0 + (i >> 2) * CS + 4 * nt + (i & 3);
#pragma unroll
                for (int e = 0; e < 4; e++) {
                    const int row = t / 2 * 32 + g * 8 + t % 2 * 4 + e;
                    if (row < r.ka && col < nc) x[e] = scale * r.init[state0 + (long long)row * r.state_row + (long long)col * r.state_col];
                }
            }
            R[t][nt] = x;
        }

    const S *const a = reinterpret_cast<const S *>(r.a) + at.start * r.a_tok + h / r.a_group * r.a_head;
    const S *const b = reinterpret_cast<const S *>(r.b) + at.start * r.b_tok + h / r.b_group * r.b_head;
    const S *const c = reinterpret_cast<const S *>(r.c) + at.start * r.c_tok + h / r.c_group * r.c_head + part * DV;
    const long long seg0 = at.seg * w.seg_len, seg1 = seg0 + w.seg_len < at.len ? seg0 + w.seg_len : at.len;
    const int nchunks = (int)((seg1 - seg0 + CH - 1) / CH);
    TileRows<S, DK, THREADS, CH> ax, bx;
    TileRows<S, DV, THREADS, CH> cx;
    auto chunk_at = [&](int step) { return seg0 + (long long)(REV ? nchunks - 1 - step : step) * CH; };
    auto chunk_rows = [&](long long t0) { return seg1 - t0 < CH ? (int)(seg1 - t0) : CH; };
    auto fetch = [&](int step) {
        const long long t0 = chunk_at(step);
        const int n = chunk_rows(t0);
        if (OUT) ax.fetch(a + t0 * r.a_tok, r.a_tok, n, r.ka);
        bx.fetch(b + t0 * r.b_tok, r.b_tok, n, r.ka);
        cx.fetch(c + t0 * r.c_tok, r.c_tok, n, nc);
    };
    if (nchunks > 0) fetch(0);
    // Backwards the first chunk may be short.  The rows that are not there are zeros, and so their weights must be finite: those of a growing
    // decay, which may be out of range, are zeros in that chunk.  (Forwards a chunk's rows meet no later ones, and the next state's weights are formed for it.)
    auto weigh = [&](int rows) {
        if (OUT)
            for (int u = threadIdx.x; u < 8 * PAIRS; u += THREADS) {
                const int first = REV ? 31 - u / 8 : u / 8 - 32, age = REV ? u % 8 - first : first - u % 8; // i - j of the eight's first j
                reinterpret_cast<float *>(pair_weights)[u] = age >= 0 && age < rows ? r.p_scale * decay_power(g2, age) : 0.0f;
            }
        for (int x = threadIdx.x; x < CH; x += THREADS) state_weights[x] = !REV || x < rows ? r.u_scale * decay_power(g2, REV ? x + 1 : CH - x) : 0.0f;
    };
    if (OUT)
        for (int x = threadIdx.x; x < CH; x += THREADS) row_weights[x] = r.w_scale * decay_power(g2, x);
    const bool cut = REV && g2 > 0.0f && nchunks > 0 && chunk_rows(chunk_at(0)) < CH;
    weigh(cut ? chunk_rows(chunk_at(0)) : CH);
    for (int step = 0; step < nchunks; step++) {
        const long long t0 = chunk_at(step);
        const int n = chunk_rows(t0);
        __syncthreads();
        if (REV && step == 1 && cut) weigh(CH);
        if (OUT) ax.template put<Lds::PK>(a_lds, n, r.ka);
        bx.template put<Lds::PK>(b_lds, n, r.ka);
        cx.template put<Lds::PV>(c_lds, n, nc);
        __syncthreads();
        if (step + 1 < nchunks) fetch(step + 1); // while this chunk is worked on

        if (OUT) {
            // ---- P, transposed (accumulator columns are the rows i, so that a lane's entries are consecutive j)
            for (int block = wave; block < Lds::P_BLOCKS; block += NW) {
                int it, ks;
                p_place<REV>(block, CH, it, ks);
                f32x4 p0 = {0, 0, 0, 0}, p1 = {0, 0, 0, 0};
                const bf16 *const arow = a_lds + (it * 16 + i) * Lds::PK + g * 8;
                const bf16 *const brow = b_lds + (ks * 32 + (i >> 2) * 8 + (i & 3)) * Lds::PK + g * 8;
#pragma unroll
                for (int kk = 0; kk < KS; kk++) {
                    Frag af[IP], b0[IP], b1[IP];
                    row_frag(af, arow + kk * 32, KP);
                    row_frag(b0, brow + kk * 32, KP);
                    row_frag(b1, brow + 4 * Lds::PK + kk * 32, KP);
                    p0 = product(b0, af, p0);
                    p1 = product(b1, af, p1);
                }
                const int first = it * 16 + i - ks * 32 - g * 8; // i - j of the lane's first j
                const f32x8 x = __builtin_shufflevector(p0, p1, 0, 1, 2, 3, 4, 5, 6, 7) * pair_weights[REV ? 31 - first : first + 32];
                Frag parts[OP];
                split(x, parts);
#pragma unroll
                for (int q = 0; q < OP; q++) p_lds[(block * OP + q) * 64 + lane] = parts[q];
            }
            __syncthreads();
        }

        Frag cf[CH / 32][NT][IP];
        auto load_columns = [&] {
#pragma unroll
            for (int ks = 0; ks < CH / 32; ks++)
#pragma unroll
                for (int nt = 0; nt < NT; nt++) col_frag<Lds::PV>(cf[ks][nt], c_lds, VP, ks * 32, col0 + 4 * nt, CS, lane);
        };
        if (!OUT) load_columns();
        if (OUT) {
            // ---- what the state gives to each row, then the pairs; transposed: a lane has consecutive columns of row i
            f32x4 y[CH / 16][NT];
#pragma unroll
            for (int it = 0; it < CH / 16; it++)
#pragma unroll
                for (int nt = 0; nt < NT; nt++) y[it][nt] = f32x4{0, 0, 0, 0};
            if (step > 0 || total || r.init) {
                // operands are read one step ahead of their products, and no further: registers are what the walk is short of
                constexpr int AHEAD = IP == 1 ? 2 : 1;
                Frag af[AHEAD][CH / 16][IP];
                const bf16 *const a0 = a_lds + i * Lds::PK + g * 8;
                auto load_rows = [&](int kk) {
#pragma unroll
                    for (int it = 0; it < CH / 16; it++) row_frag(af[kk % AHEAD][it], a0 + it * 16 * Lds::PK + kk * 32, KP);
                };
                if (AHEAD > 1) load_rows(0);
#pragma unroll
                for (int kk = 0; kk < KS; kk++) {
                    if (AHEAD == 1) load_rows(kk);
                    else if (kk + 1 < KS) load_rows(kk + 1);
                    Frag rf[NT][OP];
#pragma unroll
                    for (int nt = 0; nt < NT; nt++) split(__builtin_shufflevector(R[2 * kk][nt], R[2 * kk + 1][nt], 0, 1, 2, 3, 4, 5, 6, 7), rf[nt]);
#pragma unroll
                    for (int it = 0; it < CH / 16; it++)
#pragma unroll
                        for (int nt = 0; nt < NT; nt++) y[it][nt] = product(rf[nt], af[kk % AHEAD][it], y[it][nt]);
                    __builtin_amdgcn_sched_barrier(0);
                }
            }
            load_columns();
#pragma unroll
            for (int it = 0; it < CH / 16; it++) {
                const int row = it * 16 + i, age = REV ? n - 1 - row : row;
                const float scale = row_weights[age > 0 ? age : 0];
#pragma unroll
                for (int nt = 0; nt < NT; nt++) y[it][nt] *= scale;
#pragma unroll
                for (int ks = 0; ks < CH / 32; ks++) {
                    if (!p_has<REV>(it, ks)) continue;
                    Frag pf[OP];
#pragma unroll
                    for (int q = 0; q < OP; q++) pf[q] = p_lds[(p_block<REV>(it, ks, CH) * OP + q) * 64 + lane];
#pragma unroll
                    for (int nt = 0; nt < NT; nt++) y[it][nt] = product(cf[ks][nt], pf, y[it][nt]);
                }
                __builtin_amdgcn_sched_barrier(0);
                if (row < n) {
                    const long long to = (at.start + t0 + row) * r.y_tok + h * r.y_head + part * DV;
                    const int col = col0 + g * CS;
                    float x[NT * 4];
#pragma unroll
                    for (int e = 0; e < NT * 4; e++) x[e] = y[it][e / 4][e % 4];
                    if (col + NT * 4 <= nc) {
                        if (r.y_float) store_floats_unaligned<float, NT * 4>(reinterpret_cast<float *>(r.y) + to + col, x);
                        else store_floats_unaligned<S, NT * 4>(reinterpret_cast<S *>(r.y) + to + col, x);
                    } else {
#pragma unroll
                        for (int e = 0; e < NT * 4; e++)
                            if (col + e < nc) {
                                if (r.y_float) reinterpret_cast<float *>(r.y)[to + col + e] = x[e];
                                else reinterpret_cast<S *>(r.y)[to + col + e] = (S)x[e];
                            }
                    }
                }
            }
        }

        if (OUT && step == nchunks - 1 && !(last && r.fin)) break; // nobody needs the next state
        // ---- the next state; after the last token of a forward walk the final state, one decay short of the next chunk's
        const int ahead = !REV && last && r.fin && step == nchunks - 1 ? 1 : 0;
        const float whole = decay_power(g2, n - ahead);
#pragma unroll
        for (int t = 0; t < DK / 16; t++)
#pragma unroll
            for (int nt = 0; nt < NT; nt++) R[t][nt] *= whole;
#pragma unroll
        for (int ks = 0; ks < CH / 32; ks++) {
            f32x8 wt; // u g^(n - j'); rows past the end, where it would grow, are zeros
            if (REV || (n == CH && !ahead)) {
                wt = *reinterpret_cast<const f32x8 *>(state_weights + ks * 32 + g * 8);
            } else {
                const int first = n - ahead - ks * 32 - g * 8;
#pragma unroll
                for (int e = 0; e < 8; e++) wt[e] = first - e < 0 ? 0.0f : r.u_scale * decay_power(g2, first - e);
            }
            Frag cd[NT][OP];
#pragma unroll
            for (int nt = 0; nt < NT; nt++) split(widen(cf[ks][nt]) * wt, cd[nt]);
            constexpr int AHEAD = IP == 1 ? 2 : 1;
            Frag bf[AHEAD][IP];
            auto load_rows = [&](int t) { col_frag<Lds::PK>(bf[t % AHEAD], b_lds, KP, ks * 32, t / 2 * 32 + t % 2 * 4, 8, lane); };
            if (AHEAD > 1) load_rows(0);
#pragma unroll
            for (int t = 0; t < DK / 16; t++) {
                if (AHEAD == 1) load_rows(t);
                else if (t + 1 < DK / 16) load_rows(t + 1);
#pragma unroll
                for (int nt = 0; nt < NT; nt++) R[t][nt] = product(bf[t % AHEAD], cd[nt], R[t][nt]);
                __builtin_amdgcn_sched_barrier(0);
            }
        }
    }

    if (OUT ? r.fin && last : true) {
#pragma unroll
        for (int t = 0; t < DK / 16; t++)
#pragma unroll
            for (int nt = 0; nt < NT; nt++) {
                if (!OUT) {
                    *reinterpret_cast<f32x4 *>(total + (nt * (DK / 16) + t) * 256) = R[t][nt];
                } else {
                    const int col = col0 + (i >> 2) * CS + 4 * nt + (i & 3);
#pragma unroll
                    for (int e = 0; e < 4; e++) {
                        const int row = t / 2 * 32 + g * 8 + t % 2 * 4 + e;
                        if (row < r.ka && col < nc) r.fin[state0 + (long long)row * r.state_row + (long long)col * r.state_col] = R[t][nt][e];
                    }
                }
            }
    }
}

// grid: slots heads parts roles, in one order; the roles of a head and segment run on one XCD (of 8, dealt round robin), whose L2 has the rows
// they share
template <typename S, int DK, int DV, int NW, bool OUT>
__global__ __launch_bounds__(NW * 64, (WalkLds<S, DK, DV, NW, OUT>::per_simd)) void walk_kernel(WalkArgs w)
{
    extern __shared__ __align__(16) unsigned char lds[];
    const unsigned block = (unsigned)block_of(), group = block / (8 * w.roles), in = block % (8 * w.roles); // (2^28 at most)
    const unsigned item = group * 8 + in % 8;
    if (item >= w.slots * w.heads * w.parts) return;
    const WalkRole &r = w.role[in / 8];
    const int part = item % w.parts, h = item / w.parts % w.heads;
    const long long slot = item / w.parts / w.heads;
    const Place at = find_place(w, slot);
    if (at.seg < 0 || at.seg >= at.nseg || part * DV >= r.nc) return; // a slot that no sequence has
    if (r.reverse) walk<S, DK, DV, NW, OUT, true>(w, r, at, slot, h, part, lds);
    else walk<S, DK, DV, NW, OUT, false>(w, r, at, slot, h, part, lds);
}

// Segment totals -> incoming states, in place, in walking order: a thread has four entries of one head's state and goes
// through the segments of one sequence.  grid: (seqs heads parts times a group of 1024 entries, 1, roles)
template <int DK, int DV, int NW> __global__ __launch_bounds__(256) void carry_kernel(WalkArgs w)
{
    constexpr int NT = DV / 16 / NW, CS = NT == 2 ? 8 : 4;
    const WalkRole &r = w.role[blockIdx.z];
    constexpr int GROUPS = DK * DV / 1024;
    const unsigned item = blockIdx.x / GROUPS;
    const long long s = item / w.parts / w.heads;
    const int part = item % w.parts, h = item / w.parts % w.heads, u = blockIdx.x % GROUPS * 256 + threadIdx.x;
    long long start, len;
    span(w, s, start, len);
    const long long nseg = len > 0 ? (len + w.seg_len - 1) / w.seg_len : 1;
    const int lane = u & 63, t = u / 64 % (DK / 16), nt = u / 64 / (DK / 16) % NT, wave = u / 64 / (DK / 16) / NT, i = lane & 15;
    const float g2 = log2_decay(w.log_decay[h]);
    f32x4 x = {0, 0, 0, 0};
    if (r.init) {
        const float scale = r.reverse ? 1.0f : decay_power(g2, 1);
        const int col = part * DV + wave * NT * 16 + (i >> 2) * CS + 4 * nt + (i & 3);
        for (int e = 0; e < 4; e++) {
            const int row = t / 2 * 32 + (lane >> 4) * 8 + t % 2 * 4 + e;
            if (row < r.ka && col < r.nc) x[e] = scale * r.init[(s * w.heads + h) * (long long)r.ka * r.nc + (long long)row * r.state_row + (long long)col * r.state_col];
        }
    }
    f32x4 *const tot = reinterpret_cast<f32x4 *>(r.totals) + ((first_slot(w, s) * w.heads + h) * w.parts + part) * (long long)(DK * DV / 4) + u;
    const long long stride = (long long)w.heads * w.parts * (DK * DV / 4);
    const float whole = decay_power(g2, (int)w.seg_len);
    const float first = r.reverse ? decay_power(g2, (int)(len - (nseg - 1) * w.seg_len)) : whole; // a sequence's last segment may be shorter
    const long long dir = r.reverse ? -1 : 1, at = r.reverse ? nseg - 1 : 0;
    constexpr int AHEAD = 8; // totals in flight (the last segment in walking order has none)
    for (long long k0 = 0; k0 < nseg; k0 += AHEAD) {
        f32x4 mine[AHEAD];
#pragma unroll
        for (int k = 0; k < AHEAD; k++) mine[k] = k0 + k + 1 < nseg ? tot[(at + dir * (k0 + k)) * stride] : f32x4{0, 0, 0, 0};
#pragma unroll
        for (int k = 0; k < AHEAD; k++)
            if (k0 + k < nseg) {
                tot[(at + dir * (k0 + k)) * stride] = x;
                x = x * (k0 + k == 0 ? first : whole) + mine[k];
            }
    }
}

// lets a kernel have `bytes` of dynamic LDS, once a device (`done`: one flag for each kernel)
static int allow_lds(goom_ctx *ctx, const void *kernel, size_t bytes, std::atomic<unsigned long long> &done)
{
    const unsigned long long bit = 1ull << (ctx->device & 63);
    if (ctx->device < 64 && (done.load(std::memory_order_relaxed) & bit)) return GOOM_OK;
    if (int st = goom::check_hip(ctx, hipFuncSetAttribute(kernel, hipFuncAttributeMaxDynamicSharedMemorySize, (int)bytes), "hipFuncSetAttribute")) return st;
    done.fetch_or(bit, std::memory_order_relaxed);
    return GOOM_OK;
}

template <typename S, int DK, int DV, int NW> static int launch_walks_sized(goom_ctx *ctx, WalkArgs w, int roles, long long slots, const char *label)
{
    w.roles = roles;
    w.slots = (unsigned)slots;
    int nc = 0;
    for (int k = 0; k < roles; k++) nc = w.role[k].nc > nc ? w.role[k].nc : nc;
    w.parts = (nc + DV - 1) / DV;
    const dim3 grid = grid_of((slots * w.heads * w.parts + 7) / 8 * 8 * roles, NW * 64);
    const bool parts = w.role[0].totals != nullptr;
    if (parts) {
        auto *totals = walk_kernel<S, DK, DV, NW, false>;
        constexpr size_t bytes = WalkLds<S, DK, DV, NW, false>::bytes;
        static std::atomic<unsigned long long> done{0};
        if (int st = allow_lds(ctx, reinterpret_cast<const void *>(totals), bytes, done)) return st;
        goom::prof_begin(ctx, "linear attention: segment totals");
        totals<<<grid, NW * 64, bytes, ctx->stream>>>(w);
        goom::prof_end(ctx);
        goom::prof_begin(ctx, "linear attention: carries");
        carry_kernel<DK, DV, NW><<<dim3((unsigned)(w.seqs * w.heads * w.parts * (DK * DV / 1024)), 1, roles), 256, 0, ctx->stream>>>(w);
        goom::prof_end(ctx);
    }
    auto *walk = walk_kernel<S, DK, DV, NW, true>;
    constexpr size_t bytes = WalkLds<S, DK, DV, NW, true>::bytes;
    static std::atomic<unsigned long long> done{0};
    if (int st = allow_lds(ctx, reinterpret_cast<const void *>(walk), bytes, done)) return st;
    goom::prof_begin(ctx, label);
    walk<<<grid, NW * 64, bytes, ctx->stream>>>(w);
    goom::prof_end(ctx);
    return goom::check_hip(ctx, hipGetLastError(), label);
}

// f(DK, DV, NW): the walk's kernel for rows of ka and columns of nc entries
template <typename S, typename F> static auto with_walk(int ka, int nc, F f)
{
    constexpr int IN = Parts<S>::IN;
    auto columns = [&](auto rows) {
        constexpr int DK = decltype(rows)::value;
        if (nc <= 32) return f(rows, std::integral_constant<int, 32>(), std::integral_constant<int, 2>());
        // floats' three parts of 128 x 128 leave room for but one workgroup in a CU's LDS: two halves of the columns
        if constexpr (DK == 128 && IN == 3) return f(rows, std::integral_constant<int, 64>(), std::integral_constant<int, 4>());
        else if (nc <= 64) return f(rows, std::integral_constant<int, 64>(), std::integral_constant<int, 4>());
        else return f(rows, std::integral_constant<int, 128>(), std::integral_constant<int, 4>());
    };
    return ka <= 32 ? columns(std::integral_constant<int, 32>()) : ka <= 64 ? columns(std::integral_constant<int, 64>()) : columns(std::integral_constant<int, 128>());
}

// The roles of one launch share a kernel, of the largest size among them.  One source file for each type.
template <typename S> int launch_walks_typed(goom_ctx *ctx, const WalkArgs &w, int roles, long long slots, const char *label)
{
    int ka = 0, nc = 0;
    for (int k = 0; k < roles; k++) {
        ka = w.role[k].ka > ka ? w.role[k].ka : ka;
        nc = w.role[k].nc > nc ? w.role[k].nc : nc;
    }
    return with_walk<S>(ka, nc, [&](auto rows, auto cols, auto waves) {
        return launch_walks_sized<S, decltype(rows)::value, decltype(cols)::value, decltype(waves)::value>(ctx, w, roles, slots, label);
    });
}

// gradients of two inputs that heads share, summed over each `group` of heads: x[tokens][heads][d] floats -> y[tokens][heads / group][d]
// (goom_linear_attention.hip)
int launch_shared_sums(goom_ctx *ctx, int type, const float *x0, void *y0, int d0, const float *x1, void *y1, int d1, long long tokens, int shared_heads, int group,
                       const int64_t *offsets, long long seqs, const char *label);

template <typename S> int launch_walks_of(goom_ctx *ctx, const WalkArgs &w, int roles, long long slots, const char *label);
template <> int launch_walks_of<float>(goom_ctx *ctx, const WalkArgs &w, int roles, long long slots, const char *label);
template <> int launch_walks_of<bf16>(goom_ctx *ctx, const WalkArgs &w, int roles, long long slots, const char *label);
template <> int launch_walks_of<f16>(goom_ctx *ctx, const WalkArgs &w, int roles, long long slots, const char *label);

} // namespace goom_layer
