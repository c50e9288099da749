// The gated delta rule (Yang, Kautz and Hatamizadeh 2024, arXiv 2412.06464): a memory of one matrix per head, over sequences, forward and backward.
//
// Per head, with a_t = sigmoid(f_t), beta_t = sigmoid(b_t) and the state S [Dk][Dv] (zero before a step that starts an episode):
//   S_t = a_t (I - beta_t k_t k_t^T) S_{t-1} + beta_t k_t v_t^T,  o_t = scale S_t^T q_t.
// Over a tile of CH steps (as Yang, Wang, Zhang, Shen and Kim 2024, arXiv 2406.06484, take the rule without gates) that the state S enters, with g_i = a_1 .. a_i and G_ij = g_i / g_j (0 where an episode starts in between):
//   S_i = g_i S + sum_{j <= i} G_ij k_j u_j^T,   U = T R,   T = (I + N)^-1,   N_ij = beta_i G_ij k_i.k_j (j < i),   R_i = beta_i (v_i - g_i S^T k_i)
//   O = scale g Q S + P U,   P_ij = scale G_ij q_i.k_j (j <= i),   S' = g_C S + (G_C. K)^T U.
// Backward, from dO and the gradient D of the state that leaves:
//   dU = P^T dO + (G_C. K) D,   Y = T^T dU,   dS = g_C D + (scale g Q)^T dO - (beta g K)^T Y,   dv = beta Y,   db = (1 - beta) Y.u
//   dP = dO U^T, dN = -Y U^T:   dq = scale g S do + (dP scale G) k,   dk = (dP scale G)^T q + G_C. D u - beta g S y + (dN beta G) k + (dN beta G)^T k
// and, a_t being a factor of every G_ij with j < t <= i, of every g_i with i >= t and of every G_Cj with j < t,
//   d log a_t = sum_{j < t <= i} (dP_ij P_ij + dN_ij N_ij) + sum_{i >= t} e_i + sum_{j < t} l_j + g_C <D, S>,   df = (1 - a) d log a,
//   e_i = g_i (scale q_i.(S do_i) - beta_i k_i.(S y_i)),   l_j = G_Cj u_j.(D^T k_j).
// (Sums of do_i.o_i - dv_i.v_i, which are fewer, do not have a_t as a factor: they leave the gradient of a gate that is nearly shut as a difference of numbers
// that it has no part in.)
//
// Three kinds of launch: what a tile needs that no state has part in (T, P, the gates), all tiles at once, a wave each; the chain from state to
// state, forward or backward, a wave per 16 columns of the state; and the gradients, all tiles at once, a workgroup each.
//
// Everything but T and P is independent per column of the state.  A wave of the chain keeps its 16 columns of S, R, U, O in registers in the
// layout in which the matrix instructions leave their results; with the rows of a pair of 16 x 16 results dealt out so that a lane's eight
// numbers are eight neighbours (row 8 (l / 16) + 4 (half) + r), that is also the layout in which they take a right operand 32 deep.  So nothing is
// exchanged between lanes from state to state, and left operands (rows of K, Q, T, P in LDS) are read as they lie, 16 bytes a lane.
//
// bf16 inputs are exact operands of the bf16 instructions; a state or a U, which is fp32, is taken apart into three bf16 that are
// exactly its 24 bits, one instruction for each, where it feeds a state, into two (16 bits, and without the product of the lower ones 2^-14 of a product at
// most where both operands are such) where it only feeds results that are rounded to bf16: that changes the last bit of 0.1 % of the outputs, 0.7 % of the gradients.
// fp32 inputs go through the fp32 instructions, of a sixteenth of the rate.
#pragma once
#include "seq_common.h"

namespace seq {

constexpr int CH = 32;                 // steps of a tile
constexpr int COLS = 64;               // columns of the state of a workgroup, 16 of each wave
// A factor between steps where an episode starts in between: what it multiplies counts for nothing, whatever it is.  The 0 of gates that are shut has the other
// sign: 0 times what is not finite is a NaN, as in the definition.
constexpr uint32_t CLEARED = 0x80000000u;      // of -0.f
constexpr float LOG_LEAST = -216.f;    // of a gate, base 2; 2 to it is 0 in fp32: a gate that closes further counts as this, so that differences of sums stay finite

using f4 = vec<float, 4>;
using f8 = vec<float, 8>;
using b8 = vec<bf16, 8>;

struct Strides {
    long bs, ts, hs;                   // of a sequence, a step, a head
};

struct DeltaIn {
    const void *q, *k, *v, *f, *b;
    Strides sq, sk, sv, sf, sb;
    const uint8_t *reset;
    long reset_bs, reset_ts;
    long T, tiles;
    int B, H, Dk, Dv;
    float scale;
    int wide;                          // rows of q and k can be read 16 bytes at a time
};
struct DeltaArgs : DeltaIn {
    const float *s0;
    void *o;
    Strides so;
    float *last, *states, *records;    // states: the one that enters each tile, as waves hold it (Columns), or NULL
};
struct DeltaGradArgs : DeltaIn {
    const void *dout;
    Strides sdo;
    const float *states, *records, *dlast;
    void *dq, *dk, *dv, *df, *db;
    Strides sdq, sdk, sdv, sdf, sdb;
    float *ds0;
    float *into;                       // the gradient of the state that leaves each tile, as states
    int *again;                        // of each tile: whether its gradients hold a number that is not finite
};

// What the first launch leaves of a tile.
struct DeltaRecord {
    float t[CH * CH], p[CH * CH];
    float since[CH], until[CH], beta[CH];   // g_i, CLEARED behind an episode's start; G_Ci, CLEARED before one
    float gate[CH];                    // a
    float run_hi[CH], run_lo[CH];      // sum of log a, base 2, up to each step, as a multiple of 2^-10 and the rest
    int cut[CH];                       // episodes that have started up to each step
};
static_assert(sizeof(DeltaRecord) % 16 == 0, "records are copied 16 bytes at a time");

// ---------------------------------------------------------------- operands, 8 numbers deep a lane
// a, b of a word as their upper halves
__device__ __forceinline__ uint32_t uppers(uint32_t a, uint32_t b) { return __builtin_amdgcn_perm(b, a, 0x07060302u); }

// N bf16 whose sum is the number, exactly for N = 3 (each takes eight bits off); the last of two is rounded.
template <int N> struct Planes {
    b8 p[N];
};
template <int N> __device__ __forceinline__ Planes<N> planes(const float (&v)[8])
{
    vec<uint32_t, 4> w[N];
#pragma unroll
    for (int i = 0; i < 8; i += 2) {
        float x = v[i], y = v[i + 1];
#pragma unroll
        for (int n = 0; n < N; ++n) {
            uint32_t a = __float_as_uint(x), b = __float_as_uint(y);
            if (N == 2 && n == 1) a += 0x8000u, b += 0x8000u;
            w[n][i / 2] = uppers(a, b);
            if (n + 1 < N) {
                x -= __uint_as_float(a & 0xFFFF0000u);
                y -= __uint_as_float(b & 0xFFFF0000u);
            }
        }
    }
    Planes<N> o;
#pragma unroll
    for (int n = 0; n < N; ++n) o.p[n] = __builtin_bit_cast(b8, w[n]);
    return o;
}

__device__ __forceinline__ f4 mfma(b8 a, b8 b, f4 c) { return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0); }
__device__ __forceinline__ f4 mfma(f8 a, f8 b, f4 c)
{
#pragma unroll
    for (int i = 0; i < 8; ++i) c = __builtin_amdgcn_mfma_f32_16x16x4f32(a[i], b[i], c, 0, 0, 0);
    return c;
}

// Operands for inputs of type E.  Exact: of the inputs themselves; Split<N>: of fp32 numbers.
template <class E> struct Operand;
template <> struct Operand<bf16> {
    using Exact = b8;
    template <int N> using Split = Planes<N>;
    template <int N> static __device__ __forceinline__ Planes<N> split(const float (&v)[8]) { return planes<N>(v); }
    template <int N> static __device__ __forceinline__ f4 mul(b8 a, const Planes<N> &b, f4 c)
    {
#pragma unroll
        for (int n = N - 1; n >= 0; --n) c = mfma(a, b.p[n], c);
        return c;
    }
    template <int N> static __device__ __forceinline__ f4 mul(const Planes<N> &a, b8 b, f4 c)
    {
#pragma unroll
        for (int n = N - 1; n >= 0; --n) c = mfma(a.p[n], b, c);
        return c;
    }
    static __device__ __forceinline__ f4 mul(const Planes<2> &a, const Planes<2> &b, f4 c)
    {
        c = mfma(a.p[1], b.p[0], c);
        c = mfma(a.p[0], b.p[1], c);
        return mfma(a.p[0], b.p[0], c);
    }
    static __device__ __forceinline__ f4 mul(b8 a, b8 b, f4 c) { return mfma(a, b, c); }
};
template <> struct Operand<float> {
    using Exact = f8;
    template <int N> using Split = f8;
    template <int N> static __device__ __forceinline__ f8 split(const float (&v)[8])
    {
        f8 o;
#pragma unroll
        for (int i = 0; i < 8; ++i) o[i] = v[i];
        return o;
    }
    static __device__ __forceinline__ f4 mul(f8 a, f8 b, f4 c) { return mfma(a, b, c); }
    template <int N> static __device__ __forceinline__ f4 mul(f8 a, f8 b, f4 c) { return mfma(a, b, c); }
};

__device__ __forceinline__ f8 both(f4 a, f4 b) { return f8{a[0], a[1], a[2], a[3], b[0], b[1], b[2], b[3]}; }
template <class E, int N> __device__ __forceinline__ typename Operand<E>::template Split<N> split(f4 a, f4 b)
{
    const float v[8] = {a[0], a[1], a[2], a[3], b[0], b[1], b[2], b[3]};
    return Operand<E>::template split<N>(v);
}
template <class E, int N> __device__ __forceinline__ f4 mul(typename Operand<E>::Exact a, const typename Operand<E>::template Split<N> &b, f4 c)
{
    if constexpr (std::is_same<E, float>::value) return mfma(a, b, c);
    else return Operand<bf16>::template mul<N>(a, b, c);
}

// Loads take addresses that are always there, the last step's or column's in place of those beyond, and zeros are put in afterwards: a branch
// around each of them would wait for one before it asks for the next.

// 8 numbers of a row from column c on, zeros from D on and where the row is not real
template <class E> __device__ __forceinline__ vec<E, 8> load8(const E *p, int c, int D, bool real, int wide)
{
    vec<E, 8> v;
    if (wide) {      // D is a multiple of V
        constexpr int V = 16 / (int)sizeof(E);
#pragma unroll
        for (int i = 0; i < 8; i += V) {
            const vec<E, V> x = load<V>(p + min(c + i, D - V));
#pragma unroll
            for (int e = 0; e < V; ++e) v[i + e] = real && c + i < D ? x[e] : (E)0.f;
        }
    } else {
        E x[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) x[i] = p[min(c + i, D - 1)];
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = real && c + i < D ? x[i] : (E)0.f;
    }
    return v;
}

__device__ __forceinline__ void wave_sync() { __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront"); __builtin_amdgcn_wave_barrier(); }

__device__ __forceinline__ float power(float x) { return __builtin_amdgcn_exp2f(x); }
// The factor from step j to step i >= j of an episode: differences of the multiples of 2^-10 are exact, so that a gate that closed long before
// leaves no rounding in later ones.  The exponent x is one fp32 number, so the factor is |x| ln 2 2^-24 of itself off and what the instruction adds, 2^-23.
__device__ __forceinline__ float between(float hi_i, float lo_i, float hi_j, float lo_j) { return power((hi_i - hi_j) + (lo_i - lo_j)); }

// ---------------------------------------------------------------- T, P and the gates of every tile
// A wave per tile.  K K^T and Q K^T are a few matrix instructions; the time goes into what waits step after step: the sums of the gates' logarithms
// (in 64 bits), and the substitution that forms T's blocks on the diagonal, 16 rows one after the other.  32 x 512 x 8 x 64 in bf16, 4096 tiles: 18 us;
// 4096 of 128 columns 23.
template <class E, int DK> __global__ __launch_bounds__(256) void k_delta_tiles(DeltaIn A, DeltaRecord *records)
{
    constexpr int LN = CH + 4, KS = DK / 32;
    struct Own {
        float n[CH * LN];
        float run_hi[CH], run_lo[CH], beta[CH];
        int cut[CH];
    };
    __shared__ __align__(16) Own all[4];
    const int lane = threadIdx.x & 63, w = threadIdx.x >> 6, col = lane & 15, g = lane >> 4;
    const long id = (long)blockIdx.x * 4 + w;
    if (id >= (long)A.B * A.H * A.tiles) return;      // whole waves, and no barrier follows
    Own &s = all[w];
    const long head = id / A.tiles, tile = id % A.tiles, t0 = tile * CH;
    const int bi = (int)(head / A.H), h = (int)(head % A.H), rows = (int)min((long)CH, A.T - t0);
    DeltaRecord &out = records[id];
    const E *q = (const E *)A.q + bi * A.sq.bs + t0 * A.sq.ts + h * A.sq.hs, *k = (const E *)A.k + bi * A.sk.bs + t0 * A.sk.ts + h * A.sk.hs;
    vec<E, 8> kf[2][KS], qf[2][KS];
#pragma unroll
    for (int m = 0; m < 2; ++m)
#pragma unroll
        for (int ks = 0; ks < KS; ++ks) {
            const int r = 16 * m + col;
            kf[m][ks] = load8<E>(k + min(r, rows - 1) * A.sk.ts, 32 * ks + 8 * g, A.Dk, r < rows, A.wide);
            qf[m][ks] = load8<E>(q + min(r, rows - 1) * A.sq.ts, 32 * ks + 8 * g, A.Dk, r < rows, A.wide);
        }
    {   // both halves of the wave do the same
        const int i = lane & 31;
        const bool in = i < rows;
        const long t = t0 + min(i, rows - 1);
        const float f = (float)((const E *)A.f)[bi * A.sf.bs + t * A.sf.ts + h * A.sf.hs];
        const float b = (float)((const E *)A.b)[bi * A.sb.bs + t * A.sb.ts + h * A.sb.hs];
        const int start = A.reset ? A.reset[bi * A.reset_bs + t * A.reset_ts] : 0;
        double la = ((double)(f < 0.f ? f : 0.f) - (double)log1pf(expf(-fabsf(f)))) * 1.4426950408889634;
        la = la < LOG_LEAST ? LOG_LEAST : la;
        la = in ? la : 0.0;
        const float beta = in ? 1.f / (1.f + expf(-b)) : 0.f;
        const int cut = in && start ? 1 : 0;
        double run = la;
        int cuts = cut;
#pragma unroll
        for (int d = 1; d < CH; d *= 2) {
            const double o = __shfl_up(run, d, 32);
            const int oc = __shfl_up(cuts, d, 32);
            if (i >= d) run += o, cuts += oc;
        }
        const double whole = rint(run * 1024.0) * (1.0 / 1024.0), end = __shfl(run, CH - 1, 32);
        const int last = __shfl(cuts, CH - 1, 32);
        if (lane < CH) {
            s.run_hi[i] = out.run_hi[i] = (float)whole;
            s.run_lo[i] = out.run_lo[i] = (float)(run - whole);
            s.cut[i] = out.cut[i] = cuts;
            s.beta[i] = out.beta[i] = beta;
            out.gate[i] = power((float)la);
            out.since[i] = cuts ? -0.f : power((float)run);
            out.until[i] = in && cuts == last ? power((float)(end - run)) : -0.f;
        }
    }
    wave_sync();
    int cut_j[2];
    float hi_j[2], lo_j[2];
#pragma unroll
    for (int n = 0; n < 2; ++n) cut_j[n] = s.cut[16 * n + col], hi_j[n] = s.run_hi[16 * n + col], lo_j[n] = s.run_lo[16 * n + col];
#pragma unroll
    for (int m = 0; m < 2; ++m) {
        const vec<int, 4> cut_i = load<4>(s.cut + 16 * m + 4 * g);
        const f4 hi_i = load<4>(s.run_hi + 16 * m + 4 * g), lo_i = load<4>(s.run_lo + 16 * m + 4 * g), beta = load<4>(s.beta + 16 * m + 4 * g);
        float *p = out.p + (16 * m + 4 * g) * CH + col;
#pragma unroll
        for (int n = 0; n < 2; ++n) {
            f4 kk = {}, qk = {};
            if (n <= m)
#pragma unroll
                for (int ks = 0; ks < KS; ++ks) {
                    kk = mfma(kf[m][ks], kf[n][ks], kk);
                    qk = mfma(qf[m][ks], kf[n][ks], qk);
                }
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                const int i = 16 * m + 4 * g + r, j = 16 * n + col;
                const float b = n > m || j > i || cut_i[r] != cut_j[n] ? 0.f : between(hi_i[r], lo_i[r], hi_j[n], lo_j[n]);
                if (n <= m) s.n[i * LN + j] = j < i && b != 0.f ? -beta[r] * b * kk[r] : 0.f;
                p[r * CH + 16 * n] = b != 0.f ? A.scale * b * qk[r] : 0.f;
            }
        }
    }
    wave_sync();
    // (I + N)^-1 of the two blocks on the diagonal by forward substitution, a column per lane, in their places
    if (lane < 32) {
        float *blk = s.n + 16 * g * (LN + 1);
        float x[16];
#pragma unroll
        for (int i = 0; i < 16; ++i) {
            float v = i == col ? 1.f : 0.f;
#pragma unroll
            for (int j = 0; j < i; ++j) v = fmaf(blk[i * LN + j], x[j], v);
            x[i] = v;
        }
#pragma unroll
        for (int i = 0; i < 16; ++i) blk[i * LN + col] = x[i];
    }
    wave_sync();
    // below them T11 (-N10) T00: a result's layout is that of the next right operand, 16 deep
    f4 x = {}, y = {};
#pragma unroll
    for (int e = 0; e < 4; ++e) x = __builtin_amdgcn_mfma_f32_16x16x4f32(s.n[(16 + col) * LN + 4 * g + e], s.n[(4 * g + e) * LN + col], x, 0, 0, 0);
#pragma unroll
    for (int e = 0; e < 4; ++e) y = __builtin_amdgcn_mfma_f32_16x16x4f32(s.n[(16 + col) * LN + 16 + 4 * g + e], x[e], y, 0, 0, 0);
#pragma unroll
    for (int r = 0; r < 4; ++r) {
        const int i = 4 * g + r;
        out.t[i * CH + col] = s.n[i * LN + col];
        out.t[i * CH + 16 + col] = 0.f;
        out.t[(16 + i) * CH + col] = y[r];
        out.t[(16 + i) * CH + 16 + col] = s.n[(16 + i) * LN + 16 + col];
    }
}

// ---------------------------------------------------------------- what a workgroup holds of a tile in LDS
template <class E, int DK, int VECTORS> struct DeltaKeys {      // VECTORS: how many of the record's, from `since` on
    static constexpr int LD = DK + 16 / (int)sizeof(E), LC = CH + 4;
    static constexpr bool QUERIES = false;
    alignas(16) E k[CH * LD];
    float t[CH * LC];
    float vectors[VECTORS * CH];
    __device__ __forceinline__ const float *since() const { return vectors; }
    __device__ __forceinline__ const float *until() const { return vectors + CH; }
    __device__ __forceinline__ const float *beta() const { return vectors + 2 * CH; }
    __device__ __forceinline__ const float *gate() const { return vectors + 3 * CH; }
    __device__ __forceinline__ const float *run_hi() const { return vectors + 4 * CH; }
    __device__ __forceinline__ const float *run_lo() const { return vectors + 5 * CH; }
    __device__ __forceinline__ const int *cut() const { return reinterpret_cast<const int *>(vectors + 6 * CH); }
};
template <class E, int DK, int VECTORS> struct DeltaTile : DeltaKeys<E, DK, VECTORS> {
    using Keys = DeltaKeys<E, DK, VECTORS>;
    static constexpr bool QUERIES = true;
    alignas(16) E q[CH * Keys::LD];
    float p[CH * Keys::LC];
};

// Where a head's tensors begin, for all lanes alike, and 32-bit offsets from there: a stride from step to step is at most 2^24 elements.
template <class E> __device__ __forceinline__ const E *head_of(const void *p, const Strides &s, int bi, int h) { return (const E *)p + bi * s.bs + h * s.hs; }
template <class E> __device__ __forceinline__ E *head_of(void *p, const Strides &s, int bi, int h) { return (E *)p + bi * s.bs + h * s.hs; }
template <class T> __device__ __forceinline__ T *plus(T *p, uint32_t bytes) { return (T *)((char *)p + bytes); }
template <class T> __device__ __forceinline__ const T *plus(const T *p, uint32_t bytes) { return (const T *)((const char *)p + bytes); }

// The part of a tile that a thread of THREADS brings from memory: into registers first, so that it can arrive while another tile is worked on.
template <class E, int DK, int THREADS, int VECTORS, class Tile = DeltaTile<E, DK, VECTORS>> struct DeltaFetch {
    static constexpr int V = 16 / (int)sizeof(E), PER = DK / V, N = (CH * PER + THREADS - 1) / THREADS, NR = (CH * CH / 4 + THREADS - 1) / THREADS;
    static_assert(VECTORS * CH / 4 <= THREADS, "a thread brings one piece of the vectors");
    const E *qh, *kh;
    const DeltaRecord *records;
    int tid, rows;
    uint32_t qo[N], ko[N];
    vec<E, V> q[N], k[N];
    f4 t[NR], p[NR], vectors;
    __device__ __forceinline__ void offsets(const DeltaIn &A, int n_rows)
    {
        rows = n_rows;
#pragma unroll
        for (int n = 0; n < N; ++n) {
            const int e = tid + THREADS * n, r = min(e / PER, n_rows - 1), c = min(e % PER * V, A.wide ? A.Dk - V : A.Dk - 1);
            qo[n] = (uint32_t)(r * (int)A.sq.ts + c) * (uint32_t)sizeof(E);
            ko[n] = (uint32_t)(r * (int)A.sk.ts + c) * (uint32_t)sizeof(E);
        }
    }
    __device__ __forceinline__ void begin(const DeltaIn &A, const DeltaRecord *all, long head, int bi, int h, int thread)
    {
        qh = head_of<E>(A.q, A.sq, bi, h);
        kh = head_of<E>(A.k, A.sk, bi, h);
        records = all + head * A.tiles;
        tid = thread;
        offsets(A, CH);
    }
    __device__ __forceinline__ void load(const DeltaIn &A, long tile)
    {
        const long t0 = tile * CH;
        const int now = (int)min((long)CH, A.T - t0);
        if (now != rows) offsets(A, now);
        const E *qp = qh + t0 * A.sq.ts, *kp = kh + t0 * A.sk.ts;
        if (A.wide) {
#pragma unroll
            for (int n = 0; n < N; ++n) {
                if (Tile::QUERIES) q[n] = seq::load<V>(plus(qp, qo[n]));
                k[n] = seq::load<V>(plus(kp, ko[n]));
            }
        } else {
#pragma unroll
            for (int n = 0; n < N; ++n) {
                const int c = (tid + THREADS * n) % PER * V;
#pragma unroll
                for (int i = 0; i < V; ++i) {
                    const int more = max(0, min(i, A.Dk - 1 - c));
                    if (Tile::QUERIES) q[n][i] = plus(qp, qo[n])[more];
                    k[n][i] = plus(kp, ko[n])[more];
                }
            }
        }
        const DeltaRecord *rec = records + tile;
#pragma unroll
        for (int n = 0; n < NR; ++n) {
            const int e = min(tid + THREADS * n, CH * CH / 4 - 1);
            t[n] = seq::load<4>(rec->t + 4 * e);
            if (Tile::QUERIES) p[n] = seq::load<4>(rec->p + 4 * e);
        }
        vectors = seq::load<4>(rec->since + 4 * min(tid, VECTORS * CH / 4 - 1));
    }
    __device__ __forceinline__ void put(Tile &s, int Dk) const
    {
        const bool whole = rows == CH && Dk == DK;
#pragma unroll
        for (int n = 0; n < N; ++n) {
            const int e = tid + THREADS * n, r = e / PER, c = e % PER * V;
            vec<E, V> x{}, y = k[n];
            if (Tile::QUERIES) x = q[n];
            if (!whole)
#pragma unroll
                for (int i = 0; i < V; ++i) {
                    const bool in = r < rows && c + i < Dk;
                    x[i] = in ? x[i] : (E)0.f;
                    y[i] = in ? y[i] : (E)0.f;
                }
            if (CH * PER % THREADS == 0 || r < CH) {
                if constexpr (Tile::QUERIES) seq::store<V>(s.q + r * Tile::LD + c, x);
                seq::store<V>(s.k + r * Tile::LD + c, y);
            }
        }
#pragma unroll
        for (int n = 0; n < NR; ++n) {
            const int e = tid + THREADS * n, r = e / 8, c = e % 8 * 4;
            if (CH * CH / 4 % THREADS == 0 || r < CH) {
                seq::store<4>(s.t + r * Tile::LC + c, t[n]);
                if constexpr (Tile::QUERIES) seq::store<4>(s.p + r * Tile::LC + c, p[n]);
            }
        }
        if (tid < VECTORS * CH / 4) seq::store<4>(s.vectors + 4 * tid, vectors);
    }
};
static_assert(offsetof(DeltaRecord, cut) - offsetof(DeltaRecord, since) == 6 * CH * 4, "the vectors lie one behind the other");

template <class T> __device__ __forceinline__ vec<T, 8> eight(const T *p)
{
    constexpr int V = 16 / (int)sizeof(T);
    vec<T, 8> v;
#pragma unroll
    for (int i = 0; i < 8; i += V) {
        const vec<T, V> x = load<V>(p + i);
#pragma unroll
        for (int e = 0; e < V; ++e) v[i + e] = x[e];
    }
    return v;
}

// Rows of a matrix of steps (K, Q) as left operand: steps 16 m.., columns 32 p..
template <class E, int LD> __device__ __forceinline__ vec<E, 8> rows_of(const E *x, int m, int p, int lane)
{
    return eight(x + (16 * m + (lane & 15)) * LD + 32 * p + 8 * (lane >> 4));
}
// Columns of one as left operand, 32 steps deep in the order of a pair of results: a lane has steps 4 (l / 16).. and 16 + 4 (l / 16)... Column `i` of 16 is
// element 4 (i / 4) STRIDE + i % 4 from x on.  In bf16 by the transposing LDS read: of four rows that a group of 16 lanes points at, four lanes a row,
// each lane gets one column.
template <int STRIDE, int LD> __device__ __forceinline__ f8 columns_of(const float *x, int lane)
{
    const float *a = x + 4 * (lane >> 4) * LD + 4 * STRIDE * ((lane & 15) >> 2) + (lane & 3);
    return f8{a[0], a[LD], a[2 * LD], a[3 * LD], a[16 * LD], a[17 * LD], a[18 * LD], a[19 * LD]};
}
template <int STRIDE, int LD> __device__ __forceinline__ b8 columns_of(const bf16 *x, int lane)
{
    using s4 = vec<short, 4>;
    typedef __attribute__((address_space(3))) s4 *At;
    const bf16 *a = x + (4 * (lane >> 4) + ((lane & 15) >> 2)) * LD + 4 * STRIDE * (lane & 3);
    const s4 u = __builtin_amdgcn_ds_read_tr16_b64_v4i16((At)a), v = __builtin_amdgcn_ds_read_tr16_b64_v4i16((At)(a + 16 * LD));
    return __builtin_bit_cast(b8, (vec<short, 8>){u[0], u[1], u[2], u[3], v[0], v[1], v[2], v[3]});
}
// The columns that result n of a state's results stands for: dealt, every second four of 32
template <class E, int LD> __device__ __forceinline__ vec<E, 8> state_columns(const E *x, int n, int lane) { return columns_of<2, LD>(x + 32 * (n >> 1) + 4 * (n & 1), lane); }

__device__ __forceinline__ f4 mm4(f4 a, f4 b, f4 c)
{
#pragma unroll
    for (int e = 0; e < 4; ++e) c = __builtin_amdgcn_mfma_f32_16x16x4f32(a[e], b[e], c, 0, 0, 0);
    return c;
}
// X r and X^T r for lower triangular X (T, P) of fp32 in LDS, r a pair of results
template <int LC> __device__ __forceinline__ void lower(const float *x, const f4 (&r)[2], int lane, f4 (&out)[2])
{
    const float *a = x + (lane & 15) * LC + 4 * (lane >> 4);
    out[1] = mm4(load<4>(a + 16 * LC), r[0], out[1]);
    out[0] = mm4(load<4>(a), r[0], out[0]);
    out[1] = mm4(load<4>(a + 16 * LC + 16), r[1], out[1]);
}
template <int LC> __device__ __forceinline__ void upper(const float *x, const f4 (&r)[2], int lane, f4 (&out)[2])
{
    const float *a = x + 4 * (lane >> 4) * LC + (lane & 15), *b = a + 16 * LC;
    out[0] = mm4(f4{b[0], b[LC], b[2 * LC], b[3 * LC]}, r[1], out[0]);
    out[1] = mm4(f4{b[16], b[16 + LC], b[16 + 2 * LC], b[16 + 3 * LC]}, r[1], out[1]);
    out[0] = mm4(f4{a[0], a[LC], a[2 * LC], a[3 * LC]}, r[0], out[0]);
}
// Numbers of a step each, of the steps that a lane holds of result m
__device__ __forceinline__ f4 of_steps(const float *p, int m, int lane) { return load<4>(p + 16 * m + 4 * (lane >> 4)); }

// 0, or NaN if a number is not finite
template <int N> __device__ __forceinline__ float nothing(const f4 (&v)[N])
{
    f4 sum = {};
#pragma unroll
    for (int i = 0; i < N; ++i)
#pragma unroll
        for (int e = 0; e < 4; ++e) sum[e] = fmaf(v[i][e], 0.f, sum[e]);
    return (sum[0] + sum[1]) + (sum[2] + sum[3]);
}
__device__ __forceinline__ f4 where(f4 factor, f4 v)      // factor v, 0 where factor is CLEARED, whatever v is
{
    f4 o;
#pragma unroll
    for (int e = 0; e < 4; ++e) o[e] = __float_as_uint(factor[e]) != CLEARED ? factor[e] * v[e] : 0.f;
    return o;
}
// for a number that is the same in all lanes
__device__ __forceinline__ bool cleared(float x) { return __builtin_amdgcn_readfirstlane(__float_as_uint(x)) == CLEARED; }

// the sum over the four groups of 16 lanes, in all of them
__device__ __forceinline__ float groups_sum(float x)
{
    const auto r = __builtin_amdgcn_permlane16_swap(__float_as_int(x), __float_as_int(x), false, false);
    x = __int_as_float((int)r[0]) + __int_as_float((int)r[1]);
    float lo, hi;
    halves(x, lo, hi);
    return lo + hi;
}

__device__ __forceinline__ int blocks_of(int Dv) { return (Dv + 15) / 16; }
// A wave's 16 columns of a state: s[2 p + half][r] is row 32 p + 8 (l / 16) + 4 half + r, column l % 16; zeros from Dk and Dv on.
template <int DK> struct Columns {
    f4 s[DK / 16];
    // from and to a caller's state [Dk][Dv]
    __device__ __forceinline__ void get(const float *from, int Dk, int Dv, int c, int lane)
    {
        if (!from) return clear();
        float x[DK / 16][4];
#pragma unroll
        for (int n = 0; n < DK / 16; ++n)
#pragma unroll
            for (int e = 0; e < 4; ++e) x[n][e] = from[(uint32_t)(min(32 * (n >> 1) + 8 * (lane >> 4) + 4 * (n & 1) + e, Dk - 1) * Dv + min(c, Dv - 1))];
#pragma unroll
        for (int n = 0; n < DK / 16; ++n)
#pragma unroll
            for (int e = 0; e < 4; ++e) s[n][e] = c < Dv && 32 * (n >> 1) + 8 * (lane >> 4) + 4 * (n & 1) + e < Dk ? x[n][e] : 0.f;
    }
    __device__ __forceinline__ void put(float *to, int Dk, int Dv, int c, int lane) const
    {
#pragma unroll
        for (int n = 0; n < DK / 16; ++n)
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const int d = 32 * (n >> 1) + 8 * (lane >> 4) + 4 * (n & 1) + e;
                if (c < Dv && d < Dk) to[(uint32_t)(d * Dv + c)] = s[n][e];
            }
    }
    // from and to a state of the kernels' own: block after block of 16 columns, 16 bytes a lane
    __device__ __forceinline__ void load(const float *block, int lane)
    {
#pragma unroll
        for (int n = 0; n < DK / 16; ++n) s[n] = seq::load<4>(block + 256 * n + 4 * lane);
    }
    __device__ __forceinline__ void store(float *block, int lane) const
    {
#pragma unroll
        for (int n = 0; n < DK / 16; ++n) seq::store<4>(block + 256 * n + 4 * lane, s[n]);
    }
    // sum over rows of x_d S_dc, x a step's row of K or Q in LDS
    template <class E> __device__ __forceinline__ float dot(const E *x, int lane) const
    {
        float sum = 0.f;
#pragma unroll
        for (int n = 0; n < DK / 16; ++n)
#pragma unroll
            for (int e = 0; e < 4; ++e) sum = fmaf((float)x[32 * (n >> 1) + 8 * (lane >> 4) + 4 * (n & 1) + e], s[n][e], sum);
        return groups_sum(sum);
    }
    template <class E> __device__ __forceinline__ void add(const E *x, float y, int lane)
    {
#pragma unroll
        for (int n = 0; n < DK / 16; ++n)
#pragma unroll
            for (int e = 0; e < 4; ++e) s[n][e] = fmaf((float)x[32 * (n >> 1) + 8 * (lane >> 4) + 4 * (n & 1) + e], y, s[n][e]);
    }
    __device__ __forceinline__ void scaled(float a)
    {
#pragma unroll
        for (int n = 0; n < DK / 16; ++n) s[n] *= a;
    }
    __device__ __forceinline__ void clear()
    {
#pragma unroll
        for (int n = 0; n < DK / 16; ++n) s[n] = f4{};
    }
};

__device__ __forceinline__ bool starts(const int *cut, int i) { return cut[i] != (i ? cut[i - 1] : 0); }

// One step as its definition has it; the state after it.  -> what is written, beta (v - S^T k)
template <class Tile, int DK> __device__ __forceinline__ float delta_step(const Tile &s, const DeltaRecord &rec, Columns<DK> &S, int i, float v, int lane)
{
    if (starts(rec.cut, i)) S.clear();
    S.scaled(rec.gate[i]);
    const float u = s.beta()[i] * (v - S.dot(s.k + i * Tile::LD, lane));
    S.add(s.k + i * Tile::LD, u, lane);
    return u;
}
// and the gradient of the state before step i from that after it, do and q being the step's.  -> the gradient of v
template <class Tile, int DK> __device__ __forceinline__ float delta_step_back(const Tile &s, Columns<DK> &D, int i, float dout, float scale, int lane)
{
    D.add(s.q + i * Tile::LD, scale * dout, lane);
    const float dv = s.beta()[i] * D.dot(s.k + i * Tile::LD, lane);
    D.add(s.k + i * Tile::LD, -dv, lane);
    return dv;
}
template <int DK> __device__ __forceinline__ void delta_pass_back(const DeltaRecord &rec, Columns<DK> &D, int i)
{
    if (starts(rec.cut, i)) D.clear();
    else D.scaled(rec.gate[i]);
}

// A lane's numbers of a column of a tensor of steps [..][Dv] (V, dO): where they lie, and as they are loaded
template <class E> struct Steps {
    uint32_t at[8];
    int rows;
    E x[8];
    __device__ __forceinline__ void offsets(int ts, int c, int Dv, int n_rows, int lane)
    {
        rows = n_rows;
#pragma unroll
        for (int i = 0; i < 8; ++i) at[i] = (uint32_t)(min(16 * (i >> 2) + 4 * (lane >> 4) + (i & 3), n_rows - 1) * ts + min(c, Dv - 1)) * (uint32_t)sizeof(E);
    }
    __device__ __forceinline__ void load(const E *tile, int ts, int c, int Dv, int n_rows, int lane)
    {
        if (n_rows != rows) offsets(ts, c, Dv, n_rows, lane);
#pragma unroll
        for (int i = 0; i < 8; ++i) x[i] = *plus(tile, at[i]);
    }
    __device__ __forceinline__ void get(bool mine, int lane, f4 (&v)[2]) const
    {
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i >> 2][i & 3] = mine && 16 * (i >> 2) + 4 * (lane >> 4) + (i & 3) < rows ? (float)x[i] : 0.f;
    }
};
template <class E> __device__ __forceinline__ void put_steps(E *tile, int ts, int c, bool mine, int rows, int lane, const f4 (&v)[2])
{
    if (!mine) return;
    const uint32_t at = (uint32_t)(4 * (lane >> 4) * ts + c);
    if (rows == CH) {
#pragma unroll
        for (int i = 0; i < 8; ++i) (tile + (16 * (i >> 2) + (i & 3)) * (long)ts)[at] = (E)v[i >> 2][i & 3];
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i)
            if (16 * (i >> 2) + 4 * (lane >> 4) + (i & 3) < rows) (tile + (16 * (i >> 2) + (i & 3)) * (long)ts)[at] = (E)v[i >> 2][i & 3];
    }
}

// U of a wave's columns from the state that enters and V.
template <class E, int DK, int N, class Tile> __device__ __forceinline__ void delta_u(const Tile &s, const typename Operand<E>::template Split<N> (&S)[DK / 32], const f4 (&v)[2], int rows, int lane, f4 (&u)[2])
{
    f4 r[2], ks[2] = {};
#pragma unroll
    for (int p = 0; p < DK / 32; ++p)
#pragma unroll
        for (int m = 0; m < 2; ++m) ks[m] = mul<E, N>(rows_of<E, Tile::LD>(s.k, m, p, lane), S[p], ks[m]);
#pragma unroll
    for (int m = 0; m < 2; ++m) {
        const f4 old = where(of_steps(s.since(), m, lane), ks[m]), beta = of_steps(s.beta(), m, lane);
#pragma unroll
        for (int e = 0; e < 4; ++e) r[m][e] = 16 * m + 4 * (lane >> 4) + e < rows ? beta[e] * (v[m][e] - old[e]) : 0.f;
        u[m] = f4{};
    }
    lower<Tile::LC>(s.t, r, lane, u);
}
// kd = (G_C. K) D, then Y = T^T (pd + kd) of a wave's columns, pd = P^T dO.
template <class E, int DK, int N, class Tile>
__device__ __forceinline__ void delta_y(const Tile &s, const typename Operand<E>::template Split<N> (&D)[DK / 32], const f4 (&pd)[2], int lane, f4 (&kd)[2], f4 (&y)[2])
{
    f4 du[2];
    kd[0] = kd[1] = f4{};
#pragma unroll
    for (int p = 0; p < DK / 32; ++p)
#pragma unroll
        for (int m = 0; m < 2; ++m) kd[m] = mul<E, N>(rows_of<E, Tile::LD>(s.k, m, p, lane), D[p], kd[m]);
#pragma unroll
    for (int m = 0; m < 2; ++m) {
        kd[m] = where(of_steps(s.until(), m, lane), kd[m]);
        du[m] = kd[m] + pd[m];
        y[m] = f4{};
    }
    upper<Tile::LC>(s.t, du, lane, y);
}

// ---------------------------------------------------------------- from state to state
// A workgroup per head, range of tiles and 16 columns of each of WAVES pairs of waves.  One wave of a pair takes the state from tile to tile and
// nothing else; the other does, a tile apart, what the chain does not wait for: the outputs, or in the backward
// direction what dO alone gives.  They hand each other registers as they are, through LDS, with one barrier a tile.  Two more waves bring tiles into LDS.
// Where heads are few, a head's tiles are cut into ranges.  What a range does to the state is a linear map and an addition, S -> M S + B; a first
// launch (MAPS) finds both, M by the same chain from the unit matrix's columns, a second goes from range to range, and the last has all
// ranges' first states.
// Bound by what follows upon what within a tile: state into planes, S^T k, T, K^T u, each a few matrix instructions deep, and waiting
// for LDS: 2.6 us a tile of 64 x 64 in bf16 (256 heads of 16 tiles: forward 42 us, backward 37), 2.9 of 128 x 128 (a head of 1024 tiles in 32 ranges:
// 89 us).  With one wave for both parts of a pair 72 and 62 us; with the second waves of the pairs, which then took longer than the first, bringing the tiles 46 and 43.
// A tile whose results hold a number that is not finite is taken again step by step as the definition has it, where nothing is multiplied by the
// zeros of other steps: a NaN reaches what comes after it in its episode and nothing else.
template <class E, int DK> struct DeltaPairs {
    static constexpr int tile = (int)sizeof(DeltaTile<E, DK, 3>), pair = 2 * 64 * (DK / 16 + 2) * 16, room = 160 * 1024;
    static constexpr int waves = 3 * tile + 4 * pair <= room ? 4 : 3 * tile + 2 * pair <= room ? 2 : 1;
};
// A launch that finds the maps of the forward direction has no outputs: keys alone, and four waves of a chain that bring their tiles themselves.  So two
// workgroups fit into a compute unit, and one has what the other waits for: the same head's maps, twice the state's columns, 103 us; in pairs of waves 147.
constexpr int MAPS_WAVES = 4;
template <class E, int DK> struct DeltaMaps {
    static constexpr int WAVES = MAPS_WAVES, BRING = 0, OTHERS = 0, PER_SIMD = 2;
    using Tile = DeltaKeys<E, DK, 3>;
    Tile tiles[3];
};
template <class E, int DK> struct DeltaChain {
    using Tile = DeltaTile<E, DK, 3>;
    static constexpr int WAVES = DeltaPairs<E, DK>::waves;
    static constexpr int BRING = 2;      // waves that do nothing but bring tiles
    static constexpr int OTHERS = WAVES + BRING, PER_SIMD = 1;
    DeltaTile<E, DK, 3> tiles[3];
    f4 state[2][WAVES][DK / 16][64];      // forward: the state that enters; backward: (scale g Q)^T dO
    f4 steps[2][WAVES][2][64];            // U; P^T dO
};
// How tiles are cut into ranges, and what is kept of each: M [DK][DK], B and the state it begins with [Dk][Dv]
constexpr int MOST_RANGES = 64;
struct DeltaRanges {
    int ranges;
    long per;                             // tiles of a range, but for the last
    float *m, *b, *first;                 // [heads][ranges][..]
    float *turned;                        // M^T, the backward direction's M, for a backward call to come; or NULL
};
// A wave's place: head, range and block of 16 columns; with MAPS, forward, the blocks behind those of the state are M's.
template <class E, int DK, bool MAPS, int WAVES, bool UNITS> struct ChainPlace {
    unsigned head;
    int range, block, blocks, bi, h, c;
    long tile0, n;                        // the range's first tile, how many it has
    bool mine, unit;                      // whether the column is one of the state's; whether the block is one of M's
    __device__ __forceinline__ ChainPlace(const DeltaIn &A, const DeltaRanges &R, int w, int lane)
    {
        blocks = blocks_of(A.Dv);
        // workgroups of the same tiles on the same XCD, where there are heads and ranges for that
        const unsigned all = gridDim.x / (unsigned)((blocks + (UNITS ? DK / 16 : 0) + WAVES - 1) / WAVES), which = blockIdx.x % all;
        block = (int)(blockIdx.x / all) * WAVES + w;
        head = which / (unsigned)R.ranges;
        range = (int)(which % (unsigned)R.ranges);
        bi = (int)(head / (unsigned)A.H);
        h = (int)(head % (unsigned)A.H);
        c = 16 * block + (lane & 15);
        mine = c < A.Dv;
        unit = UNITS && block >= blocks;
        tile0 = range * R.per;
        n = min(R.per, A.tiles - tile0);
    }
    // the columns that the chain begins with
    __device__ __forceinline__ void begin(const DeltaIn &A, const DeltaRanges &R, const float *given, Columns<DK> &S, int lane) const
    {
        if (MAPS) {
            S.clear();
            if (unit)
#pragma unroll
                for (int n = 0; n < DK / 16; ++n)
#pragma unroll
                    for (int e = 0; e < 4; ++e) S.s[n][e] = 32 * (n >> 1) + 8 * (lane >> 4) + 4 * (n & 1) + e == c - 16 * blocks ? 1.f : 0.f;
        } else {
            const float *from = R.ranges > 1 ? R.first + (long)range * A.Dk * A.Dv + (long)head * R.ranges * A.Dk * A.Dv : given ? given + (long)head * A.Dk * A.Dv : nullptr;
            S.get(from, A.Dk, A.Dv, c, lane);
        }
    }
    // and ends with, in a launch that finds maps
    __device__ __forceinline__ void end(const DeltaIn &A, const DeltaRanges &R, const Columns<DK> &S, int lane) const
    {
        const long at = (long)head * R.ranges + range;
        if (!unit) S.put(R.b + at * A.Dk * A.Dv, A.Dk, A.Dv, c, lane);
        else {
            const int column = c - 16 * blocks;
            S.put(R.m + at * DK * DK, DK, DK, column, lane);
            if (R.turned && column < DK)
#pragma unroll
                for (int n = 0; n < DK / 16; ++n) store<4>(R.turned + at * DK * DK + column * DK + 32 * (n >> 1) + 8 * (lane >> 4) + 4 * (n & 1), S.s[n]);
        }
    }
};

template <class E, int DK, bool MAPS> using ForwardChain = std::conditional_t<MAPS, DeltaMaps<E, DK>, DeltaChain<E, DK>>;
template <class Chain> constexpr int threads_of = 64 * (Chain::WAVES + Chain::OTHERS);
template <class E, int DK, bool MAPS> __global__ __launch_bounds__((threads_of<ForwardChain<E, DK, MAPS>>), (ForwardChain<E, DK, MAPS>::PER_SIMD)) void k_delta(DeltaArgs A, DeltaRanges R)
{
    using Chain = ForwardChain<E, DK, MAPS>;
    using Tile = typename Chain::Tile;
    constexpr int WAVES = Chain::WAVES;
    extern __shared__ __align__(16) unsigned char lds[];
    Chain &L = *reinterpret_cast<Chain *>(lds);
    const int lane = threadIdx.x & 63, w = (threadIdx.x >> 6) % WAVES;
    const bool chain = threadIdx.x < 64 * WAVES;
    const ChainPlace<E, DK, MAPS, WAVES, MAPS> at(A, R, w, lane);
    const E *v = head_of<E>(A.v, A.sv, at.bi, at.h) + at.tile0 * CH * A.sv.ts;
    const DeltaRecord *records = (const DeltaRecord *)A.records + at.head * A.tiles + at.tile0;
    auto rows_in = [&](long tile) { return (int)min((long)CH, A.T - (at.tile0 + tile) * CH); };
    // what is brought in turn i, while tile i is worked on: tile i + 1 into LDS, i + 2 on its way
    constexpr int BRINGING = MAPS ? WAVES : Chain::BRING;
    auto bring = [&](auto &fetch, long i) {
        if (i < 0 && at.n > 0) {
            fetch.begin(A, (const DeltaRecord *)A.records, at.head, at.bi, at.h, threadIdx.x % (128 * WAVES));
            fetch.load(A, at.tile0);
        }
        if (i + 1 < at.n) fetch.put(L.tiles[(i + 1) % 3], A.Dk);
        if (i + 2 < at.n) fetch.load(A, at.tile0 + i + 2);
    };
    if (chain) {
        Columns<DK> S;
        at.begin(A, R, A.s0, S, lane);
        Steps<E> vs;
        vs.rows = 0;
        if (at.n > 0) vs.load(v, (int)A.sv.ts, at.c, A.Dv, rows_in(0), lane);
        DeltaFetch<E, DK, 64 * BRINGING, 3, Tile> fetch;
        if (MAPS) bring(fetch, -1);
        __syncthreads();
        for (long i = 0; i <= at.n; ++i) {
            if (MAPS) bring(fetch, i);
            if (i < at.n) {
                const Tile &s = L.tiles[i % 3];
                const int rows = rows_in(i);
                f4 val[2], u[2], next[DK / 16];
                vs.get(at.mine, lane, val);
                if (i + 1 < at.n) vs.load(v + (i + 1) * CH * A.sv.ts, (int)A.sv.ts, at.c, A.Dv, rows_in(i + 1), lane);
                if constexpr (!MAPS)
#pragma unroll
                    for (int n = 0; n < DK / 16; ++n) L.state[i & 1][w][n][lane] = S.s[n];
                typename Operand<E>::template Split<3> sp[DK / 32];
#pragma unroll
                for (int p = 0; p < DK / 32; ++p) sp[p] = split<E, 3>(S.s[2 * p], S.s[2 * p + 1]);
                delta_u<E, DK, 3>(s, sp, val, rows, lane, u);
                if constexpr (!MAPS) {
                    L.steps[i & 1][w][0][lane] = u[0];
                    L.steps[i & 1][w][1][lane] = u[1];
                }
                const auto up = split<E, 3>(where(of_steps(s.until(), 0, lane), u[0]), where(of_steps(s.until(), 1, lane), u[1]));
                const float left = s.since()[CH - 1];
#pragma unroll
                for (int n = 0; n < DK / 16; ++n) next[n] = left * S.s[n];
                if (cleared(left))      // whatever it was
#pragma unroll
                    for (int n = 0; n < DK / 16; ++n) next[n] = f4{};
#pragma unroll
                for (int n = 0; n < DK / 16; ++n) next[n] = mul<E, 3>(state_columns<E, Tile::LD>(s.k, n, lane), up, next[n]);
                if (__any(nothing(next) != 0.f)) {
                    for (int t = 0; t < rows; ++t) delta_step(s, records[i], S, t, at.mine ? (float)v[(i * CH + t) * A.sv.ts + at.c] : 0.f, lane);
                } else {
#pragma unroll
                    for (int n = 0; n < DK / 16; ++n) S.s[n] = next[n];
                }
            }
            lds_barrier();
        }
        if (MAPS) at.end(A, R, S, lane);
        else if (A.last && at.tile0 + at.n >= A.tiles) S.put(A.last + (long)at.head * A.Dk * A.Dv, A.Dk, A.Dv, at.c, lane);
    } else if (threadIdx.x >= 128 * WAVES) {
        DeltaFetch<E, DK, 64 * BRINGING, 3, Tile> fetch;
        bring(fetch, -1);
        __syncthreads();
        for (long i = 0; i <= at.n; ++i) {
            bring(fetch, i);
            lds_barrier();
        }
    } else if constexpr (!MAPS) {
        E *o = head_of<E>(A.o, A.so, at.bi, at.h) + at.tile0 * CH * A.so.ts;
        __syncthreads();
        for (long i = 0; i <= at.n; ++i) {
            if (i > 0) {
                const long tile = i - 1;
                const Tile &s = L.tiles[tile % 3];
                const int rows = rows_in(tile);
                Columns<DK> S;
                f4 u[2], out[2];
#pragma unroll
                for (int n = 0; n < DK / 16; ++n) S.s[n] = L.state[tile & 1][w][n][lane];
                u[0] = L.steps[tile & 1][w][0][lane];
                u[1] = L.steps[tile & 1][w][1][lane];
                if (A.states && at.block < at.blocks) S.store(A.states + ((at.head * A.tiles + at.tile0 + tile) * at.blocks + at.block) * 16 * DK, lane);
                typename Operand<E>::template Split<2> sp[DK / 32];      // o is rounded to bf16: 16 bits of the state do
#pragma unroll
                for (int p = 0; p < DK / 32; ++p) sp[p] = split<E, 2>(S.s[2 * p], S.s[2 * p + 1]);
                out[0] = out[1] = f4{};
#pragma unroll
                for (int p = 0; p < DK / 32; ++p)
#pragma unroll
                    for (int m = 0; m < 2; ++m) out[m] = mul<E, 2>(rows_of<E, Tile::LD>(s.q, m, p, lane), sp[p], out[m]);
#pragma unroll
                for (int m = 0; m < 2; ++m) out[m] = where(of_steps(s.since(), m, lane), A.scale * out[m]);
                lower<Tile::LC>(s.p, u, lane, out);
                E *to = o + tile * CH * A.so.ts;
                if (__any(nothing(out) != 0.f)) {
                    for (int t = 0; t < rows; ++t) {
                        delta_step(s, records[tile], S, t, at.mine ? (float)v[(tile * CH + t) * A.sv.ts + at.c] : 0.f, lane);
                        const float x = A.scale * S.dot(s.q + t * Tile::LD, lane);
                        if (at.mine && lane < 16) to[t * A.so.ts + at.c] = (E)x;
                    }
                } else put_steps(to, (int)A.so.ts, at.c, at.mine, rows, lane, out);
            }
            lds_barrier();
        }
    }
}

// The gradient of the state, from the last tile to the first: what leaves each tile is kept, for k_delta_grad.  A range's map is the transposed
// of its map in the other direction, which the forward call has kept; MAPS finds the additions alone.
template <class E, int DK, bool MAPS> __global__ __launch_bounds__((threads_of<DeltaChain<E, DK>>)) void k_delta_back(DeltaGradArgs A, DeltaRanges R)
{
    using Tile = DeltaTile<E, DK, 3>;
    using Chain = DeltaChain<E, DK>;
    constexpr int WAVES = Chain::WAVES;
    extern __shared__ __align__(16) unsigned char lds[];
    Chain &L = *reinterpret_cast<Chain *>(lds);
    const int lane = threadIdx.x & 63, w = (threadIdx.x >> 6) % WAVES;
    const bool chain = threadIdx.x < 64 * WAVES;
    const ChainPlace<E, DK, MAPS, WAVES, false> at(A, R, w, lane);
    const E *dout = head_of<E>(A.dout, A.sdo, at.bi, at.h) + at.tile0 * CH * A.sdo.ts;
    const DeltaRecord *records = (const DeltaRecord *)A.records + at.head * A.tiles + at.tile0;
    auto rows_in = [&](long tile) { return (int)min((long)CH, A.T - (at.tile0 + tile) * CH); };
    // turn i of the wave that prepares is for tile n - 1 - i, of the chain for the one before that; meanwhile the one after it comes into LDS
    using Fetch = DeltaFetch<E, DK, 64 * Chain::BRING, 3>;
    auto bring = [&](Fetch &fetch, long i) {
        if (i < 0 && at.n > 0) {
            fetch.begin(A, (const DeltaRecord *)A.records, at.head, at.bi, at.h, threadIdx.x % (128 * WAVES));
            fetch.load(A, at.tile0 + at.n - 1);
        }
        const long tile = at.n - 2 - i;
        if (tile >= 0) fetch.put(L.tiles[tile % 3], A.Dk);
        if (tile >= 1) fetch.load(A, at.tile0 + tile - 1);
    };
    if (threadIdx.x >= 128 * WAVES) {
        Fetch fetch;
        bring(fetch, -1);
        __syncthreads();
        for (long i = 0; i <= at.n; ++i) {
            bring(fetch, i);
            lds_barrier();
        }
    } else if (chain) {
        Columns<DK> D;
        at.begin(A, R, A.dlast, D, lane);
        __syncthreads();
        for (long i = 0; i <= at.n; ++i) {
            if (i > 0) {
                const long tile = at.n - i;
                const Tile &s = L.tiles[tile % 3];
                if (!MAPS && at.block < at.blocks) D.store(A.into + ((at.head * A.tiles + at.tile0 + tile) * at.blocks + at.block) * 16 * DK, lane);
                typename Operand<E>::template Split<3> sp[DK / 32];
#pragma unroll
                for (int p = 0; p < DK / 32; ++p) sp[p] = split<E, 3>(D.s[2 * p], D.s[2 * p + 1]);
                const f4 pd[2] = {L.steps[tile & 1][w][0][lane], L.steps[tile & 1][w][1][lane]};
                f4 kd[2], y[2], next[DK / 16];
                delta_y<E, DK, 3>(s, sp, pd, lane, kd, y);
#pragma unroll
                for (int m = 0; m < 2; ++m) y[m] = where(of_steps(s.since(), m, lane), -of_steps(s.beta(), m, lane) * y[m]);
                const auto yp = split<E, 3>(y[0], y[1]);
                const float left = s.since()[CH - 1];
#pragma unroll
                for (int n = 0; n < DK / 16; ++n) next[n] = L.state[tile & 1][w][n][lane] + left * D.s[n];
                if (cleared(left))      // whatever it was
#pragma unroll
                    for (int n = 0; n < DK / 16; ++n) next[n] = L.state[tile & 1][w][n][lane];
#pragma unroll
                for (int n = 0; n < DK / 16; ++n) next[n] = mul<E, 3>(state_columns<E, Tile::LD>(s.k, n, lane), yp, next[n]);
                if (__any(nothing(next) != 0.f)) {
                    for (int t = rows_in(tile) - 1; t >= 0; --t) {
                        delta_step_back(s, D, t, at.mine ? (float)dout[(tile * CH + t) * A.sdo.ts + at.c] : 0.f, A.scale, lane);
                        delta_pass_back(records[tile], D, t);
                    }
                } else {
#pragma unroll
                    for (int n = 0; n < DK / 16; ++n) D.s[n] = next[n];
                }
            }
            lds_barrier();
        }
        if (MAPS) at.end(A, R, D, lane);
        else if (A.ds0 && at.range == 0) D.put(A.ds0 + (long)at.head * A.Dk * A.Dv, A.Dk, A.Dv, at.c, lane);
    } else {
        Steps<E> ds;
        ds.rows = 0;
        auto get = [&](long tile) { ds.load(dout + tile * CH * A.sdo.ts, (int)A.sdo.ts, at.c, A.Dv, rows_in(tile), lane); };
        if (at.n > 0) get(at.n - 1);
        __syncthreads();
        for (long i = 0; i <= at.n; ++i) {
            const long tile = at.n - 1 - i;
            if (tile >= 0) {
                f4 out[2], pd[2] = {}, x[2];
                ds.get(at.mine, lane, out);
                if (tile > 0) get(tile - 1);
                const Tile &s = L.tiles[tile % 3];
                upper<Tile::LC>(s.p, out, lane, pd);
                L.steps[tile & 1][w][0][lane] = pd[0];
                L.steps[tile & 1][w][1][lane] = pd[1];
#pragma unroll
                for (int m = 0; m < 2; ++m) x[m] = where(of_steps(s.since(), m, lane), A.scale * out[m]);
                const auto xp = split<E, 3>(x[0], x[1]);
#pragma unroll
                for (int n = 0; n < DK / 16; ++n) L.state[tile & 1][w][n][lane] = mul<E, 3>(state_columns<E, Tile::LD>(s.q, n, lane), xp, f4{});
            }
            lds_barrier();
        }
    }
}

// From range to range: the state each begins with, forward from s0 or backward from dlast.  A workgroup per head and 16 columns, a wave per 16 rows;
// a result of 16 x 16 is the next right operand as it is, in its place in LDS.  As many waves more take it from there to memory: a wave that loads
// maps would wait for its own stores.  What enters a range with an episode's start leaves nothing, whatever it is.
// Many ranges go in groups of `span`: COMPOSE finds each group's map and addition, 16 columns of either a workgroup, from the unit matrix and zeros; then from
// group to group; then within all groups at once, `given` being what enters each.  Bound by bringing 64 KB a range (of 128 x 128) to each compute unit: 32 ranges
// of four heads one after the other 69 us, in groups of 8 18 + 31.
template <int DK, bool BACK, bool COMPOSE>
__global__ __launch_bounds__((COMPOSE ? 4 : 8) * DK) void k_delta_join(DeltaRanges R, int span, const float *given, DeltaRanges to, const DeltaRecord *records, long tiles, int Dk, int Dv)
{
    constexpr int THREADS = (COMPOSE ? 4 : 8) * DK;
    __shared__ f4 state[2][DK / 16][64];
    __shared__ int forgets[MOST_RANGES];      // whether an episode starts in a range
    const int lane = threadIdx.x & 63, w = (threadIdx.x >> 6) % (DK / 16), g = lane >> 4;
    const bool stores = threadIdx.x >= 4 * DK;
    const unsigned mine = (unsigned)blocks_of(Dv), blocks = COMPOSE ? mine + DK / 16 : mine, groups = (unsigned)((R.ranges + span - 1) / span);
    // which: head and group; its workgroups, which read the same maps, on the same XCD
    const unsigned all = gridDim.x / blocks, block = blockIdx.x / all, which = blockIdx.x % all, head = which / groups;
    const int first = (int)(which % groups) * span, n = min(span, R.ranges - first);
    const bool unit = COMPOSE && block >= mine;      // 16 columns of the map
    const int c = 16 * (int)(unit ? block - mine : block) + (lane & 15), row = 16 * w + 4 * g;
    const long size = (long)Dk * Dv, base = (long)head * R.ranges + first;
    auto in = [&](int e) { return c < Dv && row + e < Dk; };
    auto range = [&](int i) { return BACK ? n - 1 - i : i; };
    for (int r = threadIdx.x; r < n; r += THREADS) forgets[r] = 0;
    __syncthreads();
    for (long t = first * R.per + threadIdx.x; t < min(tiles, (first + n) * R.per); t += THREADS)
        if (records[head * tiles + t].cut[CH - 1]) forgets[t / R.per - first] = 1;
    if (stores) {
        for (int i = 0; i < n; ++i) {
            lds_barrier();
            const f4 S = state[i & 1][w][lane];
            float *out = R.first + (base + range(i)) * size;
#pragma unroll
            for (int e = 0; e < 4; ++e)
                if (in(e)) out[(row + e) * Dv + c] = S[e];
        }
        return;
    }
    f4 S = {}, a[DK / 16], add;
    if (!COMPOSE && given)
#pragma unroll
        for (int e = 0; e < 4; ++e)
            if (in(e)) S[e] = given[which * size + (row + e) * Dv + c];
    if (unit)
#pragma unroll
        for (int e = 0; e < 4; ++e) S[e] = row + e == c ? 1.f : 0.f;
    // a range's map is under way while the one before is applied
    auto get = [&](int i) {
        const float *m = R.m + (base + range(i)) * DK * DK + (16 * w + (lane & 15)) * DK + 4 * g, *b = R.b + (base + range(i)) * size;
#pragma unroll
        for (int kb = 0; kb < DK / 16; ++kb) a[kb] = load<4>(m + 16 * kb);
#pragma unroll
        for (int e = 0; e < 4; ++e) add[e] = b[min(row + e, Dk - 1) * Dv + min(c, Dv - 1)];
    };
    get(0);
    for (int i = 0; i < n; ++i) {
        state[i & 1][w][lane] = S;
        lds_barrier();
        if (!COMPOSE && i + 1 == n) break;
        f4 next, other = {};
#pragma unroll
        for (int e = 0; e < 4; ++e) next[e] = !unit && in(e) ? add[e] : 0.f;
        if (!forgets[range(i)]) {
#pragma unroll
            for (int kb = 0; kb < DK / 16; kb += 2) {
                next = mm4(a[kb], state[i & 1][kb][lane], next);
                other = mm4(a[kb + 1], state[i & 1][kb + 1][lane], other);
            }
            next += other;
        }
        get(min(i + 1, n - 1));      // of the last range, whose map nobody needs, too
        S = next;
    }
    if (COMPOSE) {
        float *out = unit ? to.m + (long)which * DK * DK + row * DK + c : to.b + which * size + (long)row * Dv + c;
#pragma unroll
        for (int e = 0; e < 4; ++e)
            if (unit || in(e)) out[(long)e * (unit ? DK : Dv)] = S[e];
    }
}

// Few steps, of an acting agent say: the definition, step by step, a wave per 16 columns of a head's state.  Read and written once, the state is the
// traffic: 32 x 8 x 64 x 64 and one step 6 us, most of it a launch's way to memory and back; 2048 x 8 heads 120 us, 540 MB at 4.5 TB/s.  Up to 8 steps: 2048 x 8 x 64
// x 64 take 413 us with 8, the other way 443 with 9, 32 x 8 x 64 x 64 13 and 14; at 32 x 4 x 128 x 128 the other way would be quicker from 6 steps on (8: 21 us, 9: 17).
constexpr long STEPS_MOST = 8;
template <class E, int DK> __global__ __launch_bounds__(256) void k_delta_few(DeltaArgs A)
{
    const int lane = threadIdx.x & 63, g = lane >> 4, blocks = blocks_of(A.Dv);
    const unsigned at = blockIdx.x * 4 + (threadIdx.x >> 6), head = at / (unsigned)blocks;
    if (head >= (unsigned)(A.B * A.H)) return;
    const int bi = (int)(head / (unsigned)A.H), h = (int)(head % (unsigned)A.H), c = 16 * (int)(at % (unsigned)blocks) + (lane & 15);
    const bool mine = c < A.Dv;
    const E *q = head_of<E>(A.q, A.sq, bi, h), *k = head_of<E>(A.k, A.sk, bi, h), *v = head_of<E>(A.v, A.sv, bi, h), *f = head_of<E>(A.f, A.sf, bi, h), *b = head_of<E>(A.b, A.sb, bi, h);
    E *o = head_of<E>(A.o, A.so, bi, h);
    const long size = (long)A.Dk * A.Dv;
    Columns<DK> S;
    S.get(A.s0 ? A.s0 + head * size : nullptr, A.Dk, A.Dv, c, lane);
    for (long t = 0; t < A.T; ++t) {
        vec<E, 8> kt[DK / 32], qt[DK / 32];
#pragma unroll
        for (int p = 0; p < DK / 32; ++p) {
            kt[p] = load8<E>(k + t * A.sk.ts, 32 * p + 8 * g, A.Dk, true, A.wide);
            qt[p] = load8<E>(q + t * A.sq.ts, 32 * p + 8 * g, A.Dk, true, A.wide);
        }
        const float x = (float)v[t * A.sv.ts + min(c, A.Dv - 1)], gate = 1.f / (1.f + expf(-(float)f[t * A.sf.ts])), rate = 1.f / (1.f + expf(-(float)b[t * A.sb.ts]));
        if (A.reset && A.reset[bi * A.reset_bs + t * A.reset_ts]) S.clear();
        S.scaled(gate);
        float held = 0.f, out = 0.f;
#pragma unroll
        for (int n = 0; n < DK / 16; ++n)
#pragma unroll
            for (int e = 0; e < 4; ++e) held = fmaf((float)kt[n >> 1][4 * (n & 1) + e], S.s[n][e], held);
        const float u = rate * ((mine ? x : 0.f) - groups_sum(held));
#pragma unroll
        for (int n = 0; n < DK / 16; ++n)
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                S.s[n][e] = fmaf((float)kt[n >> 1][4 * (n & 1) + e], u, S.s[n][e]);
                out = fmaf((float)qt[n >> 1][4 * (n & 1) + e], S.s[n][e], out);
            }
        out = groups_sum(out);
        if (mine && g == 0) o[t * A.so.ts + c] = (E)(A.scale * out);
    }
    if (A.last) S.put(A.last + head * size, A.Dk, A.Dv, c, lane);
}

// ---------------------------------------------------------------- gradients
// Matrices of the gradients' products, in LDS: results are put in four rows of a column at a time and read again as operands, both ways round.
// bf16 lies by columns, so that four rows are one store, and the transposing read makes rows of it; fp32, which has none, by rows.  Rounded holds fp32
// numbers, in bf16 as two planes with 16 bits together, Given an input's.
template <int R, int C> struct Plane {
    static constexpr int LD = R + 8;
    alignas(16) bf16 m[C * LD];
    using s4 = vec<short, 4>;
    // four rows, those of a group's lanes 4 x c.. to c.. + 3, of the 16 columns from i0 on: each lane gets a row of the matrix
    __device__ __forceinline__ s4 turned(int i0, int j, int lane) const
    {
        typedef __attribute__((address_space(3))) s4 *At;
        return __builtin_amdgcn_ds_read_tr16_b64_v4i16((At)(m + (j + ((lane & 15) >> 2)) * LD + i0 + 4 * (lane & 3)));
    }
    static __device__ __forceinline__ b8 joined(s4 a, s4 b) { return __builtin_bit_cast(b8, (vec<short, 8>){a[0], a[1], a[2], a[3], b[0], b[1], b[2], b[3]}); }
    __device__ __forceinline__ void put(int i, int j, uint32_t ab, uint32_t cd) { *reinterpret_cast<vec<uint32_t, 2> *>(m + j * LD + i) = vec<uint32_t, 2>{ab, cd}; }
    __device__ __forceinline__ s4 column(int i, int j) const { return load<4>(reinterpret_cast<const short *>(m) + j * LD + i); }
    __device__ __forceinline__ b8 rows(int i0, int j, int lane) const { return joined(turned(i0, j + 8 * (lane >> 4), lane), turned(i0, j + 8 * (lane >> 4) + 4, lane)); }
    __device__ __forceinline__ b8 pair(int i0, int lane) const { return joined(turned(i0, 4 * (lane >> 4), lane), turned(i0, 16 + 4 * (lane >> 4), lane)); }
    __device__ __forceinline__ b8 pair_of_columns(int j0, int lane) const { return joined(column(4 * (lane >> 4), j0 + (lane & 15)), column(16 + 4 * (lane >> 4), j0 + (lane & 15))); }
};
template <class E, int R, int C> struct Rounded;
template <int R, int C> struct Rounded<float, R, C> {
    static constexpr int LD = C + 4;
    alignas(16) float m[R * LD];
    // rows i.. to i + 3 of column j
    __device__ __forceinline__ void put(int i, int j, f4 v)
    {
#pragma unroll
        for (int e = 0; e < 4; ++e) m[(i + e) * LD + j] = v[e];
    }
    __device__ __forceinline__ f4 column(int i, int j) const { const float *a = m + i * LD + j; return f4{a[0], a[LD], a[2 * LD], a[3 * LD]}; }
    // left or right operands: row i0 + lane % 16, columns j + 8 (lane / 16)..
    __device__ __forceinline__ f8 rows(int i0, int j, int lane) const { return eight(m + (i0 + (lane & 15)) * LD + j + 8 * (lane >> 4)); }
    // that row's columns 4 (lane / 16).. and 16 + 4 (lane / 16)..
    __device__ __forceinline__ f8 pair(int i0, int lane) const
    {
        const float *a = m + (i0 + (lane & 15)) * LD + 4 * (lane >> 4);
        return both(load<4>(a), load<4>(a + 16));
    }
    // the same of the transposed matrix
    __device__ __forceinline__ f8 pair_of_columns(int j0, int lane) const { return both(column(4 * (lane >> 4), j0 + (lane & 15)), column(16 + 4 * (lane >> 4), j0 + (lane & 15))); }
};
template <int R, int C> struct Rounded<bf16, R, C> {
    Plane<R, C> p[2];
    __device__ __forceinline__ void put(int i, int j, f4 v)
    {
        uint32_t a[4], b[4];
#pragma unroll
        for (int e = 0; e < 4; ++e) a[e] = __float_as_uint(v[e]), b[e] = __float_as_uint(v[e] - __uint_as_float(a[e] & 0xFFFF0000u)) + 0x8000u;
        p[0].put(i, j, upper_halves(a[0], a[1]), upper_halves(a[2], a[3]));
        p[1].put(i, j, upper_halves(b[0], b[1]), upper_halves(b[2], b[3]));
    }
    static __device__ __forceinline__ uint32_t upper_halves(uint32_t lo, uint32_t hi) { return __builtin_amdgcn_perm(hi, lo, 0x07060302u); }
    __device__ __forceinline__ f4 column(int i, int j) const
    {
        const vec<short, 4> a = p[0].column(i, j), b = p[1].column(i, j);
        f4 o;
#pragma unroll
        for (int e = 0; e < 4; ++e) o[e] = __uint_as_float((uint32_t)(uint16_t)a[e] << 16) + __uint_as_float((uint32_t)(uint16_t)b[e] << 16);
        return o;
    }
    __device__ __forceinline__ Planes<2> rows(int i0, int j, int lane) const { return Planes<2>{{p[0].rows(i0, j, lane), p[1].rows(i0, j, lane)}}; }
    __device__ __forceinline__ Planes<2> pair(int i0, int lane) const { return Planes<2>{{p[0].pair(i0, lane), p[1].pair(i0, lane)}}; }
    __device__ __forceinline__ Planes<2> pair_of_columns(int j0, int lane) const { return Planes<2>{{p[0].pair_of_columns(j0, lane), p[1].pair_of_columns(j0, lane)}}; }
};
template <class E, int R, int C> struct Given : Rounded<float, R, C> {};
template <int R, int C> struct Given<bf16, R, C> : Plane<R, C> {
    __device__ __forceinline__ void put(int i, int j, f4 v)
    {
        Plane<R, C>::put(i, j, Rounded<bf16, R, C>::upper_halves(__float_as_uint(v[0]), __float_as_uint(v[1])), Rounded<bf16, R, C>::upper_halves(__float_as_uint(v[2]), __float_as_uint(v[3])));
    }
};
template <class E, int DK> struct DeltaGradTile {
    DeltaTile<E, DK, 7> s;
    Given<E, CH, COLS> dout;
    Rounded<E, CH, COLS> u, y;
    Rounded<E, DK, COLS> state, back;       // the state that enters, the gradient of the one that leaves
    Rounded<E, CH, CH> dp, dn;              // of P's and N's products
    float enters[DK / 16][CH], yu[2][4][CH], leaves[2][4][CH];      // sums over 16 columns each of e_i; for even and odd tiles of Y.u, l_j
    float pairs[2][2][4][16];               // for even and odd tiles, of dP P and dN N: gate_pairs'
    float ends[8];                          // of each wave: g_C <D, S>
    int wrong[8];                           // whether it has met a number that is not finite
};

// Of 16 neighbouring lanes: the sum of those before a lane; of it and those behind.
template <int CTRL> __device__ __forceinline__ float moved(float x) { return __uint_as_float(__builtin_amdgcn_update_dpp(0u, __float_as_uint(x), CTRL, 0xF, 0xF, false)); }
__device__ __forceinline__ float sum_before(float x)
{
    x = moved<0x111>(x);
    x += moved<0x111>(x);
    x += moved<0x112>(x);
    x += moved<0x114>(x);
    return x + moved<0x118>(x);
}
__device__ __forceinline__ float sum_from(float x)
{
    x += moved<0x101>(x);
    x += moved<0x102>(x);
    x += moved<0x104>(x);
    return x + moved<0x108>(x);
}
// The sums of e_ij over j < t <= i for every t, of 16 x 16 as a result holds them, rows i0.. and column j, into four rows of 16: 0 and 3 from the parts on the diagonal,
// for t of the first and the second 16 steps; from the part below it 1, for t of the first 16, and 2, the rows' sums, whose own sums from t on are for t of the second.
__device__ __forceinline__ void gate_pairs(f4 e, int i0, int j, bool diagonal, int lane, float (&out)[4][16])
{
    const int col = lane & 15;
    if (diagonal) {
        float sum = 0.f;
#pragma unroll
        for (int r = 0; r < 4; ++r) {
            const float x = sum_before(e[r]);
            sum += i0 + r >= j ? x : 0.f;
        }
        sum = groups_sum(sum);
        if (lane < 16) out[j < 16 ? 0 : 3][col] = sum;
    } else {
        const float x = sum_before(groups_sum((e[0] + e[1]) + (e[2] + e[3])));
        if (lane < 16) out[1][col] = x;
#pragma unroll
        for (int r = 0; r < 4; ++r) {
            const float sum = group_fold(e[r], 16, add);
            if (col == 0) out[2][i0 + r - 16] = sum;
        }
    }
}

// All gradients but the state's: workgroups of eight waves, `per` tiles each, one after the other, a tile's loads under way while the one before
// is worked on.  Of each 64 columns of the state four waves form U, four Y; then dP and dN; then the products over all columns, a wave having 16 of
// the columns of dq and dk for half of the steps (DK = 128: for all).
// 32 x 512 x 8 x 64 in bf16: 121 us, 16 tiles of 64 KB a compute unit, 2.2 TB/s.  What bounds it is the way through a tile, 16000 cycles in four parts between
// barriers, in which two waves a SIMD share the vector instructions.  Both directions together: with four waves a workgroup
// 461 us, with eight 313, with the next tile's loads under way and states as the waves hold them 252, with matrices by columns and arguments read anew 216; the gates'
// gradients from terms that have the gate as a factor, not from differences, took 8 us more.  The form for 128 columns needs more than the 256 registers of a wave and
// keeps 104 (bf16) or 120 bytes a lane in scratch memory: 32 x 512 x 4 x 128 in bf16 takes 175 us.
template <class E, int DK> __global__ __launch_bounds__(512, 2) void k_delta_grad(DeltaGradArgs given, int per)
{
    using Op = Operand<E>;
    using Tile = DeltaTile<E, DK, 7>;
    using Grad = DeltaGradTile<E, DK>;
    constexpr int NM = DK == 128 ? 2 : 1;
    // The arguments are more than scalar registers hold.  Each part reads them anew: kept over all of them they would be moved to vector registers' lanes
    // and back.
    auto arguments = []() -> const DeltaGradArgs & {
        auto *p = (const __attribute__((address_space(4))) DeltaGradArgs *)__builtin_amdgcn_kernarg_segment_ptr();
        asm volatile("" : "+s"(p));
        return *(const DeltaGradArgs *)p;
    };
    const DeltaGradArgs &A = arguments();
    extern __shared__ __align__(16) unsigned char lds[];
    Grad &g = *reinterpret_cast<Grad *>(lds);
    Tile &s = g.s;
    const int tid = threadIdx.x, lane = tid & 63, w = tid >> 6, wc = w & 3, grp = lane >> 4, col = lane & 15;
    const bool for_y = w >= 4;
    const unsigned all = (unsigned)(A.B * A.H * A.tiles), tiles = (unsigned)A.tiles;
    unsigned id = blockIdx.x * (unsigned)per;
    const unsigned stop = min(all, id + (unsigned)per);
    const int blocks = blocks_of(A.Dv);
    // the part of dP (waves 0..2) or dN (4..6): rows ti.., columns tj.., up to the diagonal
    const int ti = wc ? 16 : 0, tj = wc == 2 ? 16 : 0;
    // and of dq and dk: columns 16 d.., steps 16 m..
    const int d = w % (DK / 16), m0 = NM == 2 ? 0 : w / (DK / 16), dk = 16 * d + col;
    const bool has = m0 < 2;
    // what is under way: a tile, and of 64 columns V and the state that enters, or dO and the gradient of the one that leaves
    DeltaFetch<E, DK, 512, 7> fetch;
    Steps<E> in;
    Columns<DK> st;
    const E *steps = nullptr;
    const long ts = for_y ? A.sdo.ts : A.sv.ts;
    const float *states = for_y ? A.into : A.states;
    in.rows = 0;
    auto get = [&](unsigned which, int sl, bool new_head) {
        const DeltaGradArgs &A = arguments();
        const unsigned head = which / tiles, tile = which % tiles;
        const int bi = (int)(head / (unsigned)A.H), h = (int)(head % (unsigned)A.H), rows = (int)min((long)CH, A.T - (long)tile * CH), c = sl + 16 * wc + col;
        if (new_head) {
            fetch.begin(A, (const DeltaRecord *)A.records, head, bi, h, tid);
            steps = for_y ? head_of<E>(A.dout, A.sdo, bi, h) : head_of<E>(A.v, A.sv, bi, h);
        }
        if (sl == 0) fetch.load(A, tile);
        if (A.Dv > COLS) in.rows = 0;      // other columns
        in.load(steps + (long)tile * CH * ts, (int)ts, c, A.Dv, rows, lane);
        st.load(states + ((long)which * blocks + min(sl / 16 + wc, blocks - 1)) * 16 * DK, lane);
    };
    // The gradients of gates and rates are formed from the sums of all waves, a step per lane, by the last wave, one tile late, while the others have
    // dP and dN.  What that takes of the tile is kept meanwhile.
    const unsigned first = id;
    const int step = lane & 31;
    struct Gates {
        E f, b;             // the inputs, as they are: a conversion would wait for them, and with them for all that was asked for before
        E *df, *db;
        int rows;
    };
    Gates last{};
    float f_in = 0.f, b_in = 0.f;
    auto take = [&]() {         // after the wait for later loads
        f_in = (float)last.f, b_in = (float)last.b;
        asm volatile("" : "+v"(f_in), "+v"(b_in));      // here, not where they are used
    };
    auto finish = [&]() {
        const DeltaGradArgs &A = arguments();
        int again = 0;
#pragma unroll
        for (int n = 0; n < 8; ++n) again |= g.wrong[n];
        const float (&leaves)[4][CH] = g.leaves[(id - 1) & 1], (&yu)[4][CH] = g.yu[(id - 1) & 1], (&pairs)[2][4][16] = g.pairs[(id - 1) & 1];
        if (lane == 0) A.again[id - 1] = again;
        const bool second = step >= 16;
        const int at = step & 15;
        float enters = 0.f, end = 0.f;
#pragma unroll
        for (int n = 0; n < DK / 16; ++n) enters += g.enters[n][step];
#pragma unroll
        for (int n = 0; n < 8; ++n) end += g.ends[n];
        const float left = (leaves[0][step] + leaves[1][step]) + (leaves[2][step] + leaves[3][step]);
        const float own = second ? pairs[0][3][at] + pairs[1][3][at] : pairs[0][0][at] + pairs[1][0][at];
        const float other = second ? pairs[0][2][at] + pairs[1][2][at] : pairs[0][1][at] + pairs[1][1][at];
        // of the other 16 steps: what enters the second, what leaves the first.  All lanes take part in every exchange, whichever result they keep.
        const float from = sum_from(enters), before = sum_before(left), through = before + left, others = sum_from(other);
        const float entered = __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(from), 16)), passed = __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(through), 15));
        const float x = (own + (second ? others : other)) + (from + before) + (end + (second ? passed : entered));
        if (lane < last.rows && !again) {      // else k_delta_grad_steps's
            const float rate = (yu[0][step] + yu[1][step]) + (yu[2][step] + yu[3][step]);
            *last.df = (E)(x * (1.f / (1.f + expf(f_in))));
            *last.db = (E)(rate * (1.f / (1.f + expf(b_in))));
        }
    };
    if (id < stop) get(id, 0, true);
    for (; id < stop; ++id) {
        const DeltaGradArgs &A = arguments();
        const unsigned head = id / tiles, tile = id % tiles;
        const int bi = (int)(head / (unsigned)A.H), h = (int)(head % (unsigned)A.H);
        const long t0 = (long)tile * CH;
        const int rows = (int)min((long)CH, A.T - t0);
        f4 part = {}, os[NM] = {}, ys[NM] = {}, ud[NM] = {};
        float end = 0.f, wrong = 0.f;
        for (int sl = 0; sl < A.Dv; sl += COLS) {
            const int c = sl + 16 * wc + col;
            const bool mine = c < A.Dv;
            f4 val[2], res[2];         // V and U, or dO and kd
            if (sl) lds_barrier();     // of the columns before all has been read
            if (sl == 0) fetch.put(s, A.Dk);
            in.get(mine, lane, val);
            if (sl / 16 + wc >= blocks) st.clear();
            {
                auto &to = for_y ? g.back : g.state;
#pragma unroll
                for (int n = 0; n < DK / 16; ++n) to.put(32 * (n >> 1) + 8 * grp + 4 * (n & 1), 16 * wc + col, st.s[n]);
            }
            typename Op::template Split<2> sp[DK / 32];
#pragma unroll
            for (int p = 0; p < DK / 32; ++p) sp[p] = split<E, 2>(st.s[2 * p], st.s[2 * p + 1]);
            if (w == 7 && sl == 0) take();
            lds_barrier();
            if (!for_y) {
                delta_u<E, DK, 2>(s, sp, val, rows, lane, res);
                wrong += nothing(res);
#pragma unroll
                for (int m = 0; m < 2; ++m) g.u.put(16 * m + 4 * grp, 16 * wc + col, res[m]);
            } else {
                f4 y[2], dv[2], pd[2] = {};
                upper<Tile::LC>(s.p, val, lane, pd);
                delta_y<E, DK, 2>(s, sp, pd, lane, res, y);
#pragma unroll
                for (int m = 0; m < 2; ++m) {
                    dv[m] = of_steps(s.beta(), m, lane) * y[m];
                    g.dout.put(16 * m + 4 * grp, 16 * wc + col, val[m]);
                    g.y.put(16 * m + 4 * grp, 16 * wc + col, y[m]);
                }
                wrong += nothing(dv);
                put_steps(head_of<E>(A.dv, A.sdv, bi, h) + t0 * A.sdv.ts, (int)A.sdv.ts, c, mine, rows, lane, dv);
            }
            lds_barrier();
            if (!for_y) {
#pragma unroll
                for (int m = 0; m < 2; ++m) {
                    const f4 y = g.y.column(16 * m + 4 * grp, 16 * wc + col);
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        const float a = group_fold(y[e] * res[m][e], 16, add);
                        float &yu = g.yu[id & 1][wc][16 * m + 4 * grp + e];
                        if (col == 0) yu = sl ? yu + a : a;
                    }
                }
            } else {
                const float left = s.since()[CH - 1];
#pragma unroll
                for (int m = 0; m < 2; ++m) {
                    const f4 u = g.u.column(16 * m + 4 * grp, 16 * wc + col);
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        const float a = group_fold(res[m][e] * u[e], 16, add);
                        float &leaves = g.leaves[id & 1][wc][16 * m + 4 * grp + e];
                        if (col == 0) leaves = sl ? leaves + a : a;
                    }
                }
                if (!cleared(left))
#pragma unroll
                    for (int n = 0; n < DK / 16; ++n) {
                        const f4 entered = g.state.column(32 * (n >> 1) + 8 * grp + 4 * (n & 1), 16 * wc + col);
#pragma unroll
                        for (int e = 0; e < 4; ++e) end = fmaf(left * entered[e], st.s[n][e], end);
                    }
            }
            const bool same = sl + COLS < A.Dv;
            if (same || id + 1 < stop) get(same ? id : id + 1, same ? sl + COLS : 0, !same && tile + 1 == tiles);
            if (wc < 3) {
#pragma unroll
                for (int kb = 0; kb < COLS; kb += 32) {
                    const auto b = g.u.rows(tj, kb, lane);
                    if (!for_y) part = Op::mul(g.dout.rows(ti, kb, lane), b, part);
                    else part = Op::mul(g.y.rows(ti, kb, lane), b, part);
                }
            }
            // columns 16 d.. of dO S^T, Y S^T and U D^T
            if (has) {
#pragma unroll
                for (int kb = 0; kb < COLS; kb += 32) {
                    const auto sr = g.state.rows(16 * d, kb, lane), dr = g.back.rows(16 * d, kb, lane);
#pragma unroll
                    for (int m = 0; m < NM; ++m) {
                        const int i = 16 * (m0 + m);
                        os[m] = Op::mul(g.dout.rows(i, kb, lane), sr, os[m]);
                        ys[m] = Op::mul(g.y.rows(i, kb, lane), sr, ys[m]);
                        ud[m] = Op::mul(g.u.rows(i, kb, lane), dr, ud[m]);
                    }
                }
            }
        }
        if (wc < 3) {
            auto &to = for_y ? g.dn : g.dp;
            const int i0 = ti + 4 * grp, j = tj + col, cut_j = s.cut()[j];
            const vec<int, 4> cut_i = load<4>(s.cut() + i0);
            const f4 hi_i = load<4>(s.run_hi() + i0), lo_i = load<4>(s.run_lo() + i0), beta = load<4>(s.beta() + i0);
            const float hi_j = s.run_hi()[j], lo_j = s.run_lo()[j];
            f4 q, x = {};       // x: K K^T, or P
            if (for_y) {
#pragma unroll
                for (int p = 0; p < DK / 32; ++p) x = Op::mul(rows_of<E, Tile::LD>(s.k, ti / 16, p, lane), rows_of<E, Tile::LD>(s.k, tj / 16, p, lane), x);
            } else {
#pragma unroll
                for (int r = 0; r < 4; ++r) x[r] = s.p[(i0 + r) * Tile::LC + j];
            }
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                const int i = i0 + r;
                const float b = j > i || (for_y && j == i) || cut_i[r] != cut_j ? 0.f : between(hi_i[r], lo_i[r], hi_j, lo_j);
                q[r] = b == 0.f ? 0.f : (for_y ? -beta[r] : A.scale) * b * part[r];
                x[r] = b == 0.f ? 0.f : (for_y ? q[r] : part[r]) * x[r];
            }
            to.put(i0, j, q);
            gate_pairs(x, i0, j, ti == tj, lane, g.pairs[id & 1][for_y]);
        } else {
            (for_y ? g.dn : g.dp).put(4 * grp, 16 + col, f4{});     // above the diagonal
            if (for_y) {
                if (id > first) finish();
                const DeltaGradArgs &A = arguments();
                const long t = min(t0 + step, A.T - 1);
                last = Gates{((const E *)A.f)[bi * A.sf.bs + t * A.sf.ts + h * A.sf.hs], ((const E *)A.b)[bi * A.sb.bs + t * A.sb.ts + h * A.sb.hs],
                             (E *)A.df + bi * A.sdf.bs + t * A.sdf.ts + h * A.sdf.hs, (E *)A.db + bi * A.sdb.bs + t * A.sdb.ts + h * A.sdb.hs, rows};
            }
        }
        lds_barrier();
        if (has) {
            const DeltaGradArgs &A = arguments();
            const typename Op::Exact kc = columns_of<1, Tile::LD>(s.k + 16 * d, lane), qc = columns_of<1, Tile::LD>(s.q + 16 * d, lane);
            E *dq = head_of<E>(A.dq, A.sdq, bi, h) + t0 * A.sdq.ts, *dkp = head_of<E>(A.dk, A.sdk, bi, h) + t0 * A.sdk.ts;
#pragma unroll
            for (int n = 0; n < NM; ++n) {
                const int m = m0 + n, i0 = 16 * m, i = i0 + 4 * grp;
                const f4 since = of_steps(s.since(), m, lane), beta = of_steps(s.beta(), m, lane), until = of_steps(s.until(), m, lane);
                const f4 asked = where(since, A.scale * os[n]), taken = where(since, -beta * ys[n]);
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const float sum = group_fold(fmaf(asked[e], (float)s.q[(i + e) * Tile::LD + dk], taken[e] * (float)s.k[(i + e) * Tile::LD + dk]), 16, add);
                    if (col == 0) g.enters[d][i + e] = sum;
                }
                f4 r[2] = {asked, taken + where(until, ud[n])};
                r[0] = Op::mul(g.dp.pair(i0, lane), kc, r[0]);
                r[1] = Op::mul(g.dp.pair_of_columns(i0, lane), qc, r[1]);
                r[1] = Op::mul(g.dn.pair(i0, lane), kc, r[1]);
                r[1] = Op::mul(g.dn.pair_of_columns(i0, lane), kc, r[1]);
                wrong += nothing(r);
                const uint32_t qa = (uint32_t)(i * (int)A.sdq.ts + dk), ka = (uint32_t)(i * (int)A.sdk.ts + dk);
                if (rows == CH && A.Dk == DK) {
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        (dq + e * A.sdq.ts)[qa] = (E)r[0][e];
                        (dkp + e * A.sdk.ts)[ka] = (E)r[1][e];
                    }
                } else {
#pragma unroll
                    for (int e = 0; e < 4; ++e)
                        if (dk < A.Dk && i + e < rows) {
                            (dq + e * A.sdq.ts)[qa] = (E)r[0][e];
                            (dkp + e * A.sdk.ts)[ka] = (E)r[1][e];
                        }
                }
            }
        }
        end = group_fold(end, 64, add);
        wrong = wrong + end * 0.f;
        if (lane == 0) g.ends[w] = end;
        if (__any(wrong != 0.f) && lane == 0) g.wrong[w] = 1;
        else if (lane == 0) g.wrong[w] = 0;
        lds_barrier();
    }
    if (w == 7 && id > first) {
        take();
        finish();
    }
}

// The gradients of a tile's steps one by one, as the definition has them: every state is formed again from the first, which takes as many
// passes as there are steps.  For tiles with numbers that are not finite, which k_delta_grad has left: a workgroup looks at AGAIN tiles.  Such tiles are slow, one after the
// other in a workgroup: 32 x 512 x 8 x 64 in bf16 with NaN behind the ends of all sequences, a fifth of the steps, takes 16 ms with gradients, with zeros there 0.21.
constexpr int AGAIN = 64;
template <class E, int DK> struct DeltaSteps {
    DeltaTile<E, DK, 7> s;
    float sums[2][4];
    float rows[2][4][DK];               // of each wave, dq and dk of a step
};
template <class E, int DK> __device__ void delta_grad_steps(const DeltaGradArgs &A, DeltaSteps<E, DK> &g, long head, long tile)
{
    using Tile = DeltaTile<E, DK, 7>;
    const int blocks = blocks_of(A.Dv);
    const DeltaRecord &rec = ((const DeltaRecord *)A.records)[head * A.tiles + tile];
    Tile &s = g.s;
    const int tid = threadIdx.x, lane = tid & 63, w = tid >> 6, bi = (int)(head / A.H), h = (int)(head % A.H);
    const long t0 = tile * CH;
    const int rows = (int)min((long)CH, A.T - t0);
    const E *v = (const E *)A.v + bi * A.sv.bs + t0 * A.sv.ts + h * A.sv.hs, *dout = (const E *)A.dout + bi * A.sdo.bs + t0 * A.sdo.ts + h * A.sdo.hs;
    for (int t = rows - 1; t >= 0; --t) {
        float dq[DK / 16][4] = {}, dk[DK / 16][4] = {}, rate = 0.f, gate = 0.f;
        for (int c0 = 0; c0 < A.Dv; c0 += COLS) {
            const int c = c0 + 16 * w + (lane & 15);
            const bool mine = c < A.Dv;
            Columns<DK> S, D;
            const long at = ((head * A.tiles + tile) * blocks + min(c0 / 16 + w, blocks - 1)) * 16 * DK;
            S.load(A.states + at, lane);
            if (c0 / 16 + w >= blocks) S.clear();
            for (int i = 0; i < t; ++i) delta_step(s, rec, S, i, mine ? (float)v[i * A.sv.ts + c] : 0.f, lane);
            D.load(A.into + at, lane);
            if (c0 / 16 + w >= blocks) D.clear();
            for (int i = rows - 1; i > t; --i) {
                delta_step_back(s, D, i, mine ? (float)dout[i * A.sdo.ts + c] : 0.f, A.scale, lane);
                delta_pass_back(rec, D, i);
            }
            if (starts(rec.cut, t)) S.clear();
            const Columns<DK> before = S;
            S.scaled(s.gate()[t]);
            const Columns<DK> held = S;
            const float d = mine ? (float)dout[t * A.sdo.ts + c] : 0.f, gap = (mine ? (float)v[t * A.sv.ts + c] : 0.f) - S.dot(s.k + t * Tile::LD, lane);
            S.add(s.k + t * Tile::LD, s.beta()[t] * gap, lane);
            Columns<DK> full = D;
            full.add(s.q + t * Tile::LD, A.scale * d, lane);
            const float dv = delta_step_back(s, D, t, d, A.scale, lane);
            if (mine) {
                float toward = full.dot(s.k + t * Tile::LD, lane) * gap, kept = 0.f;
#pragma unroll
                for (int n = 0; n < DK / 16; ++n)
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        dq[n][e] += A.scale * S.s[n][e] * d;
                        dk[n][e] += s.beta()[t] * full.s[n][e] * gap - held.s[n][e] * dv;
                        kept += D.s[n][e] * before.s[n][e];
                    }
                if (lane < 16) {
                    rate += toward;
                    ((E *)A.dv)[bi * A.sdv.bs + (t0 + t) * A.sdv.ts + h * A.sdv.hs + c] = (E)dv;
                }
                gate += kept;
            }
        }
        __syncthreads();
#pragma unroll
        for (int n = 0; n < DK / 16; ++n)
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const float x = group_fold(dq[n][e], 16, seq::add), y = group_fold(dk[n][e], 16, seq::add);
                const int d = 32 * (n >> 1) + 8 * (lane >> 4) + 4 * (n & 1) + e;
                if ((lane & 15) == 0) g.rows[0][w][d] = x, g.rows[1][w][d] = y;
            }
        const float r = group_fold(rate, 64, seq::add), a = group_fold(gate, 64, seq::add);
        if (lane == 0) g.sums[0][w] = r, g.sums[1][w] = a;
        __syncthreads();
        if (tid < A.Dk) {
            const int d = tid;
            ((E *)A.dq)[bi * A.sdq.bs + (t0 + t) * A.sdq.ts + h * A.sdq.hs + d] = (E)((g.rows[0][0][d] + g.rows[0][1][d]) + (g.rows[0][2][d] + g.rows[0][3][d]));
            ((E *)A.dk)[bi * A.sdk.bs + (t0 + t) * A.sdk.ts + h * A.sdk.hs + d] = (E)((g.rows[1][0][d] + g.rows[1][1][d]) + (g.rows[1][2][d] + g.rows[1][3][d]));
        }
        if (tid == 0) {
            const float gt = s.gate()[t], bt = s.beta()[t];
            const float f = (float)((const E *)A.f)[bi * A.sf.bs + (t0 + t) * A.sf.ts + h * A.sf.hs], b = (float)((const E *)A.b)[bi * A.sb.bs + (t0 + t) * A.sb.ts + h * A.sb.hs];
            const float sr = (g.sums[0][0] + g.sums[0][1]) + (g.sums[0][2] + g.sums[0][3]), sa = (g.sums[1][0] + g.sums[1][1]) + (g.sums[1][2] + g.sums[1][3]);
            ((E *)A.df)[bi * A.sdf.bs + (t0 + t) * A.sdf.ts + h * A.sdf.hs] = (E)(starts(rec.cut, t) ? 0.f : gt * (1.f / (1.f + expf(f))) * sa);
            ((E *)A.db)[bi * A.sdb.bs + (t0 + t) * A.sdb.ts + h * A.sdb.hs] = (E)(bt * (1.f / (1.f + expf(b))) * sr);
        }
        __syncthreads();
    }
}
template <class E, int DK> __global__ __launch_bounds__(256) void k_delta_grad_steps(DeltaGradArgs A)
{
    extern __shared__ __align__(16) unsigned char lds[];
    DeltaSteps<E, DK> &g = *reinterpret_cast<DeltaSteps<E, DK> *>(lds);
    const long all = (long)A.B * A.H * A.tiles, first = (long)blockIdx.x * AGAIN, mine = first + (threadIdx.x & 63);
    uint64_t left = __ballot(mine < all && A.again[min(mine, all - 1)]);      // the same for all waves
    for (; left; left &= left - 1) {
        const long id = first + __ffsll((unsigned long long)left) - 1, head = id / A.tiles, tile = id % A.tiles;
        DeltaFetch<E, DK, 256, 7> fetch;
        fetch.begin(A, (const DeltaRecord *)A.records, head, (int)(head / A.H), (int)(head % A.H), threadIdx.x);
        fetch.load(A, tile);
        __syncthreads();
        fetch.put(g.s, A.Dk);
        __syncthreads();
        delta_grad_steps<E, DK>(A, g, head, tile);
    }
}

}  // namespace seq
