// The gated delta rule: a memory of one matrix per head, over sequences, forward and backward.
//
// Per head, with a_t = sigmoid(f_t), beta_t = sigmoid(b_t) and the state S [Dk][Dv] (zero before a step that starts an episode):
//   S_t = a_t (I - beta_t k_t k_t^T) S_{t-1} + beta_t k_t v_t^T,  o_t = scale S_t^T q_t.
// Over a tile of CH steps that the state S enters, with g_i = a_1 .. a_i and G_ij = g_i / g_j (0 where an episode starts in between):
//   S_i = g_i S + sum_{j <= i} G_ij k_j u_j^T,   (I + N) U = R,   N_ij = beta_i G_ij k_i.k_j (j < i),   R_i = beta_i (v_i - g_i S^T k_i)
//   O = scale g Q S + P U,   P_ij = scale G_ij q_i.k_j (j <= i),   S' = g_C S + (G_C. K)^T U.
// Backward, from dO and the gradient D of the state that leaves:
//   dU = P^T dO + (G_C. K) D,   (I + N)^T Y = dU,   dS = g_C D + (scale g Q)^T dO - (beta g K)^T Y,   dv = beta Y,   db = (1 - beta) Y.u
//   dP = dO U^T, dN = -Y U^T:   dq = scale (g S do + (dP G) k),   dk = scale (dP G)^T q + G_C. D u - beta g S y + (dN beta G) k + (dN beta G)^T k
// and, since o_i grows with a_t for every i >= t of the episode while what v_i writes does not shrink with it,
//   d log a_t = sum_{i >= t} (do_i.o_i - dv_i.v_i) + <D, S'>   (the sum ends with the episode, the last term counts if it lives on),  df = (1 - a) d log a,
// with do_i.o_i = q_i.dq_i and <D, S'> = g_C <D, S> + sum_j G_Cj u_j.(D^T k_j).
//
// All of this is independent per column of S.  A wave owns 16 columns and keeps its part of the state, of R, U, O, Y in registers in
// the layout in which the matrix instructions leave their results, which is the one in which they take their right operand; the
// left operands, K, Q, N, P, are the same for all waves and lie in LDS.  So the chain from state to state has no barrier.
#pragma once
#include "seq_common.h"

namespace seq {

constexpr int CH = 64;                 // steps of a tile
constexpr int CB = CH / 16;
constexpr int COLS = 64;               // columns of the state of a workgroup, 16 of each wave
constexpr float LOG_LEAST = -150.f;    // exp of it is 0 in fp32: a gate that closes further counts as this, so that differences of sums stay finite

using f4 = vec<float, 4>;

struct Strides {
    long bs, ts, hs;                   // of a sequence, a step, a head
};

struct DeltaArgs {
    const void *q, *k, *v, *f, *b;
    Strides sq, sk, sv, sf, sb;
    const float *s0;
    const uint8_t *reset;
    long reset_bs, reset_ts;
    void *o;
    Strides so;
    float *last, *carry;               // carry: the state that enters each tile, [B][H][tiles][Dk][Dv]
    long T, tiles;
    int B, H, Dk, Dv;
    float scale;
};

struct DeltaGradArgs {
    const void *q, *k, *v, *f, *b, *dout;
    Strides sq, sk, sv, sf, sb, sdo;
    const float *carry, *dlast;
    const uint8_t *reset;
    long reset_bs, reset_ts;
    void *dq, *dk, *dv, *df, *db;
    Strides sdq, sdk, sdv, sdf, sdb;
    float *ds0;
    float *into;                       // workspace: the gradient of the state that leaves each tile, as carry
    long T, tiles;
    int B, H, Dk, Dv;
    float scale;
};

__device__ __forceinline__ f4 mm4(f4 a, f4 b, f4 c)
{
#pragma unroll
    for (int s = 0; s < 4; ++s) c = __builtin_amdgcn_mfma_f32_16x16x4f32(a[s], b[s], c, 0, 0, 0);
    return c;
}
// 16 x 16 of a matrix in LDS as left operand: rows m0.., columns k0..; its transposed: rows m0.. are columns of the stored one
template <int LD> __device__ __forceinline__ f4 rows_of(const float *p, int m0, int k0, int lane)
{
    return *reinterpret_cast<const f4 *>(p + (m0 + (lane & 15)) * LD + k0 + 4 * (lane >> 4));
}
template <int LD> __device__ __forceinline__ f4 cols_of(const float *p, int m0, int k0, int lane)
{
    const float *a = p + (k0 + 4 * (lane >> 4)) * LD + m0 + (lane & 15);
    return f4{a[0], a[LD], a[2 * LD], a[3 * LD]};
}

// What the waves share of a tile.  Rows outside [lo, hi) are steps that do nothing: keys, queries and rates zero, gates one.
template <int DK> struct DeltaTile {
    static constexpr int LD = DK + 4, LC = CH + 4;
    float q[CH * LD], k[CH * LD];
    float n[CH * LC];                  // -N below the blocks of the diagonal, on which (I + N)^-1 of the block
    float p[CH * LC];                  // P; upper blocks are not written
    float run_hi[CH], run_lo[CH];      // sum of log a up to each step, as a multiple of 2^-10 and the rest
    float gate[CH];                    // a
    float since[CH], until[CH], beta[CH];   // g_i; G_Ci, 0 where the episode ends in the tile
    int cut[CH];                       // episodes that have started up to each step
};

// The factor from step j to step i >= j: differences of the multiples of 2^-10 are exact, so that a gate that closed long before leaves
// no rounding in later ones.
template <class Tile> __device__ __forceinline__ float between(const Tile &s, int i, int j)
{
    return s.cut[i] == s.cut[j] ? __expf((s.run_hi[i] - s.run_hi[j]) + (s.run_lo[i] - s.run_lo[j])) : 0.f;
}

// Fills the tile from step t0 on; rows outside [lo, hi) stay out of it.  Every thread of 256 takes part; the barrier before it is the caller's.
template <class E, int DK, class Args> __device__ void delta_tile(const Args &A, DeltaTile<DK> &s, int bi, int h, long t0, int lo, int hi)
{
    using Tile = DeltaTile<DK>;
    const int tid = threadIdx.x, lane = tid & 63, w = tid >> 6;
    const E *q = (const E *)A.q + bi * A.sq.bs + t0 * A.sq.ts + h * A.sq.hs;
    const E *k = (const E *)A.k + bi * A.sk.bs + t0 * A.sk.ts + h * A.sk.hs;
    for (int e = tid; e < CH * DK; e += 256) {
        const int r = e / DK, c = e % DK;
        const bool in = r >= lo && r < hi && c < A.Dk;
        s.q[r * Tile::LD + c] = in ? (float)q[r * A.sq.ts + c] : 0.f;
        s.k[r * Tile::LD + c] = in ? (float)k[r * A.sk.ts + c] : 0.f;
    }
    if (w == 0) {
        const bool in = lane >= lo && lane < hi;
        const long t = t0 + lane;
        float la = 0.f, beta = 0.f;
        int cut = 0;
        if (in) {
            const float f = (float)((const E *)A.f)[bi * A.sf.bs + t * A.sf.ts + h * A.sf.hs];
            const float b = (float)((const E *)A.b)[bi * A.sb.bs + t * A.sb.ts + h * A.sb.hs];
            la = (f < 0.f ? f : 0.f) - log1pf(expf(-fabsf(f)));
            la = la < LOG_LEAST ? LOG_LEAST : la;
            beta = 1.f / (1.f + expf(-b));
            cut = A.reset && A.reset[bi * A.reset_bs + t * A.reset_ts];
        }
        s.gate[lane] = expf(la);
        double run = la;
        int cuts = cut;
#pragma unroll
        for (int d = 1; d < CH; d *= 2) {
            const double o = __shfl_up(run, d);
            const int oc = __shfl_up(cuts, d);
            if (lane >= d) run += o, cuts += oc;
        }
        const double whole = rint(run * 1024.0) * (1.0 / 1024.0);
        s.run_hi[lane] = (float)whole;
        s.run_lo[lane] = (float)(run - whole);
        s.cut[lane] = cuts;
        s.beta[lane] = beta;
        s.since[lane] = cuts ? 0.f : expf((float)run);
        const double end = __shfl(run, CH - 1);
        const int last = __shfl(cuts, CH - 1);
        s.until[lane] = in && cuts == last ? expf((float)(end - run)) : 0.f;
    }
    __syncthreads();
    const int col = lane & 15, row = 4 * (lane >> 4);
#pragma unroll
    for (int n = 0; n < CB; ++n) {
        if (n > w) break;
        f4 kk = {}, qk = {};
#pragma unroll
        for (int kb = 0; kb < DK / 16; ++kb) {
            const f4 b = rows_of<Tile::LD>(s.k, 16 * n, 16 * kb, lane);
            kk = mm4(rows_of<Tile::LD>(s.k, 16 * w, 16 * kb, lane), b, kk);
            qk = mm4(rows_of<Tile::LD>(s.q, 16 * w, 16 * kb, lane), b, qk);
        }
#pragma unroll
        for (int r = 0; r < 4; ++r) {
            const int i = 16 * w + row + r, j = 16 * n + col;
            const float g = j <= i ? between(s, i, j) : 0.f;
            s.n[i * Tile::LC + j] = j < i && g != 0.f ? -s.beta[i] * g * kk[r] : 0.f;
            s.p[i * Tile::LC + j] = g != 0.f ? A.scale * g * qk[r] : 0.f;
        }
    }
    __syncthreads();
    // (I + N)^-1 of the blocks on the diagonal by forward substitution, a column per lane
    if (w == 0) {
        float *blk = s.n + (16 * (lane >> 4)) * (Tile::LC + 1);
        float x[16];
#pragma unroll
        for (int i = 0; i < 16; ++i) {
            float v = i == col ? 1.f : 0.f;
#pragma unroll
            for (int j = 0; j < i; ++j) v = fmaf(blk[i * Tile::LC + j], x[j], v);
            x[i] = v;
        }
#pragma unroll
        for (int i = 0; i < 16; ++i) blk[i * Tile::LC + col] = x[i];
    }
    __syncthreads();
}

template <class Tile> __device__ __forceinline__ f4 four(const float *p, int m0, int lane) { return *reinterpret_cast<const f4 *>(p + m0 + 4 * (lane >> 4)); }

// R of a wave's columns, then U in its place.  state: the state that enters, or its part of 0 where none does.
template <class E, int DK, class Args>
__device__ __forceinline__ void delta_u(const Args &A, const DeltaTile<DK> &s, const f4 (&state)[DK / 16], int bi, int h, long t0, int lo, int hi, int c, f4 (&u)[CB], f4 (*val)[CB] = nullptr)
{
    using Tile = DeltaTile<DK>;
    const int lane = threadIdx.x & 63, row = 4 * (lane >> 4);
    const E *v = (const E *)A.v + bi * A.sv.bs + t0 * A.sv.ts + h * A.sv.hs + c;
#pragma unroll
    for (int m = 0; m < CB; ++m) {
        f4 ks = {};
#pragma unroll
        for (int kb = 0; kb < DK / 16; ++kb) ks = mm4(rows_of<Tile::LD>(s.k, 16 * m, 16 * kb, lane), state[kb], ks);
        f4 r = {};
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const int i = 16 * m + row + e;
            if (i >= lo && i < hi) {
                const float x = c < A.Dv ? (float)v[i * A.sv.ts] : 0.f;
                if (val) (*val)[m][e] = x;
                r[e] = s.beta[i] * (x - (s.cut[i] ? 0.f : s.since[i] * ks[e]));
            } else if (val) (*val)[m][e] = 0.f;
        }
#pragma unroll
        for (int kb = 0; kb < m; ++kb) r = mm4(rows_of<Tile::LC>(s.n, 16 * m, 16 * kb, lane), u[kb], r);
        u[m] = mm4(rows_of<Tile::LC>(s.n, 16 * m, 16 * m, lane), r, f4{});
    }
}

template <int N> __device__ __forceinline__ bool finite(const f4 (&v)[N])
{
    bool ok = true;
#pragma unroll
    for (int i = 0; i < N; ++i)
#pragma unroll
        for (int e = 0; e < 4; ++e) ok &= fabsf(v[i][e]) < INFINITY;
    return ok;
}

// A workgroup per head and COLS columns, tile after tile.  A tile whose result holds a number that is not finite is taken again step by step,
// where nothing is multiplied by the zeros of other steps: a NaN reaches what comes after it in its episode and nothing else.
template <class E, int DK> __global__ __launch_bounds__(256) void k_delta(DeltaArgs A)
{
    using Tile = DeltaTile<DK>;
    extern __shared__ __align__(16) unsigned char lds[];
    Tile &s = *reinterpret_cast<Tile *>(lds);
    const int lane = threadIdx.x & 63, row = 4 * (lane >> 4);
    const int slices = (A.Dv + COLS - 1) / COLS, slice = blockIdx.x % slices;
    const long head = blockIdx.x / slices;
    const int bi = (int)(head / A.H), h = (int)(head % A.H), c = COLS * slice + 16 * (threadIdx.x >> 6) + (lane & 15);
    const bool mine = c < A.Dv;
    f4 state[DK / 16];
#pragma unroll
    for (int kb = 0; kb < DK / 16; ++kb)
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const int d = 16 * kb + row + e;
            state[kb][e] = A.s0 && mine && d < A.Dk ? A.s0[(head * A.Dk + d) * A.Dv + c] : 0.f;
        }
    auto put = [&](float *to) {
#pragma unroll
        for (int kb = 0; kb < DK / 16; ++kb)
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const int d = 16 * kb + row + e;
                if (mine && d < A.Dk) to[(long)d * A.Dv + c] = state[kb][e];
            }
    };
    for (long tile = 0; tile < A.tiles; ++tile) {
        const long t0 = tile * CH;
        const int rows = (int)min((long)CH, A.T - t0);
        if (A.carry) put(A.carry + (head * A.tiles + tile) * A.Dk * A.Dv);
        E *o = (E *)A.o + bi * A.so.bs + t0 * A.so.ts + h * A.so.hs + c;
        for (int lo = 0, hi = rows; lo < rows;) {
            delta_tile<E, DK>(A, s, bi, h, t0, lo, hi);
            f4 u[CB], out[CB], next[DK / 16];
            delta_u<E, DK>(A, s, state, bi, h, t0, lo, hi, c, u);
#pragma unroll
            for (int m = 0; m < CB; ++m) {
                f4 qs = {};
#pragma unroll
                for (int kb = 0; kb < DK / 16; ++kb) qs = mm4(rows_of<Tile::LD>(s.q, 16 * m, 16 * kb, lane), state[kb], qs);
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const int i = 16 * m + row + e;
                    qs[e] = s.cut[i] ? 0.f : A.scale * s.since[i] * qs[e];
                }
#pragma unroll
                for (int kb = 0; kb <= m; ++kb) qs = mm4(rows_of<Tile::LC>(s.p, 16 * m, 16 * kb, lane), u[kb], qs);
                out[m] = qs;
            }
#pragma unroll
            for (int m = 0; m < CB; ++m)
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const float left = s.until[16 * m + row + e];
                    u[m][e] = left != 0.f ? left * u[m][e] : 0.f;
                }
            const bool lives = !s.cut[CH - 1];
            const float left = s.since[CH - 1];
#pragma unroll
            for (int d = 0; d < DK / 16; ++d) {
                f4 n;
#pragma unroll
                for (int e = 0; e < 4; ++e) n[e] = lives ? left * state[d][e] : 0.f;
#pragma unroll
                for (int kb = 0; kb < CB; ++kb) n = mm4(cols_of<Tile::LD>(s.k, 16 * d, 16 * kb, lane), u[kb], n);
                next[d] = n;
            }
            const bool ok = finite(out) && finite(next);
            const bool again = __syncthreads_or(!ok) && hi - lo > 1;
            if (again) {
                hi = lo + 1;
                continue;
            }
#pragma unroll
            for (int d = 0; d < DK / 16; ++d) state[d] = next[d];
#pragma unroll
            for (int m = 0; m < CB; ++m)
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const int i = 16 * m + row + e;
                    if (mine && i >= lo && i < hi) o[i * A.so.ts] = (E)out[m][e];
                }
            lo = hi++;
        }
    }
    if (A.last) put(A.last + head * A.Dk * A.Dv);
}

// The end of the episode that step lo begins or continues, at most `rows`: for tiles that are taken again episode by episode.
template <class Args> __device__ __forceinline__ int episode_end(const Args &A, int bi, long t0, int lo, int rows)
{
    int hi = lo + 1;
    while (hi < rows && !(A.reset && A.reset[bi * A.reset_bs + (t0 + hi) * A.reset_ts])) ++hi;
    return hi;
}
// Its beginning, for an end `hi`.
template <class Args> __device__ __forceinline__ int episode_begin(const Args &A, int bi, long t0, int hi)
{
    int lo = hi - 1;
    while (lo > 0 && !(A.reset && A.reset[bi * A.reset_bs + (t0 + lo) * A.reset_ts])) --lo;
    return lo;
}

// dU, then Y in its place: (I + N)^T Y = dU from the last rows up.  out: dO of the wave's columns; D: the state's gradient or zeros.
template <int DK> __device__ __forceinline__ void delta_y(const DeltaTile<DK> &s, const f4 (&out)[CB], const f4 (&D)[DK / 16], f4 (&y)[CB], f4 (*kd)[CB] = nullptr)
{
    using Tile = DeltaTile<DK>;
    const int lane = threadIdx.x & 63, row = 4 * (lane >> 4);
#pragma unroll
    for (int m = CB - 1; m >= 0; --m) {
        f4 t = {};
#pragma unroll
        for (int kb = 0; kb < DK / 16; ++kb) t = mm4(rows_of<Tile::LD>(s.k, 16 * m, 16 * kb, lane), D[kb], t);
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const float left = s.until[16 * m + row + e];
            t[e] = left != 0.f ? left * t[e] : 0.f;
        }
        if (kd) (*kd)[m] = t;
#pragma unroll
        for (int kb = m; kb < CB; ++kb) t = mm4(cols_of<Tile::LC>(s.p, 16 * m, 16 * kb, lane), out[kb], t);
#pragma unroll
        for (int kb = m + 1; kb < CB; ++kb) t = mm4(cols_of<Tile::LC>(s.n, 16 * m, 16 * kb, lane), y[kb], t);
        y[m] = mm4(cols_of<Tile::LC>(s.n, 16 * m, 16 * m, lane), t, f4{});
    }
}

template <class E> __device__ __forceinline__ void delta_dout(const DeltaGradArgs &A, int bi, int h, long t0, int lo, int hi, int c, f4 (&d)[CB])
{
    const int lane = threadIdx.x & 63, row = 4 * (lane >> 4);
    const E *p = (const E *)A.dout + bi * A.sdo.bs + t0 * A.sdo.ts + h * A.sdo.hs + c;
#pragma unroll
    for (int m = 0; m < CB; ++m)
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const int i = 16 * m + row + e;
            d[m][e] = c < A.Dv && i >= lo && i < hi ? (float)p[i * A.sdo.ts] : 0.f;
        }
}

// The gradient of the state, from the last tile to the first: what leaves each tile is kept, for k_delta_grad.
template <class E, int DK> __global__ __launch_bounds__(256) void k_delta_back(DeltaGradArgs A)
{
    using Tile = DeltaTile<DK>;
    extern __shared__ __align__(16) unsigned char lds[];
    Tile &s = *reinterpret_cast<Tile *>(lds);
    const int lane = threadIdx.x & 63, row = 4 * (lane >> 4);
    const int slices = (A.Dv + COLS - 1) / COLS, slice = blockIdx.x % slices;
    const long head = blockIdx.x / slices;
    const int bi = (int)(head / A.H), h = (int)(head % A.H), c = COLS * slice + 16 * (threadIdx.x >> 6) + (lane & 15);
    const bool mine = c < A.Dv;
    f4 D[DK / 16];
#pragma unroll
    for (int kb = 0; kb < DK / 16; ++kb)
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const int d = 16 * kb + row + e;
            D[kb][e] = A.dlast && mine && d < A.Dk ? A.dlast[(head * A.Dk + d) * A.Dv + c] : 0.f;
        }
    auto put = [&](float *to) {
#pragma unroll
        for (int kb = 0; kb < DK / 16; ++kb)
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const int d = 16 * kb + row + e;
                if (mine && d < A.Dk) to[(long)d * A.Dv + c] = D[kb][e];
            }
    };
    for (long tile = A.tiles - 1; tile >= 0; --tile) {
        const long t0 = tile * CH;
        const int rows = (int)min((long)CH, A.T - t0);
        put(A.into + (head * A.tiles + tile) * A.Dk * A.Dv);
        for (int lo = 0, hi = rows; hi > 0;) {
            delta_tile<E, DK>(A, s, bi, h, t0, lo, hi);
            f4 out[CB], y[CB], next[DK / 16];
            delta_dout<E>(A, bi, h, t0, lo, hi, c, out);
            delta_y<DK>(s, out, D, y);
#pragma unroll
            for (int m = 0; m < CB; ++m)
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const int i = 16 * m + row + e;
                    const bool live = !s.cut[i];
                    out[m][e] = live ? A.scale * s.since[i] * out[m][e] : 0.f;
                    y[m][e] = live && i >= lo && i < hi ? -s.beta[i] * s.since[i] * y[m][e] : 0.f;
                }
            const bool lives = !s.cut[CH - 1];
            const float left = s.since[CH - 1];
#pragma unroll
            for (int d = 0; d < DK / 16; ++d) {
                f4 n;
#pragma unroll
                for (int e = 0; e < 4; ++e) n[e] = lives ? left * D[d][e] : 0.f;
#pragma unroll
                for (int kb = 0; kb < CB; ++kb) {
                    n = mm4(cols_of<Tile::LD>(s.q, 16 * d, 16 * kb, lane), out[kb], n);
                    n = mm4(cols_of<Tile::LD>(s.k, 16 * d, 16 * kb, lane), y[kb], n);
                }
                // where the first step starts an episode nothing passes it, no NaN of theirs either
                next[d] = s.cut[lo] ? f4{} : n;
            }
            const bool again = __syncthreads_or(!finite(next)) && (lo == 0 && hi == rows);
            if (again) {
                const int first = episode_begin(A, bi, t0, hi);
                if (first > 0) {
                    lo = first;
                    continue;
                }
            }
#pragma unroll
            for (int d = 0; d < DK / 16; ++d) D[d] = next[d];
            hi = lo;
            if (hi > 0) lo = episode_begin(A, bi, t0, hi);
        }
    }
    if (A.ds0) put(A.ds0 + head * A.Dk * A.Dv);
}

template <int DK> struct DeltaGradTile {
    static constexpr int LU = COLS + 4;
    DeltaTile<DK> s;
    float dout[CH * LU], u[CH * LU], y[CH * LU];
    float sums[3][4][CH];              // of each wave and row: q.dq, Y.u, dv.v
    float ends[4];                     // of each wave: <D, S'>
};

// Sums of x over the 16 lanes that share rows, in lane 0 of them
__device__ __forceinline__ float lanes16(float x)
{
    return group_fold(x, 16, add);
}

// Everything else: a workgroup per tile and head.
template <class E, int DK> __global__ __launch_bounds__(256) void k_delta_grad(DeltaGradArgs A)
{
    using Tile = DeltaTile<DK>;
    using Grad = DeltaGradTile<DK>;
    constexpr int LU = Grad::LU, ND = (DK + 63) / 64;      // tiles of 16 of a wave's columns of dq and dk
    extern __shared__ __align__(16) unsigned char lds[];
    Grad &g = *reinterpret_cast<Grad *>(lds);
    Tile &s = g.s;
    const int tid = threadIdx.x, lane = tid & 63, w = tid >> 6, row = 4 * (lane >> 4), col = lane & 15;
    const long tile = blockIdx.x % A.tiles, head = blockIdx.x / A.tiles;
    const int bi = (int)(head / A.H), h = (int)(head % A.H);
    const long t0 = tile * CH;
    const int rows = (int)min((long)CH, A.T - t0);
    const float *S = A.carry + (head * A.tiles + tile) * A.Dk * A.Dv, *Dn = A.into + (head * A.tiles + tile) * A.Dk * A.Dv;
    for (int lo = 0, hi = rows; lo < rows;) {
        delta_tile<E, DK>(A, s, bi, h, t0, lo, hi);
        // the state enters the rows from 0 on, unless the first step starts an episode; its gradient those up to the last
        const bool enters = lo == 0 && !s.cut[0], leaves = hi == rows;
        f4 dp[CB] = {}, dn[CB] = {}, os[ND][CB] = {}, ys[ND][CB] = {}, ud[ND][CB] = {};
        f4 yu[CB] = {}, vv[CB] = {};
        float end = 0.f;
        bool ok = true;
        for (int sl = 0; sl < A.Dv; sl += COLS) {
            const int c = sl + 16 * w + col;
            f4 out[CB], u[CB], y[CB], val[CB], kd[CB];
            {
                f4 st[DK / 16], D[DK / 16];
#pragma unroll
                for (int kb = 0; kb < DK / 16; ++kb)
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        const int d = 16 * kb + row + e;
                        const bool in = c < A.Dv && d < A.Dk;
                        st[kb][e] = in && enters ? S[(long)d * A.Dv + c] : 0.f;
                        D[kb][e] = in && leaves ? Dn[(long)d * A.Dv + c] : 0.f;
                    }
                delta_u<E, DK>(A, s, st, bi, h, t0, lo, hi, c, u, &val);
                delta_dout<E>(A, bi, h, t0, lo, hi, c, out);
                delta_y<DK>(s, out, D, y, &kd);
                if (enters && leaves && !s.cut[CH - 1])
#pragma unroll
                    for (int kb = 0; kb < DK / 16; ++kb)
#pragma unroll
                        for (int e = 0; e < 4; ++e) end = fmaf(s.since[CH - 1] * st[kb][e], D[kb][e], end);
            }
#pragma unroll
            for (int m = 0; m < CB; ++m)
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const int i = 16 * m + row + e;
                    const bool in = i >= lo && i < hi;
                    const float dv = s.beta[i] * y[m][e];
                    if (in) {
                        ok &= fabsf(dv) < INFINITY;
                        yu[m][e] = fmaf(y[m][e], u[m][e], yu[m][e]);
                        vv[m][e] = fmaf(dv, val[m][e], vv[m][e]);
                        end = fmaf(kd[m][e], u[m][e], end);
                        if (c < A.Dv) ((E *)A.dv)[bi * A.sdv.bs + (t0 + i) * A.sdv.ts + h * A.sdv.hs + c] = (E)dv;
                    }
                    g.dout[i * LU + 16 * w + col] = in ? out[m][e] : 0.f;
                    g.u[i * LU + 16 * w + col] = in ? u[m][e] : 0.f;
                    g.y[i * LU + 16 * w + col] = in ? y[m][e] : 0.f;
                }
            __syncthreads();
            // rows 16 w.. of dO U^T and of -Y U^T, up to the diagonal
#pragma unroll
            for (int kb = 0; kb < COLS / 16; ++kb) {
                const f4 ao = rows_of<LU>(g.dout, 16 * w, 16 * kb, lane), ay = -rows_of<LU>(g.y, 16 * w, 16 * kb, lane);
#pragma unroll
                for (int n = 0; n < CB; ++n) {
                    if (n > w) break;
                    const f4 b = rows_of<LU>(g.u, 16 * n, 16 * kb, lane);
                    dp[n] = mm4(ao, b, dp[n]);
                    dn[n] = mm4(ay, b, dn[n]);
                }
            }
            // columns 16 (w + 4 d).. of dO S^T, Y S^T and U D^T
#pragma unroll
            for (int d = 0; d < ND; ++d) {
                const int dk = 16 * (w + 4 * d) + col;
                if (16 * (w + 4 * d) >= DK) break;
#pragma unroll
                for (int kb = 0; kb < COLS / 16; ++kb) {
                    f4 st, D;
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        const int cc = sl + 16 * kb + row + e;
                        const bool in = cc < A.Dv && dk < A.Dk;
                        st[e] = in && enters ? S[(long)dk * A.Dv + cc] : 0.f;
                        D[e] = in && leaves ? Dn[(long)dk * A.Dv + cc] : 0.f;
                    }
#pragma unroll
                    for (int m = 0; m < CB; ++m) {
                        os[d][m] = mm4(rows_of<LU>(g.dout, 16 * m, 16 * kb, lane), st, os[d][m]);
                        ys[d][m] = mm4(rows_of<LU>(g.y, 16 * m, 16 * kb, lane), st, ys[d][m]);
                        ud[d][m] = mm4(rows_of<LU>(g.u, 16 * m, 16 * kb, lane), D, ud[d][m]);
                    }
                }
            }
            __syncthreads();
        }
        // the gradients of P's and N's products, in their places
#pragma unroll
        for (int n = 0; n < CB; ++n) {
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                const int i = 16 * w + row + r, j = 16 * n + col;
                const float b = n <= w && j <= i ? between(s, i, j) : 0.f;
                s.p[i * Tile::LC + j] = b != 0.f ? A.scale * b * dp[n][r] : 0.f;
                s.n[i * Tile::LC + j] = b != 0.f && j < i ? s.beta[i] * b * dn[n][r] : 0.f;
            }
        }
        __syncthreads();
        f4 qd[CB] = {};
#pragma unroll
        for (int d = 0; d < ND; ++d) {
            if (16 * (w + 4 * d) >= DK) break;
            const int dk = 16 * (w + 4 * d) + col;
#pragma unroll
            for (int m = 0; m < CB; ++m) {
                f4 dq, dkk, add_q = {}, add_k = {};
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const int i = 16 * m + row + e;
                    const bool live = !s.cut[i] && i >= lo && i < hi;
                    dq[e] = live ? A.scale * s.since[i] * os[d][m][e] : 0.f;
                    dkk[e] = (live ? -s.beta[i] * s.since[i] * ys[d][m][e] : 0.f) + (s.until[i] != 0.f ? s.until[i] * ud[d][m][e] : 0.f);
                }
#pragma unroll
                for (int kb = 0; kb < CB; ++kb) {
                    const f4 kr = cols_of<Tile::LD>(s.k, 16 * (w + 4 * d), 16 * kb, lane);
                    if (kb <= m) {
                        add_q = mm4(rows_of<Tile::LC>(s.p, 16 * m, 16 * kb, lane), kr, add_q);
                        add_k = mm4(rows_of<Tile::LC>(s.n, 16 * m, 16 * kb, lane), kr, add_k);
                    }
                    if (kb >= m) {
                        add_k = mm4(cols_of<Tile::LC>(s.p, 16 * m, 16 * kb, lane), cols_of<Tile::LD>(s.q, 16 * (w + 4 * d), 16 * kb, lane), add_k);
                        add_k = mm4(cols_of<Tile::LC>(s.n, 16 * m, 16 * kb, lane), kr, add_k);
                    }
                }
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const int i = 16 * m + row + e;
                    if (i < lo || i >= hi) continue;
                    const float x = dq[e] + add_q[e], z = dkk[e] + add_k[e];
                    ok &= fabsf(x) < INFINITY && fabsf(z) < INFINITY;
                    qd[m][e] = fmaf(x, s.q[i * Tile::LD + 16 * (w + 4 * d) + col], qd[m][e]);
                    if (dk < A.Dk) {
                        ((E *)A.dq)[bi * A.sdq.bs + (t0 + i) * A.sdq.ts + h * A.sdq.hs + dk] = (E)x;
                        ((E *)A.dk)[bi * A.sdk.bs + (t0 + i) * A.sdk.ts + h * A.sdk.hs + dk] = (E)z;
                    }
                }
            }
        }
        if (__syncthreads_or(!ok) && lo == 0 && hi == rows) {
            const int first = episode_end(A, bi, t0, 0, rows);
            if (first < rows) {       // written again, episode by episode
                hi = first;
                continue;
            }
        }
#pragma unroll
        for (int m = 0; m < CB; ++m)
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const float a = lanes16(qd[m][e]), b = lanes16(yu[m][e]), d = lanes16(vv[m][e]);
                if (col == 0) {
                    const int i = 16 * m + row + e;
                    g.sums[0][w][i] = a;
                    g.sums[1][w][i] = b;
                    g.sums[2][w][i] = d;
                }
            }
        end = group_fold(end, 64, add);
        if (lane == 0) g.ends[w] = end;
        __syncthreads();
        if (w == 0) {
            const int i = lane;
            auto all = [&](int k) { return (g.sums[k][0][i] + g.sums[k][1][i]) + (g.sums[k][2][i] + g.sums[k][3][i]); };
            const bool in = i >= lo && i < hi;
            float x = in ? all(0) - all(2) : 0.f;
            if (i == hi - 1 && leaves) x += (g.ends[0] + g.ends[1]) + (g.ends[2] + g.ends[3]);
            const int cut = s.cut[i];
#pragma unroll
            for (int d = 1; d < CH; d *= 2) {
                const float o = __shfl_down(x, d);
                const int oc = __shfl_down(cut, d);
                if (i + d < CH && oc == cut) x += o;
            }
            if (in) {
                const bool starts = A.reset && A.reset[bi * A.reset_bs + (t0 + i) * A.reset_ts];
                const float a = s.gate[i], f = (float)((const E *)A.f)[bi * A.sf.bs + (t0 + i) * A.sf.ts + h * A.sf.hs];
                const float df = starts || a == 0.f ? 0.f : x * (1.f / (1.f + expf(f)));
                const float bb = (float)((const E *)A.b)[bi * A.sb.bs + (t0 + i) * A.sb.ts + h * A.sb.hs];
                ((E *)A.df)[bi * A.sdf.bs + (t0 + i) * A.sdf.ts + h * A.sdf.hs] = (E)df;
                ((E *)A.db)[bi * A.sdb.bs + (t0 + i) * A.sdb.ts + h * A.sdb.hs] = (E)(all(1) * (1.f / (1.f + expf(bb))));
            }
        }
        if (hi >= rows) break;
        __syncthreads();
        lo = hi;
        hi = episode_end(A, bi, t0, lo, rows);
    }
}

}  // namespace seq
