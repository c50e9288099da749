// Queries and keys per head: a root-mean-square norm and the rotation by position (Su et al. 2021, arXiv 2104.09864; elements i and i + R/2 are a pair) in one
// pass, and its gradients.
//
// Per head of D elements: y = weight x rstd, then elements i and i + R/2 (i < R/2) as a point turned by position times turns_i.
// Bound by memory: everything is read once and written once.  A head belongs to a group of `lanes` lanes; a lane holds K units, a unit
// being V elements and the V they are turned with (behind R: V and the next V), V 16 bytes' worth or 1.  So a turn needs no
// exchange, and the angles of a row, 25 instructions a pair, serve all heads that a group takes.
// An angle is exact before its sine is taken: position times turns_i in 64-bit fixed point, whose upper 32 bits are the fraction of
// a full turn.  Sine and cosine of the rest of an eighth are their series, off by 2^-25 at most.
// 16384 rows of 8 + 8 heads of 64 in bf16: forward 19 us (67 MB, 3.6 TB/s), gradients 25 + 4 (101 MB, 4.0 TB/s); 30011 rows of 5 + 2 heads of 100 in fp32, 50
// of them turned, an element at a time because no partners 25 elements apart lie at multiples of 16 bytes both: 46 (168 MB, 3.7 TB/s) and 66 + 7 (252 MB, 3.8 TB/s).  A large copy reaches 5.1.
#pragma once
#include "seq_common.h"

namespace seq {

constexpr int HEADS_MAX = 256;
// Most partial sums of the weights' gradients, one per workgroup.  Wide rows take half of them: what a workgroup begins and ends with counts for more there
// (16384 x 16 x 64 in bf16: 512 25 + 4 us, 1024 32 + 6).
constexpr int HEADS_PARTS = 1024;

struct HeadsShape {
    long M;
    int Hq, Hk, D, half;               // half: R / 2
    int lanes, per_row;                // lanes of a group; groups that share a row (a power of two)
};
struct HeadsArgs {
    const void *q, *k;
    long q_rs, q_hs, k_rs, k_hs;
    const float *wq, *wk;
    const int32_t *position;
    void *yq, *yk;
    long yq_rs, yq_hs, yk_rs, yk_hs;
    float *rstd;                       // [M][Hq + Hk], or NULL
    float eps;
    HeadsShape s;
    uint64_t turns[HEADS_MAX / 2];     // per position, in units of 2^-64 of a full turn
};
struct HeadsGradArgs {
    const void *dyq, *dyk, *q, *k;
    long dyq_rs, dyq_hs, dyk_rs, dyk_hs, q_rs, q_hs, k_rs, k_hs;
    const float *wq, *wk, *rstd;
    const int32_t *position;
    void *dq, *dk;
    long dq_rs, dq_hs, dk_rs, dk_hs;
    float *part;                       // [workgroups][2][D]
    HeadsShape s;
    uint64_t turns[HEADS_MAX / 2];
};

// cosine and sine of position * turns
__device__ __forceinline__ void turned(int32_t position, uint64_t turns, float &c, float &s)
{
    const uint32_t p = (uint32_t)position, lo = (uint32_t)turns, hi = (uint32_t)(turns >> 32);
    const uint32_t f = __umulhi(p, lo) + p * hi - (position < 0 ? lo : 0u);
    const uint32_t quarter = (f + (1u << 29)) >> 30;
    const float x = (float)(int32_t)(f - (quarter << 30)) * 1.46291807926715968e-9f, xx = x * x;      // 2 pi / 2^32
    const float sn = fmaf(x * xx, fmaf(xx, fmaf(xx, fmaf(xx, 2.75573192e-6f, -1.98412698e-4f), 8.33333333e-3f), -0.166666667f), x);
    const float cs = fmaf(xx, fmaf(xx, fmaf(xx, fmaf(xx, 2.48015873e-5f, -1.38888889e-3f), 4.16666667e-2f), -0.5f), 1.f);
    const float a = quarter & 1 ? sn : cs, b = quarter & 1 ? cs : sn;
    c = (quarter + 1) & 2 ? -a : a;
    s = quarter & 2 ? -b : b;
}

// A lane's units: where each begins, where the elements it is turned with begin, and whether it is turned.
template <int V, int K> struct Units {
    int lo[K], hi[K];
    bool turn[K];
    __device__ __forceinline__ Units(const HeadsShape &s)
    {
        const int pairs = (s.half + V - 1) / V, lane = threadIdx.x & (s.lanes - 1);
#pragma unroll
        for (int j = 0; j < K; ++j) {
            const int u = lane + j * s.lanes;
            turn[j] = u < pairs;
            lo[j] = turn[j] ? u * V : 2 * s.half + 2 * (u - pairs) * V;
            hi[j] = turn[j] ? s.half + u * V : lo[j] + V;
        }
    }
};

template <class T, int V, int K> __device__ __forceinline__ void load_head(const T *p, const Units<V, K> &u, int D, bool real, vec<T, V> (&lo)[K], vec<T, V> (&hi)[K])
{
#pragma unroll
    for (int j = 0; j < K; ++j) {
        lo[j] = real && u.lo[j] < D ? load<V>(p + u.lo[j]) : vec<T, V>(0.f);
        hi[j] = real && u.hi[j] < D ? load<V>(p + u.hi[j]) : vec<T, V>(0.f);
    }
}

template <int V, int K> struct Angles {
    float c[K][V], s[K][V];
    __device__ __forceinline__ void set(const Units<V, K> &u, const uint64_t (&turns)[K][V], int32_t position)
    {
#pragma unroll
        for (int j = 0; j < K; ++j)
#pragma unroll
            for (int i = 0; i < V; ++i) turned(position, turns[j][i], c[j][i], s[j][i]);
    }
};

template <int V, int K> __device__ __forceinline__ void load_turns(const uint64_t *turns, const Units<V, K> &u, uint64_t (&t)[K][V])
{
#pragma unroll
    for (int j = 0; j < K; ++j)
#pragma unroll
        for (int i = 0; i < V; ++i) t[j][i] = u.turn[j] ? turns[u.lo[j] + i] : 0;
}

// HB heads of a group at a time, their loads ahead of everything else (an element at a time, 30011 x 7 x 100 in fp32: 4 heads 46 us, 8, with fewer waves on a
// compute unit, 55).  With the next batch's loads under way as well registers leave fewer waves, and it is no faster (50; backward, 16384 x 16 x 64 in bf16, 47 where this took 31).
template <class E, int V, int K, int HB> __device__ __forceinline__ void heads_forward(const E *x, long hs, E *y, long yhs, int H, const float (&wl)[K][V], const float (&wh)[K][V],
                                                                                      const Units<V, K> &u, const Angles<V, K> &a, const HeadsShape &s, int sub, bool row, float eps, float *rstd)
{
    for (int h0 = sub; h0 - sub < H; h0 += HB * s.per_row) {
        vec<E, V> lo[HB][K], hi[HB][K];
#pragma unroll
        for (int n = 0; n < HB; ++n) load_head<E, V, K>(x + (h0 + n * s.per_row) * hs, u, s.D, row && h0 + n * s.per_row < H, lo[n], hi[n]);
#pragma unroll
        for (int n = 0; n < HB; ++n) {
            const int h = h0 + n * s.per_row;
            float sum = 0.f;
#pragma unroll
            for (int j = 0; j < K; ++j)
#pragma unroll
                for (int i = 0; i < V; ++i) {
                    sum = fmaf((float)lo[n][j][i], (float)lo[n][j][i], sum);
                    sum = fmaf((float)hi[n][j][i], (float)hi[n][j][i], sum);
                }
            const float r = 1.f / sqrtf(group_fold(sum, s.lanes, add) / (float)s.D + eps);
            if (!row || h >= H) continue;
            if (rstd && (threadIdx.x & (s.lanes - 1)) == 0) rstd[h] = r;
#pragma unroll
            for (int j = 0; j < K; ++j) {
                float yl[V], yh[V];
#pragma unroll
                for (int i = 0; i < V; ++i) {
                    const float l = (float)lo[n][j][i] * r * wl[j][i], g = (float)hi[n][j][i] * r * wh[j][i];
                    yl[i] = u.turn[j] ? l * a.c[j][i] - g * a.s[j][i] : l;
                    yh[i] = u.turn[j] ? g * a.c[j][i] + l * a.s[j][i] : g;
                }
                if (u.lo[j] < s.D) store<V>(y + h * yhs + u.lo[j], narrow<E, V>(yl));
                if (u.hi[j] < s.D) store<V>(y + h * yhs + u.hi[j], narrow<E, V>(yh));
            }
        }
    }
}

template <int V, int K> __device__ __forceinline__ void load_weight(const float *w, const Units<V, K> &u, int D, float (&l)[K][V], float (&h)[K][V])
{
#pragma unroll
    for (int j = 0; j < K; ++j)
#pragma unroll
        for (int i = 0; i < V; ++i) {
            l[j][i] = w && u.lo[j] + i < D ? w[u.lo[j] + i] : 0.f;
            h[j][i] = w && u.hi[j] + i < D ? w[u.hi[j] + i] : 0.f;
        }
}

template <class E, int V, int K> __global__ __launch_bounds__(256) void k_heads(HeadsArgs A)
{
    const HeadsShape &s = A.s;
    const Units<V, K> u(s);
    const int group = threadIdx.x / s.lanes, groups = 256 / s.lanes, sub = group & (s.per_row - 1), rows = groups / s.per_row;
    float ql[K][V], qh[K][V], kl[K][V], kh[K][V];
    load_weight<V, K>(s.Hq ? A.wq : nullptr, u, s.D, ql, qh);
    load_weight<V, K>(s.Hk ? A.wk : nullptr, u, s.D, kl, kh);
    uint64_t t[K][V];
    load_turns<V, K>(A.turns, u, t);
    for (long m0 = (long)blockIdx.x * rows; m0 < s.M; m0 += (long)gridDim.x * rows) {
        const long m = m0 + group / s.per_row;
        const bool row = m < s.M;
        Angles<V, K> a;
        if (s.half) a.set(u, t, row ? A.position[m] : 0);
        float *rstd = A.rstd ? A.rstd + m * (s.Hq + s.Hk) : nullptr;
        heads_forward<E, V, K, V == 1 ? 4 : 2>((const E *)A.q + m * A.q_rs, A.q_hs, (E *)A.yq + m * A.yq_rs, A.yq_hs, s.Hq, ql, qh, u, a, s, sub, row, A.eps, rstd);
        heads_forward<E, V, K, V == 1 ? 4 : 2>((const E *)A.k + m * A.k_rs, A.k_hs, (E *)A.yk + m * A.yk_rs, A.yk_hs, s.Hk, kl, kh, u, a, s, sub, row, A.eps, rstd ? rstd + s.Hq : nullptr);
    }
}

// With xh = x rstd, dy turned back and g = weight dy:  dx = rstd (g - xh mean(g xh)),  dw = sum of dy xh.
template <class E, int V, int K, int HB>
__device__ __forceinline__ void heads_backward(const E *dy, long dhs, const E *x, long hs, E *dx, long xhs, int H, const float (&wl)[K][V], const float (&wh)[K][V], float (&dwl)[K][V], float (&dwh)[K][V],
                                               const Units<V, K> &u, const Angles<V, K> &a, const HeadsShape &s, int sub, bool row, const float *rstd)
{
    for (int h0 = sub; h0 - sub < H; h0 += HB * s.per_row) {
        vec<E, V> lo[HB][K], hi[HB][K], dl[HB][K], dh[HB][K];
        float rs[HB];
#pragma unroll
        for (int n = 0; n < HB; ++n) {
            const int h = h0 + n * s.per_row;
            load_head<E, V, K>(x + h * hs, u, s.D, row && h < H, lo[n], hi[n]);
            load_head<E, V, K>(dy + h * dhs, u, s.D, row && h < H, dl[n], dh[n]);
            rs[n] = row && h < H ? rstd[h] : 0.f;
        }
#pragma unroll
        for (int n = 0; n < HB; ++n) {
            const int h = h0 + n * s.per_row;
            float xl[K][V], xh[K][V], gl[K][V], gh[K][V], sum = 0.f;
#pragma unroll
            for (int j = 0; j < K; ++j)
#pragma unroll
                for (int i = 0; i < V; ++i) {
                    const float l = (float)dl[n][j][i], g = (float)dh[n][j][i];
                    const float bl = u.turn[j] ? l * a.c[j][i] + g * a.s[j][i] : l, bh = u.turn[j] ? g * a.c[j][i] - l * a.s[j][i] : g;
                    xl[j][i] = (float)lo[n][j][i] * rs[n];
                    xh[j][i] = (float)hi[n][j][i] * rs[n];
                    dwl[j][i] = fmaf(bl, xl[j][i], dwl[j][i]);
                    dwh[j][i] = fmaf(bh, xh[j][i], dwh[j][i]);
                    gl[j][i] = bl * wl[j][i];
                    gh[j][i] = bh * wh[j][i];
                    sum = fmaf(gl[j][i], xl[j][i], fmaf(gh[j][i], xh[j][i], sum));
                }
            const float mean = group_fold(sum, s.lanes, add) / (float)s.D;
            if (!row || h >= H) continue;
#pragma unroll
            for (int j = 0; j < K; ++j) {
                float ol[V], oh[V];
#pragma unroll
                for (int i = 0; i < V; ++i) {
                    ol[i] = rs[n] * (gl[j][i] - xl[j][i] * mean);
                    oh[i] = rs[n] * (gh[j][i] - xh[j][i] * mean);
                }
                if (u.lo[j] < s.D) store<V>(dx + h * xhs + u.lo[j], narrow<E, V>(ol));
                if (u.hi[j] < s.D) store<V>(dx + h * xhs + u.hi[j], narrow<E, V>(oh));
            }
        }
    }
}

template <class E, int V, int K> __global__ __launch_bounds__(256) void k_heads_grad(HeadsGradArgs A)
{
    __shared__ float sh[4][4][HEADS_MAX / 2];
    const HeadsShape &s = A.s;
    const Units<V, K> u(s);
    const int group = threadIdx.x / s.lanes, groups = 256 / s.lanes, sub = group & (s.per_row - 1), rows = groups / s.per_row;
    float ql[K][V], qh[K][V], kl[K][V], kh[K][V], dq[2][K][V] = {}, dk[2][K][V] = {};
    load_weight<V, K>(s.Hq ? A.wq : nullptr, u, s.D, ql, qh);
    load_weight<V, K>(s.Hk ? A.wk : nullptr, u, s.D, kl, kh);
    uint64_t t[K][V];
    load_turns<V, K>(A.turns, u, t);
    for (long m0 = (long)blockIdx.x * rows; m0 < s.M; m0 += (long)gridDim.x * rows) {
        const long m = m0 + group / s.per_row;
        const bool row = m < s.M;
        Angles<V, K> a;
        if (s.half) a.set(u, t, row ? A.position[m] : 0);
        const float *rstd = A.rstd + m * (s.Hq + s.Hk);
        heads_backward<E, V, K, V == 1 ? 4 : 2>((const E *)A.dyq + m * A.dyq_rs, A.dyq_hs, (const E *)A.q + m * A.q_rs, A.q_hs, (E *)A.dq + m * A.dq_rs, A.dq_hs, s.Hq, ql, qh, dq[0], dq[1], u, a, s, sub, row, rstd);
        heads_backward<E, V, K, V == 1 ? 4 : 2>((const E *)A.dyk + m * A.dyk_rs, A.dyk_hs, (const E *)A.k + m * A.k_rs, A.k_hs, (E *)A.dk + m * A.dk_rs, A.dk_hs, s.Hk, kl, kh, dk[0], dk[1], u, a, s, sub, row, rstd + s.Hq);
    }
    // the groups' sums, of a wave's groups lane by lane, then of the four waves
    float *part = A.part + (long)blockIdx.x * 2 * s.D;
    const int lane = threadIdx.x & 63, w = threadIdx.x >> 6;
#pragma unroll
    for (int j = 0; j < K; ++j)
#pragma unroll
        for (int i = 0; i < V; ++i) {
            float v[4] = {dq[0][j][i], dq[1][j][i], dk[0][j][i], dk[1][j][i]};
            for (int d = s.lanes; d < 64; d *= 2)
#pragma unroll
                for (int n = 0; n < 4; ++n) v[n] += __shfl_xor(v[n], d);
            if (lane < s.lanes)
#pragma unroll
                for (int n = 0; n < 4; ++n) sh[w][n][(j * V + i) * s.lanes + lane] = v[n];
        }
    __syncthreads();
    const int count = K * V * s.lanes, pairs = (s.half + V - 1) / V;
    for (int e = threadIdx.x; e < 4 * count; e += 256) {
        const int which = e / count, at = e % count, i = at / s.lanes % V, unit = at / s.lanes / V * s.lanes + at % s.lanes;
        const int lo = unit < pairs ? unit * V : 2 * s.half + 2 * (unit - pairs) * V, hi = unit < pairs ? s.half + unit * V : lo + V;
        const int c = (which & 1 ? hi : lo) + i;
        if (c < s.D) part[(which >> 1) * s.D + c] = (sh[0][which][at] + sh[1][which][at]) + (sh[2][which][at] + sh[3][which][at]);
    }
}

// The sum of the workgroups' parts, 16 columns a workgroup, in a fixed order.
__global__ __launch_bounds__(1024) void k_heads_join(const float *part, int parts, int D, float *dwq, float *dwk)
{
    __shared__ float sh[64][17];
    const int c = blockIdx.x * 16 + (threadIdx.x & 15), g = threadIdx.x >> 4;
    float sum = 0.f;
    if (c < 2 * D)
        for (int p = g; p < parts; p += 64) sum += part[(long)p * 2 * D + c];
    sh[g][threadIdx.x & 15] = sum;
    __syncthreads();
    if (g == 0 && c < 2 * D) {
        sum = 0.f;
        for (int p = 0; p < 64; ++p) sum += sh[p][threadIdx.x & 15];
        if (float *to = c < D ? dwq : dwk) to[c < D ? c : c - D] = sum;
    }
}

}  // namespace seq
