// Root-mean-square norm with the residual's addition, its gradients, and rows of 8-bit numbers.
//
// All of it is bound by memory: every element is read once and written once, a row being kept in registers between its
// sums and its results.  A row belongs to W waves (1, 4 or 16), a lane holding K times V consecutive elements; V is 16
// bytes' worth, or 1 where the size, a stride or an address does not allow that.  Short rows (K = 1) share a wave.
// Measured: 16384 rows of 512 in bf16 with a residual 12.2 us forward (5.5 TB/s) and 16.7 backward (5.0); 30011 rows of
// 1001 in fp32 81 us (5.9 TB/s) and 103 (5.8); a copy reaches 5.2.
#pragma once
#include "seq_common.h"

namespace seq {

struct NormArgs {
    const void *x, *residual;
    long x_rs, residual_rs;
    const float *weight;   // NULL: the rows are only converted (no norm)
    float eps;
    void *r, *y;
    long r_rs, y_rs;
    uint8_t *q;
    long q_rs;
    float *scale, *rstd;
    long M;
    int C, lanes;   // lanes of a row: 64, or a smaller power of two
};
struct NormGradArgs {
    const void *dy, *x, *residual, *dr;
    long dy_rs, x_rs, residual_rs, dr_rs;
    const float *weight, *rstd;
    void *dx;
    long dx_rs;
    float *dw, *part;
    long M;
    int C, lanes;
};

constexpr int NORM_PARTS = 512;   // most partial sums of the weight's gradient, one per workgroup
constexpr int NORM_ROWS = 16;      // rows that are worth a partial sum

// The W waves of a row add up (or fold by f) a value; `sh` holds W floats and must not be written again before all have
// read it: two in turn do.
template <int W, class F> __device__ __forceinline__ float row_fold(float v, int lanes, float *sh, F f)
{
    v = group_fold(v, W == 1 ? lanes : 64, f);
    if constexpr (W > 1) {
        if ((threadIdx.x & 63) == 0) sh[threadIdx.x >> 6] = v;
        lds_barrier();
        v = sh[0];
#pragma unroll
        for (int w = 1; w < W; ++w) v = f(v, sh[w]);
    }
    return v;
}

// Where a thread stands: its row among those that a workgroup has at a time, and its column of the k-th V elements.
template <int V, int W> struct Spot {
    int row, first, stride;
    __device__ __forceinline__ Spot(int lanes)
    {
        const int t = threadIdx.x;
        row = W > 1 ? 0 : t / lanes;
        first = (W > 1 ? t : t & (lanes - 1)) * V;
        stride = (W > 1 ? 64 * W : 64) * V;
    }
    __device__ __forceinline__ int col(int k) const { return first + k * stride; }
    static __device__ __forceinline__ int rows(int lanes) { return W > 1 ? 1 : 256 / lanes; }
};

template <class E, int V, int K, int W> __device__ __forceinline__ void load_row(const E *p, const Spot<V, W> &s, int C, vec<E, V> (&v)[K])
{
#pragma unroll
    for (int k = 0; k < K; ++k)
        v[k] = s.col(k) < C ? load<V>(p + s.col(k)) : vec<E, V>(0.f);
}

template <class E, int V, int K, int W, bool EIGHT> __global__ __launch_bounds__(W == 1 ? 256 : 64 * W) void k_norm(NormArgs A)
{
    __shared__ float sh[4][W];
    const Spot<V, W> s(A.lanes);
    const int rows = s.rows(A.lanes), pad = (A.C + 15) & ~15;
    const bool normed = A.weight;
    float w[K][V];
#pragma unroll
    for (int k = 0; k < K; ++k) {
        const auto v = normed && s.col(k) < A.C ? load<V>(A.weight + s.col(k)) : vec<float, V>(1.f);
#pragma unroll
        for (int i = 0; i < V; ++i) w[k][i] = v[i];
    }
    int turn = 0;
    for (long m0 = (long)blockIdx.x * rows; m0 < A.M; m0 += (long)gridDim.x * rows, turn ^= 2) {
        const long m = m0 + s.row;
        if (W == 1 && m >= A.M) break;   // no barrier follows: with W = 1 rows do not meet
        vec<E, V> x[K], res[K];
        float r[K][V];
        load_row<E, V, K, W>((const E *)A.x + m * A.x_rs, s, A.C, x);
        if (A.residual) load_row<E, V, K, W>((const E *)A.residual + m * A.residual_rs, s, A.C, res);
        float sum = 0.f;
#pragma unroll
        for (int k = 0; k < K; ++k)
#pragma unroll
            for (int i = 0; i < V; ++i) {
                r[k][i] = (float)x[k][i] + (A.residual ? (float)res[k][i] : 0.f);
                sum = fmaf(r[k][i], r[k][i], sum);
            }
        if (A.r) {
#pragma unroll
            for (int k = 0; k < K; ++k)
                if (s.col(k) < A.C) store<V>((E *)A.r + m * A.r_rs + s.col(k), narrow<E, V>(r[k]));
        }
        if (normed) {
            const float rstd = 1.f / sqrtf(row_fold<W>(sum, A.lanes, sh[turn], add) / (float)A.C + A.eps);
            if (A.rstd && s.first == 0) A.rstd[m] = rstd;
#pragma unroll
            for (int k = 0; k < K; ++k)
#pragma unroll
                for (int i = 0; i < V; ++i) r[k][i] = r[k][i] * rstd * w[k][i];
        }
        if constexpr (EIGHT) {
            float top = 0.f;
#pragma unroll
            for (int k = 0; k < K; ++k)
#pragma unroll
                for (int i = 0; i < V; ++i) top = nan_max(top, fabsf(r[k][i]));
            top = row_fold<W>(top, A.lanes, sh[turn + 1], nan_max);
            if (!(top <= 3.4028234e38f)) top = __builtin_nanf("");
            if (top > 0.f) top = fmaxf(top, E4M3_LEAST);
            const float inv = top == 0.f ? 0.f : 1.f / top * E4M3_MAX;
            if (s.first == 0) A.scale[m] = top * (1.f / E4M3_MAX);
#pragma unroll
            for (int k = 0; k < K; ++k) {
                if (s.col(k) >= pad) continue;
                float q[V < 4 ? 4 : V] = {};
#pragma unroll
                for (int i = 0; i < V; ++i) q[i] = s.col(k) < A.C ? fminf(fmaxf(r[k][i] * inv, -E4M3_MAX), E4M3_MAX) : 0.f;
                uint8_t *p = A.q + m * A.q_rs + s.col(k);
                if constexpr (V == 1) *p = (uint8_t)pack_e4m3(q[0], 0.f, 0.f, 0.f);
                else {
                    vec<uint32_t, V / 4> o;
#pragma unroll
                    for (int i = 0; i < V; i += 4) o[i / 4] = pack_e4m3(q[i], q[i + 1], q[i + 2], q[i + 3]);
                    *reinterpret_cast<vec<uint32_t, V / 4> *>(p) = o;
                }
            }
        } else {
#pragma unroll
            for (int k = 0; k < K; ++k)
                if (s.col(k) < A.C) store<V>((E *)A.y + m * A.y_rs + s.col(k), narrow<E, V>(r[k]));
        }
    }
}

// Gradients.  A workgroup goes through rows blockIdx.x, + gridDim.x, ... and adds up its part of the weight's gradient in
// registers; the parts are joined by k_norm_grad_join in a fixed order.  r is formed again as the forward call did, from
// x and the residual where they were rounded to be stored: the sum of the two as one number would be a bf16 off in dw.
template <class E, int V, int K, int W> __global__ __launch_bounds__(W == 1 ? 256 : 64 * W) void k_norm_grad(NormGradArgs A)
{
    __shared__ float sh[2][W];
    __shared__ float parts[W == 1 ? 4 : 1][W == 1 ? 64 * V * K : 1];
    const Spot<V, W> s(A.lanes);
    const int rows = s.rows(A.lanes);
    float w[K][V], dw[K][V];
#pragma unroll
    for (int k = 0; k < K; ++k) {
        const auto v = s.col(k) < A.C ? load<V>(A.weight + s.col(k)) : vec<float, V>(0.f);
#pragma unroll
        for (int i = 0; i < V; ++i) { w[k][i] = v[i]; dw[k][i] = 0.f; }
    }
    const float mean = 1.f / (float)A.C;
    int turn = 0;
    for (long m0 = (long)blockIdx.x * rows; m0 < A.M; m0 += (long)gridDim.x * rows, turn ^= 1) {
        const long m = m0 + s.row;
        if (W == 1 && m >= A.M) break;
        vec<E, V> dy[K], x[K], res[K], dr[K];
        load_row<E, V, K, W>((const E *)A.dy + m * A.dy_rs, s, A.C, dy);
        load_row<E, V, K, W>((const E *)A.x + m * A.x_rs, s, A.C, x);
        if (A.residual) load_row<E, V, K, W>((const E *)A.residual + m * A.residual_rs, s, A.C, res);
        if (A.dr) load_row<E, V, K, W>((const E *)A.dr + m * A.dr_rs, s, A.C, dr);
        const float rstd = A.rstd[m];
        float xh[K][V], sum = 0.f;
#pragma unroll
        for (int k = 0; k < K; ++k)
#pragma unroll
            for (int i = 0; i < V; ++i) {
                xh[k][i] = ((float)x[k][i] + (A.residual ? (float)res[k][i] : 0.f)) * rstd;
                const float d = (float)dy[k][i] * xh[k][i];
                dw[k][i] += d;
                sum = fmaf(d, w[k][i], sum);
            }
        sum = row_fold<W>(sum, A.lanes, sh[turn], add) * mean;
#pragma unroll
        for (int k = 0; k < K; ++k) {
            if (s.col(k) >= A.C) continue;
            float dx[V];
#pragma unroll
            for (int i = 0; i < V; ++i) {
                dx[i] = rstd * ((float)dy[k][i] * w[k][i] - xh[k][i] * sum);
                if (A.dr) dx[i] += (float)dr[k][i];
            }
            store<V>((E *)A.dx + m * A.dx_rs + s.col(k), narrow<E, V>(dx));
        }
    }
    float *part = A.part + (long)blockIdx.x * A.C;
    if constexpr (W > 1) {
#pragma unroll
        for (int k = 0; k < K; ++k)
            if (s.col(k) < A.C) store<V>(part + s.col(k), narrow<float, V>(dw[k]));
    } else {
        const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
#pragma unroll
        for (int k = 0; k < K; ++k) {
#pragma unroll
            for (int i = 0; i < V; ++i)
                for (int o = 32; o >= A.lanes; o >>= 1) dw[k][i] += __shfl_xor(dw[k][i], o);   // the rows of a wave
            if (lane < A.lanes) store<V>(&parts[wave][s.col(k)], narrow<float, V>(dw[k]));
        }
        __syncthreads();
        for (int c = threadIdx.x; c < A.C; c += 256) part[c] = (parts[0][c] + parts[1][c]) + (parts[2][c] + parts[3][c]);
    }
}

// dw: the sum of `parts` rows; a workgroup takes 16 columns, a thread every 64th row of one of them
__global__ __launch_bounds__(1024) void k_norm_grad_join(const float *part, int parts, int C, float *dw)
{
    __shared__ float sh[64][17];
    const int c = threadIdx.x & 15, g = threadIdx.x >> 4, col = blockIdx.x * 16 + c;
    float s = 0.f;
    if (col < C)
#pragma unroll 8
        for (int p = g; p < parts; p += 64) s += part[(long)p * C + col];
    sh[g][c] = s;
    for (int o = 32; o; o >>= 1) {
        __syncthreads();
        if (g < o) sh[g][c] += sh[g + o][c];
    }
    if (g == 0 && col < C) dw[col] = sh[0][c];
}

}  // namespace seq
