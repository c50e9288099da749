// Root-mean-square norm with the residual's addition, its gradients, and rows of 8-bit numbers.
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
    int C;
};
struct NormGradArgs {
    const void *dy, *r, *dr;
    long dy_rs, r_rs, dr_rs;
    const float *weight, *rstd;
    void *dx;
    long dx_rs;
    float *dw, *part;
    long M;
    int C, parts;
};

constexpr int NORM_PARTS = 512;   // most partial sums of the weight's gradient

template <class F> __device__ __forceinline__ float block_fold(float v, float *sh, F f)
{
    for (int o = 32; o; o >>= 1) v = f(v, __shfl_xor(v, o));
    __syncthreads();
    if ((threadIdx.x & 63) == 0) sh[threadIdx.x >> 6] = v;
    __syncthreads();
    v = sh[0];
    for (int w = 1; w < (int)(blockDim.x >> 6); ++w) v = f(v, sh[w]);
    return v;
}
__device__ __forceinline__ float add(float a, float b) { return a + b; }

// one workgroup per row, the row read again for each of its uses
template <class E> __global__ __launch_bounds__(256) void k_norm(NormArgs A)
{
    __shared__ float sh[4];
    const long m = blockIdx.x;
    const E *x = (const E *)A.x + m * A.x_rs, *res = A.residual ? (const E *)A.residual + m * A.residual_rs : nullptr;
    auto at = [&](int c) { return (float)x[c] + (res ? (float)res[c] : 0.f); };
    float rstd = 1.f;
    if (A.weight) {
        float s = 0.f;
        for (int c = threadIdx.x; c < A.C; c += 256) s += at(c) * at(c);
        rstd = 1.f / sqrtf(block_fold(s, sh, add) / (float)A.C + A.eps);
        if (A.rstd && threadIdx.x == 0) A.rstd[m] = rstd;
    }
    auto out = [&](int c) { return A.weight ? at(c) * rstd * A.weight[c] : at(c); };
    float inv = 0.f;
    if (A.q) {
        float top = 0.f;
        for (int c = threadIdx.x; c < A.C; c += 256) top = nan_max(top, fabsf(out(c)));
        top = block_fold(top, sh, nan_max);
        if (!(top <= 3.4e38f)) top = __builtin_nanf("");
        inv = top == 0.f ? 0.f : E4M3_MAX / top;
        if (threadIdx.x == 0) A.scale[m] = top / E4M3_MAX;
        const int pad = (A.C + 15) & ~15;
        for (int c = threadIdx.x; c < pad; c += 256)
            A.q[m * A.q_rs + c] = c < A.C ? (uint8_t)pack_e4m3(fminf(fmaxf(out(c) * inv, -E4M3_MAX), E4M3_MAX), 0.f, 0.f, 0.f) : 0;
    }
    for (int c = threadIdx.x; c < A.C; c += 256) {   // r may lie where x or the residual does: a thread's own elements, and last
        const float v = at(c), o = out(c);
        if (A.y) ((E *)A.y + m * A.y_rs)[c] = (E)o;
        if (A.r) ((E *)A.r + m * A.r_rs)[c] = (E)v;
    }
}

template <class E> __global__ __launch_bounds__(256) void k_norm_grad(NormGradArgs A)
{
    __shared__ float sh[4];
    const long m = blockIdx.x;
    const E *dy = (const E *)A.dy + m * A.dy_rs, *r = (const E *)A.r + m * A.r_rs, *dr = A.dr ? (const E *)A.dr + m * A.dr_rs : nullptr;
    const float rstd = A.rstd[m];
    float s = 0.f;
    for (int c = threadIdx.x; c < A.C; c += 256) s += (float)dy[c] * A.weight[c] * (float)r[c] * rstd;
    s = block_fold(s, sh, add) / (float)A.C;
    for (int c = threadIdx.x; c < A.C; c += 256) {
        const float d = rstd * ((float)dy[c] * A.weight[c] - (float)r[c] * rstd * s) + (dr ? (float)dr[c] : 0.f);
        ((E *)A.dx + m * A.dx_rs)[c] = (E)d;
    }
}

// part[p][c]: sum over the rows p, p + parts, ...
template <class E> __global__ __launch_bounds__(256) void k_norm_grad_weight(NormGradArgs A)
{
    const int c = blockIdx.x * 256 + threadIdx.x, p = blockIdx.y;
    if (c >= A.C) return;
    float s = 0.f;
    for (long m = p; m < A.M; m += A.parts) s += (float)((const E *)A.dy + m * A.dy_rs)[c] * (float)((const E *)A.r + m * A.r_rs)[c] * A.rstd[m];
    A.part[(long)p * A.C + c] = s;
}
inline __global__ __launch_bounds__(256) void k_norm_grad_join(const float *part, int parts, int C, float *dw)
{
    const int c = blockIdx.x * 256 + threadIdx.x;
    if (c >= C) return;
    float s = 0.f;
    for (int p = 0; p < parts; ++p) s += part[(long)p * C + c];
    dw[c] = s;
}

}  // namespace seq
