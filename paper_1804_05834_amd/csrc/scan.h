// Gated linear recurrence over time, h_t = a_t k_t h_{t-1} + (1 - a_t) x_t, and its gradients.
#pragma once
#include "seq_common.h"

namespace seq {

struct ScanArgs {
    const void *f, *x;
    long f_bs, f_ts, x_bs, x_ts;
    const float *h0;
    const uint8_t *reset;
    long r_bs, r_ts;
    void *h;
    long h_bs, h_ts;
    float *h_last, *carry;
    long T;
    int B, C;
};
struct ScanGradArgs {
    const void *f, *x, *dh;
    long f_bs, f_ts, x_bs, x_ts, dh_bs, dh_ts;
    const float *carry, *dlast;
    const uint8_t *reset;
    long r_bs, r_ts;
    void *df, *dx;
    long df_bs, df_ts, dx_bs, dx_ts;
    float *dh0;
    long T;
    int B, C;
};

constexpr int SCAN_CARRY = 16;   // steps between two states of `carry`

// sigmoid(f) and 1 - sigmoid(f).  The second is computed apart: 1 - a of an `a` near one, a memory that lasts, would keep
// few of its digits.
__device__ __forceinline__ void gates(float f, float &a, float &i)
{
    const float e = __builtin_amdgcn_exp2f(-1.44269504088896341f * fabsf(f));
    const float r = __builtin_amdgcn_rcpf(1.f + e), s = e * r;
    a = f < 0.f ? s : r;
    i = f < 0.f ? r : s;
}

// one thread per channel of a sequence
template <class E> __global__ __launch_bounds__(64) void k_scan(ScanArgs A)
{
    const int c = blockIdx.x * 64 + threadIdx.x, b = blockIdx.y;
    if (c >= A.C) return;
    const E *f = (const E *)A.f + b * A.f_bs + c, *x = (const E *)A.x + b * A.x_bs + c;
    E *h = (E *)A.h + b * A.h_bs + c;
    float s = A.h0 ? A.h0[(long)b * A.C + c] : 0.f;
    const long tiles = (A.T + SCAN_CARRY - 1) / SCAN_CARRY;
    for (long t = 0; t < A.T; ++t) {
        if (A.carry && t % SCAN_CARRY == 0) A.carry[(b * tiles + t / SCAN_CARRY) * A.C + c] = s;
        if (A.reset && A.reset[b * A.r_bs + t * A.r_ts]) s = 0.f;
        float a, i;
        gates((float)f[t * A.f_ts], a, i);
        s = fmaf(a, s, i * (float)x[t * A.x_ts]);
        h[t * A.h_ts] = (E)s;
    }
    if (A.h_last) A.h_last[(long)b * A.C + c] = s;
}

template <class E> __global__ __launch_bounds__(64) void k_scan_grad(ScanGradArgs A)
{
    const int c = blockIdx.x * 64 + threadIdx.x, b = blockIdx.y;
    if (c >= A.C) return;
    const E *f = (const E *)A.f + b * A.f_bs + c, *x = (const E *)A.x + b * A.x_bs + c, *dh = (const E *)A.dh + b * A.dh_bs + c;
    E *df = (E *)A.df + b * A.df_bs + c, *dx = (E *)A.dx + b * A.dx_bs + c;
    float mu = A.dlast ? A.dlast[(long)b * A.C + c] : 0.f;
    const long tiles = (A.T + SCAN_CARRY - 1) / SCAN_CARRY;
    for (long q = tiles - 1; q >= 0; --q) {
        float s = A.carry[(b * tiles + q) * A.C + c], before[SCAN_CARRY];
        for (int j = 0; j < SCAN_CARRY; ++j) {
            const long t = q * SCAN_CARRY + j;
            if (t >= A.T) break;
            if (A.reset && A.reset[b * A.r_bs + t * A.r_ts]) s = 0.f;
            before[j] = s;
            float a, i;
            gates((float)f[t * A.f_ts], a, i);
            s = fmaf(a, s, i * (float)x[t * A.x_ts]);
        }
        for (int j = SCAN_CARRY - 1; j >= 0; --j) {
            const long t = q * SCAN_CARRY + j;
            if (t >= A.T) continue;
            float a, i;
            gates((float)f[t * A.f_ts], a, i);
            const float l = (float)dh[t * A.dh_ts] + mu;
            dx[t * A.dx_ts] = (E)(i * l);
            df[t * A.df_ts] = (E)(l * (before[j] - (float)x[t * A.x_ts]) * a * i);
            mu = A.reset && A.reset[b * A.r_bs + t * A.r_ts] ? 0.f : a * l;
        }
    }
    if (A.dh0) A.dh0[(long)b * A.C + c] = mu;
}

}  // namespace seq
