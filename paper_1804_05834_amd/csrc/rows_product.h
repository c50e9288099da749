// Product of 8-bit rows with 8-bit weights.
#pragma once
#include "seq_common.h"

namespace seq {

struct ProductArgs {
    const uint8_t *a, *w;
    long a_rs, w_rs;
    const float *a_scale, *w_scale, *bias;
    void *y;
    long y_rs, M;
    int N, K;
};

// the 8 bytes of a row from k on, those from K on set to zero (k is a multiple of 8, a row may be read up to the next
// multiple of 16)
__device__ __forceinline__ long row_bytes(const uint8_t *row, int k, int K)
{
    if (k >= K) return 0;
    const unsigned long v = *reinterpret_cast<const unsigned long *>(row + k);
    return (long)(K - k >= 8 ? v : v & ~(~0ul << 8 * (K - k)));
}

// eight e4m3 numbers as bf16, exactly
__device__ __forceinline__ vec<bf16, 8> widen(long v)
{
    vec<bf16, 8> o;
#pragma unroll
    for (int w = 0; w < 2; ++w) {
        const int x = (int)(v >> 32 * w);
        const auto lo = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(x, 1.f, false), hi = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(x, 1.f, true);
        o[4 * w] = lo[0]; o[4 * w + 1] = lo[1]; o[4 * w + 2] = hi[0]; o[4 * w + 3] = hi[1];
    }
    return o;
}

// s + sum over 32 k.  The matrix instructions on e4m3 keep about 16 bits of a sum (measured, 16 x 16 outputs: 1.5e-5 off in
// the 2-norm at every K, where the same numbers as bf16 are 5e-8 off).  An output that is rounded to bf16 loses a
// hundred times that anyway and takes them; an fp32 output takes the numbers as bf16, at half the rate.
template <class E> __device__ __forceinline__ vec<float, 4> mac(long a, long w, vec<float, 4> s)
{
    if constexpr (sizeof(E) == 2) return __builtin_amdgcn_mfma_f32_16x16x32_fp8_fp8(a, w, s, 0, 0, 0);
    else return __builtin_amdgcn_mfma_f32_16x16x32_bf16(widen(a), widen(w), s, 0, 0, 0);
}

// One wave per 16 x 16 outputs, operands from memory into registers.  A lane holds row lane % 16 of both operands,
// bytes 8 (lane / 16) to + 7 of every 32; it gets column lane % 16 of rows 4 (lane / 16) to + 3.
template <class E> __global__ __launch_bounds__(64) void k_product(ProductArgs A)
{
    const int lane = threadIdx.x, i = lane & 15, g = lane >> 4;
    const long m0 = (long)blockIdx.x * 16;
    const int n0 = blockIdx.y * 16;
    const uint8_t *a = A.a + min(m0 + i, A.M - 1) * A.a_rs, *w = A.w + (long)min(n0 + i, A.N - 1) * A.w_rs;
    vec<float, 4> s = {0.f, 0.f, 0.f, 0.f};
    for (int k = 0; k < A.K; k += 32) s = mac<E>(row_bytes(a, k + 8 * g, A.K), row_bytes(w, k + 8 * g, A.K), s);
    const int n = n0 + i;
    if (n >= A.N) return;
    const float sw = A.w_scale[n], bias = A.bias ? A.bias[n] : 0.f;
    for (int j = 0; j < 4; ++j) {
        const long m = m0 + 4 * g + j;
        if (m < A.M) ((E *)A.y + m * A.y_rs)[n] = (E)(s[j] * A.a_scale[m] * sw + bias);
    }
}

}  // namespace seq
