// AdamW over many tensors in one launch, moments in 32 or 8 bits.
#pragma once
#include "seq_common.h"
#include "sumtree.h"

namespace seq {

constexpr int ADAM_BLOCK = 256;          // elements that share a scale: one wave, four elements per lane
constexpr int ADAM_CHUNK = 2048;         // elements of a workgroup

struct AdamTensor {
    float *param;
    const void *grad;
    uint16_t *copy;
    long n, at;      // elements; place of its moments in the buffers of moments
    float decay;
    int wide;        // every pointer allows four elements at a time
};
struct AdamChunk {
    int tensor, block;   // first block of the chunk within the tensor, in units of ADAM_CHUNK
};
struct AdamArgs {
    const AdamTensor *tensors;
    const AdamChunk *chunks;
    void *m, *v;
    float *ms, *vs;
    float lr, b1, c1, b2, c2, eps, rate, root;   // c = 1 - b; rate = lr / (1 - b1^t); root = 1 / sqrt(1 - b2^t)
    uint64_t seed;
};

// |x| >= 0 to MANTISSA bits (below 2^LOWEST: to multiples of the smallest number of the type), up where the 16 random
// bits are the larger and down where they are not, so that x is kept on average
template <int MANTISSA, int LOWEST> __device__ __forceinline__ float rounded(float x, uint32_t bits)
{
    constexpr int drop = 23 - MANTISSA;
    const float unit = __int_as_float((127 + LOWEST - MANTISSA) << 23);   // 2^(LOWEST - MANTISSA)
    const float normal = __uint_as_float((__float_as_uint(x) + (bits << (drop - 16))) & ~((1u << drop) - 1));
    const float small = floorf(x * (1.f / unit) + (float)bits * (1.f / 65536.f)) * unit;
    return x < __int_as_float((127 + LOWEST) << 23) ? small : normal;
}

// The new moments, every product and sum rounded by itself (no contraction into fused forms): what is rounded to 8 bits at
// random afterwards is then the same number in every correct implementation.
__device__ __forceinline__ void moments(float &m, float &v, float g, float b1, float c1, float b2, float c2)
{
#pragma clang fp contract(off)
    m = m * b1 + g * c1;
    v = v * b2 + g * g * c2;
}
__device__ __forceinline__ float product(float a, float b)
{
#pragma clang fp contract(off)
    return a * b;
}

template <class G, int BITS> __global__ __launch_bounds__(256) void k_adamw(AdamArgs A)
{
    const AdamChunk ch = A.chunks[blockIdx.x];
    const AdamTensor T = A.tensors[ch.tensor];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const G *grad = (const G *)T.grad;
    const float keep = 1.f - A.lr * T.decay;
    for (int k = wave; k < ADAM_CHUNK / ADAM_BLOCK; k += 4) {
        const long first = (long)ch.block * ADAM_CHUNK + (long)k * ADAM_BLOCK + 4 * lane;   // in the tensor
        if (first - 4 * lane >= T.n) break;
        const long place = T.at + first;
        const int count = (int)min(4l, max(0l, T.n - first));
        float p[4], g[4], m[4], v[4], ms = 0.f, vs = 0.f;
        for (int j = 0; j < 4; ++j) {
            p[j] = j < count ? T.param[first + j] : 0.f;
            g[j] = j < count ? (float)grad[first + j] : 0.f;
            m[j] = v[j] = 0.f;
        }
        if constexpr (BITS == 8) {
            ms = A.ms[place / ADAM_BLOCK];
            vs = A.vs[place / ADAM_BLOCK];
            unpack_e4m3(((const uint32_t *)A.m)[place / 4], m);
            unpack_e5m2(((const uint32_t *)A.v)[place / 4], v);
            for (int j = 0; j < 4; ++j) { m[j] = product(m[j], ms); v[j] = product(v[j], vs); }
        } else {
            for (int j = 0; j < count; ++j) { m[j] = ((const float *)A.m)[place + j]; v[j] = ((const float *)A.v)[place + j]; }
        }
        float mt = 0.f, vt = 0.f;
        for (int j = 0; j < 4; ++j) {
            moments(m[j], v[j], g[j], A.b1, A.c1, A.b2, A.c2);
            if (j >= count) m[j] = v[j] = 0.f;
            mt = nan_max(mt, fabsf(m[j]));
            vt = nan_max(vt, v[j]);
            p[j] = p[j] * keep - A.rate * m[j] / (sqrtf(v[j]) * A.root + A.eps);
            if (j < count) {
                T.param[first + j] = p[j];
                if (T.copy) ((bf16 *)T.copy)[first + j] = (bf16)p[j];
            }
        }
        if constexpr (BITS == 8) {
            for (int o = 32; o; o >>= 1) { mt = nan_max(mt, __shfl_xor(mt, o)); vt = nan_max(vt, __shfl_xor(vt, o)); }
            const float mi = mt > 0.f ? product(1.f / mt, E4M3_MAX) : 0.f, vi = vt > 0.f ? product(1.f / vt, E5M2_MAX) : 0.f;
            float mq[4], vq[4];
            for (int j = 0; j < 4; ++j) {
                const uint64_t z = misc::mix64(A.seed, (uint64_t)(place + j) >> 1);
                const uint32_t bits = (uint32_t)(j & 1 ? z >> 32 : z);
                mq[j] = copysignf(fminf(rounded<3, -6>(fabsf(product(m[j], mi)), bits & 0xFFFF), E4M3_MAX), m[j]);
                vq[j] = fminf(rounded<2, -14>(product(v[j], vi), bits >> 16), E5M2_MAX);
                if (v[j] > 0.f) vq[j] = fmaxf(vq[j], 1.f / 65536.f);
            }
            if (count) {
                ((uint32_t *)A.m)[place / 4] = pack_e4m3(mq[0], mq[1], mq[2], mq[3]);
                ((uint32_t *)A.v)[place / 4] = pack_e5m2(vq[0], vq[1], vq[2], vq[3]);
            }
            if (lane == 0) { A.ms[place / ADAM_BLOCK] = mt * (1.f / E4M3_MAX); A.vs[place / ADAM_BLOCK] = vt * (1.f / E5M2_MAX); }
        } else {
            for (int j = 0; j < count; ++j) { ((float *)A.m)[place + j] = m[j]; ((float *)A.v)[place + j] = v[j]; }
        }
    }
}

}  // namespace seq
