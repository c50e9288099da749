// AdamW over many tensors in one launch, moments in 32 or 8 bits.
//
// Bound by memory: 28 bytes per element with 32-bit moments and fp32 gradients, 14.06 with 8-bit moments and bf16 gradients.
// A wave takes blocks of 256 elements, four per lane: the elements that share a scale, so that the largest is found within
// the wave.  A workgroup's share, a chunk, has a record of its own in the plan (addresses, length, decay): a look-up
// of the chunk's tensor and then of the tensor would be two trips to memory before the first element is asked for.
// Measured: 100M parameters in 150 tensors, 8 bits, bf16 gradients 263 us (5.3 TB/s); the Q-network's 1.7M in 32 bits 8.9.
#pragma once
#include "seq_common.h"
#include "sumtree.h"

namespace seq {

constexpr int ADAM_BLOCK = 256;   // elements that share a scale: one wave, four elements per lane
constexpr int ADAM_DEEP = 2;      // blocks of a wave, all of whose loads are in flight together
constexpr int ADAM_CHUNK = 4 * ADAM_DEEP * ADAM_BLOCK;   // elements of a workgroup of four waves

struct AdamChunk {
    float *param;
    const void *grad;
    uint16_t *copy;
    long at;         // place of its first moment in the buffers of moments
    int n;           // elements, up to ADAM_CHUNK
    float decay;
    int wide, pad;   // whether every pointer allows four elements at a time
};
struct AdamArgs {
    const AdamChunk *chunks;
    void *m, *v;
    float *ms, *vs;
    float lr, b1, c1, b2, c2, eps, rate, root;   // c = 1 - b; rate = lr / (1 - b1^t); root = 1 / sqrt(1 - b2^t)
    uint64_t seed;
};

// |x| to MANTISSA bits (below 2^LOWEST: to multiples of the smallest number of the type), up where the 16 random bits are
// the larger and down where they are not, so that x is kept on average.  Numbers that small are rare: a wave
// without any skips their form (zero comes out of both).
template <int MANTISSA, int LOWEST> __device__ __forceinline__ void rounded(float (&x)[4], const uint32_t (&bits)[4])
{
    constexpr int drop = 23 - MANTISSA;
    const float lowest = __int_as_float((127 + LOWEST) << 23), unit = __int_as_float((127 + LOWEST - MANTISSA) << 23);
    float y[4];
    bool small = false;
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        y[j] = __uint_as_float((__float_as_uint(x[j]) + (bits[j] << (drop - 16))) & ~((1u << drop) - 1));
        small |= x[j] < lowest && x[j] != 0.f;
    }
    if (__any(small)) {
#pragma unroll
        for (int j = 0; j < 4; ++j)
            if (x[j] < lowest) y[j] = floorf(x[j] * (1.f / unit) + (float)bits[j] * (1.f / 65536.f)) * unit;
    }
#pragma unroll
    for (int j = 0; j < 4; ++j) x[j] = y[j];
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
__device__ __forceinline__ float larger(float a, float b) { return __builtin_elementwise_maximum(a, b); }   // a NaN if one is a NaN

// sqrt(v) root + eps.  The instruction takes a v below 2^-126 for zero, and a small eps would be all that is left.
__device__ __forceinline__ float root_plus(float v, float root, float eps)
{
    const bool small = v < 0x1p-96f;
    return fmaf(__builtin_amdgcn_sqrtf(small ? v * 0x1p64f : v), small ? root * 0x1p-32f : root, eps);
}

// An address that comes from memory could be one in LDS for all that the compiler knows; these are not.
template <class T> using Global = __attribute__((address_space(1))) T;
template <class T> __device__ __forceinline__ Global<T> *global(T *p) { return (Global<T> *)(uintptr_t)p; }

// What a lane holds of a block: four elements and their moments.
template <class G, int BITS> struct AdamLane {
    using Word = std::conditional_t<BITS == 8, uint32_t, vec<float, 4>>;
    vec<float, 4> p;
    vec<G, 4> g;
    Word m, v;
    float ms, vs;
    int first, count;   // place in the chunk, elements of the lane
    bool whole;         // of the wave's whole block: four elements at a time

    __device__ __forceinline__ void fetch(const AdamArgs &A, const AdamChunk &ch, int block)
    {
        const int base = block * ADAM_BLOCK;
        first = base + 4 * (threadIdx.x & 63);
        count = min(4, max(0, ch.n - first));
        whole = ch.wide && ch.n >= base + ADAM_BLOCK;
        if (whole) {
            p = *reinterpret_cast<const Global<vec<float, 4>> *>(global(ch.param) + first);
            g = *reinterpret_cast<const Global<vec<G, 4>> *>(global((const G *)ch.grad) + first);
        } else {
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                p[j] = j < count ? global(ch.param)[first + j] : 0.f;
                g[j] = j < count ? global((const G *)ch.grad)[first + j] : (G)0.f;
            }
        }
        const long place = ch.at + first;     // the buffers of moments go on to the end of the block
        m = reinterpret_cast<const Word *>(A.m)[place / 4];
        v = reinterpret_cast<const Word *>(A.v)[place / 4];
        if constexpr (BITS == 8) {
            ms = A.ms[place / ADAM_BLOCK];
            vs = A.vs[place / ADAM_BLOCK];
        }
    }

    __device__ __forceinline__ void step(const AdamArgs &A, const AdamChunk &ch, float decay, int lane)
    {
        float mn[4], vn[4];
        if constexpr (BITS == 8) {
            unpack_e4m3(m, mn);
            unpack_e5m2(v, vn);
#pragma unroll
            for (int j = 0; j < 4; ++j) { mn[j] = product(mn[j], ms); vn[j] = product(vn[j], vs); }
        } else {
#pragma unroll
            for (int j = 0; j < 4; ++j) { mn[j] = m[j]; vn[j] = v[j]; }
        }
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            moments(mn[j], vn[j], (float)g[j], A.b1, A.c1, A.b2, A.c2);
            // the whole change first: 1 - lr decay as one number would keep few digits of a small decay, or none
            p[j] -= fmaf(decay, p[j], A.rate * mn[j] * __builtin_amdgcn_rcpf(root_plus(vn[j], A.root, A.eps)));
        }
        if (whole) {
            *reinterpret_cast<Global<vec<float, 4>> *>(global(ch.param) + first) = p;
            if (ch.copy) *reinterpret_cast<Global<vec<bf16, 4>> *>(global((bf16 *)ch.copy) + first) = __builtin_convertvector(p, vec<bf16, 4>);
        } else {
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                if (j < count) {
                    global(ch.param)[first + j] = p[j];
                    if (ch.copy) global((bf16 *)ch.copy)[first + j] = (bf16)p[j];
                } else {
                    mn[j] = vn[j] = 0.f;
                }
            }
        }
        const long place = ch.at + first;
        if constexpr (BITS == 8) {
            float mt = 0.f, vt = 0.f;
#pragma unroll
            for (int j = 0; j < 4; ++j) { mt = larger(mt, fabsf(mn[j])); vt = larger(vt, vn[j]); }
            mt = group_fold(mt, 64, larger);
            vt = group_fold(vt, 64, larger);
            if (mt > 0.f) mt = fmaxf(mt, E4M3_LEAST);
            if (vt > 0.f) vt = fmaxf(vt, E5M2_LEAST);
            const float mi = mt > 0.f ? product(1.f / mt, E4M3_MAX) : 0.f, vi = vt > 0.f ? product(1.f / vt, E5M2_MAX) : 0.f;
            const uint64_t z0 = misc::mix64(A.seed, (uint64_t)place / 2), z1 = misc::mix64(A.seed, (uint64_t)place / 2 + 1);
            uint32_t mb[4], vb[4];
            float mq[4], vq[4];
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const uint64_t z = j < 2 ? z0 : z1;
                const uint32_t bits = (uint32_t)(j & 1 ? z >> 32 : z);
                mb[j] = bits & 0xFFFF;
                vb[j] = bits >> 16;
                mq[j] = fabsf(product(mn[j], mi));
                vq[j] = product(vn[j], vi);
            }
            rounded<3, -6>(mq, mb);
            rounded<2, -14>(vq, vb);
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                mq[j] = copysignf(fminf(mq[j], E4M3_MAX), mn[j]);
                vq[j] = fminf(vn[j] > 0.f ? fmaxf(vq[j], 1.f / 65536.f) : vq[j], E5M2_MAX);   // one that is not zero does not become zero
            }
            if (count) {
                reinterpret_cast<uint32_t *>(A.m)[place / 4] = pack_e4m3(mq[0], mq[1], mq[2], mq[3]);
                reinterpret_cast<uint32_t *>(A.v)[place / 4] = pack_e5m2(vq[0], vq[1], vq[2], vq[3]);
            }
            if (lane == 0) {
                A.ms[place / ADAM_BLOCK] = mt * (1.f / E4M3_MAX);
                A.vs[place / ADAM_BLOCK] = vt * (1.f / E5M2_MAX);
            }
        } else if (count) {
            reinterpret_cast<vec<float, 4> *>(A.m)[place / 4] = vec<float, 4>{mn[0], mn[1], mn[2], mn[3]};
            reinterpret_cast<vec<float, 4> *>(A.v)[place / 4] = vec<float, 4>{vn[0], vn[1], vn[2], vn[3]};
        }
    }
};

template <class G, int BITS> __global__ __launch_bounds__(256) void k_adamw(AdamArgs A)
{
    const AdamChunk ch = A.chunks[blockIdx.x];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const float decay = A.lr * ch.decay;
    const int first = wave * ADAM_DEEP, blocks = min(ADAM_DEEP, (ch.n + ADAM_BLOCK - 1) / ADAM_BLOCK - first);
    AdamLane<G, BITS> b[ADAM_DEEP];
    if (blocks == ADAM_DEEP) {
#pragma unroll
        for (int k = 0; k < ADAM_DEEP; ++k) b[k].fetch(A, ch, first + k);
#pragma unroll
        for (int k = 0; k < ADAM_DEEP; ++k) b[k].step(A, ch, decay, lane);
    } else {
        for (int k = 0; k < blocks; ++k) {
            b[0].fetch(A, ch, first + k);
            b[0].step(A, ch, decay, lane);
        }
    }
}

}  // namespace seq
