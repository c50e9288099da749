// What the kernels of the recurrent network's operators share: elements in fp32 or bf16, 8-bit
// numbers, and the host side's errors.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

#include <type_traits>

namespace seq {

using bf16 = __bf16;
template <class T, int N> using vec = T __attribute__((ext_vector_type(N)));

constexpr float E4M3_MAX = 448.f, E5M2_MAX = 57344.f;
// The least value that the largest of the numbers that share a scale counts as, unless all are zero.  Below it the scale would
// lose its digits (it is 2^-125.8 there) and its inverse would be infinite, times zero a NaN.
constexpr float E4M3_LEAST = 0x1p-117f, E5M2_LEAST = 0x1p-110f;

// bytes a and b of a word as e4m3 / e5m2 numbers, and back.  The conversions to 8 bits are exact where the value is a
// number of the type, else to the nearest, ties to even; nothing above the largest number is passed to them.
__device__ __forceinline__ uint32_t pack_e4m3(float a, float b, float c, float d)
{
    int w = __builtin_amdgcn_cvt_pk_fp8_f32(a, b, 0, false);
    return (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(c, d, w, true);
}
__device__ __forceinline__ uint32_t pack_e5m2(float a, float b, float c, float d)
{
    int w = __builtin_amdgcn_cvt_pk_bf8_f32(a, b, 0, false);
    return (uint32_t)__builtin_amdgcn_cvt_pk_bf8_f32(c, d, w, true);
}
__device__ __forceinline__ void unpack_e4m3(uint32_t w, float (&o)[4])
{
    const auto lo = __builtin_amdgcn_cvt_pk_f32_fp8((int)w, false), hi = __builtin_amdgcn_cvt_pk_f32_fp8((int)w, true);
    o[0] = lo[0]; o[1] = lo[1]; o[2] = hi[0]; o[3] = hi[1];
}
__device__ __forceinline__ void unpack_e5m2(uint32_t w, float (&o)[4])
{
    const auto lo = __builtin_amdgcn_cvt_pk_f32_bf8((int)w, false), hi = __builtin_amdgcn_cvt_pk_f32_bf8((int)w, true);
    o[0] = lo[0]; o[1] = lo[1]; o[2] = hi[0]; o[3] = hi[1];
}

// Barrier that orders LDS traffic only: global loads and stores stay in flight across it.
__device__ __forceinline__ void lds_barrier() { asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory"); }

// Loaded values that have to be here before what follows, a barrier say: it need not wait for loads.
__device__ __forceinline__ void arrived(float v) { asm volatile("" ::"v"(v) : "memory"); }
template <int V> __device__ __forceinline__ void arrived(const float (&v)[V])
{
#pragma unroll
    for (int k = 0; k < V; ++k) arrived(v[k]);
}

// the larger one, or a NaN if one is a NaN
__device__ __forceinline__ float nan_max(float a, float b) { return a != a ? a : (b > a || b != b) ? b : a; }

__device__ __forceinline__ float add(float a, float b) { return a + b; }

// V elements from or to an address that allows V at once
template <int V, class T> __device__ __forceinline__ vec<T, V> load(const T *p)
{
    if constexpr (V == 1) return vec<T, 1>{*p};
    else return *reinterpret_cast<const vec<T, V> *>(p);
}
template <int V, class T> __device__ __forceinline__ void store(T *p, vec<T, V> v)
{
    if constexpr (V == 1) *p = v[0];
    else *reinterpret_cast<vec<T, V> *>(p) = v;
}
template <class E, int V> __device__ __forceinline__ vec<E, V> narrow(const float (&v)[V])
{
    vec<E, V> o;
#pragma unroll
    for (int k = 0; k < V; ++k) o[k] = (E)v[k];
    return o;
}

// x of the lower and of the upper half of the wave, in both
__device__ __forceinline__ void halves(float x, float &lo, float &hi)
{
    const auto r = __builtin_amdgcn_permlane32_swap(__float_as_int(x), __float_as_int(x), false, false);
    lo = __int_as_float((int)r[0]);
    hi = __int_as_float((int)r[1]);
}

// f over the values of a group of `lanes` (a power of two) neighbouring lanes, in all of them, f commutative.  By operand
// permutations and swaps: each is a few cycles, an exchange through LDS about a hundred.
template <int CTRL> __device__ __forceinline__ float permuted(float v)
{
    return __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(v), CTRL, 0xF, 0xF, true));
}
template <class F> __device__ __forceinline__ float group_fold(float v, int lanes, F f)
{
    if (lanes > 1) v = f(v, permuted<0xB1>(v));     // lane ^ 1
    if (lanes > 2) v = f(v, permuted<0x4E>(v));     // lane ^ 2
    if (lanes > 4) v = f(v, permuted<0x141>(v));    // 7 - lane of eight: the other four hold one value
    if (lanes > 8) v = f(v, permuted<0x140>(v));    // 15 - lane of sixteen
    if (lanes > 16) {
        const auto r = __builtin_amdgcn_permlane16_swap(__float_as_int(v), __float_as_int(v), false, false);
        v = f(__int_as_float((int)r[0]), __int_as_float((int)r[1]));
    }
    if (lanes > 32) {
        float lo, hi;
        halves(v, lo, hi);
        v = f(lo, hi);
    }
    return v;
}

}  // namespace seq

// Sets what dqn_last_error(NULL) says on this thread and returns `code`.
int32_t dqn_seq_fail(int32_t code, const char *call, const char *why);
