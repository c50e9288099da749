// What the kernels of the recurrent network's operators share: elements in fp32 or bf16, 8-bit
// numbers, and the host side's errors.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

namespace seq {

using bf16 = __bf16;
template <class T, int N> using vec = T __attribute__((ext_vector_type(N)));

constexpr float E4M3_MAX = 448.f, E5M2_MAX = 57344.f;

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

// the larger one, or a NaN if one is a NaN
__device__ __forceinline__ float nan_max(float a, float b) { return a != a ? a : (b > a || b != b) ? b : a; }

}  // namespace seq

// Sets what dqn_last_error(NULL) says on this thread and returns `code`.
int32_t dqn_seq_fail(int32_t code, const char *call, const char *why);
