// Rows of a vocabulary as the kernels over logits read and write them: eight tokens of a lane at a time, rows that start anywhere, a grid of
// slices by rows; a workgroup's barrier and a wavefront's lanes by DPP.
#pragma once
#include "device_math.h"

namespace mamba {
namespace {

typedef float f32x4_any __attribute__((ext_vector_type(4), aligned(4)));      // rows of V elements start anywhere
typedef int32_t i32x4_any __attribute__((ext_vector_type(4), aligned(4)));
typedef uint32_t u32x4_any __attribute__((ext_vector_type(4), aligned(2)));

__device__ __forceinline__ void load8(const float *p, float *x)
{
    const f32x4_any a = *reinterpret_cast<const f32x4_any *>(p), b = *reinterpret_cast<const f32x4_any *>(p + 4);
#pragma unroll
    for (int i = 0; i < 4; ++i) x[i] = a[i], x[4 + i] = b[i];
}
__device__ __forceinline__ void load8(const bf16_t *p, float *x)
{
    const u32x4_any a = *reinterpret_cast<const u32x4_any *>(p);
#pragma unroll
    for (int i = 0; i < 4; ++i) x[2 * i] = bf16_lo(a[i]), x[2 * i + 1] = bf16_hi(a[i]);
}
__device__ __forceinline__ void load8(const int32_t *p, int32_t *x)
{
    const i32x4_any a = *reinterpret_cast<const i32x4_any *>(p), b = *reinterpret_cast<const i32x4_any *>(p + 4);
#pragma unroll
    for (int i = 0; i < 4; ++i) x[i] = a[i], x[4 + i] = b[i];
}
__device__ __forceinline__ void store8(float *p, const float *x)
{
    f32x4_any a, b;
#pragma unroll
    for (int i = 0; i < 4; ++i) a[i] = x[i], b[i] = x[4 + i];
    *reinterpret_cast<f32x4_any *>(p) = a;
    *reinterpret_cast<f32x4_any *>(p + 4) = b;
}
__device__ __forceinline__ void store8(bf16_t *p, const float *x)
{
    u32x4_any a;
#pragma unroll
    for (int i = 0; i < 4; ++i) a[i] = f32x2_to_bf16x2(x[2 * i], x[2 * i + 1]);
    *reinterpret_cast<u32x4_any *>(p) = a;
}

// What the workgroup wrote to LDS is there for all of it.  (Its stores to memory and loads from there stay under way: nothing but LDS goes from thread to
// thread in these kernels, and a barrier that waits for stores costs a microsecond each time.)
__device__ __forceinline__ void lds_barrier()
{
    __builtin_amdgcn_fence(__ATOMIC_RELEASE, "workgroup", "local");
    __builtin_amdgcn_s_barrier();
    __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "workgroup", "local");
}

// lanes of a wavefront by DPP: what comes from `CTRL`'s lane, where ROWS has the row, else what `other` says
template <int CTRL, int ROWS = 0xf> __device__ __forceinline__ uint32_t from_lane(uint32_t other, uint32_t v)
{
    return (uint32_t)__builtin_amdgcn_update_dpp((int)other, (int)v, CTRL, ROWS, 0xf, false);
}
// A grid of slices by rows has the rows in two of its dimensions: no number of a workgroup is divided.
constexpr int64_t kRowsY = 65535;
__device__ __forceinline__ int64_t row_of_block() { return (int64_t)blockIdx.z * kRowsY + blockIdx.y; }

}  // namespace
}  // namespace mamba
