// The way into low-rank adapters of many requests (mamba_linear_adapted_fwd): t[m, r] = scale[a] sum_k x[m, k] A[a, r, k], a = idx[m] the
// adapter of row m.  The way out, t B^T, is part of the shared product's own kernel (linear.hip).
//
// t leaves as two bfloat16 terms, high and low, side by side: the product with B has its 16 bits then, more than the output keeps.
#include "device_math.h"
#include "launch.h"

namespace mamba {
namespace {

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef float f32x4v __attribute__((ext_vector_type(4)));
typedef unsigned int u32x4 __attribute__((ext_vector_type(4)));

__device__ __forceinline__ int32_t wave_min(int32_t v)
{
#pragma unroll
    for (int d = 32; d; d >>= 1) v = min(v, __shfl_xor(v, d));
    return v;
}

// One workgroup per 16 rows and all ranks (RT tiles of 16), its NW wavefronts share the k range in steps of 32, every NW-th each.  Rows of several
// adapters are multiplied by each of them, and a row takes the sums of its own.
template <int RT, int NW>
__global__ void __launch_bounds__(64 * NW)
down_kernel(const bf16_t *__restrict__ x, const bf16_t *__restrict__ a, const float *__restrict__ scale, const int32_t *__restrict__ idx,
            bf16_t *__restrict__ t, int64_t M, int K, int rank, int adapters)
{
    __shared__ float part[NW][RT * 256];
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, li = lane & 15, lg = lane >> 4;
    const int64_t m0 = (int64_t)blockIdx.x * 16;
    const int32_t id = lane < 16 && m0 + lane < M ? idx[m0 + lane] : -1;
    const bf16_t *row = x + min(m0 + li, M - 1) * K;
    f32x4v sum[RT];
#pragma unroll
    for (int r = 0; r < RT; ++r) sum[r] = f32x4v(0.0f);
    auto next = [&](int32_t last) { return wave_min(id > last && id < adapters ? id : adapters); };
    bool any = false;
    for (int32_t cur = next(-1); cur < adapters; cur = next(cur)) {
        any = true;
        const uint64_t rows = __ballot(id == cur);
        const bf16_t *w = a + (int64_t)cur * rank * K;
        f32x4v d[RT];
#pragma unroll
        for (int r = 0; r < RT; ++r) d[r] = f32x4v(0.0f);
        for (int k = wave * 32 + lg * 8; k < (K + 31) / 32 * 32; k += NW * 32) {
            const bool in = k < K;                                   // (K is a multiple of 8)
            const u32x4 raw = *reinterpret_cast<const u32x4 *>(row + (in ? k : 0));
            const bf16x8 xf = __builtin_bit_cast(bf16x8, in ? raw : u32x4(0u));
#pragma unroll
            for (int r = 0; r < RT; ++r) {
                const u32x4 wr = *reinterpret_cast<const u32x4 *>(w + (int64_t)min(16 * r + li, rank - 1) * K + (in ? k : 0));
                d[r] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(xf, __builtin_bit_cast(bf16x8, in ? wr : u32x4(0u)), d[r], 0, 0, 0);
            }
        }
#pragma unroll
        for (int r = 0; r < RT; ++r)
#pragma unroll
            for (int i = 0; i < 4; ++i) sum[r][i] = rows >> (4 * lg + i) & 1 ? d[r][i] : sum[r][i];
    }
    if (!any) return;                                                // (the same in all wavefronts)
    // sum[r][i] is t[4 (lane / 16) + i][16 r + lane % 16]
#pragma unroll
    for (int r = 0; r < RT; ++r)
#pragma unroll
        for (int i = 0; i < 4; ++i) part[wave][(r * 4 + i) * 64 + lane] = sum[r][i];
    __syncthreads();
    for (int e = tid; e < RT * 256; e += 64 * NW) {
        float v = 0.0f;
#pragma unroll
        for (int q = 0; q < NW; ++q) v += part[q][e];
        const int l = e & 63, r = (e >> 8) * 16 + (l & 15), mr = 4 * (l >> 4) + (e >> 6 & 3);
        const int64_t m = m0 + mr;
        const int32_t of = m < M ? idx[m] : -1;
        if (of < 0 || of >= adapters || r >= rank) continue;
        if (scale) v *= scale[of];
        const uint32_t high = f32_to_bf16(v);
        const float low = v - bf16_to_f32(high);
        t[m * (2 * rank) + r] = (bf16_t)high;
        t[m * (2 * rank) + rank + r] = (bf16_t)f32_to_bf16(low == low ? low : 0.0f);   // (an infinity has no low term)
    }
}

}  // namespace

hipError_t launch_adapters_down(const void *x, const AdapterArgs &l, int64_t M, int64_t K, hipStream_t stream)
{
    const bf16_t *xp = static_cast<const bf16_t *>(x), *a = static_cast<const bf16_t *>(l.a);
    const unsigned grid = (unsigned)((M + 15) / 16);
#define MAMBA_DOWN(RT) \
    down_kernel<RT, 8><<<grid, 512, 0, stream>>>(xp, a, l.scale, l.idx, static_cast<bf16_t *>(l.t), M, (int)K, (int)l.rank, (int)l.adapters)
    if (l.rank <= 16) MAMBA_DOWN(1);
    else if (l.rank <= 32) MAMBA_DOWN(2);
    else if (l.rank <= 64) MAMBA_DOWN(4);
    else MAMBA_DOWN(8);
#undef MAMBA_DOWN
    return hipGetLastError();
}

}  // namespace mamba
