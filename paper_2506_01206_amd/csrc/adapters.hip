// The way into low-rank adapters of many requests (mamba_linear_adapted_fwd): t[m, r] = scale[a] sum_k x[m, k] A[a, r, k], a = idx[m] the
// adapter of row m.  The way out, t B^T, is part of the shared product's own kernel (linear.hip; for one row both are).
//
// t leaves as two bfloat16 terms, high and low, side by side: the product with B has its 16 bits then, more than the output keeps.
#include "device_math.h"
#include "launch.h"

namespace mamba {
namespace {

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef float f32x4v __attribute__((ext_vector_type(4)));
typedef unsigned int u32x4 __attribute__((ext_vector_type(4)));

constexpr int64_t kEnough = 256;                                      // workgroups, one to a compute unit
constexpr int kLine = 128;                                           // 64 k of a row in LDS

// 16 bytes a lane from an address of its own into LDS at lds_addr + 16 lane (see linear.hip: the waits for them are explicit)
__device__ __forceinline__ void load_to_lds16(const void *from, uint32_t lds_addr)
{
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, off" ::"s"(lds_addr), "v"(from) : "memory");
}
__device__ __forceinline__ void lds_barrier()
{
    __builtin_amdgcn_fence(__ATOMIC_RELEASE, "workgroup", "local");
    __builtin_amdgcn_s_barrier();
    __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "workgroup", "local");
}

// A workgroup has 16 G rows and RT tiles of 16 ranks of one adapter: of those that its rows have, in the rows' order, every gridDim.y-th from the
// blockIdx.y-th on, so that rows of many adapters are not multiplied by one after the other.  A row's sums are written by who has its adapter.
// Of the W wavefronts G go by rows, W / G by k: slabs of as many k as give each of those 32, four of them in LDS, straight from memory, a
// row's 16-byte slot c at c ^ (row / 2 & 7).
// Bound by x from memory where there are many rows, by trips to memory where there are few.  us: 24 rows, K = 768, 8 adapters of rank 16 4.3; 333 rows, K = 768, rank 16
// 4.3; 4097 rows, K = 1024, 16 adapters of rank 64 in runs 9.2; 16384 rows, K = 2048, 32 of rank 32 32 (2.1 TB/s; 64 rows to a workgroup 37, slabs of
// twice the k 34, workgroups that begin at different k, for the sake of the memory's channels, the same).
template <int RT, int G, int W>
__global__ void __launch_bounds__(64 * W)
down_kernel(const bf16_t *__restrict__ x, const bf16_t *__restrict__ a, const float *__restrict__ scale, const int32_t *__restrict__ idx,
            bf16_t *__restrict__ t, uint32_t *__restrict__ zeros, int64_t M, int K, int rank, int adapters)
{
    constexpr int kWaves = W, kThreads = 64 * W, kStages = 4;
    constexpr int BM = 16 * G, BN = 16 * RT, S = W / G, kBlocks = S > 2 ? S / 2 : 1, kStep = 64 * kBlocks;   // blocks of 64 k to a slab
    constexpr int kStage = (BM + BN) * kLine * kBlocks;
    constexpr int kGroups = (BM + BN) / 8 * kBlocks, NL = (kGroups + kWaves - 1) / kWaves;   // loads of 8 rows, and of a wavefront
    constexpr int kPart = S * BM * BN * 4;
    __shared__ __attribute__((aligned(1024))) unsigned char lds[kStages * kStage > kPart ? kStages * kStage : kPart];
    const int tid = threadIdx.x, lane = tid & 63, li = lane & 15, lg = lane >> 4;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6), group = wave % G, split = wave / G;
    const int64_t m0 = (int64_t)blockIdx.x * BM;
    const int rank0 = (int)blockIdx.z * BN, ranks = min(rank - rank0, BN);
    if (blockIdx.x == 0 && blockIdx.y == 0 && blockIdx.z == 0 && tid < 32) zeros[tid] = 0;
    const int32_t id = lane < BM && m0 + lane < M ? idx[m0 + lane] : -1;
    const uint32_t lds0 = (uint32_t)(size_t)(__attribute__((address_space(3))) unsigned char *)lds;
    const int slabs = (K + kStep - 1) / kStep, chunks = K / 8;
    int turn = 0;
    for (uint64_t left = __ballot(id >= 0 && id < adapters); left; ++turn) {
        const int32_t cur = __builtin_amdgcn_readlane(id, __builtin_ctzll(left));
        left &= ~__ballot(id == cur);
        if (turn % (int)gridDim.y != (int)blockIdx.y) continue;
        // what this lane brings: of load i rows 8 g .. 8 g + 7 of a block, x's first
        const bf16_t *row[NL];
        int chunk[NL];
        uint32_t to[NL];
#pragma unroll
        for (int i = 0; i < NL; ++i) {
            const int g = min(i * kWaves + wave, kGroups - 1), block = g / ((BM + BN) / 8), r = g % ((BM + BN) / 8) * 8 + (lane >> 3);
            row[i] = r < BM ? x + min(m0 + r, M - 1) * K : a + ((int64_t)cur * rank + rank0 + min(r - BM, ranks - 1)) * K;
            chunk[i] = 8 * block + ((lane & 7) ^ (r >> 1 & 7));
            to[i] = (uint32_t)g * 1024;
        }
        auto request = [&](int slab, int stage) __attribute__((always_inline)) {
#pragma unroll
            for (int i = 0; i < NL; ++i) {
                const int c = slab * (kStep / 8) + chunk[i];
                load_to_lds16(row[i] + (c < chunks ? c : 0) * 8, lds0 + stage * kStage + to[i]);   // (behind K: something, see below)
            }
        };
        // until no more than the loads of `slabs_under_way` slabs are under way (vmcnt is split over bits 3:0 and 15:14), and no LDS read (lgkmcnt(0)):
        // behind the barrier other wavefronts' loads overwrite a stage, and keep no order with one
        auto wait_for = [&](int slabs_under_way) __attribute__((always_inline)) {
            static_assert((kStages - 2) * NL < 64 && kStages == 4, "fits the counter");
            if (slabs_under_way >= 2) __builtin_amdgcn_s_waitcnt(0x0070 | ((2 * NL) & 15) | (((2 * NL) >> 4) << 14));
            else if (slabs_under_way >= 1) __builtin_amdgcn_s_waitcnt(0x0070 | (NL & 15) | ((NL >> 4) << 14));
            else __builtin_amdgcn_s_waitcnt(0x0070);
        };
        f32x4v d[RT];
#pragma unroll
        for (int r = 0; r < RT; ++r) d[r] = f32x4v(0.0f);
        __builtin_amdgcn_s_waitcnt(0xC07F);                          // lgkmcnt(0): the last adapter's sums are read
        lds_barrier();
#pragma unroll
        for (int i = 0; i < kStages - 1; ++i)
            if (i < slabs) request(i, i);
        int stage = 0;
#pragma unroll 1
        for (int s = 0; s < slabs; ++s) {
            wait_for(min(slabs - 1 - s, kStages - 2));
            lds_barrier();                                           // slab s is there, slab s - 1 is read
            if (s + kStages - 1 < slabs) request(s + kStages - 1, (stage + kStages - 1) % kStages);
            const unsigned char *from = lds + stage * kStage;
#pragma unroll
            for (int h = 0; h < 2 * kBlocks / S; ++h) {              // steps of 32 k
                const int block = (split + S * h) >> 1, c = 4 * ((split + S * h) & 1) + lg;
                const bool in = s * (kStep / 8) + 8 * block + c < chunks;
                auto fragment = [&](int r) __attribute__((always_inline)) {
                    const u32x4 v = *reinterpret_cast<const u32x4 *>(from + (block * (BM + BN) + r) * kLine + ((c ^ (r >> 1 & 7)) << 4));
                    return __builtin_bit_cast(bf16x8, in ? v : u32x4(0u));
                };
                const bf16x8 xf = fragment(16 * group + li);
#pragma unroll
                for (int r = 0; r < RT; ++r) d[r] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(xf, fragment(BM + 16 * r + li), d[r], 0, 0, 0);
            }
            stage = stage + 1 == kStages ? 0 : stage + 1;
        }
        lds_barrier();
        // d[r][i] is t[4 (lane / 16) + i][16 r + lane % 16] of the group's rows
        float *part = reinterpret_cast<float *>(lds) + split * (BM * BN);
#pragma unroll
        for (int r = 0; r < RT; ++r)
#pragma unroll
            for (int i = 0; i < 4; ++i) part[(16 * group + 4 * lg + i) * BN + 16 * r + li] = d[r][i];
        lds_barrier();
        const float by = scale ? scale[cur] : 1.0f;
        for (int e = tid; e < BM * BN / 2; e += kThreads) {          // two ranks of a row
            const int mr = e / (BN / 2), r = 2 * (e % (BN / 2));
            const int64_t m = m0 + mr;
            if (m >= M || r >= ranks || idx[m] != cur) continue;
            float v[2] = {0.0f, 0.0f};
#pragma unroll
            for (int q = 0; q < S; ++q) {
                const float2 p = *reinterpret_cast<const float2 *>(reinterpret_cast<const float *>(lds) + q * (BM * BN) + mr * BN + r);
                v[0] += p.x, v[1] += p.y;
            }
            float low[2];
            uint32_t high[2];
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                v[i] *= by;
                high[i] = f32_to_bf16(v[i]);
                const float rest = v[i] - bf16_to_f32(high[i]);
                low[i] = rest == rest ? rest : 0.0f;                 // (an infinity has no low term)
            }
            *reinterpret_cast<uint32_t *>(t + m * (2 * rank) + rank0 + r) = high[0] | high[1] << 16;
            *reinterpret_cast<uint32_t *>(t + m * (2 * rank) + rank + rank0 + r) = f32x2_to_bf16x2(low[0], low[1]);
        }
    }
}

// Adapters of a workgroup's rows at once: up to 16 while workgroups are fewer than a quarter of the CUs, and rows of many adapters would be one product
// after the other; up to 4 beyond, where a workgroup without a turn is one more to be run through.  us, up to 4 | 16, K = 1024, 64 adapters:
//   rows                 64          333         512         1024        2048        4097        16384
//   rank 16, no order    9.3| 4.7    10.6| 5.7   10.6| 5.8   10.8| 7.7   13.4|12.6   25.2|28.9   101|98
//   rank 16, runs        9.4| 4.7     4.2| 4.2    4.1| 4.1    4.1| 4.0    4.0| 4.0    5.3| 7.4   10.0|12.7
//   rank 64, no order    9.4| 4.8    14.2|10.8   14.4|13.3   19.1|22.9   33.2|32.2   62.6|70.0   267|251
//   rank 64, runs        9.5| 5.0     5.1| 6.0    5.0| 6.0    6.1| 7.2    6.3| 8.3   12.7|19.4   17.9|24.1
template <int RT, int G, int W> hipError_t launch(const bf16_t *x, const AdapterArgs &l, int64_t M, int64_t K, hipStream_t stream)
{
    const int64_t tiles = (M + 16 * G - 1) / (16 * G), parts = (l.rank + 16 * RT - 1) / (16 * RT);
    const int64_t turns = tiles * parts >= kEnough / 4 ? 4 : 16;     // adapters of a workgroup's rows at once
    const dim3 grid((unsigned)tiles, (unsigned)(l.adapters < turns ? l.adapters : turns), (unsigned)parts);
    down_kernel<RT, G, W><<<grid, 64 * W, 0, stream>>>(x, static_cast<const bf16_t *>(l.a), l.scale, l.idx, static_cast<bf16_t *>(l.t),
                                                       static_cast<uint32_t *>(l.zeros), M, (int)K, (int)l.rank, (int)l.adapters);
    return hipGetLastError();
}

}  // namespace

// Ranks are split over workgroups, 16 of them or more to one, while there are not enough of those: x is read again from the second-level cache then.
// Up to 64 rows eight wavefronts share k, four beyond.  us, eight | four: K = 2048, rank 16 1 row 4.5|5.3, 64 4.7|5.6, 256 4.8|5.6; eight adapters of rank
// 64 24 rows 5.1|5.7, 128 5.4|5.9, 256 7.5|7.5; K = 768 the same to 0.1, but 256 rows of those 5.4|4.7.
// From 6144 rows a workgroup has 32 of them, 16 below, so that A comes half as often.  us, 16 | 32 rows, K = 2048, runs of 8 to 32 adapters (no order):
//   rows       4097                    6144                  8192                   16384
//   rank 16     7.8| 9.5 (44|69)        8.6| 9.4 (47|65)      9.8| 9.7 (65|91)      17.8|13.7 (157|207)
//   rank 64    15.4|15.3 (67|69)       14.5|15.3 (90|73)     17.6|15.4 (124|124)    29.5|19.5 (227|232)
//   rank 128   30.2|21.0               28.1|21.0             36.6|20.9              71.6|27.6
hipError_t launch_adapters_down(const void *x, const AdapterArgs &l, int64_t M, int64_t K, hipStream_t stream)
{
    const bf16_t *xp = static_cast<const bf16_t *>(x);
    if (M <= 64) return launch<1, 1, 8>(xp, l, M, K, stream);
    if (M >= 6144) {
        if (l.rank <= 16) return launch<1, 2, 4>(xp, l, M, K, stream);
        if (l.rank <= 32) return launch<2, 2, 4>(xp, l, M, K, stream);
        if (l.rank <= 64) return launch<4, 2, 4>(xp, l, M, K, stream);
        return launch<8, 2, 4>(xp, l, M, K, stream);
    }
    const int64_t tiles = (M + 15) / 16, parts = (kEnough + tiles - 1) / tiles;   // (of the ranks)
    if (l.rank <= 16 * parts) return launch<1, 1, 4>(xp, l, M, K, stream);
    if (l.rank <= 32 * parts) return launch<2, 1, 4>(xp, l, M, K, stream);
    if (l.rank <= 64 * parts) return launch<4, 1, 4>(xp, l, M, K, stream);
    return launch<8, 1, 4>(xp, l, M, K, stream);
}

}  // namespace mamba
