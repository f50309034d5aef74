// Gated-delta layer core for gfx950: the scalar-decay layer (ssd.hip) with the delta rule's write, a state of the same shape
// (Yang, Kautz & Hatamizadeh, "Gated Delta Networks: Improving Mamba2 with Delta Rule", 2024).  Per value head, P x N state S:
//
//   a = exp(softplus(dt + dt_bias) A), b = sigmoid(beta), k and q divided by their lengths
//   S <- a S (I - b k k^T) + b v k^T   =   a S + u k^T,  u = b (v - a S k)
//   o  = scale S q                     =   scale (a S_before q + u (k . q));   out = rmsnorm(o) norm_w silu(z)
#include "device_math.h"
#include "launch.h"
#include "routes.h"

namespace mamba {
namespace {

constexpr int kThreads = 256;

// what a token does to a head besides q, k and v
struct DeltaOptions {
    float scale, eps;
    int softplus, sigmoid, qk_norm;
};

template <int CTRL> __device__ __forceinline__ float lane_add(float v)
{
    return v + __builtin_bit_cast(float, __builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, v), CTRL, 0xf, 0xf, false));
}
// sum over 16 lanes, in all of them: quad_perm [1,0,3,2], [2,3,0,1], row_half_mirror, row_mirror
__device__ __forceinline__ float sum16(float v) { return lane_add<0x140>(lane_add<0x141>(lane_add<0x4e>(lane_add<0xb1>(v)))); }

__device__ __forceinline__ void load4(const float *p, float *v)
{
    const float4 f = *reinterpret_cast<const float4 *>(p);
    v[0] = f.x, v[1] = f.y, v[2] = f.z, v[3] = f.w;
}
__device__ __forceinline__ void load4(const bf16_t *p, float *v)
{
    const uint2 f = *reinterpret_cast<const uint2 *>(p);
    v[0] = bf16_lo(f.x), v[1] = bf16_hi(f.x), v[2] = bf16_lo(f.y), v[3] = bf16_hi(f.y);
}

__device__ __forceinline__ float sigmoid_f32(float v) { return rcp_hw(1.0f + exp2_hw(-v * kLog2e)); }

// ---------------------------------------------------------------------------------------------------
// Token after token as the equations stand: one workgroup has a head of one row, its state in registers (16 lanes to a row of S,
// P / 16 rows to a thread).  For single tokens this is all there is to do: a state is read and written once, both dot products
// of a row with it come out of one reduction, and the head's P outputs are together for the norm.
// (The states come first and are an aggregate: arguments fetched by the kernel, as in the other steps, see build.py.)
// grid: (H, rows)
template <typename T, int N, int P>
__global__ void __launch_bounds__(kThreads)
delta_recurrent_kernel(StepStates h, const int32_t *__restrict__ parent, const T *__restrict__ q, const T *__restrict__ k,
                       const T *__restrict__ v, const T *__restrict__ dt, const T *__restrict__ beta, const T *__restrict__ z,
                       const float *__restrict__ A, const float *__restrict__ norm_w, const float *__restrict__ dt_bias, T *__restrict__ out,
                       int64_t n_in, int64_t L, int64_t H, int64_t group, DeltaOptions o)
{
    constexpr int F = N / 16, R = P / 16;
    typedef float f32x4 __attribute__((ext_vector_type(4)));
    const int tid = threadIdx.x, l = tid & 15, p0 = (tid >> 4) * R;
    const int64_t hh = blockIdx.x, j = blockIdx.y, Hk = H / group, hk = hh / group;
    const int64_t from = parent ? (int64_t)parent[j] : j;
    const bool known = from >= 0 && from < n_in;
    float S[R][F];
    if (h.in) {
        const float *src = h.in + (((known ? from : 0) * H + hh) * P + p0) * N + 4 * l;
#pragma unroll
        for (int i = 0; i < R; ++i)
#pragma unroll
            for (int f = 0; f < F; f += 4) {
                const f32x4 w = __builtin_nontemporal_load(reinterpret_cast<const f32x4 *>(src + i * N + f * 16));
                S[i][f] = w.x, S[i][f + 1] = w.y, S[i][f + 2] = w.z, S[i][f + 3] = w.w;
            }
    } else {
#pragma unroll
        for (int i = 0; i < R; ++i)
#pragma unroll
            for (int f = 0; f < F; ++f) S[i][f] = 0.0f;
    }
    const float a2 = A[hh] * kLog2e, bias = dt_bias ? dt_bias[hh] : 0.0f;
    __shared__ float squares[2][kThreads / 64];
    for (int64_t t = 0; t < L; ++t) {
        const int64_t tok = j * L + t;
        float kv[F], qv[F], vv[R];
#pragma unroll
        for (int f = 0; f < F; f += 4) {
            load4(k + (tok * Hk + hk) * N + f * 16 + 4 * l, kv + f);
            load4(q + (tok * Hk + hk) * N + f * 16 + 4 * l, qv + f);
        }
#pragma unroll
        for (int i = 0; i < R; i += 4) load4(v + (tok * H + hh) * P + p0 + i, vv + i);
        const float x = ld_io(dt, tok * H + hh) + bias, w = ld_io(beta, tok * H + hh);
        const float a = exp2_hw((o.softplus ? softplus_f32(x) : x) * a2), b = o.sigmoid ? sigmoid_f32(w) : w;
        float kk = 0.0f, qq = 0.0f, kq = 0.0f, sk[R], sq[R];
#pragma unroll
        for (int f = 0; f < F; ++f) kk = fmaf(kv[f], kv[f], kk), qq = fmaf(qv[f], qv[f], qq), kq = fmaf(kv[f], qv[f], kq);
#pragma unroll
        for (int i = 0; i < R; ++i) {
            sk[i] = sq[i] = 0.0f;
#pragma unroll
            for (int f = 0; f < F; ++f) sk[i] = fmaf(S[i][f], kv[f], sk[i]), sq[i] = fmaf(S[i][f], qv[f], sq[i]);
        }
        kk = sum16(kk), qq = sum16(qq), kq = sum16(kq);
        const float rk = o.qk_norm ? 1.0f / sqrtf(kk + o.eps) : 1.0f, rq = (o.qk_norm ? 1.0f / sqrtf(qq + o.eps) : 1.0f) * o.scale;
        float y[R], ss = 0.0f;
#pragma unroll
        for (int i = 0; i < R; ++i) {
            const float u = b * (vv[i] - a * rk * sum16(sk[i])) * rk;
#pragma unroll
            for (int f = 0; f < F; ++f) S[i][f] = fmaf(a, S[i][f], u * kv[f]);
            y[i] = fmaf(u, kq, a * sum16(sq[i])) * rq;
            ss = fmaf(y[i], y[i], ss);
        }
        float norm = 1.0f;
        if (norm_w) {
            ss += __shfl_xor(ss, 16, 64);
            ss += __shfl_xor(ss, 32, 64);
            if ((tid & 63) == 0) squares[t & 1][tid >> 6] = ss;
            __syncthreads();                                         // (the next token's go to the other half)
            norm = 1.0f / sqrtf(((squares[t & 1][0] + squares[t & 1][1]) + (squares[t & 1][2] + squares[t & 1][3])) / P + o.eps);
        }
        // the 16 lanes of a row group have its R outputs: one each
        float mine = 0.0f;
#pragma unroll
        for (int i = 0; i < R; ++i)
            if (l == i) mine = y[i];
        if (l < R) {
            const int p = p0 + l;
            if (norm_w) mine *= norm * norm_w[p];
            if (z) mine *= silu_f32(ld_io(z, (tok * H + hh) * P + p));
            st_io(out, (tok * H + hh) * P + p, known ? mine : __int_as_float(0x7fc00000));
        }
    }
    if (!h.out) return;
    float *dst = h.out + ((j * H + hh) * P + p0) * N + 4 * l;
#pragma unroll
    for (int i = 0; i < R; ++i)
#pragma unroll
        for (int f = 0; f < F; f += 4) {
            const float nan = __int_as_float(0x7fc00000);
            f32x4 w;
            w.x = known ? S[i][f] : nan, w.y = known ? S[i][f + 1] : nan, w.z = known ? S[i][f + 2] : nan, w.w = known ? S[i][f + 3] : nan;
            __builtin_nontemporal_store(w, reinterpret_cast<f32x4 *>(dst + i * N + f * 16));
        }
}

template <typename T, int N, int P> hipError_t recurrent(const DeltaArgs &a, hipStream_t stream)
{
    delta_recurrent_kernel<T, N, P><<<dim3((unsigned)a.H, (unsigned)a.rows), kThreads, 0, stream>>>(
        StepStates{a.h_out, a.h_in}, a.parent, static_cast<const T *>(a.q), static_cast<const T *>(a.k), static_cast<const T *>(a.v),
        static_cast<const T *>(a.dt), static_cast<const T *>(a.beta), static_cast<const T *>(a.z), a.A, a.norm_w, a.dt_bias,
        static_cast<T *>(a.out), a.n_in, a.L, a.H, a.H / a.Hk, DeltaOptions{a.scale, a.eps, a.dt_softplus, a.beta_sigmoid, a.qk_norm});
    return hipGetLastError();
}

// ---------------------------------------------------------------------------------------------------
// A context in chunks of 64 tokens on the matrix cores.  With G_t the running sum of delta A inside a chunk and S the state at its
// start, the writes u_t = b_t (v_t - a_t S_{t-1} k_t) of a chunk solve a triangular system,
//   T[t,s] = b_t exp(G_t - G_s) k_t . k_s  (s < t),   X = (I + T)^-1 diag(b),   U = X (V - diag(exp G) K S^T)
//   O = diag(exp G) Q S^T + M U,   M[t,s] = exp(G_t - G_s) q_t . k_s  (s <= t)
//   S <- exp(G_end) S + sum_s exp(G_end - G_s) u_s k_s^T
// X and M do not depend on the state: delta_prepare_kernel forms them for all chunks at once.  What is left goes chunk after chunk, but
// every row of S (a value channel) by itself: delta_walk_kernel gives a workgroup 16 PT channels of a head.
// The lengths of q and k are float32 factors of rows and columns, so that k and q enter the products as they were given, exact in
// bfloat16.  Of two factors that are both computed (X, R, U, M, S) each is carried as two bfloat16 terms, the rounded value and
// the remainder, and a product takes three of the four: the states are float32 results, and single terms are off by 2^-9.
// The triangular systems are solved, not expanded: powers of T grow like binomials where keys lean to one side, the inverse does not.
// Fragments of v_mfma_f32_16x16x32_bf16: lane l has row (or column) l % 16 and eight consecutive k from 8 (l / 16); of the result
// column l % 16, rows 4 (l / 16) .. + 3.  What the preparation leaves for the walk is stored in that order, a kilobyte a fragment.
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef float f32x4_t __attribute__((ext_vector_type(4)));

constexpr int kC = 64;                                            // tokens of a chunk
constexpr int kTiles = 6;                                         // 16 x 32 fragments of a lower triangle: 1, 1, 2, 2 to a row of tiles
constexpr int kFrag = 512;                                        // bf16 of a fragment
constexpr int kTri = kTiles * kFrag;
constexpr int kScalars = 256;                                     // floats: factors of k S, of q S, of the write to the state (64 each), decay
constexpr int kChunkHalves = 4 * kTri + 2 * kScalars;             // 16-bit words of a chunk and head: X and M in two terms each, scalars
__device__ __forceinline__ int tile_at(int t_tile, int k_step) { return (t_tile < 2 ? t_tile : 2 * t_tile - 2) + k_step; }

__device__ __forceinline__ bf16x8 as_frag(uint4 q) { return __builtin_bit_cast(bf16x8, q); }
__device__ __forceinline__ bf16x8 lds_frag(const uint16_t *p) { return as_frag(*reinterpret_cast<const uint4 *>(p)); }
__device__ __forceinline__ f32x4_t mma(bf16x8 a, bf16x8 b, f32x4_t c) { return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0); }
__device__ __forceinline__ f32x4_t mma(float a, float b, f32x4_t c) { return __builtin_amdgcn_mfma_f32_16x16x4f32(a, b, c, 0, 0, 0); }

// four values -> their bf16 roundings and the bf16 of what the roundings dropped
__device__ __forceinline__ void split4(f32x4_t v, uint16_t *top, uint16_t *rem)
{
    const uint32_t t01 = f32x2_to_bf16x2(v[0], v[1]), t23 = f32x2_to_bf16x2(v[2], v[3]);
    *reinterpret_cast<uint2 *>(top) = make_uint2(t01, t23);
    *reinterpret_cast<uint2 *>(rem) = make_uint2(f32x2_to_bf16x2(v[0] - bf16_lo(t01), v[1] - bf16_hi(t01)),
                                                 f32x2_to_bf16x2(v[2] - bf16_lo(t23), v[3] - bf16_hi(t23)));
}

// Workgroup barrier for what is exchanged through LDS; global loads and stores in flight stay there.
__device__ __forceinline__ void lds_barrier()
{
    __builtin_amdgcn_fence(__ATOMIC_RELEASE, "workgroup", "local");
    __builtin_amdgcn_s_barrier();
    __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "workgroup", "local");
}

// grid: (chunks, H, batch)
template <int N>
__global__ void __launch_bounds__(kThreads)
delta_prepare_kernel(const bf16_t *__restrict__ q, const bf16_t *__restrict__ k, const bf16_t *__restrict__ dt, const bf16_t *__restrict__ beta,
                     const float *__restrict__ A, const float *__restrict__ dt_bias, uint16_t *__restrict__ ws, uint16_t *__restrict__ kt,
                     int64_t L, int64_t H, int64_t group, DeltaOptions o)
{
    constexpr int kRow = N + 8, kSys = kC + 4;
    __shared__ __attribute__((aligned(16))) uint16_t ks[kC * kRow], qs[kC * kRow];
    __shared__ __attribute__((aligned(16))) float sys[kC * kSys], inv[kC * kSys];
    __shared__ __attribute__((aligned(16))) float rk[kC], rq[kC], G[kC], bt[kC];
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), c16 = lane & 15, g4 = lane >> 4;
    const int64_t chunk = blockIdx.x, n_chunks = gridDim.x, h = blockIdx.y, b = blockIdx.z;
    const int64_t Hk = H / group, hk = h / group, tok0 = chunk * kC;
    const int live = (int)min((int64_t)kC, L - tok0);             // tokens of this chunk
    ws += ((b * H + h) * n_chunks + chunk) * kChunkHalves;

    // keys and queries into LDS, and one over their lengths (rows behind the end: zeros)
    constexpr int kPieces = N / 8;                                // 16-byte pieces of a row, on as many adjacent lanes
    {
        uint4 kp[kC * kPieces / kThreads], qp[kC * kPieces / kThreads];
#pragma unroll
        for (int i = 0; i < kC * kPieces / kThreads; ++i) {
            const int id = i * kThreads + tid, row = id / kPieces, piece = id % kPieces;
            const int64_t at = ((b * L + tok0 + min(row, live - 1)) * Hk + hk) * N + piece * 8;
            kp[i] = *reinterpret_cast<const uint4 *>(k + at);
            qp[i] = *reinterpret_cast<const uint4 *>(q + at);
        }
#pragma unroll
        for (int i = 0; i < kC * kPieces / kThreads; ++i) {
            const int id = i * kThreads + tid, row = id / kPieces, piece = id % kPieces;
            if (row >= live) kp[i] = qp[i] = make_uint4(0, 0, 0, 0);
            float sk = 0.0f, sq = 0.0f;
            const uint32_t kw[4] = {kp[i].x, kp[i].y, kp[i].z, kp[i].w}, qw[4] = {qp[i].x, qp[i].y, qp[i].z, qp[i].w};
#pragma unroll
            for (int w = 0; w < 4; ++w) {
                sk = fmaf(bf16_lo(kw[w]), bf16_lo(kw[w]), fmaf(bf16_hi(kw[w]), bf16_hi(kw[w]), sk));
                sq = fmaf(bf16_lo(qw[w]), bf16_lo(qw[w]), fmaf(bf16_hi(qw[w]), bf16_hi(qw[w]), sq));
            }
            sk = lane_add<0x141>(lane_add<0x4e>(lane_add<0xb1>(sk)));    // 8 lanes
            sq = lane_add<0x141>(lane_add<0x4e>(lane_add<0xb1>(sq)));
            if constexpr (kPieces == 16) sk = lane_add<0x140>(sk), sq = lane_add<0x140>(sq);
            *reinterpret_cast<uint4 *>(&ks[row * kRow + piece * 8]) = kp[i];
            *reinterpret_cast<uint4 *>(&qs[row * kRow + piece * 8]) = qp[i];
            if (piece == 0) {
                rk[row] = row >= live ? 0.0f : o.qk_norm ? 1.0f / sqrtf(sk + o.eps) : 1.0f;
                rq[row] = row >= live ? 0.0f : (o.qk_norm ? 1.0f / sqrtf(sq + o.eps) : 1.0f) * o.scale;
            }
        }
    }
    // running sum of delta A (in powers of two) and the write strengths; tokens behind the end neither decay nor write
    if (wave == 0) {
        const int64_t at = (b * L + tok0 + min(lane, live - 1)) * H + h;
        const float x = bf16_to_f32(dt[at]) + (dt_bias ? dt_bias[h] : 0.0f), w = bf16_to_f32(beta[at]);
        float sc = lane < live ? (o.softplus ? softplus_f32(x) : x) * A[h] * kLog2e : 0.0f;
        sc += __builtin_bit_cast(float, __builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, sc), 0x111, 0xf, 0xf, false));
        sc += __builtin_bit_cast(float, __builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, sc), 0x112, 0xf, 0xf, false));
        sc += __builtin_bit_cast(float, __builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, sc), 0x114, 0xf, 0xf, false));
        sc += __builtin_bit_cast(float, __builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, sc), 0x118, 0xf, 0xf, false));
        const float r0 = __builtin_bit_cast(float, __builtin_amdgcn_readlane(__builtin_bit_cast(int, sc), 15));
        const float r1 = __builtin_bit_cast(float, __builtin_amdgcn_readlane(__builtin_bit_cast(int, sc), 31));
        const float r2 = __builtin_bit_cast(float, __builtin_amdgcn_readlane(__builtin_bit_cast(int, sc), 47));
        sc += g4 == 0 ? 0.0f : g4 == 1 ? r0 : g4 == 2 ? r0 + r1 : (r0 + r1) + r2;
        G[lane] = sc;
        bt[lane] = lane < live ? (o.sigmoid ? sigmoid_f32(w) : w) : 0.0f;
    }
    lds_barrier();

    // T and M, tile by tile of 16 x 16: lane has token t = l % 16 of the tile and four s.  A wavefront has a row of tiles of T and
    // the row of M as far from the other end: five tiles each.
    auto tiles = [&](const uint16_t *rows, int t_tile, auto put) {
        bf16x8 of_t[N / 32];
#pragma unroll
        for (int i = 0; i < N / 32; ++i) of_t[i] = lds_frag(&rows[(t_tile * 16 + c16) * kRow + i * 32 + g4 * 8]);
        const int t = t_tile * 16 + c16;
        const float Gt = G[t];
        for (int s_tile = 0; s_tile <= (t_tile | 1); ++s_tile) {
            f32x4_t acc = {0.0f, 0.0f, 0.0f, 0.0f};
            const int s0 = s_tile * 16 + 4 * g4;
            if (s_tile <= t_tile) {
                bf16x8 of_s[N / 32];
#pragma unroll
                for (int i = 0; i < N / 32; ++i) of_s[i] = lds_frag(&ks[(s_tile * 16 + c16) * kRow + i * 32 + g4 * 8]);
#pragma unroll
                for (int i = 0; i < N / 32; ++i) acc = mma(of_s[i], of_t[i], acc);
                const float4 Gs = *reinterpret_cast<const float4 *>(&G[s0]), rs = *reinterpret_cast<const float4 *>(&rk[s0]);
                acc[0] *= exp2_hw(Gt - Gs.x) * rs.x, acc[1] *= exp2_hw(Gt - Gs.y) * rs.y;
                acc[2] *= exp2_hw(Gt - Gs.z) * rs.z, acc[3] *= exp2_hw(Gt - Gs.w) * rs.w;
            }
            put(t, s_tile, s0, acc);
        }
    };
    tiles(ks, wave, [&](int t, int, int s0, f32x4_t v) {
        const float f = bt[t] * rk[t];
#pragma unroll
        for (int i = 0; i < 4; ++i) v[i] = s0 + i < t ? v[i] * f : 0.0f;
        *reinterpret_cast<f32x4_t *>(&sys[t * kSys + s0]) = v;
    });
    tiles(qs, 3 - wave, [&](int t, int s_tile, int s0, f32x4_t v) {
        const float f = rq[t];
#pragma unroll
        for (int i = 0; i < 4; ++i) v[i] = s0 + i <= t ? v[i] * f : 0.0f;
        const int at = tile_at(t >> 4, s_tile >> 1) * kFrag + (c16 + 16 * ((s_tile & 1) * 2 + (g4 >> 1))) * 8 + 4 * (g4 & 1);
        split4(v, ws + 2 * kTri + at, ws + 3 * kTri + at);
    });
    // the keys the other way round, for the write to the state: once for the value heads that share them
    if (h % group == 0) {
        uint16_t *to = kt + ((b * Hk + hk) * n_chunks + chunk) * (N * kC);
        for (int f = wave; f < N / 8; f += 4) {
            const int n = (f >> 1) * 16 + c16, s0 = (f & 1) * 32 + g4 * 8;
            uint32_t w[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) w[i] = ks[(s0 + 2 * i) * kRow + n] | (uint32_t)ks[(s0 + 2 * i + 1) * kRow + n] << 16;
            *reinterpret_cast<uint4 *>(to + f * kFrag + lane * 8) = make_uint4(w[0], w[1], w[2], w[3]);
        }
    }
    lds_barrier();

    // (I + T)^-1: the four 16 x 16 blocks on the diagonal by substitution, a column to a lane ...
    {
        const float *d = sys + wave * 16 * kSys + wave * 16;
        float x[16];
#pragma unroll
        for (int i = 0; i < 16; ++i) {
            float v = i == c16 ? 1.0f : 0.0f;
#pragma unroll
            for (int j = 0; j < i; ++j) v = fmaf(-d[i * kSys + j], x[j], v);
            x[i] = v;
        }
        float *to = inv + wave * 16 * kSys + wave * 16 + c16;
#pragma unroll
        for (int i = 0; i < 16; ++i)
            if ((i & 3) == g4) to[i * kSys] = x[i];
    }
    lds_barrier();
    // ... then what stands below them, X21 = -X22 T21 X11, in float32 on the matrix cores.  The contraction takes the four k of a step from
    // the four lane groups, 4 g + i in step i: so a result is the next product's operand as it lies in the registers.
    auto times_block = [&](int row, int mid, int col, f32x4_t y) {   // y + T[row, mid] X[mid, col] of 16 x 16 blocks
        const f32x4_t a = *reinterpret_cast<const f32x4_t *>(&sys[(row * 16 + c16) * kSys + mid * 16 + 4 * g4]);
#pragma unroll
        for (int i = 0; i < 4; ++i) y = mma(a[i], inv[(mid * 16 + 4 * g4 + i) * kSys + col * 16 + c16], y);
        return y;
    };
    auto times_inverse = [&](int row, int mid, f32x4_t y, f32x4_t acc) {   // acc - X[row, mid] y
        const f32x4_t a = *reinterpret_cast<const f32x4_t *>(&inv[(row * 16 + c16) * kSys + mid * 16 + 4 * g4]);
#pragma unroll
        for (int i = 0; i < 4; ++i) acc = mma(-a[i], y[i], acc);
        return acc;
    };
    auto store_block = [&](int row, int col, f32x4_t v) {
#pragma unroll
        for (int i = 0; i < 4; ++i) inv[(row * 16 + 4 * g4 + i) * kSys + col * 16 + c16] = v[i];
    };
    const f32x4_t zero = {0.0f, 0.0f, 0.0f, 0.0f};
    if (wave < 2) {
        const int r = 2 * wave + 1, c = 2 * wave;
        store_block(r, c, times_inverse(r, r, times_block(r, c, c, zero), zero));
    }
    lds_barrier();
    {
        const int r = 2 + (wave >> 1), c = wave & 1;
        f32x4_t y = times_block(2, 1, c, zero);
        if (c == 0) y = times_block(2, 0, 0, y);
        f32x4_t acc = times_inverse(r, 2, y, zero);
        if (r == 3) {
            y = times_block(3, 1, c, zero);
            if (c == 0) y = times_block(3, 0, 0, y);
            acc = times_inverse(3, 3, y, acc);
        }
        store_block(r, c, acc);
    }
    lds_barrier();
    // X in two terms, and the factors of rows
    for (int step = 0; step <= wave >> 1; ++step) {
        const int t = wave * 16 + c16, s0 = step * 32 + g4 * 8, at = tile_at(wave, step) * kFrag + lane * 8;
#pragma unroll
        for (int i = 0; i < 8; i += 4) {
            f32x4_t v = *reinterpret_cast<const f32x4_t *>(&inv[t * kSys + s0 + i]);
            const float4 w = *reinterpret_cast<const float4 *>(&bt[s0 + i]);
            v[0] = s0 + i <= t ? v[0] * w.x : 0.0f, v[1] = s0 + i + 1 <= t ? v[1] * w.y : 0.0f;
            v[2] = s0 + i + 2 <= t ? v[2] * w.z : 0.0f, v[3] = s0 + i + 3 <= t ? v[3] * w.w : 0.0f;
            split4(v, ws + at + i, ws + kTri + at + i);
        }
    }
    if (wave == 0) {
        float *f = reinterpret_cast<float *>(ws + 4 * kTri);
        const float e = exp2_hw(G[lane]), end = G[kC - 1];
        f[lane] = rk[lane] * e;
        f[kC + lane] = rq[lane] * e;
        f[2 * kC + lane] = rk[lane] * exp2_hw(end - G[lane]);
        if (lane == 0) f[3 * kC] = exp2_hw(end);
    }
}

// The chunks of one (batch row, head) in order, for 16 PT of its channels, whose rows of S stay in MFMA accumulators (transposed: lane
// has a channel and four adjacent states).  Four wavefronts; three phases of a chunk, each ending in a barrier:
//   1  wavefront w has tokens 16 w .. + 15: R = V - diag K S^T and the first half of the outputs, Q S^T
//   2  U = X R of its tokens
//   3  the second half of the outputs, M U; and the write to the state, N / 64 tiles of 16 states each
// All operands but S, R and U come from memory as fragments, requested as soon as the chunk before has used up their registers.
// grid: 8 channel blocks (heads / 8 rounded up); the blocks of a head, which read the same fragments, are 8 apart: on one XCD
template <int N, int PT>
__global__ void __launch_bounds__(kThreads) __attribute__((amdgpu_waves_per_eu(1, 2)))
delta_walk_kernel(const bf16_t *q, const bf16_t *k, const bf16_t *v, const bf16_t *z, const uint16_t *ws, const uint16_t *kt, const float *h0,
                  float *h_final, bf16_t *out, float *raw, int64_t L, int64_t H, int64_t group, int P, int64_t heads, int64_t n_chunks)
{
    constexpr int kRowS = N + 8, kRowU = kC + 8, kSteps = N / 32, kNT = N / 64;
    __shared__ __attribute__((aligned(16))) uint16_t s_hi[16 * PT * kRowS], s_lo[16 * PT * kRowS];          // S as [channel][state]
    __shared__ __attribute__((aligned(16))) uint16_t r_hi[16 * PT * kRowU], r_lo[16 * PT * kRowU];          // R as [channel][token]
    __shared__ __attribute__((aligned(16))) uint16_t u_hi[16 * PT * kRowU], u_lo[16 * PT * kRowU];          // U
    __shared__ __attribute__((aligned(16))) uint16_t w_hi[16 * PT * kRowU], w_lo[16 * PT * kRowU];          // U times the decay to the end
    const uint32_t blocks = (uint32_t)P / (16 * PT), place = blockIdx.x >> 3;
    const int64_t hb = (int64_t)(place / blocks) * 8 + (blockIdx.x & 7);
    if (hb >= heads) return;
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), c16 = lane & 15, g4 = lane >> 4;
    const int64_t b = hb / H, h = hb - b * H, Hk = H / group, hk = h / group;
    const int p0 = (int)(place % blocks) * 16 * PT;
    const int t_own = wave * 16 + c16;                            // as a row of K and Q, and as the column of outputs

    const uint16_t *own = ws + hb * n_chunks * kChunkHalves;
    const uint16_t *own_kt = kt + (b * Hk + hk) * n_chunks * (N * kC) + wave * kNT * 2 * kFrag + lane * 8;
    // What is requested of a chunk; past the last one, the last one's again.
    uint4 kf[kSteps], qf[kSteps], xh[2], xl[2], mh[2], ml[2], ktf[kNT][2];
    uint16_t vf[PT][4];
    float4 k_factor, w_factor;
    float q_factor, decay;
    auto token = [&](int64_t chunk, int t) { return b * L + min(chunk * kC + t, L - 1); };
    auto fetch_1 = [&](int64_t chunk) {
        chunk = min(chunk, n_chunks - 1);
        const int64_t at = (token(chunk, t_own) * Hk + hk) * N + g4 * 8;
#pragma unroll
        for (int i = 0; i < kSteps; ++i) kf[i] = *reinterpret_cast<const uint4 *>(k + at + i * 32), qf[i] = *reinterpret_cast<const uint4 *>(q + at + i * 32);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const bf16_t *row = v + (token(chunk, wave * 16 + 4 * g4 + i) * H + h) * P + p0 + c16;
#pragma unroll
            for (int p = 0; p < PT; ++p) vf[p][i] = row[p * 16];
        }
        const float *f = reinterpret_cast<const float *>(own + chunk * kChunkHalves + 4 * kTri);
        k_factor = *reinterpret_cast<const float4 *>(f + wave * 16 + 4 * g4);
    };
    auto fetch_2 = [&](int64_t chunk) {
        const uint16_t *x = own + min(chunk, n_chunks - 1) * kChunkHalves + lane * 8;
#pragma unroll
        for (int i = 0; i < 2; ++i)
            if (i <= wave >> 1) {
                xh[i] = *reinterpret_cast<const uint4 *>(x + tile_at(wave, i) * kFrag);
                xl[i] = *reinterpret_cast<const uint4 *>(x + kTri + tile_at(wave, i) * kFrag);
            }
        w_factor = *reinterpret_cast<const float4 *>(reinterpret_cast<const float *>(own + min(chunk, n_chunks - 1) * kChunkHalves + 4 * kTri) + 2 * kC + wave * 16 + 4 * g4);
    };
    auto fetch_3 = [&](int64_t chunk) {
        chunk = min(chunk, n_chunks - 1);
        const uint16_t *x = own + chunk * kChunkHalves + 2 * kTri + lane * 8;
#pragma unroll
        for (int i = 0; i < 2; ++i)
            if (i <= wave >> 1) {
                mh[i] = *reinterpret_cast<const uint4 *>(x + tile_at(wave, i) * kFrag);
                ml[i] = *reinterpret_cast<const uint4 *>(x + kTri + tile_at(wave, i) * kFrag);
            }
#pragma unroll
        for (int j = 0; j < kNT; ++j)
#pragma unroll
            for (int i = 0; i < 2; ++i) ktf[j][i] = *reinterpret_cast<const uint4 *>(own_kt + chunk * (N * kC) + (j * 2 + i) * kFrag);
        const float *f = reinterpret_cast<const float *>(own + chunk * kChunkHalves + 4 * kTri);
        q_factor = f[kC + t_own];
        decay = f[3 * kC];
    };
    fetch_1(0);
    fetch_2(0);
    fetch_3(0);

    f32x4_t acc[kNT][PT];                                         // [j][p][i]: state 16 (kNT wave + j) + 4 g4 + i of channel p0 + 16 p + c16
    auto park_state = [&]() {
#pragma unroll
        for (int j = 0; j < kNT; ++j)
#pragma unroll
            for (int p = 0; p < PT; ++p) {
                const int at = (p * 16 + c16) * kRowS + (wave * kNT + j) * 16 + 4 * g4;
                split4(acc[j][p], &s_hi[at], &s_lo[at]);
            }
    };
#pragma unroll
    for (int j = 0; j < kNT; ++j)
#pragma unroll
        for (int p = 0; p < PT; ++p) {
            acc[j][p] = f32x4_t{0.0f, 0.0f, 0.0f, 0.0f};
            if (h0) acc[j][p] = *reinterpret_cast<const f32x4_t *>(h0 + (hb * P + p0 + p * 16 + c16) * N + (wave * kNT + j) * 16 + 4 * g4);
        }
    park_state();
    lds_barrier();

    for (int64_t chunk = 0; chunk < n_chunks; ++chunk) {
        f32x4_t o[PT];
#pragma unroll
        for (int p = 0; p < PT; ++p) {
            bf16x8 sh[kSteps], sl[kSteps];
#pragma unroll
            for (int i = 0; i < kSteps; ++i) {
                sh[i] = lds_frag(&s_hi[(p * 16 + c16) * kRowS + i * 32 + g4 * 8]);
                sl[i] = lds_frag(&s_lo[(p * 16 + c16) * kRowS + i * 32 + g4 * 8]);
            }
            f32x4_t r = {0.0f, 0.0f, 0.0f, 0.0f};
            o[p] = r;
#pragma unroll
            for (int i = 0; i < kSteps; ++i) r = mma(as_frag(kf[i]), sh[i], r);
#pragma unroll
            for (int i = 0; i < kSteps; ++i) r = mma(as_frag(kf[i]), sl[i], r);
#pragma unroll
            for (int i = 0; i < kSteps; ++i) o[p] = mma(sh[i], as_frag(qf[i]), o[p]);
#pragma unroll
            for (int i = 0; i < kSteps; ++i) o[p] = mma(sl[i], as_frag(qf[i]), o[p]);
            r[0] = fmaf(-k_factor.x, r[0], bf16_to_f32(vf[p][0])), r[1] = fmaf(-k_factor.y, r[1], bf16_to_f32(vf[p][1]));
            r[2] = fmaf(-k_factor.z, r[2], bf16_to_f32(vf[p][2])), r[3] = fmaf(-k_factor.w, r[3], bf16_to_f32(vf[p][3]));
            const int at = (p * 16 + c16) * kRowU + wave * 16 + 4 * g4;
            split4(r, &r_hi[at], &r_lo[at]);
        }
        fetch_1(chunk + 1);
        lds_barrier();
#pragma unroll
        for (int p = 0; p < PT; ++p) {
            f32x4_t u = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
            for (int i = 0; i < 2; ++i)
                if (i <= wave >> 1) {
                    const bf16x8 rh = lds_frag(&r_hi[(p * 16 + c16) * kRowU + i * 32 + g4 * 8]), rl = lds_frag(&r_lo[(p * 16 + c16) * kRowU + i * 32 + g4 * 8]);
                    u = mma(as_frag(xh[i]), rh, u);
                    u = mma(as_frag(xh[i]), rl, u);
                    u = mma(as_frag(xl[i]), rh, u);
                }
            const int at = (p * 16 + c16) * kRowU + wave * 16 + 4 * g4;
            split4(u, &u_hi[at], &u_lo[at]);
            u[0] *= w_factor.x, u[1] *= w_factor.y, u[2] *= w_factor.z, u[3] *= w_factor.w;
            split4(u, &w_hi[at], &w_lo[at]);
        }
        fetch_2(chunk + 1);
        lds_barrier();
#pragma unroll
        for (int p = 0; p < PT; ++p) {
            bf16x8 wh[2], wl[2];
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                wh[i] = lds_frag(&w_hi[(p * 16 + c16) * kRowU + i * 32 + g4 * 8]);
                wl[i] = lds_frag(&w_lo[(p * 16 + c16) * kRowU + i * 32 + g4 * 8]);
            }
#pragma unroll
            for (int j = 0; j < kNT; ++j) {
                acc[j][p] *= decay;
#pragma unroll
                for (int i = 0; i < 2; ++i) {
                    acc[j][p] = mma(as_frag(ktf[j][i]), wh[i], acc[j][p]);
                    acc[j][p] = mma(as_frag(ktf[j][i]), wl[i], acc[j][p]);
                }
            }
            o[p] *= q_factor;
#pragma unroll
            for (int i = 0; i < 2; ++i)
                if (i <= wave >> 1) {
                    const bf16x8 uh = lds_frag(&u_hi[(p * 16 + c16) * kRowU + i * 32 + g4 * 8]), ul = lds_frag(&u_lo[(p * 16 + c16) * kRowU + i * 32 + g4 * 8]);
                    o[p] = mma(uh, as_frag(mh[i]), o[p]);
                    o[p] = mma(ul, as_frag(mh[i]), o[p]);
                    o[p] = mma(uh, as_frag(ml[i]), o[p]);
                }
        }
        park_state();
        fetch_3(chunk + 1);
        if (chunk * kC + t_own < L) {
            const int64_t at = ((b * L + chunk * kC + t_own) * H + h) * P + p0 + 4 * g4;
#pragma unroll
            for (int p = 0; p < PT; ++p) {
                if (raw) {
                    *reinterpret_cast<f32x4_t *>(raw + at + p * 16) = o[p];
                    continue;
                }
                float y[4] = {o[p][0], o[p][1], o[p][2], o[p][3]};
                if (z) {
                    float g[4];
                    load4(z + at + p * 16, g);
#pragma unroll
                    for (int i = 0; i < 4; ++i) y[i] *= silu_f32(g[i]);
                }
                *reinterpret_cast<uint2 *>(out + at + p * 16) = make_uint2(f32x2_to_bf16x2(y[0], y[1]), f32x2_to_bf16x2(y[2], y[3]));
            }
        }
        lds_barrier();
    }
    if (!h_final) return;
#pragma unroll
    for (int j = 0; j < kNT; ++j)
#pragma unroll
        for (int p = 0; p < PT; ++p)
            *reinterpret_cast<f32x4_t *>(h_final + (hb * P + p0 + p * 16 + c16) * N + (wave * kNT + j) * 16 + 4 * g4) = acc[j][p];
}

// The norm over a head's channels, which the walk's workgroups have in parts, and the gate: P / 4 lanes to a (token, head).
template <int P>
__global__ void __launch_bounds__(kThreads)
delta_norm_kernel(const float *__restrict__ raw, const bf16_t *__restrict__ z, const float *__restrict__ norm_w, bf16_t *__restrict__ out, int64_t n,
                  float eps)
{
    const int64_t at = (int64_t)blockIdx.x * kThreads + threadIdx.x;
    const int64_t safe = min(at, n - 1);
    const int p = (int)(safe % (P / 4)) * 4;
    float y[4], w[4], g[4] = {0.0f, 0.0f, 0.0f, 0.0f};
    load4(raw + safe * 4, y);
    load4(norm_w + p, w);
    if (z) load4(z + safe * 4, g);
    float ss = sum16(fmaf(y[0], y[0], fmaf(y[1], y[1], fmaf(y[2], y[2], y[3] * y[3]))));
    if constexpr (P == 128) ss += __shfl_xor(ss, 16, 64);
    const float f = 1.0f / sqrtf(ss / P + eps);
#pragma unroll
    for (int i = 0; i < 4; ++i) y[i] *= f * w[i] * (z ? silu_f32(g[i]) : 1.0f);
    if (at < n) *reinterpret_cast<uint2 *>(out + at * 4) = make_uint2(f32x2_to_bf16x2(y[0], y[1]), f32x2_to_bf16x2(y[2], y[3]));
}

// Where the parts of the workspace lie (bytes from its start): fragments of a chunk and value head, transposed keys of a chunk and key
// head, outputs ahead of their norm.
struct DeltaPlan {
    int64_t chunks, kt_at, raw_at, bytes;
};
DeltaPlan delta_plan(int64_t batch, int64_t L, int64_t H, int64_t Hk, int64_t P, int64_t N)
{
    DeltaPlan p;
    p.chunks = (L + kC - 1) / kC;
    p.kt_at = batch * H * p.chunks * kChunkHalves * 2;
    p.raw_at = p.kt_at + batch * Hk * p.chunks * N * kC * 2;
    p.bytes = p.raw_at + batch * L * H * P * 4;
    return p;
}

template <int N, int PT> void walk(const DeltaArgs &a, const DeltaPlan &p, float *raw, hipStream_t stream)
{
    const char *ws = reinterpret_cast<const char *>(a.ws);
    const int64_t heads = a.rows * a.H;
    delta_walk_kernel<N, PT><<<(unsigned)((heads + 7) / 8 * 8 * (a.P / (16 * PT))), kThreads, 0, stream>>>(
        static_cast<const bf16_t *>(a.q), static_cast<const bf16_t *>(a.k), static_cast<const bf16_t *>(a.v), static_cast<const bf16_t *>(a.z),
        reinterpret_cast<const uint16_t *>(ws), reinterpret_cast<const uint16_t *>(ws + p.kt_at), a.h_in, a.h_out, static_cast<bf16_t *>(a.out),
        raw, a.L, a.H, a.H / a.Hk, a.P, heads, p.chunks);
}

template <int N> hipError_t chunked(const DeltaArgs &a, hipStream_t stream)
{
    const DeltaPlan p = delta_plan(a.rows, a.L, a.H, a.Hk, a.P, a.N);
    char *ws = reinterpret_cast<char *>(a.ws);
    delta_prepare_kernel<N><<<dim3((unsigned)p.chunks, (unsigned)a.H, (unsigned)a.rows), kThreads, 0, stream>>>(
        static_cast<const bf16_t *>(a.q), static_cast<const bf16_t *>(a.k), static_cast<const bf16_t *>(a.dt), static_cast<const bf16_t *>(a.beta),
        a.A, a.dt_bias, reinterpret_cast<uint16_t *>(ws), reinterpret_cast<uint16_t *>(ws + p.kt_at), a.L, a.H, a.H / a.Hk,
        DeltaOptions{a.scale, a.eps, a.dt_softplus, a.beta_sigmoid, a.qk_norm});
    if (hipError_t e = hipGetLastError()) return e;
    float *raw = a.norm_w ? reinterpret_cast<float *>(ws + p.raw_at) : nullptr;
    walk<N, 2>(a, p, raw, stream);
    if (hipError_t e = hipGetLastError()) return e;
    if (raw) {
        const int64_t n = a.rows * a.L * a.H * a.P / 4;
        const unsigned grid = (unsigned)((n + kThreads - 1) / kThreads);
        const bf16_t *z = static_cast<const bf16_t *>(a.z);
        if (a.P == 64) delta_norm_kernel<64><<<grid, kThreads, 0, stream>>>(raw, z, a.norm_w, static_cast<bf16_t *>(a.out), n, a.eps);
        else delta_norm_kernel<128><<<grid, kThreads, 0, stream>>>(raw, z, a.norm_w, static_cast<bf16_t *>(a.out), n, a.eps);
    }
    return hipGetLastError();
}

}  // namespace

hipError_t launch_gated_delta_step(const DeltaArgs &a, hipStream_t stream)
{
#define MAMBA_DELTA(T) (a.N == 64 ? a.P == 64 ? recurrent<T, 64, 64>(a, stream) : recurrent<T, 64, 128>(a, stream) \
                                  : a.P == 64 ? recurrent<T, 128, 64>(a, stream) : recurrent<T, 128, 128>(a, stream))
    return a.io == kIoBf16 ? MAMBA_DELTA(bf16_t) : MAMBA_DELTA(float);
#undef MAMBA_DELTA
}

size_t gated_delta_workspace_bytes(int64_t batch, int64_t L, int64_t H, int64_t Hk, int64_t P, int64_t N)
{
    return (size_t)delta_plan(batch, L, H, Hk, P, N).bytes;
}

hipError_t launch_gated_delta(const DeltaArgs &a, hipStream_t stream)
{
    if (a.io != kIoBf16) return launch_gated_delta_step(a, stream);
    return a.N == 64 ? chunked<64>(a, stream) : chunked<128>(a, stream);
}

}  // namespace mamba
