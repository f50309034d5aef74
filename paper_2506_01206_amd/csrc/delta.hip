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

}  // namespace

hipError_t launch_gated_delta_step(const DeltaArgs &a, hipStream_t stream)
{
#define MAMBA_DELTA(T) (a.N == 64 ? a.P == 64 ? recurrent<T, 64, 64>(a, stream) : recurrent<T, 64, 128>(a, stream) \
                                  : a.P == 64 ? recurrent<T, 128, 64>(a, stream) : recurrent<T, 128, 128>(a, stream))
    return a.io == kIoBf16 ? MAMBA_DELTA(bf16_t) : MAMBA_DELTA(float);
#undef MAMBA_DELTA
}

size_t gated_delta_workspace_bytes(int64_t, int64_t, int64_t, int64_t, int64_t, int64_t) { return 0; }

hipError_t launch_gated_delta(const DeltaArgs &a, hipStream_t stream) { return launch_gated_delta_step(a, stream); }

}  // namespace mamba
