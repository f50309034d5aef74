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
// a double of the lane that CTRL names within a row of 16 (0: none such), and of one lane
template <int CTRL> __device__ __forceinline__ double lanes_back(double v)
{
    const uint64_t bits = __builtin_bit_cast(uint64_t, v);
    const uint32_t lo = __builtin_amdgcn_update_dpp(0, (int)(uint32_t)bits, CTRL, 0xf, 0xf, false);
    const uint32_t hi = __builtin_amdgcn_update_dpp(0, (int)(uint32_t)(bits >> 32), CTRL, 0xf, 0xf, false);
    return __builtin_bit_cast(double, (uint64_t)hi << 32 | lo);
}
__device__ __forceinline__ double of_lane(double v, int lane)
{
    const uint64_t bits = __builtin_bit_cast(uint64_t, v);
    const uint32_t lo = __builtin_amdgcn_readlane((int)(uint32_t)bits, lane), hi = __builtin_amdgcn_readlane((int)(uint32_t)(bits >> 32), lane);
    return __builtin_bit_cast(double, (uint64_t)hi << 32 | lo);
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

// Four values as they lie in memory.
template <typename T> struct RawOf;
template <> struct RawOf<float> { typedef float4 type; };
template <> struct RawOf<bf16_t> { typedef uint2 type; };
template <typename T> using Raw4 = typename RawOf<T>::type;
template <typename T> __device__ __forceinline__ Raw4<T> raw4(const T *p) { return *reinterpret_cast<const Raw4<T> *>(p); }
__device__ __forceinline__ void unpack4(float4 w, float *v) { v[0] = w.x, v[1] = w.y, v[2] = w.z, v[3] = w.w; }
__device__ __forceinline__ void unpack4(uint2 w, float *v)
{
    v[0] = bf16_lo(w.x), v[1] = bf16_hi(w.x), v[2] = bf16_lo(w.y), v[3] = bf16_hi(w.y);
}

__device__ __forceinline__ bool finite(float v) { return __builtin_isfinite(v); }
__device__ __forceinline__ float sigmoid_f32(float v) { return rcp_hw(1.0f + exp2_hw(-v * kLog2e)); }

// ---------------------------------------------------------------------------------------------------
// Token after token as the equations stand: one workgroup has a head of one row, its state in registers (16 lanes to a row of S,
// P / 16 rows to a thread).  For single tokens this is all there is to do: a state is read and written once, both dot products
// of a row with it come out of one reduction, and the head's P outputs are together for the norm.
// A new state is written past the caches (nobody reads it in this launch), but an old one is read through them: children of one parent
// read it one after the other.  128 branches of 64 parents, 32 heads of 128 x 128: 74 us; both past the caches 93, both through them 88.
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
                const f32x4 w = *reinterpret_cast<const f32x4 *>(src + i * N + f * 16);
                S[i][f] = w.x, S[i][f + 1] = w.y, S[i][f + 2] = w.z, S[i][f + 3] = w.w;
            }
    } else {
#pragma unroll
        for (int i = 0; i < R; ++i)
#pragma unroll
            for (int f = 0; f < F; ++f) S[i][f] = 0.0f;
    }
    const float a2 = A[hh] * kLog2e, bias = dt_bias ? dt_bias[hh] : 0.0f;
    // The 16 lanes of a row group have its R outputs: one each (the rest repeat the last).
    const int mine = l < R ? l : R - 1;
    const float weight = norm_w ? norm_w[p0 + mine] : 1.0f;
    // All that a token brings, as it lies in memory: the next token's is on its way while this one is worked on.
    struct Token {
        Raw4<T> k[F / 4], q[F / 4], v[R / 4];
        T dt, beta, z;
    };
    auto fetch = [&](int64_t t) __attribute__((always_inline)) {
        Token w;
        const int64_t tok = j * L + t;
#pragma unroll
        for (int f = 0; f < F / 4; ++f) {
            w.k[f] = raw4(k + (tok * Hk + hk) * N + f * 64 + 4 * l);
            w.q[f] = raw4(q + (tok * Hk + hk) * N + f * 64 + 4 * l);
        }
#pragma unroll
        for (int i = 0; i < R / 4; ++i) w.v[i] = raw4(v + (tok * H + hh) * P + p0 + 4 * i);
        w.dt = dt[tok * H + hh], w.beta = beta[tok * H + hh];
        w.z = z ? z[(tok * H + hh) * P + p0 + mine] : T{};
        return w;
    };
    __shared__ float squares[2][kThreads / 64];
    Token next = fetch(0);
    for (int64_t t = 0; t < L; ++t) {
        const int64_t tok = j * L + t;
        const Token c = next;
        if (t + 1 < L) next = fetch(t + 1);
        float kv[F], qv[F], vv[R];
#pragma unroll
        for (int f = 0; f < F / 4; ++f) unpack4(c.k[f], kv + 4 * f), unpack4(c.q[f], qv + 4 * f);
#pragma unroll
        for (int i = 0; i < R / 4; ++i) unpack4(c.v[i], vv + 4 * i);
        const float x = ld_io(&c.dt, 0) + bias, w = ld_io(&c.beta, 0);
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
        float r = y[0];
#pragma unroll
        for (int i = 1; i < R; ++i) r = l == i ? y[i] : r;
        if (norm_w) r *= norm * weight;
        if (z) r *= silu_f32(ld_io(&c.z, 0));
        if (l < R) st_io(out, (tok * H + hh) * P + p0 + l, known ? r : __int_as_float(0x7fc00000));
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
//   T[t,s] = b_t exp(G_t - G_s) k_t . k_s  (s < t),   X = (I + T)^-1 diag(b),   R = V - diag(exp G) K S^T,   U = X R
//   M[t,s] = exp(G_t - G_s) q_t . k_s  (s <= t),      O = diag(exp G) Q S^T + (M X) R
//   S <- exp(G_end) S + sum_s (exp(G_end - G_s) u_s) k_s^T
// X and M X do not depend on the state: delta_prepare_kernel forms them for all chunks at once.  What is left goes chunk after chunk,
// but every row of S (a value channel) by itself: delta_walk_kernel gives a workgroup 16 channels of a head.
// The lengths of q and k are float32 factors of rows and columns, so that k and q enter the products as they were given, exact in
// bfloat16.  A computed factor (X, R, U, S) is carried as three bfloat16 terms, which hold all of a float32 (8 bits each, cut off, not
// rounded, so that what is left is exact), and of the products of two such all but the three smallest are formed: states and outputs are
// float32 results.  Two terms were off by 3e-6 of a state; an output is the difference of Q S^T and (M X) R, and where values of a
// thousandth replaced what the state held, two terms of S, R and M X lost a tenth of it.
// The triangular systems are solved, not expanded: powers of T grow like binomials where keys lean to one side, the inverse does not.
// Fragments of v_mfma_f32_16x16x32_bf16: lane l has row (or column) l % 16 and eight consecutive k from 8 (l / 16); of the result
// column l % 16, rows 4 (l / 16) .. + 3.  What the preparation leaves for the walk is stored in that order, a kilobyte a fragment.
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef float f32x4_t __attribute__((ext_vector_type(4)));

constexpr int kC = kDeltaChunk;                                   // tokens of a chunk
constexpr int kTiles = 6;                                         // 16 x 32 fragments of a lower triangle: 1, 1, 2, 2 to a row of tiles
constexpr int kFrag = 512;                                        // bf16 of a fragment
constexpr int kTri = kTiles * kFrag;
constexpr int kScalars = 256;                                     // floats, four to a token: its factors of k S and of q S, the chunk's decay
// 16-bit words of a chunk and head: X times the decay to the end, M X (three terms each), scalars
constexpr int kAtMX = 3 * kTri, kAtScalars = 6 * kTri, kChunkHalves = 6 * kTri + 2 * kScalars;
static_assert(kC == 64 && kChunkHalves == kDeltaChunkHalves, "as the workspace is planned");
__device__ __forceinline__ int tile_at(int t_tile, int k_step) { return (t_tile < 2 ? t_tile : 2 * t_tile - 2) + k_step; }

__device__ __forceinline__ bf16x8 as_frag(uint4 q) { return __builtin_bit_cast(bf16x8, q); }
__device__ __forceinline__ bf16x8 as_frag(uint2 a, uint2 b) { return as_frag(make_uint4(a.x, a.y, b.x, b.y)); }
__device__ __forceinline__ bf16x8 lds_frag(const uint16_t *p) { return as_frag(*reinterpret_cast<const uint4 *>(p)); }
__device__ __forceinline__ f32x4_t mma(bf16x8 a, bf16x8 b, f32x4_t c) { return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0); }
__device__ __forceinline__ f32x4_t mma(float a, float b, f32x4_t c) { return __builtin_amdgcn_mfma_f32_16x16x4f32(a, b, c, 0, 0, 0); }

// the upper halves of four values, in order, and what they leave of them
__device__ __forceinline__ uint2 take_top(f32x4_t &v)
{
    const uint32_t a = __float_as_uint(v[0]), b = __float_as_uint(v[1]), c = __float_as_uint(v[2]), d = __float_as_uint(v[3]);
    const uint2 top = make_uint2(__builtin_amdgcn_perm(b, a, 0x07060302), __builtin_amdgcn_perm(d, c, 0x07060302));
    v[0] -= __uint_as_float(a & 0xffff0000u), v[1] -= __uint_as_float(b & 0xffff0000u);
    v[2] -= __uint_as_float(c & 0xffff0000u), v[3] -= __uint_as_float(d & 0xffff0000u);
    return top;
}
// four values as three bfloat16 terms
struct Terms {
    uint2 hi, mid, lo;
};
__device__ __forceinline__ Terms terms_of(f32x4_t v)
{
    Terms t;
    t.hi = take_top(v);
    t.mid = take_top(v);
    t.lo = take_top(v);
    return t;
}
__device__ __forceinline__ void put(uint16_t *p, uint2 v) { *reinterpret_cast<uint2 *>(p) = v; }

// Workgroup barrier for what is exchanged through LDS; global loads and stores in flight stay there.
__device__ __forceinline__ void lds_barrier()
{
    __builtin_amdgcn_fence(__ATOMIC_RELEASE, "workgroup", "local");
    __builtin_amdgcn_s_barrier();
    __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "workgroup", "local");
}

// 16-bit words of a chunk and key head: K and Q as fragments
template <int N> constexpr int kKeyHalves = 2 * N * kC;
// x[i] += t[i] of lane J (of its 16) times x[J], for the rows i behind J, and on with the next row: a unit lower triangular system, the
// right-hand side's rows in x, minus the matrix's rows in t
template <int J> __device__ __forceinline__ void substitute(const float (&t)[16], float (&x)[16])
{
    if constexpr (J < 15) {
#pragma unroll
        for (int i = J + 1; i < 16; ++i) {
            const float row = __builtin_bit_cast(float, __builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, t[i]), 0x150 + J, 0xf, 0xf, true));
            x[i] = fmaf(row, x[J], x[i]);
        }
        substitute<J + 1>(t, x);
    }
}
// The state that row `row` of tile `tile` of 16 stands for: with 128 states pairs of tiles take turns of four, so that a lane's four of
// both are eight adjacent ones, as a fragment of K has them.
template <int N> __device__ __forceinline__ int state_of(int tile, int row)
{
    return N == 64 ? tile * 16 + row : (tile >> 1) * 32 + (row >> 2) * 8 + (tile & 1) * 4 + (row & 3);
}

// One chunk of one head.  Eight wavefronts, and what the chain of phases needs comes first: T by all of them; then one inverts the blocks
// on its diagonal while the others form M and write the fragments of keys and queries.
// Bound by the latency of those phases, three workgroups to a CU: one chunk 6.9 us, 768 chunks (24 heads, N = 128) 16.9, 1504 (32 heads, N = 128)
// 29, which then write their 82 MB at 2.8 TB/s.
// grid: (chunks of the slab, H, batch); tok_slab: the slab's first token
constexpr int kPrepThreads = 512;
template <int N>
__global__ void __launch_bounds__(kPrepThreads) __attribute__((amdgpu_waves_per_eu(6)))
delta_prepare_kernel(const bf16_t *__restrict__ q, const bf16_t *__restrict__ k, const bf16_t *__restrict__ dt, const bf16_t *__restrict__ beta,
                     const float *__restrict__ A, const float *__restrict__ dt_bias, uint16_t *__restrict__ ws, uint16_t *__restrict__ frags,
                     int64_t tok_slab, int64_t L, int64_t H, int64_t group, DeltaOptions o)
{
    constexpr int kRow = N + 8, kSys = kC + 4;
    // T, then M X; K, then (I + T)^-1; Q, then M: 53 KB, so that three workgroups share a CU
    __shared__ __attribute__((aligned(16))) float sys[kC * kSys], inv[kC * kSys], mq[kC * kSys];
    __shared__ __attribute__((aligned(16))) float rk[kC], rq[kC], G[kC], G_rest[kC], bt[kC];
    uint16_t *ks = reinterpret_cast<uint16_t *>(inv), *qs = reinterpret_cast<uint16_t *>(mq);
    static_assert(sizeof(uint16_t) * kC * kRow <= sizeof(mq), "k and q share their places");
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), c16 = lane & 15, g4 = lane >> 4;
    const int64_t chunk = blockIdx.x, n_chunks = gridDim.x, h = blockIdx.y, b = blockIdx.z;
    const int64_t Hk = H / group, hk = h / group, tok0 = tok_slab + chunk * kC;
    const int live = (int)min((int64_t)kC, L - tok0);             // tokens of this chunk
    ws += ((b * H + h) * n_chunks + chunk) * kChunkHalves;

    // keys and queries into LDS (rows behind the end: zeros)
    constexpr int kPieces = N / 8, kMine = kC * kPieces / kPrepThreads;   // 16-byte pieces of a row, on as many adjacent lanes
    uint4 kp[kMine], qp[kMine];
    const int64_t first = ((b * L + tok0) * Hk + hk) * N;
#pragma unroll
    for (int i = 0; i < kMine; ++i) {
        const int id = i * kPrepThreads + tid, row = id / kPieces, piece = id % kPieces;
        const uint32_t at = (uint32_t)min(row, live - 1) * (uint32_t)(Hk * N) + (uint32_t)(piece * 8);
        kp[i] = *reinterpret_cast<const uint4 *>(k + first + at);
        qp[i] = *reinterpret_cast<const uint4 *>(q + first + at);
    }
    // running sum of delta A (in powers of two) and the write strengths; tokens behind the end neither decay nor write.  The decay from a token
    // to another is a difference of two sums, and a token that resets the state leaves large ones behind it: they are formed in
    // float64 and kept as two float32, of which the differences are formed one by one (a single float32 was off by 5e-4 of the decays
    // behind one of 2^-10000).  A token's exponent ends at -160, which leaves nothing of anything: no infinities are subtracted (a NaN passes).
    if (wave == 7) {
        const int64_t at = (b * L + tok0 + min(lane, live - 1)) * H + h;
        const float x = bf16_to_f32(dt[at]) + (dt_bias ? dt_bias[h] : 0.0f), w = bf16_to_f32(beta[at]);
        const float own = lane < live ? (o.softplus ? softplus_f32(x) : x) * A[h] * kLog2e : 0.0f;
        double sum = own < -160.0f ? -160.0f : own;
        sum += lanes_back<0x111>(sum);
        sum += lanes_back<0x112>(sum);
        sum += lanes_back<0x114>(sum);
        sum += lanes_back<0x118>(sum);
        const double r0 = of_lane(sum, 15), r1 = of_lane(sum, 31), r2 = of_lane(sum, 47);
        sum += g4 == 0 ? 0.0 : g4 == 1 ? r0 : g4 == 2 ? r0 + r1 : (r0 + r1) + r2;
        G[lane] = (float)sum;
        G_rest[lane] = (float)(sum - (double)(float)sum);
        const float b = lane < live ? (o.sigmoid ? sigmoid_f32(w) : w) : 0.0f;
        bt[lane] = finite((float)sum) ? b : __int_as_float(0x7fc00000);
    }
#pragma unroll
    for (int i = 0; i < kMine; ++i) {
        const int id = i * kPrepThreads + tid, row = id / kPieces, piece = id % kPieces;
        if (row >= live) kp[i] = qp[i] = make_uint4(0, 0, 0, 0);
        *reinterpret_cast<uint4 *>(&ks[row * kRow + piece * 8]) = kp[i];
        *reinterpret_cast<uint4 *>(&qs[row * kRow + piece * 8]) = qp[i];
    }
    lds_barrier();
    // one over the lengths of keys (wavefronts 0 .. 3) and queries: the diagonal of a tile of K K^T or Q Q^T
    {
        const int t_tile = wave & 3, t = t_tile * 16 + c16;
        const uint16_t *rows = wave < 4 ? ks : qs;
        f32x4_t acc = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
        for (int i = 0; i < N / 32; ++i) {
            const bf16x8 f = lds_frag(&rows[t * kRow + i * 32 + g4 * 8]);
            // (where no lengths are asked for, times zeros: 0, or NaN for a row that is no numbers, however long)
            acc = mma(f, o.qk_norm ? f : as_frag(make_uint4(0, 0, 0, 0)), acc);
        }
        const float square = (c16 & 2) ? (c16 & 1) ? acc[3] : acc[2] : (c16 & 1) ? acc[1] : acc[0];
        const float inverse = t >= live ? 0.0f : o.qk_norm ? 1.0f / sqrtf(square + o.eps) : 1.0f;
        if (g4 == c16 >> 2) (wave < 4 ? rk : rq)[t] = wave >= 4 ? inverse * o.scale : finite(square) ? inverse : __int_as_float(0x7fc00000);
    }
    lds_barrier();
    // From the first token on whose key, decay or write strength is not a number the state is none either, and so are the outputs: such tokens
    // are left out of the chunk's systems, where products with the zeros above a diagonal would take them to the tokens ahead, and their
    // factors say so.  (A query is a row of its own, a value a channel: the walk sees to it.)
    const uint64_t no_key = __ballot(!finite(rk[lane])), none = no_key | __ballot(!finite(bt[lane]));
    const int good = none ? __builtin_ctzll(none) : kC, keys = no_key ? __builtin_ctzll(no_key) : kC;
    auto row_end = [&](int t, int end) { return t < good ? end : 0; };

    // T and M, tile by tile of 16 x 16: lane has token t = l % 16 of the tile and four s.  The ten tiles of a lower triangle by number:
    // row 0 of tiles, row 1, ...
    auto tile_row = [](int i) { return i < 1 ? 0 : i < 3 ? 1 : i < 6 ? 2 : 3; };
    auto tile = [&](const uint16_t *rows, int t_tile, int s_tile) {
        const int t = t_tile * 16 + c16, s0 = s_tile * 16 + 4 * g4;
        bf16x8 of_s[N / 32], of_t[N / 32];
#pragma unroll
        for (int i = 0; i < N / 32; ++i) {
            of_s[i] = lds_frag(&ks[(s_tile * 16 + c16) * kRow + i * 32 + g4 * 8]);
            of_t[i] = lds_frag(&rows[t * kRow + i * 32 + g4 * 8]);
        }
        const float4 Gs = *reinterpret_cast<const float4 *>(&G[s0]), Gr = *reinterpret_cast<const float4 *>(&G_rest[s0]);
        const float4 rs = *reinterpret_cast<const float4 *>(&rk[s0]);
        const float Gt = G[t], Gtr = G_rest[t];
        f32x4_t acc = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
        for (int i = 0; i < N / 32; ++i) acc = mma(of_s[i], of_t[i], acc);
        acc[0] *= exp2_hw((Gt - Gs.x) + (Gtr - Gr.x)) * rs.x, acc[1] *= exp2_hw((Gt - Gs.y) + (Gtr - Gr.y)) * rs.y;
        acc[2] *= exp2_hw((Gt - Gs.z) + (Gtr - Gr.z)) * rs.z, acc[3] *= exp2_hw((Gt - Gs.w) + (Gtr - Gr.w)) * rs.w;
        return acc;
    };
    for (int i = wave; i < 10; i += 8) {
        const int t_tile = tile_row(i), s_tile = i - t_tile * (t_tile + 1) / 2, t = t_tile * 16 + c16, s0 = s_tile * 16 + 4 * g4;
        f32x4_t v = tile(ks, t_tile, s_tile);
        const float f = bt[t] * rk[t];
#pragma unroll
        for (int j = 0; j < 4; ++j) v[j] = s0 + j < row_end(t, t) ? v[j] * f : 0.0f;
        *reinterpret_cast<f32x4_t *>(&sys[t * kSys + s0]) = v;
    }
    lds_barrier();

    f32x4_t m[2];                                                 // wavefronts 1 .. 7: tiles wave - 1 and wave + 6 of M
    float x[16];                                                  // wavefront 0: a column of a block of (I + T)^-1
    if (wave == 0) {
        // (I + T)^-1: the four 16 x 16 blocks on the diagonal by substitution, a block to 16 lanes and a column to a lane.  A lane has its
        // column of T as well, and hands its entry of a row to the 15 others as the operand of their multiplication.
        const float *d = sys + g4 * 16 * kSys + g4 * 16 + c16;
        float t[16];
#pragma unroll
        for (int i = 0; i < 16; ++i) t[i] = -d[i * kSys], x[i] = i == c16 ? 1.0f : 0.0f;
        substitute<0>(t, x);
    } else {
#pragma unroll
        for (int j = 0; j < 2; ++j) {
            const int i = 7 * j + wave - 1;
            if (i >= 10) continue;
            const int t_tile = tile_row(i), s_tile = i - t_tile * (t_tile + 1) / 2, t = t_tile * 16 + c16, s0 = s_tile * 16 + 4 * g4;
            m[j] = tile(qs, t_tile, s_tile);
            const float f = rq[t];
#pragma unroll
            for (int n = 0; n < 4; ++n) m[j][n] = s0 + n < row_end(t, t + 1) ? m[j][n] * f : 0.0f;
        }
        // keys and queries as the fragments that the walk takes: once for the value heads that share them
        if (h % group == 0) {
            uint16_t *to = frags + ((b * Hk + hk) * n_chunks + chunk) * kKeyHalves<N> + lane * 8;
            for (int f = wave - 1; f < N / 8; f += 7) {
                // K: rows are tokens, columns the states of the walk's wavefront f / (N / 32); with 64 states two tiles of tokens side by side
                // (none of those from the first on that is not a number)
                uint4 piece;
                if constexpr (N == 128) {
                    piece = *reinterpret_cast<const uint4 *>(&ks[((f & 3) * 16 + c16) * kRow + (f >> 2) * 32 + 8 * g4]);
                    if ((f & 3) * 16 + c16 >= keys) piece = make_uint4(0, 0, 0, 0);
                } else {
                    const uint16_t *at = &ks[((f & 1) * 32 + c16) * kRow + (f >> 1) * 16 + 4 * g4];
                    const uint2 lo = *reinterpret_cast<const uint2 *>(at), hi = *reinterpret_cast<const uint2 *>(at + 16 * kRow);
                    piece = make_uint4(lo.x, lo.y, hi.x, hi.y);
                    if ((f & 1) * 32 + c16 >= keys) piece.x = piece.y = 0;
                    if ((f & 1) * 32 + 16 + c16 >= keys) piece.z = piece.w = 0;
                }
                *reinterpret_cast<uint4 *>(to + f * kFrag) = piece;
                // Q: rows are tokens, columns states
                *reinterpret_cast<uint4 *>(to + N * kC + f * kFrag) =
                    *reinterpret_cast<const uint4 *>(&qs[((f / (N / 32)) * 16 + c16) * kRow + (f % (N / 32)) * 32 + 8 * g4]);
            }
        }
    }
    lds_barrier();
    if (wave == 0) {
        float *to = inv + g4 * 16 * kSys + g4 * 16 + c16;
#pragma unroll
        for (int i = 0; i < 16; ++i) to[i * kSys] = x[i];
    } else {
#pragma unroll
        for (int j = 0; j < 2; ++j) {
            const int i = 7 * j + wave - 1, t_tile = tile_row(i), s_tile = i - t_tile * (t_tile + 1) / 2;
            if (i < 10) *reinterpret_cast<f32x4_t *>(&mq[(t_tile * 16 + c16) * kSys + s_tile * 16 + 4 * g4]) = m[j];
        }
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
    if (wave < 4) {
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
    // M X, block by block into T's place (lane has token t and four adjacent s), the longer sums by the wavefronts that have no X to write
    auto out_block = [&](int row, int col) {
        f32x4_t acc = zero;
        for (int mid = col; mid <= row; ++mid) {
            const f32x4_t a = *reinterpret_cast<const f32x4_t *>(&mq[(row * 16 + c16) * kSys + mid * 16 + 4 * g4]);
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const int j = mid * 16 + 4 * g4 + i, s = col * 16 + c16;
                acc = mma(s <= j ? inv[j * kSys + s] : 0.0f, a[i], acc);
            }
        }
        *reinterpret_cast<f32x4_t *>(&sys[(row * 16 + c16) * kSys + col * 16 + 4 * g4]) = acc;
    };
    // a fragment of a lower triangle of LDS, its columns times the write strengths, its rows times f, in terms
    auto fragment = [&](const float *rows, int t, int s0, float f, Terms (&w)[2]) {
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            f32x4_t v = *reinterpret_cast<const f32x4_t *>(&rows[t * kSys + s0 + 4 * i]);
            const f32x4_t strength = *reinterpret_cast<const f32x4_t *>(&bt[s0 + 4 * i]);
#pragma unroll
            for (int j = 0; j < 4; ++j) v[j] = s0 + 4 * i + j < row_end(t, t + 1) ? v[j] * strength[j] * f : 0.0f;
            w[i] = terms_of(v);
        }
    };
    auto write = [&](int at, uint2 lo, uint2 hi) { *reinterpret_cast<uint4 *>(ws + at) = make_uint4(lo.x, lo.y, hi.x, hi.y); };
    const float end = G[kC - 1], end_rest = G_rest[kC - 1];
    if (wave < 4) {
        // X times the decay to the end of the chunk, in three terms
        const int t = wave * 16 + c16;
        const float f = rk[t] * exp2_hw((end - G[t]) + (end_rest - G_rest[t]));
        for (int step = 0; step <= wave >> 1; ++step) {
            const int at = tile_at(wave, step) * kFrag + lane * 8;
            Terms w[2];
            fragment(inv, t, step * 32 + g4 * 8, f, w);
            write(at, w[0].hi, w[1].hi), write(kTri + at, w[0].mid, w[1].mid), write(2 * kTri + at, w[0].lo, w[1].lo);
        }
        if (wave == 0) out_block(3, 2);
        else if (wave == 1) out_block(3, 3), out_block(2, 2);
        else if (wave == 2) out_block(1, 1);
    } else if (wave == 4) {
        out_block(3, 0);
    } else if (wave == 5) {
        out_block(3, 1), out_block(0, 0);
    } else if (wave == 6) {
        out_block(2, 0);
        const float e = exp2_hw(G[lane]);
        const float nan = __int_as_float(0x7fc00000);
        reinterpret_cast<float4 *>(ws + kAtScalars)[lane] =
            make_float4(lane < good ? rk[lane] * e : 0.0f, lane < good ? rq[lane] * e : nan, good == kC ? exp2_hw(end) : nan, 0.0f);
    } else {
        out_block(1, 0), out_block(2, 1);
    }
    lds_barrier();
    if (wave < kTiles) {
        const int t_tile = wave < 2 ? wave : wave < 4 ? 2 : 3, step = wave < 2 ? 0 : wave & 1, at = kAtMX + wave * kFrag + lane * 8;
        Terms w[2];
        fragment(sys, t_tile * 16 + c16, step * 32 + g4 * 8, 1.0f, w);
        write(at, w[0].hi, w[1].hi), write(kTri + at, w[0].mid, w[1].mid), write(2 * kTri + at, w[0].lo, w[1].lo);
    }
}

// The chunks of one (batch row, head) in order, for 16 of its channels.  Two roles of four wavefronts, three barriers to a chunk:
//   chain    wavefront w keeps the states n of the w-th quarter in MFMA accumulators (lane: a channel, four adjacent states), which are
//            the right operand of K S^T as they lie there: the contraction over n takes a lane group's states in any order, if K is
//            read in the same one.  Every wavefront leaves its part of K S^T for all 64 tokens in LDS                        | A
//            adds up the parts of the 16 tokens 16 w ..: R, three terms                                                   | B
//            U = X R of those tokens, with their decay to the end                                                         | C
//            the write to its states
//   outputs  wavefront w has the tokens 16 w ..: Q S^T after B, (M X) R after C, gate and store, with the next chunk under way in the chain
// All operands but S, R and U come from memory, requested a chunk ahead, into the registers that the last use has just left: with two sets used in
// turn a wavefront has more than 128 registers, a CU holds one workgroup, and 4 contexts of 1000 tokens of 16 heads of 128 x 128 took 48 us
// where they took 39 with one; alone on its CU a workgroup is no slower for it.
// Bound by the latency of a chunk's chain: N = 64 1.1, N = 128 1.25 us (3000 cycles: terms of S 360, K S^T 400, sum, K^T and R 520, U 220 to 350, its
// terms 250, the write to S 690, the rest barriers); 24 heads of N = 128, P = 64 and 2048 tokens 43 us, of which the matrix cores of the CUs that
// have a workgroup are busy for a third.  With two workgroups to a CU (the 4 contexts: 42 us) they are for 42 %.
struct WalkArgs {
    const bf16_t *v, *z;
    const uint16_t *ws, *frags;
    const float *h0;
    float *h_final;
    bf16_t *out;
    float *raw;
    float *starts, *map;                                          // of parts of the slab
    int64_t L, H, group, heads, tok0, n_chunks, part;             // (of the slab: its first token and its chunks; chunks of a part)
    uint32_t first_part, walked, maps;                            // the parts walked for their outputs, and how many of those from 1 on for their maps
    int P;
};
constexpr int kWalkPlain = 0, kWalkGate = 1, kWalkRaw = 2;        // outputs as they are, gated, or in float32 for the norm
constexpr int kRowV = kC + 4;
// What is exchanged lies in LDS as the fragments that will be read, a kilobyte each: whole lines both ways, no bank conflicts.
template <int N> struct __attribute__((aligned(16))) WalkLds {
    float part[4 * 4 * 256];                                      // parts of K S^T, [token tile][wavefront][lane][4]
    uint16_t s_hi[N / 32 * kFrag], s_mid[N / 32 * kFrag], s_lo[N / 32 * kFrag];   // S, channels by states
    uint16_t r_hi[2 * kFrag], r_mid[2 * kFrag], r_lo[2 * kFrag];  // R, channels by tokens
    uint16_t u_hi[2 * kFrag], u_mid[2 * kFrag], u_lo[2 * kFrag];  // decayed U
    uint16_t v[2][16 * kRowV];                                    // V, [channel][token], two chunks
    float factors[2][3][kC];                                      // of the rows of K S^T and of Q S^T; the chunk's decay
    float o[4][16 * 16];                                          // a wavefront's outputs, [token][channel]
    int ended[4];                                                 // has a wavefront come by a value that is not a number
    int ends[16];                                                 // if one has: a channel's first token (of the part) with such a value
};
// Where a workgroup and a lane are.
template <int N> struct WalkPlace {
    int lane, wave, c16, g4, p0;
    int unit;                                                     // the first of the 16 unit vectors that are the start; -1: none
    int64_t hb, b, h, Hk, hk;
    int64_t tok0, first, n_chunks;                                // its part of the slab: first token, chunks ahead of it, chunks
    const float *h0;                                              // the 16 rows of the state that it has, ahead and behind (or NULL)
    float *h_final;
    const uint16_t *own, *frags;                                  // the head's and the key head's parts of the workspace
    uint32_t value_row;                                           // elements of a token
    // where the four adjacent k from 16 tile + 4 g4 of row c16 lie in fragments, and where a lane's eight of fragment i
    __device__ __forceinline__ int in_frags(int tile) const { return (tile >> 1) * kFrag + (c16 + 16 * ((tile & 1) * 2 + (g4 >> 1))) * 8 + 4 * (g4 & 1); }
    __device__ __forceinline__ int of_lane(int i) const { return i * kFrag + lane * 8; }
};
// A request for a later chunk goes out where its registers are free, and stays there: the compiler would move it.
__device__ __forceinline__ void requested() { __builtin_amdgcn_sched_barrier(0); }
// An operand of the chunks in order, by running address (an address formed anew from the chunk's number is some 20 scalar instructions
// of a wavefront that has none to spare); behind the last chunk it stays there.
template <typename T> struct Cursor {
    const T *p;
    int64_t stride;
    int left;                                                     // chunks behind this one
    __device__ __forceinline__ void advance()
    {
        p += left > 0 ? stride : 0;
        left -= left > 0;
    }
};

template <int N> __device__ __forceinline__ bool any_ended(const WalkLds<N> &lds)
{
    return __builtin_amdgcn_readfirstlane(lds.ended[0] | lds.ended[1] | lds.ended[2] | lds.ended[3]) != 0;
}

// TWO: the wavefront's row of tiles has two fragments of 32 columns (wavefronts 2 and 3)
template <int N, bool TWO> __device__ __forceinline__ void walk_chain(const WalkArgs &a, const WalkPlace<N> &me, WalkLds<N> &lds)
{
    constexpr int kNT = N / 64, kX = TWO ? 2 : 1;
    const f32x4_t zero = {0.0f, 0.0f, 0.0f, 0.0f};
    const int n_chunks = (int)me.n_chunks;
    const uint32_t lane8 = (uint32_t)me.lane * 8;
    // (the state ahead of the operands: what the loop waits for at its head is then never what it has just requested)
    f32x4_t acc[kNT];                                             // [j][i]: state_of(kNT wave + j, 4 g4 + i) of channel p0 + c16
#pragma unroll
    for (int j = 0; j < kNT; ++j) {
        const int n = state_of<N>(me.wave * kNT + j, 4 * me.g4);
        acc[j] = zero;
        if (me.h0) acc[j] = *reinterpret_cast<const f32x4_t *>(me.h0 + me.c16 * N + n);
#pragma unroll
        for (int i = 0; i < 4; ++i)
            if (me.unit >= 0 && n + i == me.unit + me.c16) acc[j][i] = 1.0f;
    }
    struct Operands {
        uint2 k[4][kNT];
        uint4 x[3][kX];
    };
    Cursor<uint16_t> keys{me.frags + me.wave * kNT * 2 * kFrag, kKeyHalves<N>, n_chunks - 1}, xs{me.own, kChunkHalves, n_chunks - 1};
    auto fetch_k = [&](Operands &f) {
        if constexpr (kNT == 2) {
#pragma unroll
            for (int t = 0; t < 4; ++t) {
                const uint4 both_tiles = *reinterpret_cast<const uint4 *>(keys.p + t * kFrag + lane8);
                f.k[t][0] = make_uint2(both_tiles.x, both_tiles.y), f.k[t][1] = make_uint2(both_tiles.z, both_tiles.w);
            }
        } else {
#pragma unroll
            for (int t = 0; t < 4; t += 2) {
                const uint4 two_rows = *reinterpret_cast<const uint4 *>(keys.p + t / 2 * kFrag + lane8);
                f.k[t][0] = make_uint2(two_rows.x, two_rows.y), f.k[t + 1][0] = make_uint2(two_rows.z, two_rows.w);
            }
        }
        keys.advance();
        requested();
    };
    auto fetch_x = [&](Operands &f) {
#pragma unroll
        for (int n = 0; n < 3; ++n)
#pragma unroll
            for (int i = 0; i < kX; ++i) f.x[n][i] = *reinterpret_cast<const uint4 *>(xs.p + n * kTri + tile_at(me.wave, i) * kFrag + lane8);
        xs.advance();
        requested();
    };
    // K^T of the wavefront's states is its K times a choice of columns: a product gives it exactly, lane a state, four adjacent tokens
    bf16x8 choice[kNT];
#pragma unroll
    for (int j = 0; j < kNT; ++j) {
        const uint32_t one = me.g4 == me.c16 >> 2 ? (me.c16 & 1 ? 0x3f800000u : 0x3f80u) : 0u, lo = me.c16 & 2 ? 0u : one, hi = me.c16 & 2 ? one : 0u;
        choice[j] = j == 0 ? as_frag(make_uint2(lo, hi), make_uint2(0, 0)) : as_frag(make_uint2(0, 0), make_uint2(lo, hi));
    }
    auto transposed = [&](const Operands &f, int t, int j) {
        const f32x4_t d = mma(kNT == 2 ? as_frag(f.k[t][0], f.k[t][kNT - 1]) : as_frag(f.k[t][0], f.k[t][0]), choice[j], zero);
        return make_uint2(__builtin_amdgcn_perm(__float_as_uint(d[1]), __float_as_uint(d[0]), 0x07060302),
                          __builtin_amdgcn_perm(__float_as_uint(d[3]), __float_as_uint(d[2]), 0x07060302));
    };
    Operands f;
    fetch_k(f), fetch_x(f);
    __builtin_amdgcn_s_setprio(1);                                // the chain's instructions ahead of the other role's
    const int at = me.in_frags(me.wave);
    // the write to the state takes the tokens of two tiles in turns of four, as K^T comes out of its products
    const int u_at = me.of_lane(me.wave >> 1) + 4 * (me.wave & 1);
    // (requests go out where the wavefront waits for LDS anyway: a request holds its wavefront for some 14 cycles, and 12 of them at once
    // are a sixth of a chunk)
    auto step = [&](int parity) __attribute__((always_inline)) {
        Terms s[kNT];
#pragma unroll
        for (int j = 0; j < kNT; ++j) s[j] = terms_of(acc[j]);
        if constexpr (kNT == 2) {
            *reinterpret_cast<uint4 *>(&lds.s_hi[me.of_lane(me.wave)]) = make_uint4(s[0].hi.x, s[0].hi.y, s[1].hi.x, s[1].hi.y);
            *reinterpret_cast<uint4 *>(&lds.s_mid[me.of_lane(me.wave)]) = make_uint4(s[0].mid.x, s[0].mid.y, s[1].mid.x, s[1].mid.y);
            *reinterpret_cast<uint4 *>(&lds.s_lo[me.of_lane(me.wave)]) = make_uint4(s[0].lo.x, s[0].lo.y, s[1].lo.x, s[1].lo.y);
        } else {
            put(&lds.s_hi[at], s[0].hi);
            put(&lds.s_mid[at], s[0].mid);
            put(&lds.s_lo[at], s[0].lo);
        }
        f32x4_t sum[4];
        if constexpr (kNT == 2) {
#pragma unroll
            for (int t = 0; t < 4; ++t) sum[t] = mma(as_frag(f.k[t][0], f.k[t][1]), as_frag(s[0].lo, s[1].lo), zero);
#pragma unroll
            for (int t = 0; t < 4; ++t) sum[t] = mma(as_frag(f.k[t][0], f.k[t][1]), as_frag(s[0].mid, s[1].mid), sum[t]);
#pragma unroll
            for (int t = 0; t < 4; ++t) sum[t] = mma(as_frag(f.k[t][0], f.k[t][1]), as_frag(s[0].hi, s[1].hi), sum[t]);
        } else {                                                  // 16 states a wavefront: two terms to a product, the keys twice
#pragma unroll
            for (int t = 0; t < 4; ++t) sum[t] = mma(as_frag(f.k[t][0], f.k[t][0]), as_frag(s[0].lo, make_uint2(0, 0)), zero);
#pragma unroll
            for (int t = 0; t < 4; ++t) sum[t] = mma(as_frag(f.k[t][0], f.k[t][0]), as_frag(s[0].mid, s[0].hi), sum[t]);
        }
#pragma unroll
        for (int t = 0; t < 4; ++t) *reinterpret_cast<f32x4_t *>(&lds.part[(t * 4 + me.wave) * 256 + me.lane * 4]) = sum[t];
        lds_barrier();                                            // A
        f32x4_t r[4];
#pragma unroll
        for (int w = 0; w < 4; ++w) r[w] = *reinterpret_cast<const f32x4_t *>(&lds.part[(me.wave * 4 + w) * 256 + me.lane * 4]);
        const uint2 values = *reinterpret_cast<const uint2 *>(&lds.v[parity][me.c16 * kRowV + me.wave * 16 + 4 * me.g4]);
        const f32x4_t k_factor = *reinterpret_cast<const f32x4_t *>(&lds.factors[parity][0][me.wave * 16 + 4 * me.g4]);
        const float decay = lds.factors[parity][2][0];
        uint2 kt[4][kNT];
#pragma unroll
        for (int t = 0; t < 4; ++t)
#pragma unroll
            for (int j = 0; j < kNT; ++j) kt[t][j] = transposed(f, t, j);
        fetch_k(f);
        r[0] = (r[0] + r[1]) + (r[2] + r[3]);
        r[0][0] = fmaf(-k_factor[0], r[0][0], bf16_lo(values.x)), r[0][1] = fmaf(-k_factor[1], r[0][1], bf16_hi(values.x));
        r[0][2] = fmaf(-k_factor[2], r[0][2], bf16_lo(values.y)), r[0][3] = fmaf(-k_factor[3], r[0][3], bf16_hi(values.y));
        const Terms rt = terms_of(r[0]);
        put(&lds.r_hi[at], rt.hi);
        put(&lds.r_mid[at], rt.mid);
        put(&lds.r_lo[at], rt.lo);
        lds_barrier();                                            // B
        bf16x8 rf[3][kX];
#pragma unroll
        for (int i = 0; i < kX; ++i) {
            const int from = me.of_lane(i);
            rf[0][i] = lds_frag(&lds.r_hi[from]), rf[1][i] = lds_frag(&lds.r_mid[from]), rf[2][i] = lds_frag(&lds.r_lo[from]);
        }
        f32x4_t u[2] = {zero, zero};
#pragma unroll
        for (int i = 0; i < kX; ++i) {
            const bf16x8 xh = as_frag(f.x[0][i]), xm = as_frag(f.x[1][i]), xl = as_frag(f.x[2][i]);
            u[1] = mma(xl, rf[0][i], u[1]);
            u[0] = mma(xm, rf[0][i], u[0]);
            u[1] = mma(xh, rf[2][i], u[1]);
            u[0] = mma(xh, rf[1][i], u[0]);
            u[1] = mma(xm, rf[1][i], u[1]);
            u[0] = mma(xh, rf[0][i], u[0]);
        }
        const Terms ut = terms_of(u[0] + u[1]);
        put(&lds.u_hi[u_at], ut.hi);
        put(&lds.u_mid[u_at], ut.mid);
        put(&lds.u_lo[u_at], ut.lo);
#pragma unroll
        for (int j = 0; j < kNT; ++j) acc[j] *= decay;
        lds_barrier();                                            // C
        bf16x8 uf[3][2];
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            const int from = me.of_lane(i);
            uf[0][i] = lds_frag(&lds.u_lo[from]), uf[1][i] = lds_frag(&lds.u_mid[from]), uf[2][i] = lds_frag(&lds.u_hi[from]);
        }
        fetch_x(f);
#pragma unroll
        for (int n = 0; n < 3; ++n)
#pragma unroll
            for (int i = 0; i < 2; ++i)
#pragma unroll
                for (int j = 0; j < kNT; ++j) acc[j] = mma(as_frag(kt[2 * i][j], kt[2 * i + 1][j]), uf[n][i], acc[j]);
    };
    int left = n_chunks;
    for (; left > 1; left -= 2) {
        step(0);
        step(1);
    }
    if (left > 0) step(0);
    lds_barrier();                                                // (a value that is not a number: the other role says whether, and then where)
    if (any_ended(lds)) {
        __syncthreads();
        if (lds.ends[me.c16] != INT32_MAX)
#pragma unroll
            for (int j = 0; j < kNT; ++j) acc[j] = zero + __int_as_float(0x7fc00000);
    }
    if (me.h_final)
#pragma unroll
        for (int j = 0; j < kNT; ++j)
            *reinterpret_cast<f32x4_t *>(me.h_final + me.c16 * N + state_of<N>(me.wave * kNT + j, 4 * me.g4)) = acc[j];
}

// OUT: or no outputs, only the values for the other role
template <int N, int MODE, bool TWO, bool OUT> __device__ __forceinline__ void walk_outputs(const WalkArgs &a, const WalkPlace<N> &me, WalkLds<N> &lds)
{
    constexpr int kSteps = N / 32, kX = TWO ? 2 : 1;
    const f32x4_t zero = {0.0f, 0.0f, 0.0f, 0.0f};
    const int n_chunks = (int)me.n_chunks;
    const uint32_t lane8 = (uint32_t)me.lane * 8;
    // V, the gates and the outputs: token lane / 4 of the wavefront's 16, four channels, so that four adjacent lanes have a row's 32 bytes
    // (a request costs a cycle for every run of adjacent lanes that reads adjacent bytes: 64 of them as a fragment has its rows).
    // Behind the end: the last token again.
    const int t_own = me.wave * 16 + (me.lane >> 2), p_own = 4 * (me.lane & 3);
    const uint32_t live = (uint32_t)min((int64_t)kC, a.L - me.tok0 - (int64_t)(n_chunks - 1) * kC);
    const uint32_t value_at = (uint32_t)t_own * me.value_row + (uint32_t)p_own, value_last = min((uint32_t)t_own, live - 1) * me.value_row + (uint32_t)p_own;
    const int64_t first = ((me.b * a.L + me.tok0) * a.H + me.h) * a.P + me.p0, chunk_values = (int64_t)kC * me.value_row;
    struct Operands {
        uint2 z, v;
        float factor;                                             // number lane % 4 of token lane / 4
    };
    uint4 q[kSteps], mx[3][kX];                                   // (one set: the next chunk's are requested when this one's have been used)
    Cursor<uint16_t> queries{me.frags + N * kC + me.wave * kSteps * kFrag, kKeyHalves<N>, n_chunks - 1};
    Cursor<bf16_t> values{a.v + first, chunk_values, n_chunks - 1}, gates{MODE == kWalkGate ? a.z + first : nullptr, chunk_values, n_chunks - 1};
    Cursor<uint16_t> xs{me.own + kAtMX, kChunkHalves, n_chunks - 1};
    Cursor<float> factors{reinterpret_cast<const float *>(me.own + kAtScalars) + me.wave * 64, kChunkHalves / 2, n_chunks - 1};
    auto fetch_q = [&]() {
#pragma unroll
        for (int i = 0; i < kSteps; ++i) q[i] = *reinterpret_cast<const uint4 *>(queries.p + i * kFrag + lane8);
        queries.advance();
        requested();
    };
    auto fetch_mx = [&]() {
#pragma unroll
        for (int n = 0; n < 3; ++n)
#pragma unroll
            for (int i = 0; i < kX; ++i) mx[n][i] = *reinterpret_cast<const uint4 *>(xs.p + n * kTri + tile_at(me.wave, i) * kFrag + lane8);
        xs.advance();
        requested();
    };
    auto fetch_v = [&](Operands &f) {
        f.v = *reinterpret_cast<const uint2 *>(values.p + (values.left > 0 ? value_at : value_last));
        f.factor = factors.p[(uint32_t)me.lane];
        values.advance(), factors.advance();
        requested();
    };
    auto fetch_z = [&](Operands &f) {
        if constexpr (MODE == kWalkGate) {
            f.z = *reinterpret_cast<const uint2 *>(gates.p + (gates.left > 0 ? value_at : value_last));
            gates.advance();
            requested();
        }
    };
    // A value that is not a number ends its channel: the outputs are none from its token on, nor is the state at the end.  The walk takes a 0 for
    // it, which the zeros above the diagonals of X and M X leave alone, and remembers only that there was one: 9 instructions a chunk, without a
    // branch (one that found the token at once took 250 cycles of a chunk's 3000); ends_of_channels has the rest, seldom called.
    uint32_t ended = 0;                                           // bits 15 and 31
    auto number = [&](uint32_t &pair) {
        typedef int16_t short2_t __attribute__((ext_vector_type(2)));
        const uint32_t top = (pair & 0x7f807f80u) + 0x00800080u;  // an exponent of ones carries into the bit above it
        pair &= ~__builtin_bit_cast(uint32_t, __builtin_bit_cast(short2_t, top) >> 15);
        ended |= top;
    };
    auto numbers = [&](Operands &f) { number(f.v.x), number(f.v.y); };
    auto say_ended = [&]() {
        const bool some = __any((ended & 0x80008000u) != 0);
        if (me.lane == 0) lds.ended[me.wave] = (OUT || me.unit < 0) && some;
    };
    // V of a chunk, the other way round, and the factors of its rows
    auto park_v = [&](int parity, const Operands &f) {
        uint16_t *to = &lds.v[parity][p_own * kRowV + t_own];
        const uint32_t x = OUT || me.unit < 0 ? f.v.x : 0u, y = OUT || me.unit < 0 ? f.v.y : 0u;
        to[0] = (uint16_t)x, to[kRowV] = (uint16_t)(x >> 16), to[2 * kRowV] = (uint16_t)y, to[3 * kRowV] = (uint16_t)(y >> 16);
        if ((me.lane & 3) < 3) lds.factors[parity][me.lane & 3][t_own] = f.factor;
    };
    // Where there were such values: each wavefront looks for the first in four of the channels, and writes their outputs anew.
    auto ends_of_channels = [&]() {
        const int64_t tokens = min((int64_t)n_chunks * kC, a.L - me.tok0);
        const bf16_t *v = a.v + first + 4 * me.wave;
        int64_t ends[4] = {tokens, tokens, tokens, tokens};
        for (int64_t t0 = 0; t0 < tokens; t0 += 64) {
            const int64_t t = t0 + me.lane;
            const uint2 w = t < tokens ? *reinterpret_cast<const uint2 *>(v + t * me.value_row) : make_uint2(0, 0);
            const float x[4] = {bf16_lo(w.x), bf16_hi(w.x), bf16_lo(w.y), bf16_hi(w.y)};
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const uint64_t none = __ballot(!finite(x[i]));
                if (none && ends[i] == tokens) ends[i] = t0 + __builtin_ctzll(none);
            }
        }
#pragma unroll
        for (int i = 0; i < 4; ++i) lds.ends[4 * me.wave + i] = ends[i] < tokens ? (int)ends[i] : INT32_MAX;
        __threadfence();                                          // the outputs as they are, of all wavefronts, are written
        __syncthreads();
        if constexpr (!OUT) return;
        const int64_t at = (MODE == kWalkRaw ? ((me.b * a.n_chunks + me.first) * kC * a.H + me.h) * a.P + me.p0 : first) + 4 * me.wave;
#pragma unroll
        for (int i = 0; i < 4; ++i)
            for (int64_t t = ends[i] + me.lane; t < tokens; t += 64) {
                if constexpr (MODE == kWalkRaw) a.raw[at + i + t * me.value_row] = __int_as_float(0x7fc00000);
                else a.out[at + i + t * me.value_row] = 0x7fc0;
            }
    };
    Operands even, odd;
    if constexpr (!OUT) {
        fetch_v(even), fetch_v(odd);
        numbers(even);
        park_v(0, even);
        fetch_v(even);
        auto step = [&](int parity, Operands &other) __attribute__((always_inline)) {
            numbers(other);
            lds_barrier();                                        // A
            park_v(parity ^ 1, other);
            fetch_v(other);
            lds_barrier();                                        // B
            lds_barrier();                                        // C
        };
        int left = n_chunks;
        for (; left > 1; left -= 2) {
            step(0, odd);
            step(1, even);
        }
        if (left > 0) step(0, odd);
        say_ended();
        lds_barrier();
        if (any_ended(lds)) ends_of_channels();
        return;
    }
    fetch_v(even), fetch_v(odd), fetch_q(), fetch_mx(), fetch_z(even);
    numbers(even), numbers(odd);
    park_v(0, even);
    fetch_v(even);
    // this lane's outputs of the chunk (ahead of a norm they go into a buffer of the slab)
    int64_t to = (MODE == kWalkRaw ? ((me.b * a.n_chunks + me.first) * kC * a.H + me.h) * a.P + me.p0 : first) + value_at;
    // (what this role requests goes out where the chain has more to do: all of it behind C made the chain wait there)
    auto step = [&](int parity, bool stores, Operands &f, Operands &other) __attribute__((always_inline)) {
        lds_barrier();                                            // A
        park_v(parity ^ 1, other);
        fetch_v(other);
        fetch_z(other);
        // (the lowest terms of S ahead of B, where LDS is less used: 2048 tokens of N = 128 64.9 -> 60.7 us)
        f32x4_t o = zero, o2 = zero;
#pragma unroll
        for (int i = 0; i < kSteps; ++i) o2 = mma(lds_frag(&lds.s_lo[me.of_lane(i)]), as_frag(q[i]), o2);
        lds_barrier();                                            // B (the chain is short between the two, and would wait for this role)
        const float q_factor = lds.factors[parity][1][me.wave * 16 + me.c16];
#pragma unroll
        for (int i = 0; i < kSteps; ++i) {
            const int from = me.of_lane(i);
            o2 = mma(lds_frag(&lds.s_mid[from]), as_frag(q[i]), o2);
            o = mma(lds_frag(&lds.s_hi[from]), as_frag(q[i]), o);
        }
        o = (o + o2) * q_factor;
        o2 = zero;
        lds_barrier();                                            // C
        fetch_q();
        numbers(f);
#pragma unroll
        for (int i = 0; i < kX; ++i) {
            const int from = me.of_lane(i);
            const bf16x8 rh = lds_frag(&lds.r_hi[from]), rm = lds_frag(&lds.r_mid[from]), rl = lds_frag(&lds.r_lo[from]);
            const bf16x8 xh = as_frag(mx[0][i]), xm = as_frag(mx[1][i]), xl = as_frag(mx[2][i]);
            o2 = mma(rh, xl, o2);
            o = mma(rh, xm, o);
            o2 = mma(rl, xh, o2);
            o = mma(rm, xh, o);
            o2 = mma(rm, xm, o2);
            o = mma(rh, xh, o);
        }
        fetch_mx();
        o += o2;
        // a lane has a token's four channels 4 g4 ..: to the order of the rows, within the wavefront
        *reinterpret_cast<f32x4_t *>(&lds.o[me.wave][me.c16 * 16 + 4 * me.g4]) = o;
        __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront", "local");
        __builtin_amdgcn_wave_barrier();
        __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront", "local");
        o = *reinterpret_cast<const f32x4_t *>(&lds.o[me.wave][me.lane * 4]);
        if constexpr (MODE == kWalkGate) {
            o[0] *= silu_f32(bf16_lo(f.z.x)), o[1] *= silu_f32(bf16_hi(f.z.x));
            o[2] *= silu_f32(bf16_lo(f.z.y)), o[3] *= silu_f32(bf16_hi(f.z.y));
        }
        if (stores) {
            if constexpr (MODE == kWalkRaw) *reinterpret_cast<f32x4_t *>(a.raw + to) = o;
            else *reinterpret_cast<uint2 *>(a.out + to) = make_uint2(f32x2_to_bf16x2(o[0], o[1]), f32x2_to_bf16x2(o[2], o[3]));
        }
        to += chunk_values;
    };
    // (the last chunk, which may be short, by itself: at every other turn all lanes store, and the compiler knows what is in flight)
    int left = n_chunks;
    for (; left > 2; left -= 2) {
        step(0, true, even, odd);
        step(1, true, odd, even);
    }
    const bool last = (uint32_t)t_own < live;
    if (left == 2) {
        step(0, true, even, odd);
        step(1, last, odd, even);
    } else {
        step(0, last, even, odd);
    }
    say_ended();
    lds_barrier();
    if (any_ended(lds)) ends_of_channels();
}

// Heads that leave CUs free have their slab in parts of `part` chunks, several at once: what a part makes of a state is a linear map,
// S -> S F + C, whose C is the walk from nothing and whose F is the walk of the unit vectors without values.  A first launch walks the
// first part for its outputs and the others but the last for their maps; delta_join_kernel takes the states through the maps; a second
// launch walks the parts from the second on for their outputs, from their own states.
// grid: 8 blocks of 16 rows (heads parts / 8 rounded up), first those of the parts for their outputs, then those for their maps; the blocks of
// a head's part, which read the same fragments, are 8 apart: on one XCD, and the maps begin on the XCD behind the last of the others
template <int N, int MODE>
__global__ void __launch_bounds__(2 * kThreads) delta_walk_kernel(WalkArgs a)
{
    __shared__ WalkLds<N> lds;
    const uint32_t heads = (uint32_t)a.heads, values = (uint32_t)a.P / 16, walks = (heads * a.walked + 7) / 8 * 8 * values;
    const bool maps = blockIdx.x >= walks;
    const uint32_t index = maps ? blockIdx.x - walks : blockIdx.x, blocks = maps ? values + N / 16 : values, place = index >> 3;
    const uint32_t pair = place / blocks * 8 + ((maps ? index - heads * a.walked : index) & 7), block = place % blocks, turn = pair / heads;
    if (turn >= (maps ? a.maps : a.walked)) return;
    const bool unit = block >= values;
    const uint32_t part = turn + (maps ? 1 : a.first_part);
    WalkPlace<N> at;
    at.hb = pair - turn * heads;
    const int role = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6);
    at.lane = threadIdx.x & 63, at.wave = role & 3, at.c16 = at.lane & 15, at.g4 = at.lane >> 4;
    at.b = at.hb / a.H, at.h = at.hb - at.b * a.H, at.Hk = a.H / a.group, at.hk = at.h / a.group;
    at.p0 = unit ? 0 : (int)block * 16;
    at.unit = unit ? (int)(block - values) * 16 : -1;
    at.first = part * a.part, at.n_chunks = min(a.part, a.n_chunks - at.first), at.tok0 = a.tok0 + at.first * kC;
    at.own = a.ws + (at.hb * a.n_chunks + at.first) * kChunkHalves;
    at.frags = a.frags + ((at.b * at.Hk + at.hk) * a.n_chunks + at.first) * kKeyHalves<N>;
    at.value_row = (uint32_t)(a.H * a.P);
    // (a.starts: of the parts from the second on)
    const bool last = at.first + at.n_chunks == a.n_chunks;
    const int64_t rows = (at.hb * a.P + at.p0) * N, each = a.heads * a.P * N;
    at.h0 = maps ? nullptr : part > 0 ? a.starts + (part - 1) * each + rows : a.h0 ? a.h0 + rows : nullptr;
    at.h_final = unit ? a.map + ((turn * a.heads + at.hb) * N + at.unit) * N : last ? a.h_final ? a.h_final + rows : nullptr
                 : maps || part == 0 ? a.starts + part * each + rows : nullptr;
    if (maps) {
        if (role < 2) walk_chain<N, false>(a, at, lds);
        else if (role < 4) walk_chain<N, true>(a, at, lds);
        else walk_outputs<N, MODE, false, false>(a, at, lds);
        return;
    }
    if (role < 2) walk_chain<N, false>(a, at, lds);
    else if (role < 4) walk_chain<N, true>(a, at, lds);
    else if (role < 6) walk_outputs<N, MODE, false, true>(a, at, lds);
    else walk_outputs<N, MODE, true, true>(a, at, lds);
}

// The states at the starts of the parts, from that of the second on: S[i + 1] = S[i] F[i] + C[i], C[i] where S[i + 1] will be.  A workgroup
// has 16 rows of a head and a wavefront 16 of the N columns, in float32: of S^T = F^T S^T + C^T a lane has four adjacent columns of
// row l % 16, just as the next product's right operand needs them (k in the order 16 q + 4 (l / 16) + j).
// Bound by the float32 matrix rate of a CU (N = 128: 0.9 us a step) and the exchange: 0.75 us a step with N = 64, 2 with N = 128.
// grid: (heads P / 16); rows: of all heads, head_rows: of one; steps > 0
template <int N>
__global__ void __launch_bounds__(4 * N)
delta_join_kernel(const float *__restrict__ map, float *states, int64_t rows, int64_t head_rows, int steps)
{
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, c16 = lane & 15, g4 = lane >> 4;
    const int64_t row = (int64_t)blockIdx.x * 16 + c16, hb = (int64_t)blockIdx.x * 16 / head_rows;
    const int64_t f_step = rows / head_rows * N * N, s_step = rows * N;
    __shared__ f32x4_t tiles[2][N / 16][64];
    const float *f = map + (hb * N + 4 * g4) * N + wave * 16 + c16;
    float *s = states + row * N + wave * 16 + 4 * g4;
    f32x4_t now = *reinterpret_cast<const f32x4_t *>(s);
    const float *c = s + s_step;
    struct Operands {
        float f[N / 4];
        f32x4_t c;
    };
    int left = steps;                                             // that are to be fetched
    auto fetch = [&](Operands &w) __attribute__((always_inline)) {
#pragma unroll
        for (int i = 0; i < N / 4; ++i) w.f[i] = f[(i / 4 * 16 + i % 4) * N];
        w.c = *reinterpret_cast<const f32x4_t *>(c);
        --left;
        f += left > 0 ? f_step : 0, c += left > 0 ? s_step : 0;
    };
    auto step = [&](int parity, Operands &w) __attribute__((always_inline)) {
        tiles[parity][wave][lane] = now;
        __syncthreads();                                          // (the next step's go to the other half)
        now = w.c;
#pragma unroll
        for (int q = 0; q < N / 16; ++q) {
            const f32x4_t right = tiles[parity][q][lane];
#pragma unroll
            for (int j = 0; j < 4; ++j) now = mma(w.f[q * 4 + j], right[j], now);
        }
        s += s_step;
        *reinterpret_cast<f32x4_t *>(s) = now;
        fetch(w);
    };
    Operands even, odd;
    fetch(even), fetch(odd);
    for (int i = 0; i < steps; i += 2) {
        step(0, even);
        if (i + 1 < steps) step(1, odd);
    }
}

// The norm over a head's channels, which the walk's workgroups have in parts, and the gate: P / 4 lanes to a (token, head).  Bound by bytes:
// 3008 tokens of 32 heads of 128 channels, 99 MB, in 15 us.
// grid: (workgroups, batch); n: quadruples of a batch row, raw_row and row those from one batch row to the next
template <int P>
__global__ void __launch_bounds__(kThreads)
delta_norm_kernel(const float *__restrict__ raw, const bf16_t *__restrict__ z, const float *__restrict__ norm_w, bf16_t *__restrict__ out, int64_t n,
                  int64_t raw_row, int64_t row, float eps)
{
    const int64_t at = (int64_t)blockIdx.x * kThreads + threadIdx.x;
    const int64_t safe = min(at, n - 1);
    const int64_t from = (int64_t)blockIdx.y * raw_row + safe, to = (int64_t)blockIdx.y * row + safe;
    const int p = (int)(safe % (P / 4)) * 4;
    float y[4], w[4], g[4] = {0.0f, 0.0f, 0.0f, 0.0f};
    load4(raw + from * 4, y);
    load4(norm_w + p, w);
    if (z) load4(z + to * 4, g);
    float ss = sum16(fmaf(y[0], y[0], fmaf(y[1], y[1], fmaf(y[2], y[2], y[3] * y[3]))));
    if constexpr (P == 128) ss += __shfl_xor(ss, 16, 64);
    const float f = 1.0f / sqrtf(ss / P + eps);
#pragma unroll
    for (int i = 0; i < 4; ++i) y[i] *= f * w[i] * (z ? silu_f32(g[i]) : 1.0f);
    if (at < n) *reinterpret_cast<uint2 *>(out + to * 4) = make_uint2(f32x2_to_bf16x2(y[0], y[1]), f32x2_to_bf16x2(y[2], y[3]));
}

template <int N> hipError_t walk(const WalkArgs &w, hipStream_t stream)
{
    const int64_t blocks = delta_walk_blocks(w.heads, w.P, N, w.walked, w.maps);
    // Two workgroups fit on a CU, but each takes its time then: where a CU can be had for each, LDS that nobody uses keeps the second away
    // (8191 tokens of 12 heads of N = 64, P = 128: 138 -> 130 us; without it two go to one CU while others stay empty).
    const unsigned alone = delta_fullest_xcd(w.heads, w.P, N, w.walked, w.maps) <= 32 ? 40960 : 0;
    if (w.raw) delta_walk_kernel<N, kWalkRaw><<<(unsigned)blocks, 2 * kThreads, alone, stream>>>(w);
    else if (w.z) delta_walk_kernel<N, kWalkGate><<<(unsigned)blocks, 2 * kThreads, alone, stream>>>(w);
    else delta_walk_kernel<N, kWalkPlain><<<(unsigned)blocks, 2 * kThreads, alone, stream>>>(w);
    return hipGetLastError();
}

template <int N> hipError_t chunked(const DeltaArgs &a, hipStream_t stream)
{
    const DeltaPlan p = delta_plan(a.rows, a.L, a.H, a.Hk, a.P, a.N);
    char *ws = reinterpret_cast<char *>(a.ws);
    uint16_t *frags = reinterpret_cast<uint16_t *>(ws + p.frags_at);
    float *raw = a.norm_w ? reinterpret_cast<float *>(ws + p.raw_at) : nullptr;
    float *state = a.h_out ? a.h_out : reinterpret_cast<float *>(ws + p.state_at);
    const bf16_t *z = static_cast<const bf16_t *>(a.z);
    bf16_t *out = static_cast<bf16_t *>(a.out);
    for (int64_t first = 0; first < p.chunks; first += p.slab) {
        const DeltaSlab slab = delta_slab(p, first);
        const int64_t n = slab.chunks, tok0 = first * kC;
        const bool last = first + n == p.chunks;
        delta_prepare_kernel<N><<<dim3((unsigned)n, (unsigned)a.H, (unsigned)a.rows), kPrepThreads, 0, stream>>>(
            static_cast<const bf16_t *>(a.q), static_cast<const bf16_t *>(a.k), static_cast<const bf16_t *>(a.dt), static_cast<const bf16_t *>(a.beta),
            a.A, a.dt_bias, reinterpret_cast<uint16_t *>(ws), frags, tok0, a.L, a.H, a.H / a.Hk,
            DeltaOptions{a.scale, a.eps, a.dt_softplus, a.beta_sigmoid, a.qk_norm});
        if (hipError_t e = hipGetLastError()) return e;
        const int64_t heads = a.rows * a.H;
        const uint32_t parts = (uint32_t)slab.parts;
        float *starts = reinterpret_cast<float *>(ws + p.parts_at), *map = reinterpret_cast<float *>(ws + p.map_at);
        WalkArgs w{static_cast<const bf16_t *>(a.v), z, reinterpret_cast<const uint16_t *>(ws), frags, first == 0 ? a.h_in : state,
                   last ? a.h_out : state, out, raw, starts, map, a.L, a.H, a.H / a.Hk, heads, tok0, n, p.part, 0, 1, (uint32_t)slab.maps, a.P};
        if (hipError_t e = walk<N>(w, stream)) return e;
        if (w.maps > 0) {
            delta_join_kernel<N><<<(unsigned)(heads * a.P / 16), 4 * N, 0, stream>>>(map, starts, heads * a.P, a.P, (int)w.maps);
            if (hipError_t e = hipGetLastError()) return e;
        }
        if (parts > 1) {
            w.first_part = 1, w.walked = parts - 1, w.maps = 0;
            if (hipError_t e = walk<N>(w, stream)) return e;
        }
        if (!raw) continue;
        const int64_t token = a.H * a.P / 4, tokens = last ? a.L - tok0 : n * kC;
        const dim3 grid((unsigned)((tokens * token + kThreads - 1) / kThreads), (unsigned)a.rows);
        const bf16_t *gates = z ? z + tok0 * token * 4 : nullptr;
        bf16_t *to = out + tok0 * token * 4;
        if (a.P == 64) delta_norm_kernel<64><<<grid, kThreads, 0, stream>>>(raw, gates, a.norm_w, to, tokens * token, n * kC * token, a.L * token, a.eps);
        else delta_norm_kernel<128><<<grid, kThreads, 0, stream>>>(raw, gates, a.norm_w, to, tokens * token, n * kC * token, a.L * token, a.eps);
        if (hipError_t e = hipGetLastError()) return e;
    }
    return hipSuccess;
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
    if (delta_few_tokens(batch, L, H)) return 0;
    return (size_t)delta_plan(batch, L, H, Hk, P, N).bytes;
}

hipError_t launch_gated_delta(const DeltaArgs &a, hipStream_t stream)
{
    if (a.io != kIoBf16 || delta_few_tokens(a.rows, a.L, a.H)) return launch_gated_delta_step(a, stream);
    return a.N == 64 ? chunked<64>(a, stream) : chunked<128>(a, stream);
}

}  // namespace mamba
