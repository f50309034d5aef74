// Which path of a drafted tree a target accepts (appendix, verification algorithm, for every node of a tree in place of a chain): the host's
// sd_verify on the device, so that no probability leaves it.
//
//   at a node, children c_1 .. c_N drawn from q without replacement:   P = p, Q = q
//   c_j is accepted where u_j < min(1, P(c_j) / Q(c_j)), and the walk goes on at its node
//   else  P = (P - Q)_+ / its sum (P as it was where that is zero),   Q = q without c_1 .. c_j / its sum
//   no child accepted: a token is drawn from P, and the walk ends;  a leaf reached: a token is drawn from its p
//
// P and Q are formed again from p and q wherever they are looked at, from the sums of the rejections before; all of it in float64, since which
// token a sum passes its bound at is decided by its last bits.
#include "device_math.h"
#include "launch.h"
#include "logit_rows.h"

namespace mamba {
namespace {

constexpr int kThreads = 1024, kWaves = kThreads / 64;
constexpr int kTile = kThreads * 4;                                  // tokens that the workgroup adds up together
constexpr int kMaxTiles = (1 << 25) / kTile;

struct Shared {
    double tile[kMaxTiles];                                          // sums of P by tiles
    double part[2][kWaves];
    double sum[2];
    int32_t token, where;
};

// The children of one node that were rejected so far, and what P and Q became by them.
struct Rejections {
    int n = 0;
    int32_t token[kMaxFan];
    double of_gap[kMaxFan], of_rest[kMaxFan];                        // 1 / sums; 0: the sum was zero

    // P - Q ahead of the division, P and Q of a token with probabilities p and q; `left`: q of the token while it is not rejected
    __device__ __forceinline__ void at(double p, double q, int32_t v, double *P, double *Q, double *left) const
    {
        double Pv = p, Qv = q;
#pragma unroll
        for (int i = 0; i < kMaxFan; ++i) {
            if (i < n) {
                const double gap = fmax(Pv - Qv, 0.0);
                Pv = of_gap[i] > 0.0 ? gap * of_gap[i] : Pv;
                q = v == token[i] ? 0.0 : q;
                Qv = q * of_rest[i];
            }
        }
        *P = Pv, *Q = Qv, *left = q;
    }
};

__device__ __forceinline__ double wave_sum(double v)
{
#pragma unroll
    for (int d = 32; d; d >>= 1) v += __shfl_xor(v, d);
    return v;
}

// four tokens of a row from v0 on, zeros behind its end
__device__ __forceinline__ void load4(const float *row, int32_t v0, int32_t V, float *x)
{
    if (v0 + 4 <= V) {
        const f32x4_any a = *reinterpret_cast<const f32x4_any *>(row + v0);
#pragma unroll
        for (int i = 0; i < 4; ++i) x[i] = a[i];
    } else {
#pragma unroll
        for (int i = 0; i < 4; ++i) x[i] = v0 + i < V ? row[v0 + i] : 0.0f;
    }
}

// One workgroup to a sequence.
__global__ void __launch_bounds__(kThreads) verify_kernel(VerifyArgs a)
{
    __shared__ Shared s;
    const int64_t b = blockIdx.x;
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const int32_t V = (int32_t)a.V;
    const float *p_rows = a.p + b * a.nodes * a.V, *q_rows = a.q + b * a.inner * a.V;
    const int32_t *tokens = a.tokens + b * (a.nodes - 1);
    const float *u_accept = a.u_accept + b * (a.nodes - 1);
    int32_t *out = a.out + b * (a.gamma + 1), *node = a.node + b * a.gamma;

    // sums over the row of what f gives for a token, in an order that depends on V alone; the first of the two by tiles too
    auto sums = [&](const float *p, const float *q, auto f) {
        double total[2] = {0.0, 0.0};
        for (int t = 0; t * kTile < V; ++t) {
            const int32_t v0 = t * kTile + tid * 4;
            float pv[4] = {}, qv[4] = {};
            load4(p, v0, V, pv);
            if (q) load4(q, v0, V, qv);
            double x[2] = {0.0, 0.0};
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                double y[2] = {0.0, 0.0};
                f((double)pv[i], (double)qv[i], v0 + i, y);
                x[0] += y[0], x[1] += y[1];
            }
            __syncthreads();
            x[0] = wave_sum(x[0]), x[1] = wave_sum(x[1]);
            if (lane == 0) s.part[0][wave] = x[0], s.part[1][wave] = x[1];
            __syncthreads();
            double y[2] = {0.0, 0.0};
            for (int w = 0; w < kWaves; ++w) y[0] += s.part[0][w], y[1] += s.part[1][w];
            if (tid == 0) s.tile[t] = y[0];
            total[0] += y[0], total[1] += y[1];
        }
        s.sum[0] = total[0], s.sum[1] = total[1];                    // (the same from all threads)
        __syncthreads();
    };
    // the token at which the sums of f pass u times `total`, the tiles' sums of f in s.tile
    auto drawn = [&](const float *p, const float *q, double total, float u, auto f) -> int32_t {
        if (!(total > 0.0)) return -1;
        const double bound = (double)u * total;
        const int tiles = (V + kTile - 1) / kTile;
        int t = 0;
        double before = 0.0;
        for (; t < tiles - 1 && !(before + s.tile[t] > bound); ++t) before += s.tile[t];
        int32_t last = -1;                                           // of those with any weight
        for (; t < tiles; ++t) {
            const int32_t v0 = t * kTile + tid * 4;
            float pv[4] = {}, qv[4] = {};
            load4(p, v0, V, pv);
            if (q) load4(q, v0, V, qv);
            double x[4], mine = 0.0;
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                double y[2] = {0.0, 0.0};
                f((double)pv[i], (double)qv[i], v0 + i, y);
                x[i] = y[0];
                mine += y[0];
            }
            double to = mine;
#pragma unroll
            for (int d = 1; d < 64; d <<= 1) {
                const double o = __shfl_up(to, d);
                to += lane >= d ? o : 0.0;
            }
            __syncthreads();
            if (lane == 63) s.part[0][wave] = to;
            if (tid == 0) s.token = V, s.where = -1;
            __syncthreads();
            double from = before;
            for (int w = 0; w < wave; ++w) from += s.part[0][w];
            double at = from + (to - mine);
            int32_t first = V, some = -1;
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                at += x[i];
                if (x[i] > 0.0) {
                    some = v0 + i;
                    if (at > bound && first == V) first = v0 + i;
                }
            }
            if (first < V) atomicMin(&s.token, first);
            if (some >= 0) atomicMax(&s.where, some);
            __syncthreads();
            if (s.where >= 0) last = s.where;
            if (s.token < V) return s.token;
            before += s.tile[t];
            __syncthreads();
        }
        return last;                                                 // (the last bits of the sums)
    };

    int64_t row = 0, rows = 1, nodes = 0, children = 0;              // of the node, of its position, ahead of that
    int depth = 0;
    int32_t token = -1;
    for (; depth < a.gamma; ++depth) {
        const int fan = a.tree[depth];
        const float *p = p_rows + (nodes + row) * a.V, *q = q_rows + (nodes + row) * a.V;
        const int64_t first = children + row * fan;
        Rejections r;
        double sum = 1.0;
        bool fresh = false;                                          // s.tile has the sums of the last gap
        int taken = -1;
        int32_t c = -1;
        for (int j = 0; j < fan; ++j) {
            c = tokens[first + j];
            if (c < 0 || c >= V) continue;
            double P, Q, left;
            r.at((double)p[c], (double)q[c], c, &P, &Q, &left);
            const double ratio = Q > 0.0 ? P / Q : P > 0.0 ? 1.0 : 0.0;
            if ((double)u_accept[first + j] < (ratio < 1.0 ? ratio : 1.0)) {
                taken = j;
                break;
            }
            sums(p, q, [&](double pv, double qv, int32_t v, double (&y)[2]) {
                double Pv, Qv, rest;
                r.at(pv, qv, v, &Pv, &Qv, &rest);
                y[0] = fmax(Pv - Qv, 0.0), y[1] = v == c ? 0.0 : rest;
            });
            sum = s.sum[0];
            const double rest = s.sum[1];
#pragma unroll
            for (int i = 0; i < kMaxFan; ++i)
                if (i == r.n) r.token[i] = c, r.of_gap[i] = sum > 0.0 ? 1.0 / sum : 0.0, r.of_rest[i] = rest > 0.0 ? 1.0 / rest : 0.0;
            ++r.n;
            fresh = sum > 0.0;
        }
        if (taken >= 0) {
            if (tid == 0) out[depth] = c, node[depth] = (int32_t)(row * fan + taken);
            nodes += rows, children += rows * fan, row = row * fan + taken, rows *= fan;
            continue;
        }
        auto residual = [&](double pv, double qv, int32_t v, double (&y)[2]) {
            double Pv, Qv, rest;
            if (fresh) {                                             // ahead of its division: what the tiles hold
                --r.n;
                r.at(pv, qv, v, &Pv, &Qv, &rest);
                ++r.n;
                y[0] = fmax(Pv - Qv, 0.0);
            } else {
                r.at(pv, qv, v, &Pv, &Qv, &rest);
                y[0] = Pv;
            }
        };
        if (!fresh) {
            sums(p, q, residual);
            sum = s.sum[0];
        }
        token = drawn(p, q, sum, a.u_sample[b], residual);
        break;
    }
    if (depth == a.gamma) {
        const float *p = p_rows + (nodes + row) * a.V;
        auto itself = [](double pv, double, int32_t, double (&y)[2]) { y[0] = pv; };
        sums(p, nullptr, itself);
        token = drawn(p, nullptr, s.sum[0], a.u_sample[b], itself);
    }
    if (tid == 0) {
        out[depth] = token;
        a.count[b] = depth + 1;
        for (int i = depth + 1; i <= a.gamma; ++i) out[i] = -1;
        for (int i = depth; i < a.gamma; ++i) node[i] = -1;
    }
}

}  // namespace

hipError_t launch_verify(const VerifyArgs &a, hipStream_t stream)
{
    verify_kernel<<<(unsigned)a.n_seq, kThreads, 0, stream>>>(a);
    return hipGetLastError();
}

}  // namespace mamba
