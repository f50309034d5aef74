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
constexpr int kTrip = 64 * 4;                                        // tokens that a wavefront has at once

// The children of a node that were rejected so far, and what P and Q became by them.
struct Rejections {
    int32_t token[kMaxFan];
    double of_gap[kMaxFan], of_rest[kMaxFan];                        // 1 / sums; 0: the sum was zero
};
struct Shared {
    double part[2][2][kWaves];                                       // sums of the wavefronts' ranges, in turn: the others may still be being read
    Rejections rejected;
};

// What is added up over the tokens of a row: P after the first `levels` rejections, or where `gap` says so what P is ahead of Q there (then of q too what
// is left beside the rejected children and `token`).  (One function for all passes, not inlined: its instructions are fetched once.)
struct Weighing {
    const float *p, *q;                                              // q: nullptr: zeros
    int levels;
    bool gap;
    int32_t token;
};

__device__ __forceinline__ double wave_sum(double v)
{
#pragma unroll
    for (int d = 32; d; d >>= 1) v += __shfl_xor(v, d);
    return v;
}

// P and Q of four tokens with probabilities p and q; `left`: q while the token is not rejected
__device__ __forceinline__ void after_rejections(const Rejections &r, int levels, int32_t v0, double (&P)[4], double (&Q)[4], double (&left)[4])
{
#pragma unroll 1
    for (int l = 0; l < levels; ++l) {
        const int32_t token = r.token[l];
        const double of_gap = r.of_gap[l], of_rest = r.of_rest[l];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const double gap = fmax(P[i] - Q[i], 0.0);
            P[i] = of_gap > 0.0 ? gap * of_gap : P[i];
            left[i] = v0 + i == token ? 0.0 : left[i];
            Q[i] = left[i] * of_rest;
        }
    }
}
// x: what is added up of four tokens, y: of q
__device__ __forceinline__ void weigh(const Rejections &r, const Weighing &w, const f32x4_any &pv, const f32x4_any &qv, int32_t v0, double (&x)[4], double (&y)[4])
{
    double P[4], Q[4], left[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) P[i] = pv[i], left[i] = Q[i] = qv[i];
    after_rejections(r, w.levels, v0, P, Q, left);
#pragma unroll
    for (int i = 0; i < 4; ++i) x[i] = w.gap ? fmax(P[i] - Q[i], 0.0) : P[i], y[i] = v0 + i == w.token ? 0.0 : left[i];
}
// four tokens of a row from v on, zeros from `end` on
__device__ __forceinline__ f32x4_any load4(const float *row, int32_t v, int32_t end)
{
    if (v + 4 <= end) return *reinterpret_cast<const f32x4_any *>(row + v);
    f32x4_any x;
#pragma unroll
    for (int i = 0; i < 4; ++i) x[i] = v + i < end ? row[v + i] : 0.0f;
    return x;
}

// Tokens from .. from + length - 1 added up: by wavefronts, which have `per_of(length)` each in one piece, and all together, in an order that depends on
// the numbers alone.
struct Sums {
    const double *by_wave;                                           // of the first
    double first, second;
};
__device__ __forceinline__ int32_t per_of(int32_t length) { return ((length + kWaves - 1) / kWaves + 3) / 4 * 4; }
__device__ __attribute__((noinline)) Sums sums_of(Shared &s, int turn, Weighing w, int32_t from, int32_t length)
{
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6);
    const int32_t per = per_of(length), begin = from + min(wave * per, length), end = from + min((wave + 1) * per, length);
    constexpr int kAhead = 4;
    double x = 0.0, y = 0.0;
#pragma unroll 1
    for (int32_t v0 = begin; v0 < end; v0 += kAhead * kTrip) {
        f32x4_any pv[kAhead], qv[kAhead];
#pragma unroll
        for (int j = 0; j < kAhead; ++j) {
            const int32_t v = v0 + j * kTrip + lane * 4;
            pv[j] = load4(w.p, v, end);
            qv[j] = w.q ? load4(w.q, v, end) : f32x4_any(0.0f);
        }
#pragma unroll 1
        for (int j = 0; j < kAhead; ++j) {
            double xs[4], ys[4];
            weigh(s.rejected, w, pv[0], qv[0], v0 + j * kTrip + lane * 4, xs, ys);
#pragma unroll
            for (int i = 0; i < 4; ++i) x += xs[i], y += ys[i];
#pragma unroll
            for (int i = 0; i + 1 < kAhead; ++i) pv[i] = pv[i + 1], qv[i] = qv[i + 1];
        }
    }
    x = wave_sum(x), y = wave_sum(y);
    double(*part)[kWaves] = s.part[turn];
    if (lane == 0) part[0][wave] = x, part[1][wave] = y;
    __syncthreads();
    Sums r{part[0], 0.0, 0.0};
#pragma unroll
    for (int i = 0; i < kWaves; ++i) r.first += part[0][i], r.second += part[1][i];
    return r;
}

// One workgroup to a sequence.  A pass over a row of p and q is what a rejection takes: every wavefront has a sixteenth of it, in one piece, so that
// its sum is also where the search for a drawn token begins, which goes on in sixteenths of a sixteenth.  Bound by what one CU brings in: a pass
// over 50280 tokens reads 400 KB.
__global__ void __launch_bounds__(kThreads) verify_kernel(VerifyArgs a)
{
    __shared__ Shared s;
    const int64_t b = blockIdx.x;
    const int tid = threadIdx.x, lane = tid & 63;
    const int32_t V = (int32_t)a.V;
    const float *p_rows = a.p + b * a.nodes * a.V, *q_rows = a.q + b * a.inner * a.V;
    const int32_t *tokens = a.tokens + b * (a.nodes - 1);
    const float *u_accept = a.u_accept + b * (a.nodes - 1);
    int32_t *out = a.out + b * (a.gamma + 1), *node = a.node + b * a.gamma;
    int turn = 0;
    auto sums = [&](const Weighing &w, int32_t from, int32_t length) { return sums_of(s, turn ^= 1, w, from, length); };

    int64_t row = 0, rows = 1, nodes = 0, children = 0;              // of the node, of its position, ahead of that
    int depth = 0;
    Weighing w{};                                                    // of the token that is drawn
    Sums all{};                                                      // and its sums over the row, where there are some
    bool known = false;
#pragma unroll 1
    for (; depth < a.gamma; ++depth) {
        const int fan = a.tree[depth];
        const float *p = p_rows + (nodes + row) * a.V, *q = q_rows + (nodes + row) * a.V;
        const int64_t first = children + row * fan;
        int n = 0, taken = -1;                                       // rejections; the child that was accepted
        int32_t c = -1;
        known = false;
#pragma unroll 1
        for (int j = 0; j < fan; ++j) {
            c = tokens[first + j];
            const float u = u_accept[first + j];
            if (c < 0 || c >= V) continue;
            double P[4] = {p[c], 0.0, 0.0, 0.0}, Q[4] = {q[c], 0.0, 0.0, 0.0}, left[4] = {Q[0], 0.0, 0.0, 0.0};
            after_rejections(s.rejected, n, c, P, Q, left);
            const double ratio = Q[0] > 0.0 ? P[0] / Q[0] : P[0] > 0.0 ? 1.0 : 0.0;
            if ((double)u < (ratio < 1.0 ? ratio : 1.0)) {
                taken = j;
                break;
            }
            w = Weighing{p, q, n, true, c};
            all = sums(w, 0, V);
            known = all.first > 0.0;
            if (tid == 0) {
                s.rejected.token[n] = c;
                s.rejected.of_gap[n] = known ? 1.0 / all.first : 0.0;
                s.rejected.of_rest[n] = all.second > 0.0 ? 1.0 / all.second : 0.0;
            }
            ++n;
            __syncthreads();
        }
        if (taken < 0) {
            // from what P is ahead of Q at the last rejection, undivided, or where that was nothing from P
            if (!known) w = Weighing{p, q, n, false, -1};
            break;
        }
        if (tid == 0) out[depth] = c, node[depth] = (int32_t)(row * fan + taken);
        __syncthreads();                                             // (what the rejections are read by is over)
        nodes += rows, children += rows * fan, row = row * fan + taken, rows *= fan;
    }
    if (depth == a.gamma) w = Weighing{p_rows + (nodes + row) * a.V, nullptr, 0, false, -1}, known = false;

    // ---- the token at which the sums pass u times their total
    int32_t token = -1, from = 0, length = V;
    double before = 0.0, bound = 0.0;
#pragma unroll 1
    for (bool whole = true;; whole = false) {                        // the range in which they do; the last that has any (the last bits of the sums)
        if (!known) all = sums(w, from, length);
        known = false;
        if (whole) bound = (double)a.u_sample[b] * all.first;
        if (whole && !(all.first > 0.0)) {
            length = 0;
            break;
        }
        const int32_t per = per_of(length);
        int at = -1;
        double at_before = before;
#pragma unroll 1
        for (int i = 0; i < kWaves; ++i) {
            const double x = all.by_wave[i];
            if (x > 0.0) {
                at = i, at_before = before;
                if (before + x > bound) break;
            }
            before += x;
        }
        if (at < 0) {
            length = 0;
            break;
        }
        before = at_before;
        from += min(at * per, length), length = min(per, length - min(at * per, length));
        if (length <= kTrip) break;
    }
    if (length > 0) {                                                // (every wavefront looks through the same tokens)
        const int32_t v0 = from + lane * 4, end = from + length;
        double x[4], y[4], mine = 0.0;
        weigh(s.rejected, w, load4(w.p, v0, end), w.q ? load4(w.q, v0, end) : f32x4_any(0.0f), v0, x, y);
#pragma unroll
        for (int i = 0; i < 4; ++i) x[i] = v0 + i < end ? x[i] : 0.0, mine += x[i];
        double to = mine;
#pragma unroll
        for (int d = 1; d < 64; d <<= 1) {
            const double o = __shfl_up(to, d);
            to += lane >= d ? o : 0.0;
        }
        double at = before + (to - mine);
        int32_t there = -1, some = -1;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            at += x[i];
            if (x[i] > 0.0) {
                some = v0 + i;
                if (at > bound && there < 0) there = v0 + i;
            }
        }
        const uint64_t is = __ballot(there >= 0), any = __ballot(some >= 0);
        token = is ? __builtin_amdgcn_readlane(there, __builtin_ctzll(is)) : any ? __builtin_amdgcn_readlane(some, 63 - __builtin_clzll(any)) : -1;
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
