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
//
// Decisions are a few numbers, but a rejection needs sums over a row of p and q, which takes one CU 10 us (400 KB for 50280 tokens) and many CUs two.  So a
// launch goes on with the walk until a row is to be added up, and adds it up, a workgroup to a piece of it; the next launch begins by
// what that gave.  All workgroups of a sequence walk, each for itself and all alike.  There are as many launches as a tree may have rejections on one way
// and one more, up to kMostRounds; draw_kernel ends the walk, adding up by itself what is left, and draws.  us, a call (one
// workgroup to a sequence from beginning to end): one tree (3,2,2,1,1) of 50280 23.5 (58), 32 chains of five of 131071 23.2 (44).
//
// Bound by the launches and what follows one another in them, for many sequences by memory.  A launch of one tree is 4.0 us: the walk read 1.0, a
// node's tokens and their probabilities 0.9, the row added up 1.6, results 0.4.  Of 32 x 131071 it is 14 (33.5 MB: 2.4 TB/s), and the draw 10.
#include "device_math.h"
#include "launch.h"
#include "logit_rows.h"

namespace mamba {
namespace {

constexpr int kThreads = 256, kWaves = kThreads / 64, kTrip = kThreads * 8;   // tokens that a workgroup has at once
constexpr int kMostPieces = 256;
constexpr int kMostRounds = 8;

typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));

// What is added up over the tokens of a row: P after the first `levels` rejections, or where `gap` says so what P is ahead of Q there (then of q too what
// is left beside the rejected children and `token`).
struct Weighing {
    int64_t p_row, q_row;                                            // of a sequence's rows (q: -1: zeros)
    int32_t levels, gap, token;
};

// A walk between two launches.
constexpr int kWalking = 0, kWaiting = 1, kDecided = 2;              // (on its way to the next sums; for those of `w` as a rejection; as what is drawn from)
struct Walk {
    int64_t row, rows, nodes, children;                              // of the node, of its position, ahead of that
    int32_t depth, phase;
    int32_t n, next;                                                 // rejections of the node, its next child
    int32_t known;                                                   // the sums of w: 0 not there, 1 there
    int32_t turn;                                                    // in which of the two buffers
    Weighing w;
    int32_t token[kMaxFan];                                          // the rejected children, and what P and Q became by them:
    double of_gap[kMaxFan], of_rest[kMaxFan];                        // 1 / sums; 0: the sum was zero
};

struct Sums {
    double first, second;
};

// (by DPP: six trips through LDS for a sum were a sixth of a launch of few sequences)
template <int CTRL, int ROWS = 0xf> __device__ __forceinline__ double plus_lane(double v)
{
    const u32x2 u = __builtin_bit_cast(u32x2, v);
    return v + __builtin_bit_cast(double, u32x2{from_lane<CTRL, ROWS>(0, u.x), from_lane<CTRL, ROWS>(0, u.y)});
}
// prefix sums with the lane's own: row_shr 1, 2, 4, 8, row_bcast 15, 31
__device__ __forceinline__ double wave_prefix(double v)
{
    return plus_lane<0x143, 0xc>(plus_lane<0x142, 0xa>(plus_lane<0x118>(plus_lane<0x114>(plus_lane<0x112>(plus_lane<0x111>(v))))));
}
__device__ __forceinline__ double lane_of(double v, int lane)
{
    const u32x2 u = __builtin_bit_cast(u32x2, v);
    return __builtin_bit_cast(double, u32x2{(uint32_t)__builtin_amdgcn_readlane((int)u.x, lane), (uint32_t)__builtin_amdgcn_readlane((int)u.y, lane)});
}
__device__ __forceinline__ double wave_sum(double v) { return lane_of(wave_prefix(v), 63); }

// P and Q of N tokens, from v0 on, with probabilities p and q; `left`: q while the token is not rejected
template <int N> __device__ __forceinline__ void after_rejections(const Walk &s, int levels, int32_t v0, double (&P)[N], double (&Q)[N], double (&left)[N])
{
#pragma unroll 1
    for (int l = 0; l < levels; ++l) {
        const int32_t token = s.token[l];
        const double of_gap = s.of_gap[l], of_rest = s.of_rest[l];
#pragma unroll
        for (int i = 0; i < N; ++i) {
            const double gap = fmax(P[i] - Q[i], 0.0);
            P[i] = of_gap > 0.0 ? gap * of_gap : P[i];
            left[i] = v0 + i == token ? 0.0 : left[i];
            Q[i] = left[i] * of_rest;
        }
    }
}
// x: what is added up of four tokens, y: of q
__device__ __forceinline__ void weigh(const Walk &s, const f32x4_any &pv, const f32x4_any &qv, int32_t v0, double (&x)[4], double (&y)[4])
{
    double P[4], Q[4], left[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) P[i] = pv[i], left[i] = Q[i] = qv[i];
    after_rejections(s, s.w.levels, v0, P, Q, left);
#pragma unroll
    for (int i = 0; i < 4; ++i) x[i] = s.w.gap ? fmax(P[i] - Q[i], 0.0) : P[i], y[i] = v0 + i == s.w.token ? 0.0 : left[i];
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

// One sequence's inputs.
struct Sequence {
    const float *p, *q;
    const int32_t *tokens;
    const float *u_accept;
    int32_t V;
    __device__ __forceinline__ Sequence(const VerifyArgs &a, int64_t b)
        : p(a.p + b * a.nodes * a.V), q(a.q + b * a.inner * a.V), tokens(a.tokens + b * (a.nodes - 1)), u_accept(a.u_accept + b * (a.nodes - 1)), V((int32_t)a.V)
    {
    }
    __device__ __forceinline__ const float *p_of(const Weighing &w) const { return p + w.p_row * V; }
    __device__ __forceinline__ const float *q_of(const Weighing &w) const { return w.q_row >= 0 ? q + w.q_row * V : nullptr; }
};

// Tokens from .. end - 1 added up by the workgroup, in an order that depends on their number alone; `part`: 2 kWaves numbers that nobody reads any more.
__device__ __forceinline__ Sums add_up(const Walk &s, const Sequence &in, int32_t from, int32_t end, double *part)
{
    const float *p = in.p_of(s.w), *q = in.q_of(s.w);
    const int tid = threadIdx.x;
    double x = 0.0, y = 0.0;
#pragma unroll 1
    for (int32_t v0 = from; v0 < end; v0 += kTrip) {
        f32x4_any pv[2], qv[2];
#pragma unroll
        for (int j = 0; j < 2; ++j) {
            const int32_t v = v0 + (j * kThreads + tid) * 4;
            pv[j] = load4(p, v, end);
            qv[j] = q ? load4(q, v, end) : f32x4_any(0.0f);
        }
#pragma unroll
        for (int j = 0; j < 2; ++j) {
            double xs[4], ys[4];
            weigh(s, pv[j], qv[j], v0 + (j * kThreads + tid) * 4, xs, ys);
#pragma unroll
            for (int i = 0; i < 4; ++i) x += xs[i], y += ys[i];
        }
    }
    x = wave_sum(x), y = wave_sum(y);
    if ((tid & 63) == 0) part[tid >> 6] = x, part[kWaves + (tid >> 6)] = y;
    lds_barrier();
    Sums r{0.0, 0.0};
#pragma unroll
    for (int i = 0; i < kWaves; ++i) r.first += part[i], r.second += part[kWaves + i];
    return r;
}

// The sums of all pieces, by every wavefront.
__device__ __forceinline__ Sums total_of(const Sums *pieces, int n)
{
    const int lane = threadIdx.x & 63;
    double x = 0.0, y = 0.0;
#pragma unroll
    for (int i = 0; i < kMostPieces / 64; ++i) {
        const bool in = i * 64 + lane < n;
        const Sums v = pieces[in ? i * 64 + lane : 0];
        x += in ? v.first : 0.0, y += in ? v.second : 0.0;
    }
    return Sums{wave_sum(x), wave_sum(y)};
}

// The walk from where it is to where sums are needed, by all threads alike (`s` in LDS; thread 0 writes it and the accepted tokens).  `got`: the sums
// it waited for.
__device__ __forceinline__ void go_on(Walk &s, const VerifyArgs &a, const Sequence &in, Sums got, int32_t *out, int32_t *node, unsigned first_block)
{
    const int lane = threadIdx.x & 63;
    const bool writes = threadIdx.x == 0;                            // (the walk; accepted tokens, which the others come to as well, one workgroup)
    lds_barrier();
    int32_t n = s.n, next = s.next, depth = s.depth, known = s.known;
    int64_t row = s.row, rows = s.rows, nodes = s.nodes, children = s.children;
    const bool waited = s.phase == kWaiting;
    lds_barrier();
    if (waited) {
        if (writes) {
            s.token[n] = s.w.token;
            s.of_gap[n] = got.first > 0.0 ? 1.0 / got.first : 0.0;
            s.of_rest[n] = got.second > 0.0 ? 1.0 / got.second : 0.0;
        }
        known = got.first > 0.0;
        ++n, ++next;
        lds_barrier();
    }
    int phase = kWalking;
    Weighing w = s.w;
    while (phase == kWalking) {
        if (depth == a.gamma) {
            w = Weighing{nodes + row, -1, 0, 0, -1}, known = 0, phase = kDecided;
            break;
        }
        const int fan = a.tree[depth];
        const int64_t first = children + row * fan;
        const float *p = in.p + (nodes + row) * in.V, *q = in.q + (nodes + row) * in.V;
        // a lane to a child
        const int32_t mine = lane < fan ? in.tokens[first + lane] : -1;
        const float u_mine = lane < fan ? in.u_accept[first + lane] : 0.0f;
        const bool real = mine >= 0 && mine < in.V;
        const float p_mine = p[real ? mine : 0], q_mine = q[real ? mine : 0];
        int taken = -1;
        for (; next < fan; ++next) {
            const int32_t c = __builtin_amdgcn_readlane(mine, next);
            if (c < 0 || c >= in.V) continue;
            double P[1] = {__builtin_bit_cast(float, __builtin_amdgcn_readlane(__builtin_bit_cast(int, p_mine), next))};
            double Q[1] = {__builtin_bit_cast(float, __builtin_amdgcn_readlane(__builtin_bit_cast(int, q_mine), next))}, left[1] = {Q[0]};
            after_rejections(s, n, c, P, Q, left);
            // (what is no number accepts nothing: no comparison with it is true)
            const double ratio = Q[0] > 0.0 ? P[0] / Q[0] : Q[0] <= 0.0 && P[0] > 0.0 ? 1.0 : 0.0;
            const float u = __builtin_bit_cast(float, __builtin_amdgcn_readlane(__builtin_bit_cast(int, u_mine), next));
            if (u < 1.0f && (double)u < ratio) {
                taken = next;
                if (writes && blockIdx.x == first_block) out[depth] = c, node[depth] = (int32_t)(row * fan + taken);
                break;
            }
            w = Weighing{nodes + row, nodes + row, n, 1, c}, phase = kWaiting;
            break;
        }
        if (phase == kWaiting) break;
        if (taken < 0) {
            // from what P is ahead of Q at the last rejection, undivided: its sums are there; or where that was nothing from P
            if (!known) w = Weighing{nodes + row, nodes + row, n, 0, -1};
            phase = kDecided;
            break;
        }
        nodes += rows, children += rows * fan, row = row * fan + taken, rows *= fan;
        ++depth, n = 0, next = 0, known = 0;
    }
    lds_barrier();
    if (writes) {
        s.row = row, s.rows = rows, s.nodes = nodes, s.children = children;
        s.depth = depth, s.phase = phase, s.n = n, s.next = next, s.known = known, s.w = w;
    }
    lds_barrier();
}

__device__ __forceinline__ void begin(Walk &s, const Walk *from)
{
    if (threadIdx.x == 0) {
        if (from) {
            s = *from;
        } else {
            s.row = s.nodes = s.children = 0, s.rows = 1;
            s.depth = 0, s.phase = kWalking, s.n = 0, s.next = 0, s.known = 0, s.turn = 0;
        }
    }
    lds_barrier();
}

// pieces: (2, n_seq, kMostPieces), walks: (2, n_seq), in turn: the other launch's are being read
struct Between {
    Sums *pieces;
    Walk *walks;
};

// One round of a sequence: a workgroup to a piece of a row.
__global__ void __launch_bounds__(kThreads) round_kernel(VerifyArgs a, Between between, int round, int32_t per)
{
    __shared__ Walk s;
    __shared__ double part[2 * kWaves];
    const int64_t b = row_of_block();
    if (b >= a.n_seq) return;
    const int pieces = gridDim.x, turn = round & 1;
    Walk *to = between.walks + (turn * a.n_seq + b);
    begin(s, round > 0 ? between.walks + ((1 - turn) * a.n_seq + b) : nullptr);
    const Sequence in(a, b);
    Sums got{0.0, 0.0};
    const bool over = s.phase == kDecided && s.known;                // (what is drawn from is there; it only goes on to the next launch)
    if (!over) {
        if (s.phase == kWaiting) got = total_of(between.pieces + ((1 - turn) * a.n_seq + b) * kMostPieces, pieces);
        go_on(s, a, in, got, a.out + b * (a.gamma + 1), a.node + b * a.gamma, 0);
        if (!(s.phase == kDecided && s.known)) {
            const int32_t from = (int32_t)blockIdx.x * per;
            const Sums mine = add_up(s, in, from, min(from + per, in.V), part);
            if (threadIdx.x == 0) between.pieces[(turn * a.n_seq + b) * kMostPieces + blockIdx.x] = mine;
            if (threadIdx.x == 0) {
                s.turn = turn;
                if (s.phase == kDecided) s.known = 1;                // (or nothing, if their sum turns out to be)
            }
        }
    }
    if (blockIdx.x == 0) {
        lds_barrier();
        if (threadIdx.x == 0) *to = s;
    }
}

// The end of a walk: what the rounds left to be added up, and the token that is drawn.  One workgroup to a sequence.
__global__ void __launch_bounds__(kThreads) draw_kernel(VerifyArgs a, Between between, int rounds, int pieces, int32_t per)
{
    __shared__ Walk s;
    __shared__ double part[2][2 * kWaves];
    __shared__ Sums own[kMostPieces];
    __shared__ double before_piece;
    __shared__ int32_t piece, found, last;
    const int64_t b = blockIdx.x;
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const int turn = rounds & 1;                                     // (of the last round: 1 - turn)
    int32_t *out = a.out + b * (a.gamma + 1), *node = a.node + b * a.gamma;
    begin(s, between.walks + ((1 - turn) * a.n_seq + b));
    const Sequence in(a, b);
    const float u = a.u_sample[b];
    // sums of the pieces of a row by this workgroup alone
    auto add_all = [&]() {
        for (int i = 0; i < pieces; ++i) {
            const Sums v = add_up(s, in, i * per, min((i + 1) * per, in.V), part[i & 1]);
            if (tid == 0) own[i] = v;
        }
        lds_barrier();
    };
    if (s.phase == kWaiting) {
        Sums got = total_of(between.pieces + (s.turn * a.n_seq + b) * kMostPieces, pieces);
        go_on(s, a, in, got, out, node, blockIdx.x);
#pragma unroll 1
        while (s.phase == kWaiting) {                                // (a tree with more rejections than there were rounds)
            add_all();
            got = total_of(own, pieces);
            go_on(s, a, in, got, out, node, blockIdx.x);
            if (tid == 0 && s.phase == kDecided && s.known) s.turn = -1;
            lds_barrier();
        }
    }
    if (!s.known) {
        add_all();
        if (tid == 0) s.turn = -1;
        lds_barrier();
    }
    for (int i = tid; i < pieces && s.turn >= 0; i += kThreads) own[i] = between.pieces[(s.turn * a.n_seq + b) * kMostPieces + i];
    lds_barrier();

    // ---- the piece in which the sums pass u times their total; the last that has any (the last bits of the sums)
    const double total = total_of(own, pieces).first, bound = (double)u * total;
    if (wave == 0) {
        double before = 0.0, at_before = 0.0;
        int at = -1;
        for (int i0 = 0; i0 < pieces && (at < 0 || !(at_before + own[at].first > bound)); i0 += 64) {
            const double x = i0 + lane < pieces ? own[i0 + lane].first : 0.0;
            const double to = wave_prefix(x);
            const uint64_t some = __ballot(x > 0.0), there = __ballot(x > 0.0 && before + (to - x) + x > bound);
            const int l = there ? __builtin_ctzll(there) : some ? 63 - __builtin_clzll(some) : -1;
            if (l >= 0) at = i0 + l, at_before = before + lane_of(to - x, l);
            before += lane_of(to, 63);
        }
        if (lane == 0) piece = total > 0.0 ? at : -1, before_piece = at_before;
    }
    lds_barrier();
    int32_t token = -1;
    if (piece >= 0) {
        const float *p = in.p_of(s.w), *q = in.q_of(s.w);
        const int32_t end = min((piece + 1) * per, in.V);
        double before = before_piece;
#pragma unroll 1
        for (int32_t v0 = piece * per; v0 < end; v0 += kTrip) {
            double x[8], mine = 0.0;
            const int32_t v = v0 + tid * 8;
#pragma unroll
            for (int j = 0; j < 2; ++j) {
                double xs[4], ys[4];
                weigh(s, load4(p, v + 4 * j, end), q ? load4(q, v + 4 * j, end) : f32x4_any(0.0f), v + 4 * j, xs, ys);
#pragma unroll
                for (int i = 0; i < 4; ++i) x[4 * j + i] = v + 4 * j + i < end ? xs[i] : 0.0, mine += x[4 * j + i];
            }
            const double to = wave_prefix(mine);
            lds_barrier();
            if (lane == 63) part[0][wave] = to;
            if (tid == 0) found = INT32_MAX, last = -1;
            lds_barrier();
            double at = before + (to - mine);
#pragma unroll
            for (int w = 0; w < kWaves; ++w) at += w < wave ? part[0][w] : 0.0, before += part[0][w];
            int32_t there = INT32_MAX, some = -1;
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                at += x[i];
                if (x[i] > 0.0) {
                    some = v + i;
                    if (at > bound) there = min(there, v + i);
                }
            }
            if (there < INT32_MAX) atomicMin(&found, there);
            if (some >= 0) atomicMax(&last, some);
            lds_barrier();
            if (found < INT32_MAX) token = found;
            else if (last >= 0) token = last;
            if (found < INT32_MAX) break;
        }
    }
    if (tid == 0) {
        const int depth = s.depth;
        out[depth] = token;
        a.count[b] = depth + 1;
        for (int i = depth + 1; i <= a.gamma; ++i) out[i] = -1;
        for (int i = depth; i < a.gamma; ++i) node[i] = -1;
    }
}

int32_t piece_of(int64_t V) { return (int32_t)((V + (int64_t)kTrip * kMostPieces - 1) / ((int64_t)kTrip * kMostPieces)) * kTrip; }

}  // namespace

// (a launch has fewer than 2^32 threads)
bool verify_fits(int64_t n_seq, int64_t V) { return n_seq <= (0xffffffff / kThreads) / ((V + piece_of(V) - 1) / piece_of(V)); }

size_t verify_workspace_bytes(int64_t n_seq) { return (size_t)n_seq * 2 * (kMostPieces * sizeof(Sums) + sizeof(Walk)); }

hipError_t launch_verify(const VerifyArgs &a, void *ws, hipStream_t stream)
{
    const int32_t per = piece_of(a.V);
    const int pieces = (int)((a.V + per - 1) / per);
    int rounds = 1;
    for (int i = 0; i < a.gamma; ++i) rounds += a.tree[i] - 1;
    if (rounds > kMostRounds) rounds = kMostRounds;
    const Between between{static_cast<Sums *>(ws), reinterpret_cast<Walk *>(static_cast<unsigned char *>(ws) + (size_t)a.n_seq * 2 * kMostPieces * sizeof(Sums))};
    const dim3 grid((unsigned)pieces, (unsigned)(a.n_seq < kRowsY ? a.n_seq : kRowsY), (unsigned)((a.n_seq + kRowsY - 1) / kRowsY));
    for (int r = 0; r < rounds; ++r) round_kernel<<<grid, kThreads, 0, stream>>>(a, between, r, per);
    draw_kernel<<<(unsigned)a.n_seq, kThreads, 0, stream>>>(a, between, rounds, pieces, per);
    return hipGetLastError();
}

}  // namespace mamba
