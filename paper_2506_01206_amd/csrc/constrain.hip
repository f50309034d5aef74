// Logits under the rules that a verifier decodes by (penalties for repeated tokens, biases, grammar masks), and the children that a
// draft tree's branches propose under them (Sec. 4.1: a drafted token that the verifier's rules forbid is never accepted).
//
//   c = occurrences of v in the generated text of the row's sequence and in the row's own path through the tree
//   x = x > 0 ? x / repetition : x * repetition      where c > 0 or v stands in the prompt
//   x = (x - frequency c) - presence                 where c > 0
//   x = x + bias[v]
//   not allowed by the row's mask: -inf, and no candidate
//
// Every operation is one float32 operation, rounded: which of two tokens is ahead does not depend on how the compiler contracts.
#include "device_math.h"
#include "launch.h"
#include "logit_rows.h"

#include <type_traits>

namespace mamba {
namespace {

constexpr int kThreads = 256;
// A lane has one vector of 8 tokens.  What it does with a vector is long (quotients that round right, the rules, the search), and more vectors
// repeat it in the code, which a workgroup fetches as it goes: 3 children of one row of 50280 5.9 us with one, 8.2 with two, 13.3 with
// four (4.4 with one since the search is without branches); logits of 19 rows 3.6, 4.2 and 5.8.
constexpr int kSlice = kThreads * 8;                                 // tokens to a workgroup
constexpr int32_t kNoKey = INT32_MIN;                                // below every key

// What holds for one row of logits.
struct RowRules {
    bool known;                                                      // its indices are in range
    float repetition, presence, frequency;
    const int32_t *counts;
    const uint8_t *mask;                                             // nullptr: everything is allowed
};
template <bool COUNTS, bool MASK> __device__ __forceinline__ RowRules rules_of(const ConstrainArgs &c, int64_t m)
{
    RowRules r{true, 1.0f, 0.0f, 0.0f, nullptr, nullptr};
    if (c.penalties || c.counts) {
        const int64_t s = c.seq_idx ? c.seq_idx[m] : c.n_seq == 1 ? 0 : m;
        r.known = s >= 0 && s < c.n_seq;
        const int64_t safe = r.known ? s : 0;
        if (c.penalties) r.repetition = c.penalties[3 * safe], r.presence = c.penalties[3 * safe + 1], r.frequency = c.penalties[3 * safe + 2];
        if constexpr (COUNTS) r.counts = c.counts + safe * c.V;
    }
    if constexpr (MASK) {
        const int64_t g = c.mask_idx ? c.mask_idx[m] : c.n_masks == 1 ? 0 : m;
        r.known = r.known && g >= -1 && g < c.n_masks;
        if (r.known && g >= 0) r.mask = reinterpret_cast<const uint8_t *>(c.mask + g * ((c.V + 31) / 32));
    }
    return r;
}

// x / d rounded to nearest from y = 1 / d rounded to nearest: two corrections of x y by the exact remainder (P. Markstein, Computation of
// elementary functions on the IBM RISC System/6000 processor, 1990: with y so rounded and q off by less than one unit, q + (x - q d) y is
// rounded right).  Holds where nothing over- or underflows on the way; elsewhere the division itself.
__device__ __forceinline__ float divided(float x, float d, float y)
{
    float q = x * y;
    q = fmaf(fmaf(-q, d, x), y, q);
    return fmaf(fmaf(-q, d, x), y, q);
}
constexpr float kLeast = 0x1p-40f, kMost = 0x1p40f;

// The penalties on a lane's n logits.  Without branches, as a wavefront has tokens of all kinds.
template <int n> __device__ __forceinline__ void penalise(const RowRules &r, float (&x)[n], const int32_t (&count)[n])
{
#pragma clang fp contract(off)
    const float y = 1.0f / r.repetition;
    // Only what is above zero is divided.  As unsigned integers less one such values are in order, and zeros, negative values and NaN are beyond them:
    // a zero does not send its wavefront to the slow division (2 children of 96 rows with zeros among them 18.7 -> 16.5 us).
    uint32_t least = UINT32_MAX;
    float less[n], most = kLeast;
#pragma unroll
    for (int i = 0; i < n; ++i) {
        least = min(least, __float_as_uint(x[i]) - 1u), most = fmaxf(most, x[i]);
        less[i] = divided(x[i], r.repetition, y);
    }
    if (!__all(least >= __builtin_bit_cast(uint32_t, kLeast) - 1u && most <= kMost && r.repetition >= kLeast && r.repetition <= kMost)) {
#pragma unroll 1
        for (int i = 0; i < n; ++i) {                                // (rolled up: seldom run, and not to be fetched by the others)
            const float first = x[0], q = first / r.repetition;
#pragma unroll
            for (int j = 0; j + 1 < n; ++j) less[j] = less[j + 1], x[j] = x[j + 1];
            less[n - 1] = q, x[n - 1] = first;
        }
    }
#pragma unroll
    for (int i = 0; i < n; ++i) {
        const int32_t times = count[i] & 0x7fffffff;
        float v = x[i] > 0.0f ? less[i] : x[i] * r.repetition;
        v = count[i] != 0 ? v : x[i];
        const float f = r.frequency * (float)times;
        float w = v - f;
        w = w - r.presence;
        x[i] = times > 0 ? w : v;
    }
}

// A lane's 8 tokens of a slice of a row: their adjusted logits, and which of them count (allowed, of this row and no other lane's).
// Everything is requested ahead of the first use, at addresses that do not depend on a condition: a vector past the row's end is the last 8
// tokens of the row again, of which those that stand in the vector before it are left out.  (A row of fewer than 8 tokens is read token by
// token.)
// COUNTS: penalties with counts; BIAS, MASK: there are such
template <typename T, bool COUNTS, bool BIAS, bool MASK> struct Share {
    int32_t start;                                                   // first token of the vector as it was read
    float x[8];
    uint32_t valid;

    __device__ __forceinline__ void load(const ConstrainArgs &c, const T *row, int64_t m, int32_t slice, RowRules &r)
    {
        int32_t counts[8];
        float bias[8];
        uint32_t mask[2];
        const int32_t v0 = slice * kSlice + (int32_t)threadIdx.x * 8, V = (int32_t)c.V;
        if (V >= 8) {
            start = min(v0, V - 8);
            load8(row + start, x);
            if constexpr (BIAS) load8(c.bias + start, bias);
            r = rules_of<COUNTS, MASK>(c, m);
            if constexpr (COUNTS) load8(r.counts + start, counts);
            if constexpr (MASK) {
                const int32_t last = (V + 31) / 32 * 4 - 1, at = start >> 3;
                const uint8_t *bits = r.mask ? r.mask : reinterpret_cast<const uint8_t *>(c.mask);
                mask[0] = bits[at], mask[1] = bits[min(at + 1, last)];
            }
            __builtin_amdgcn_sched_barrier(0);
        } else {
            r = rules_of<COUNTS, MASK>(c, m);
            start = v0;
            if constexpr (MASK) mask[0] = mask[1] = r.mask ? r.mask[0] : 0;   // (the second is not looked at)
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const int32_t v = min(i, V - 1);                     // (only the first vector counts)
                x[i] = ld_io(row, v);
                if constexpr (BIAS) bias[i] = c.bias[v];
                if constexpr (COUNTS) counts[i] = r.counts[v];
            }
        }
        if constexpr (!COUNTS) {
#pragma unroll
            for (int i = 0; i < 8; ++i) counts[i] = 0;
        }
        // The row's path: a lane of each wavefront has a token of it, and those that stand in this slice are handed to all lanes.
        if (c.path && c.penalties) {
            for (int64_t t0 = 0; t0 < c.path_len; t0 += 64) {
                const int64_t t = t0 + (threadIdx.x & 63);
                const int32_t token = t < c.path_len ? c.path[m * c.path_len + t] : -1;
                uint64_t here = __ballot(token >= 0 && token < V && token / kSlice == slice);
                while (here) {
                    const int32_t one = __builtin_amdgcn_readlane(token, __builtin_ctzll(here));
                    here &= here - 1;
#pragma unroll
                    for (int i = 0; i < 8; ++i) counts[i] += start + i == one && (counts[i] & 0x7fffffff) != 0x7fffffff;
                }
            }
        }
        valid = 0xff;
        if constexpr (MASK) valid = r.mask ? (mask[0] | mask[1] << 8) >> (start & 7) & 0xff : 0xff;
        if (V >= 8) valid &= v0 < V ? 0xffu << (v0 - start) : 0u;    // (the shift is 0 but in a row's last vector)
        else valid &= v0 == 0 ? 0xffu >> (8 - V) : 0u;
        if (!r.known) valid = 0;
        if (c.penalties) penalise(r, x, counts);
#pragma unroll
        for (int i = 0; i < 8; ++i)
            if constexpr (BIAS) x[i] = x[i] + bias[i];
    }
};

// Bound by bytes where there are many rows: 128 rows of 131071 float32 logits with counts and masks, 201 MB, in 35.7 us (5.6 TB/s, what a large
// copy reaches); few rows are a launch and three dependent trips to memory (19 rows of 50280 in bfloat16: 3.6 us).
// grid: slices and rows (see row_of_block); out may be logits (a thread writes what it alone has read)
template <typename T, bool COUNTS, bool BIAS, bool MASK>
__global__ void __launch_bounds__(kThreads) constrain_kernel(const T *logits, T *out, ConstrainArgs c, int64_t M)
{
    const int64_t m = row_of_block();
    if (m >= M) return;
    const int32_t slice = blockIdx.x, v = slice * kSlice + (int32_t)threadIdx.x * 8, V = (int32_t)c.V;
    RowRules r;
    Share<T, COUNTS, BIAS, MASK> s;
    s.load(c, logits + m * c.V, m, slice, r);
    T *to = out + m * c.V;
#pragma unroll
    for (int i = 0; i < 8; ++i) s.x[i] = !r.known ? __int_as_float(0x7fc00000) : (s.valid >> i & 1) ? s.x[i] : -INFINITY;
    if (v + 8 <= V) {
        store8(to + v, s.x);
    } else if (v < V) {                                              // (the end of a row: only what is not another lane's)
        const int32_t first = V >= 8 ? v - s.start : 0, end = V >= 8 ? 8 : V;
#pragma unroll
        for (int i = 0; i < 8; ++i)
            if (i >= first && i < end) st_io(to, s.start + i, s.x[i]);
    }
}

template <int CTRL> __device__ __forceinline__ int32_t lane_max(int32_t v)
{
    return max(v, __builtin_amdgcn_update_dpp(INT32_MIN, v, CTRL, 0xf, 0xf, false));
}
// largest of the 64 lanes: quad_perm [1,0,3,2], [2,3,0,1], row_half_mirror, row_mirror, row_bcast:15, row_bcast:31
__device__ __forceinline__ int32_t wave_max(int32_t v)
{
    v = lane_max<0x140>(lane_max<0x141>(lane_max<0x4e>(lane_max<0xb1>(v))));
    return __builtin_amdgcn_readlane(lane_max<0x143>(lane_max<0x142>(v)), 63);
}
// Keys order as signed integers like the values (NaN as -inf, -0 as +0).
__device__ __forceinline__ int32_t key_of(float x)
{
    const float v = x != x ? -INFINITY : x + 0.0f;
    const int32_t b = __float_as_int(v);
    return b ^ ((b >> 31) & 0x7fffffff);
}
__device__ __forceinline__ float value_of(int32_t key) { return __int_as_float(key ^ ((key >> 31) & 0x7fffffff)); }

// child n of row m, by a whole wavefront: token, value, and the path that leads to it
__device__ __forceinline__ void write_child(const ConstrainArgs &c, int64_t m, int n, int k, int32_t key, int32_t token, int32_t *idx, float *val,
                                            int32_t *path_out, int lane)
{
    const bool some = key != kNoKey;
    const int64_t at = m * k + n;
    if (lane == 0) {
        idx[at] = some ? token : -1;
        val[at] = some ? value_of(key) : -INFINITY;
    }
    if (path_out)
        for (int64_t t = lane; t <= c.path_len; t += 64)
            path_out[at * (c.path_len + 1) + t] = t < c.path_len ? c.path[m * c.path_len + t] : some ? token : -1;
}

// The k best of one slice of one row.  A lane keeps its 8 tokens' keys in registers and offers the best; the workgroup's best is
// found k times, and only the wavefront that owned it looks through its registers again.  Bound by vector instructions, some 400 for a lane's
// 8 tokens: 2 children of 96 rows of 50280 10.0 us; a single row 4.4.
// grid: slices and rows; with one slice the result is the row's, with more the slices' go to `part` and merge_kernel takes over
template <typename T, bool COUNTS, bool BIAS, bool MASK>
__global__ void __launch_bounds__(kThreads)
children_kernel(const T *__restrict__ logits, int32_t *__restrict__ idx, float *__restrict__ val, int32_t *__restrict__ path_out,
                int2 *__restrict__ part, ConstrainArgs c, int64_t M, int k)
{
    const int64_t m = row_of_block(), slices = gridDim.x;
    if (m >= M) return;
    const int32_t slice = blockIdx.x;
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    RowRules r;
    Share<T, COUNTS, BIAS, MASK> s;
    s.load(c, logits + m * c.V, m, slice, r);
    int32_t key[8], best = kNoKey, best_at = 0;                      // first of the lane's largest
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const int32_t on = (int32_t)(s.valid << (31 - i)) >> 31;     // (all bits of one: no branch)
        key[i] = (key_of(s.x[i]) & on) | (kNoKey & ~on);
        const bool ahead = key[i] > best;
        best = max(best, key[i]), best_at = ahead ? i : best_at;
    }
    __shared__ int2 heads[2][kThreads / 64];
    for (int n = 0; n < k; ++n) {
        // (lanes, and wavefronts, have the tokens in their order: the first of equals has the lowest)
        const int32_t wk = wave_max(best), wt = __builtin_amdgcn_readlane(s.start + best_at, __builtin_ctzll(__ballot(best == wk)));
        if (lane == 0) heads[n & 1][wave] = make_int2(wk, wt);       // (the other half may still be being read)
        __syncthreads();
        int32_t win = kNoKey, token = -1;
#pragma unroll
        for (int w = 0; w < kThreads / 64; ++w) {
            const int2 h = heads[n & 1][w];
            if (h.x > win) win = h.x, token = h.y;
        }
        if (wave == 0) {
            if (slices == 1) write_child(c, m, n, k, win, token, idx, val, path_out, lane);
            else if (lane == 0) part[(m * slices + slice) * k + n] = make_int2(win, token);
        }
        if (best == win && s.start + best_at == token) {             // the owner's next
            const int32_t taken = best_at;
            best = kNoKey, best_at = 0;
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                key[i] = taken == i ? kNoKey : key[i];
                const bool ahead = key[i] > best;
                best = max(best, key[i]), best_at = ahead ? i : best_at;
            }
        }
    }
}

// The k best of a row's slices: one wavefront, which goes through the slices' candidates (k each: 75 for 3 children of a row of 50280)
// for the best one behind the one taken last.  A launch of one or two trips to memory: 2.5 us.
__global__ void __launch_bounds__(64)
merge_kernel(const int2 *__restrict__ part, int32_t *__restrict__ idx, float *__restrict__ val, int32_t *__restrict__ path_out, ConstrainArgs c,
             int64_t slices, int k)
{
    const int64_t m = blockIdx.x, n_part = slices * k;
    const int lane = threadIdx.x;
    part += m * n_part;
    const int2 first = lane < n_part ? part[lane] : make_int2(kNoKey, 0);
    int32_t win = INT32_MAX, token = -1;
    for (int n = 0; n < k; ++n) {
        int32_t best = kNoKey, best_token = INT32_MAX;
        auto offer = [&](int2 p) {
            if ((p.x < win || (p.x == win && p.y > token)) && (p.x > best || (p.x == best && p.y < best_token))) best = p.x, best_token = p.y;
        };
        offer(first);
        for (int64_t e = lane + 64; e < n_part; e += 64) offer(part[e]);
        win = wave_max(best);
        token = ~wave_max(best == win ? ~best_token : INT32_MIN);
        write_child(c, m, n, k, win, token, idx, val, path_out, lane);
        if (win == kNoKey) token = INT32_MAX;                        // nothing is left: no entry is behind this
    }
}

// Occurrences of every token in its sequence.  A workgroup has a range of the vocabulary and counts in LDS, over all of the
// sequence's tokens (numbers outside the vocabulary, such as the -1 of a padded row, are in no range), and writes its range whole:
// no clearing beforehand, and integer sums, whatever their order.  Bound by trips to memory one behind the other (its wavefronts wait for 76 % of
// their cycles): 1 sequence of 333 tokens 2.8 us, 8 of 8000 4.1 to 5.3.
// Narrow ranges while all their workgroups, two to a CU, are there at once: every one reads all of its sequence's tokens, but clears and
// writes a quarter.  Narrow | wide (us), a vocabulary of 50280: 1 sequence of 333 tokens 2.9 | 4.1, 8 of 8000 4.7 | 5.8, 16 of 8000
// 5.7 | 6.0, 32 of 16000 11.9 | 7.8, 64 of 2000 11.5 | 7.8.
constexpr int kCountThreads = 1024, kCountRange = 8192, kCountNarrow = 2048;
__global__ void __launch_bounds__(kCountThreads)
token_counts_kernel(const int32_t *__restrict__ tokens, int32_t *__restrict__ counts, int64_t L, int64_t V, int32_t range, int64_t n_seq, int accumulate, int prompt)
{
    __shared__ int32_t n[kCountRange];
    const int64_t s = row_of_block(), v0 = (int64_t)blockIdx.x * range;
    if (s >= n_seq) return;
    const int len = (int)min((int64_t)range, V - v0);
    for (int i = threadIdx.x; i < len; i += kCountThreads) n[i] = 0;
    __syncthreads();
    constexpr int kAhead = 8;
    for (int64_t t0 = threadIdx.x; t0 < L; t0 += kCountThreads * kAhead) {
        int64_t v[kAhead];
#pragma unroll
        for (int i = 0; i < kAhead; ++i) v[i] = t0 + i * kCountThreads < L ? (int64_t)tokens[s * L + t0 + i * kCountThreads] - v0 : -1;
#pragma unroll
        for (int i = 0; i < kAhead; ++i)
            if (v[i] >= 0 && v[i] < len) atomicAdd(&n[v[i]], 1);
    }
    __syncthreads();
    for (int i = threadIdx.x; i < len; i += kCountThreads) {
        const uint32_t old = accumulate ? (uint32_t)counts[s * V + v0 + i] : 0u, more = (uint32_t)n[i];
        const uint32_t sum = min((old & 0x7fffffffu) + more, 0x7fffffffu);
        counts[s * V + v0 + i] = (int32_t)(prompt ? old | (more ? 0x80000000u : 0u) : (old & 0x80000000u) | sum);
    }
}

int64_t slices_of(int64_t V) { return (V + kSlice - 1) / kSlice; }

}  // namespace

// (a launch has fewer than 2^32 threads)
bool constrain_grid_ok(int64_t M, int64_t V) { return M <= (0xffffffff / kThreads) / (slices_of(V) > 0 ? slices_of(V) : 1); }
bool token_counts_grid_ok(int64_t n_seq, int64_t V) { return n_seq <= (0xffffffff / kCountThreads) / ((V + kCountRange - 1) / kCountRange); }

size_t children_workspace_bytes(int64_t M, int64_t V, int k)
{
    const int64_t slices = slices_of(V);
    return slices > 1 ? (size_t)(M * slices * k) * sizeof(int2) : 0;
}

namespace {
dim3 grid_of(int64_t M, int64_t V)
{
    return dim3((unsigned)slices_of(V), (unsigned)(M < kRowsY ? M : kRowsY), (unsigned)((M + kRowsY - 1) / kRowsY));
}

// F with the rules that a call has as constants: their absence costs nothing then, and what there is is requested without conditions
template <typename F> auto with_rules(const ConstrainArgs &c, F f)
{
    const int rules = (c.counts && c.penalties ? 1 : 0) | (c.bias ? 2 : 0) | (c.mask ? 4 : 0);
    switch (rules) {
    case 0: return f(std::false_type(), std::false_type(), std::false_type());
    case 1: return f(std::true_type(), std::false_type(), std::false_type());
    case 2: return f(std::false_type(), std::true_type(), std::false_type());
    case 3: return f(std::true_type(), std::true_type(), std::false_type());
    case 4: return f(std::false_type(), std::false_type(), std::true_type());
    case 5: return f(std::true_type(), std::false_type(), std::true_type());
    case 6: return f(std::false_type(), std::true_type(), std::true_type());
    default: return f(std::true_type(), std::true_type(), std::true_type());
    }
}
}  // namespace

hipError_t launch_constrain(const void *logits, void *out, const ConstrainArgs &c, int64_t M, int io, hipStream_t stream)
{
    const dim3 grid = grid_of(M, c.V);
    return with_rules(c, [&](auto counts, auto bias, auto mask) {
        if (io == kIoBf16)
            constrain_kernel<bf16_t, counts.value, bias.value, mask.value>
                <<<grid, kThreads, 0, stream>>>(static_cast<const bf16_t *>(logits), static_cast<bf16_t *>(out), c, M);
        else
            constrain_kernel<float, counts.value, bias.value, mask.value>
                <<<grid, kThreads, 0, stream>>>(static_cast<const float *>(logits), static_cast<float *>(out), c, M);
        return hipGetLastError();
    });
}

hipError_t launch_children(const void *logits, int32_t *idx, float *val, int32_t *path_out, void *ws, const ConstrainArgs &c, int64_t M, int k, int io,
                           hipStream_t stream)
{
    const int64_t slices = slices_of(c.V);
    const dim3 grid = grid_of(M, c.V);
    int2 *part = static_cast<int2 *>(ws);
    const hipError_t e = with_rules(c, [&](auto counts, auto bias, auto mask) {
        if (io == kIoBf16)
            children_kernel<bf16_t, counts.value, bias.value, mask.value>
                <<<grid, kThreads, 0, stream>>>(static_cast<const bf16_t *>(logits), idx, val, path_out, part, c, M, k);
        else
            children_kernel<float, counts.value, bias.value, mask.value>
                <<<grid, kThreads, 0, stream>>>(static_cast<const float *>(logits), idx, val, path_out, part, c, M, k);
        return hipGetLastError();
    });
    if (e != hipSuccess || slices == 1) return e;
    merge_kernel<<<(unsigned)M, 64, 0, stream>>>(part, idx, val, path_out, c, slices, k);
    return hipGetLastError();
}

hipError_t launch_token_counts(const int32_t *tokens, int32_t *counts, int64_t n_seq, int64_t L, int64_t V, int accumulate, int prompt,
                               hipStream_t stream)
{
    const int64_t narrow = (V + kCountNarrow - 1) / kCountNarrow;
    const int range = n_seq * narrow <= 512 ? kCountNarrow : kCountRange;
    const dim3 grid((unsigned)((V + range - 1) / range), (unsigned)(n_seq < kRowsY ? n_seq : kRowsY), (unsigned)((n_seq + kRowsY - 1) / kRowsY));
    token_counts_kernel<<<grid, kCountThreads, 0, stream>>>(tokens, counts, L, V, range, n_seq, accumulate, prompt);
    return hipGetLastError();
}

}  // namespace mamba
