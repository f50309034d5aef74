// Children drawn from the drafter's distribution (Sec. 4.1: a node's N_i children are samples of q_i), and the next tokens that a verifier
// draws, from given random numbers.  Of a row of logits x, T the temperature:
//
//   w = exp((x - max x) / T)                     T = 0: one for the first of the largest, zero for all others
//   kept: the tokens with w >= min_p; of those the top_k largest; of those the fewest, largest first, that make up top_p of their sum
//   q = w / (sum over what is kept)
//   child j: the first token, in the order of the vocabulary, up to which the w of what is kept and not drawn yet add up to more
//   than u_j of their sum
//
// Tokens are in the order of their logits, ties in the order of the vocabulary: what is kept is everything down to one token of that order, the cut.
//
// Whether a token is the one at which a sum passes its bound is a matter of the last bits of that sum, and float32 has too few of them for some ten
// thousand tokens.  So weights are formed in float64 and added up as whole multiples of 2^-s, s as large as 64 bits hold the sum of a row
// and float64 the multiples (47 for 50280 tokens, 51 at most).  Integer sums do not depend on their order.
//
// A row is cut into chunks.  bins_kernel has a chunk each: its weights, relative to its own largest, by bins of an eighth of an octave and more, whose borders
// are the same for all chunks.  From their sums plan_kernel, a workgroup to a row, sees in which bins a cut may lie; gather_kernel, again by chunks,
// brings the tokens of those bins together, and draw_kernel finds the cuts among them and draws.  Only dist_kernel writes a row.
#include "device_math.h"
#include "launch.h"
#include "logit_rows.h"

// Every operation is one rounding: kernels that form the same weights and sums come to the same units.
#pragma clang fp contract(off)

namespace mamba {
namespace {

typedef unsigned long long u64;

constexpr int kThreads = 256;                                        // of the kernels that have a chunk of a row
constexpr int kSlice = kThreads * 8;                                 // tokens of a chunk
constexpr int kMaxChunks = 1024;
constexpr int kBins = 128;                                           // of the weights of a row or chunk
constexpr int kWide = 1024, kWideWaves = kWide / 64;                 // threads of the kernel that has a row
constexpr int kList = 7168;                                          // tokens of bins with a cut that are brought together (more, in flat rows: scan_cut)

// Tokens in order: a larger number is ahead.  Logits order as signed integers (-0 as +0), ties by the lower index.
__device__ __forceinline__ uint32_t key_of(float x)
{
    const int32_t b = __float_as_int(x + 0.0f);
    return (uint32_t)(b ^ ((b >> 31) & 0x7fffffff)) ^ 0x80000000u;
}
// A token's place in that order: its logit's key, and below it `bits` bits of the index.  A bfloat16 logit has 16 bits of a key.
template <typename T> struct Order {
    static constexpr bool kShort = sizeof(T) == 2;
    int bits;
    __device__ __forceinline__ u64 place(float x, int32_t token) const
    {
        return (u64)(kShort ? key_of(x) >> 16 : key_of(x)) << bits | (((u64)1 << bits) - 1 - (u64)token);
    }
    __device__ __forceinline__ uint32_t key(u64 place) const { return (uint32_t)(place >> bits); }
    __device__ __forceinline__ float logit(u64 place) const
    {
        uint32_t k = key(place);
        if (kShort) k = k << 16 | (k & 0x8000u ? 0u : 0xffffu);
        const int32_t b = (int32_t)(k ^ 0x80000000u);
        return __int_as_float(b ^ ((b >> 31) & 0x7fffffff));
    }
    __device__ __forceinline__ int32_t token(u64 place) const { return (int32_t)(((u64)1 << bits) - 1 - (place & (((u64)1 << bits) - 1))); }
};

__device__ __forceinline__ bool counts(float x) { return x > -INFINITY; }   // (no NaN, which is as -inf)

// Weight of x relative to `most`, the largest logit (of the row, of a chunk, of what is left): 2^y, y = (x - most) log2 e / T, as 2^n 2^f with
// |f| <= 1/2 and 2^f by its Taylor series, whose next term is below 2^-47 of it.  (An infinite logit leaves the others nothing.)
// The coefficients are held in scalar registers: as literals of the multiply-adds each would be brought into a pair of vector registers first, for every
// weight again (66 instructions a token of bins_kernel instead of 37).
constexpr int kTerms = 11;
struct Weights {
    double rate;                                                     // log2 e / T
    double c[kTerms];                                                // ln 2 ^ i / i!, the last first
    __device__ __forceinline__ void set(float T)
    {
        rate = 1.4426950408889634074 / (double)T;
        constexpr double k1 = 0.69314718055994530942, k2 = k1 * k1 / 2, k3 = k2 * k1 / 3, k4 = k3 * k1 / 4, k5 = k4 * k1 / 5, k6 = k5 * k1 / 6, k7 = k6 * k1 / 7,
                         k8 = k7 * k1 / 8, k9 = k8 * k1 / 9, k10 = k9 * k1 / 10, k11 = k10 * k1 / 11;
        constexpr double k[kTerms] = {k11, k10, k9, k8, k7, k6, k5, k4, k3, k2, k1};
#pragma unroll
        for (int i = 0; i < kTerms; ++i) {
            c[i] = k[i];
            asm("" : "+s"(c[i]));
        }
    }
    __device__ __forceinline__ double power(float x, float most, double *n) const   // 2^f of a finite most
    {
        const double y = fmax(((double)x - (double)most) * rate, -1100.0);
        *n = __builtin_rint(y);
        const double f = y - *n;
        double e = c[0];
#pragma unroll
        for (int i = 1; i < kTerms; ++i) e = __builtin_fma(e, f, c[i]);
        return __builtin_fma(e, f, 1.0);
    }
    __device__ __forceinline__ double of(float x, float most) const
    {
        double n;
        const double e = power(x, most, &n);
        return most < INFINITY ? __builtin_ldexp(e, (int)n) : x == most ? 1.0 : 0.0;
    }
    // the same in units of 2^-scale, rounded (to even: 2^52 is added, which leaves the units as the last bits)
    __device__ __forceinline__ u64 units(float x, float most, int scale) const
    {
        double n;
        const double e = power(x, most, &n), v = __builtin_ldexp(e, (int)n + scale) + 0x1p52;
        return most < INFINITY ? (u64)__builtin_bit_cast(int64_t, v) - 0x4330000000000000ull : x == most ? (u64)1 << scale : 0;
    }
};

// What a row is drawn by.
struct Settings {
    Weights weights;
    float T;                                                         // 1 where a row is greedy
    float per_bin;                                                   // bins to a unit of logits
    float min_p, top_p;                                              // 0 or less: off; 1 or more: off
    int32_t top_k;                                                   // 0: off
    bool known;                                                      // its index is in range and its numbers are numbers
};
__device__ __forceinline__ Settings settings_of(const SampleArgs &a, int64_t m)
{
    const int64_t s = a.seq_idx ? a.seq_idx[m] : a.n_seq == 1 ? 0 : m;
    const bool in = s >= 0 && s < a.n_seq;
    const int64_t safe = in ? s : 0;
    const float T = a.params[3 * safe], top_p = a.params[3 * safe + 1], min_p = a.params[3 * safe + 2];
    const int32_t top_k = a.top_k ? a.top_k[safe] : 0;
    Settings r;
    r.known = in && T >= 0.0f && top_p == top_p && min_p == min_p;
    const bool greedy = r.known && T == 0.0f, drawn = r.known && !greedy;   // greedy: the first of the largest; a row that is not known is not looked at
    r.T = drawn ? T : 1.0f;
    r.weights.set(r.T);
    r.per_bin = fminf(fmaxf((float)(r.weights.rate * 8.0), 1e-30f), 1e30f);   // eighths of an octave
    r.min_p = drawn ? fminf(min_p, 1.0f) : 0.0f;
    r.top_p = drawn ? top_p : 1.0f;
    r.top_k = greedy ? 1 : drawn && top_k > 0 ? top_k : 0;
    return r;
}

// Marks are whole eighths of an octave of x / T, whatever the largest logit is.  Bins go down from the largest's mark, rounded up to a whole octave: a
// mark each for ten octaves, two for nine, eight for twelve, so that a bin of one largest is made up of whole bins of any smaller one; the last has all
// below.  (The flatter a row, the more of its tokens are in an octave, and the fewer octaves it takes down to where top-p cuts it: 131071 normally
// distributed logits, divided by T, with a deviation of 1.3 have 3400 tokens in the bin of the cut, with 2 4500, with 4 1200.)
constexpr float kEndMark = 0x1p29f;                              // (marks of a row are 2^30 apart at most: their differences are integers too)
__device__ __forceinline__ float scale_of(float x, float per_bin) { return __builtin_amdgcn_fmed3f(x * per_bin, -kEndMark, kEndMark); }
__device__ __forceinline__ int mark_of(float x, float per_bin) { return (int)floorf(scale_of(x, per_bin)); }
__device__ __forceinline__ int top_mark_of(float x, float per_bin) { return (mark_of(x, per_bin) + 7) & ~7; }
constexpr int kOnes = 80, kTwos = 36, kAfterOnes = kOnes, kAfterTwos = kOnes + 2 * kTwos;   // bins, and marks down to their end
__device__ __forceinline__ int bin_at(int below)
{
    const int b = below < kAfterOnes ? below : below < kAfterTwos ? kOnes + ((below - kAfterOnes) >> 1) : kOnes + kTwos + ((below - kAfterTwos) >> 3);
    return max(min(b, kBins - 1), 0);
}
__device__ __forceinline__ int bin_of(int mark, int top_mark) { return bin_at(top_mark - mark); }
__device__ __forceinline__ int start_of(int bin)                     // its first mark, down from the top
{
    return bin <= kOnes ? bin : bin <= kOnes + kTwos ? kAfterOnes + 2 * (bin - kOnes) : kAfterTwos + 8 * (bin - kOnes - kTwos);
}

// A lane's 8 tokens: a vector past the row's end is the last 8 of the row again, of which those that stand in the vector before it are left out.
struct Eight {
    int32_t start;
    uint32_t valid;
    float x[8];
    template <typename T> __device__ __forceinline__ void load(const T *row, int32_t v0, int32_t V)
    {
        if (V >= 8) {
            start = min(v0, V - 8);
            load8(row + start, x);
            valid = v0 < V ? 0xffu << (v0 - start) & 0xffu : 0u;
        } else {
            start = 0;
#pragma unroll
            for (int i = 0; i < 8; ++i) x[i] = ld_io(row, min(i, V - 1));
            valid = v0 == 0 ? 0xffu >> (8 - V) : 0u;
        }
    }
    // what does not count as -inf (the largest of a NaN and a number is the number)
    __device__ __forceinline__ void settle()
    {
#pragma unroll
        for (int i = 0; i < 8; ++i) x[i] = fmaxf(x[i], -INFINITY);
        if (valid != 0xff) {
#pragma unroll
            for (int i = 0; i < 8; ++i) x[i] = valid >> i & 1 ? x[i] : -INFINITY;
        }
    }
};

template <int CTRL, int ROWS = 0xf> __device__ __forceinline__ u64 plus_lane(u64 v)
{
    return v + ((u64)from_lane<CTRL, ROWS>(0, (uint32_t)(v >> 32)) << 32 | from_lane<CTRL, ROWS>(0, (uint32_t)v));
}
// prefix sums with the lane's own: row_shr 1, 2, 4, 8, row_bcast 15, 31
__device__ __forceinline__ u64 wave_prefix(u64 v)
{
    return plus_lane<0x143, 0xc>(plus_lane<0x142, 0xa>(plus_lane<0x118>(plus_lane<0x114>(plus_lane<0x112>(plus_lane<0x111>(v))))));
}
__device__ __forceinline__ u64 lane_of(u64 v, int lane)
{
    return (u64)(uint32_t)__builtin_amdgcn_readlane((int)(v >> 32), lane) << 32 | (uint32_t)__builtin_amdgcn_readlane((int)v, lane);
}
__device__ __forceinline__ u64 wave_sum(u64 v) { return lane_of(wave_prefix(v), 63); }
template <int CTRL> __device__ __forceinline__ uint32_t max_lane(uint32_t v) { return max(v, from_lane<CTRL>(v, v)); }
// the largest of the wavefront: quad_perm [1,0,3,2], [2,3,0,1], row_half_mirror, row_mirror, row_bcast 15, 31
__device__ __forceinline__ uint32_t wave_max(uint32_t v)
{
    v = max_lane<0x143>(max_lane<0x142>(max_lane<0x140>(max_lane<0x141>(max_lane<0x4e>(max_lane<0xb1>(v))))));
    return (uint32_t)__builtin_amdgcn_readlane((int)v, 63);
}
__device__ __forceinline__ float wave_max(float v)
{
    const uint32_t k = wave_max(key_of(v));                          // (no NaN here)
    const int32_t b = (int32_t)(k ^ 0x80000000u);
    return __int_as_float(b ^ ((b >> 31) & 0x7fffffff));
}

// What bins_kernel leaves of every chunk: its largest logit, and up to each of its bins (from its own largest's down) the units relative to that logit
// and the number of tokens.
struct Chunks {
    u64 *mass;                                                       // (chunks, kBins)
    uint32_t *number;                                                // the same; only where the row has a top-k
    float *most;                                                     // (chunks)
};

// ---- the weights of a chunk by bins: a workgroup to a chunk, a thread to eight tokens
// Bound by float64 arithmetic and LDS: some forty instructions and two atomics a token.  128 rows of 131071 float32 logits 36 us (1.9 TB/s; the loads
// alone 17), 96 of 50280 bfloat16 ones 14, one row 4 to 5.  (The last bin, which may have most of a row, is added up in registers: atomics on one
// address follow one another.)
template <typename T>
__global__ void __launch_bounds__(kThreads) bins_kernel(const T *__restrict__ logits, Chunks to, SampleArgs a, int scale)
{
    const int64_t m = row_of_block(), chunk = m * gridDim.x + blockIdx.x;
    if (m >= a.M) return;
    __shared__ float part[kThreads / 64];
    __shared__ u64 mass[kBins];
    __shared__ uint32_t number[kBins];
    __shared__ u64 first_mass;
    __shared__ uint32_t first_number;
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    Eight e;
    e.load(logits + m * a.V, (int32_t)blockIdx.x * kSlice + tid * 8, (int32_t)a.V);
    const Settings r = settings_of(a, m);
    if (tid < kBins) mass[tid] = 0, number[tid] = 0;
    e.settle();
    float top = -INFINITY;
#pragma unroll
    for (int j = 0; j < 8; ++j) top = fmaxf(top, e.x[j]);
    top = wave_max(top);
    if (lane == 0) part[wave] = top;
    lds_barrier();
    top = fmaxf(fmaxf(part[0], part[1]), fmaxf(part[2], part[3]));
    const int top_mark = top_mark_of(top, r.per_bin);
    u64 last_mass = 0;                                               // (of the last bin: it may have most of the tokens)
    uint32_t last_number = 0;
    u64 w[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) w[j] = r.weights.units(e.x[j], top, scale);   // (-infinity: none, as its weight is; in the last bin)
#pragma unroll
    for (int j = 0; j < 8; ++j) {
        const int b = bin_of(mark_of(e.x[j], r.per_bin), top_mark);
        if (b < kBins - 1) {
            atomicAdd(&mass[b], w[j]);
            if (r.top_k > 0) atomicAdd(&number[b], 1u);
        } else {
            last_mass += w[j], last_number += counts(e.x[j]);
        }
    }
    last_mass = wave_sum(last_mass);
    if (lane == 0) atomicAdd(&mass[kBins - 1], last_mass);
    if (r.top_k > 0) {
        last_number = (uint32_t)wave_sum((u64)last_number);
        if (lane == 0) atomicAdd(&number[kBins - 1], last_number);
    }
    lds_barrier();
    u64 v = 0, n = 0;
    if (wave < 2) {
        v = wave_prefix(mass[tid]);
        n = r.top_k > 0 ? wave_prefix((u64)number[tid]) : 0;
        if (tid == 63) first_mass = v, first_number = (uint32_t)n;
    }
    lds_barrier();
    if (wave == 1) v += first_mass, n += first_number;
    if (tid < kBins) {
        to.mass[chunk * kBins + tid] = v;
        if (r.top_k > 0) to.number[chunk * kBins + tid] = (uint32_t)n;
    }
    if (tid == 0) to.most[chunk] = top;
}

constexpr int kNoChunk = 1 << 20;
// the bin of a chunk up to which it stands ahead of the row's mark `below` (-1: no bin does)
__device__ __forceinline__ int chunk_bin(int below, int shift) { return below > shift ? bin_at(below - shift) - 1 : -1; }
__device__ __forceinline__ u64 scaled(u64 v, double factor) { return (u64)((double)v * factor + 0.5); }

// Bins that a cut of the row may lie in, ahead of knowing the cuts: min-p's from its border (a float32 neighbourhood of it), top-k's from the
// numbers, top-p's from the least and the most that may be left of the others' cuts.
struct CutBins {
    int min_first, min_last;                                         // bins before the first pass min-p whole, behind the last none (-1, kBins - 1: off)
    float min_above;                                                 // what passes has a larger logit, or stands in one of these bins
    int k_bin, p_first, p_last;                                      // (-1: off)
    __device__ __forceinline__ bool any() const { return min_first >= 0 || k_bin >= 0 || p_first >= 0; }
    __device__ __forceinline__ bool has(int b) const { return (b >= min_first && b <= min_last && min_first >= 0) || b == k_bin || (b >= p_first && b <= p_last && p_first >= 0); }
};
// What plan_kernel leaves of a row.
struct RowBins {
    u64 mass[kBins];                                                 // up to each bin over all chunks, in units relative to the row's largest logit
    uint32_t number[kBins];
    CutBins cuts;
    float top, per_bin;                                              // the largest logit, bins to a unit of logits
    uint32_t listed;                                                 // tokens of those bins
};
// and of each of its chunks
struct ChunkScale {
    double factor;                                                   // the weight of its largest logit
    float most;
    int shift;                                                       // by how many marks it is behind (kNoChunk: it has none)
};

// the first bin up to which the sums are `need` or more (the last bin where there is none), by a whole wavefront
template <typename N> __device__ __forceinline__ int reaching_bin(const N *upto, u64 need, int lane)
{
    const uint64_t lower = __ballot(upto[lane] >= need), upper = __ballot(upto[lane + 64] >= need);
    return lower ? __builtin_ctzll(lower) : upper ? 64 + __builtin_ctzll(upper) : kBins - 1;
}
template <typename N> __device__ __forceinline__ u64 ahead_of(const N *upto, int bin) { return bin > 0 ? (u64)upto[bin - 1] : 0; }

// v p rounded up, at least one, exactly: p has 24 bits
__device__ __forceinline__ u64 share_of(u64 v, float p)
{
    if (!(p > 0.0f)) return 1;
    const u64 f = (u64)((double)p * 18446744073709551616.0), high = __umul64hi(v, f);   // 2^64, p < 1
    return max(high + (v * f != 0), (u64)1);
}

template <typename T> __device__ __forceinline__ CutBins cut_bins(const RowBins &s, const Settings &r, float top, int lane)
{
    CutBins c{-1, kBins - 1, 0.0f, -1, -1, -1};
    const int top_mark = top_mark_of(top, r.per_bin);
    if (r.min_p > 0.0f) {
        const float away = r.T * (log2_hw(r.min_p) * kLn2), border = top + away;
        // (roundings of these, and the logarithm's: near one, where a weight's own rounding counts too, not relative to it)
        const float around = fmaxf(fmaxf(fabsf(border), fabsf(top)), fabsf(away)) * 0x1p-18f + r.T * 0x1p-20f;
        float above = border + around;
        // (a logit of the row's type, so that what is above it has a larger key)
        if (Order<T>::kShort) above = above >= 0.0f ? __uint_as_float((__float_as_uint(above) + 0xffffu) & 0xffff0000u) : __uint_as_float(__float_as_uint(above) & 0xffff0000u);
        if (above < INFINITY && border - around > -INFINITY && log2_hw(r.min_p) > -INFINITY) {
            c.min_first = bin_of(mark_of(above, r.per_bin), top_mark);
            c.min_last = bin_of(mark_of(border - around, r.per_bin), top_mark);
            c.min_above = above;
        } else {
            c.min_first = 0;
        }
    }
    u64 least = c.min_first >= 0 ? ahead_of(s.mass, c.min_first) : s.mass[kBins - 1], most = s.mass[c.min_last];
    if (r.top_k > 0 && (u64)r.top_k < s.number[c.min_last]) {
        c.k_bin = reaching_bin(s.number, (u64)r.top_k, lane);
        least = min(least, ahead_of(s.mass, c.k_bin)), most = min(most, s.mass[c.k_bin]);
    }
    if (r.top_p < 1.0f) {
        c.p_first = reaching_bin(s.mass, share_of(least, r.top_p), lane);
        c.p_last = max(reaching_bin(s.mass, share_of(most, r.top_p), lane), c.p_first);
    }
    return c;
}

// ---- the sums of a row, and in which bins its cuts lie: one workgroup to a row
// Bound by trips to memory, one after the other: the chunks' largest logits, then their bins.  One row of 50280 5.9 us, 128 of 131071 8.2.
template <typename T>
__global__ void __launch_bounds__(kWide) plan_kernel(Chunks from, RowBins *__restrict__ rows, ChunkScale *__restrict__ scales, SampleArgs a, int chunks)
{
    constexpr int kGroups = kWide / kBins, kAhead = 8;
    __shared__ RowBins s;
    __shared__ ChunkScale scale[kMaxChunks];
    __shared__ u64 mass_part[kWide];
    __shared__ uint32_t number_part[kWide];
    __shared__ float part[kWideWaves];
    const int64_t m = blockIdx.x;
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, bin = tid & (kBins - 1), group = tid / kBins;
    const float own = tid < chunks ? from.most[m * chunks + tid] : -INFINITY;
    const Settings r = settings_of(a, m);
    float top = wave_max(own);
    if (lane == 0) part[wave] = top;
    lds_barrier();
    top = wave_max(part[lane & (kWideWaves - 1)]);
    const int top_mark = top_mark_of(top, r.per_bin);
    if (tid < chunks) {
        const bool some = counts(own);
        const ChunkScale mine{some ? r.weights.of(own, top) : 0.0, own, some ? min(top_mark - top_mark_of(own, r.per_bin), kNoChunk - 1) : kNoChunk};
        scale[tid] = mine;
        scales[m * chunks + tid] = mine;
    }
    lds_barrier();
    u64 v = 0;
    uint32_t n = 0;
#pragma unroll 1
    for (int i0 = group; i0 < chunks; i0 += kGroups * kAhead) {
        u64 mass[kAhead];
        uint32_t number[kAhead];
#pragma unroll
        for (int j = 0; j < kAhead; ++j) {
            const int i = min(i0 + j * kGroups, chunks - 1), shift = scale[i].shift, b = bin == kBins - 1 ? bin : chunk_bin(start_of(bin + 1), shift);
            const bool is = i0 + j * kGroups < chunks && shift < kNoChunk && b >= 0;
            const int64_t at = (m * chunks + i) * kBins + (is ? b : 0);
            mass[j] = is ? from.mass[at] : 0;
            number[j] = is && r.top_k > 0 ? from.number[at] : 0;
        }
#pragma unroll
        for (int j = 0; j < kAhead; ++j) v += scaled(mass[j], scale[min(i0 + j * kGroups, chunks - 1)].factor), n += number[j];
    }
    mass_part[tid] = v;
    number_part[tid] = n;
    lds_barrier();
    if (tid < kBins) {
#pragma unroll
        for (int g = 1; g < kGroups; ++g) v += mass_part[g * kBins + tid], n += number_part[g * kBins + tid];
        s.mass[tid] = v, s.number[tid] = n;
        rows[m].mass[tid] = v, rows[m].number[tid] = n;
    }
    lds_barrier();
    if (wave == 0) {
        CutBins c{-1, kBins - 1, 0.0f, -1, -1, -1};
        if (r.known && counts(top)) c = cut_bins<T>(s, r, top, lane);
        if (lane == 0) rows[m].cuts = c, rows[m].top = top, rows[m].per_bin = r.per_bin, rows[m].listed = 0;
    }
}

// ---- the tokens of those bins: a workgroup to a chunk
// The row once more, against a range of marks for every cut.  128 rows of 131071 float32 logits 13 us (5.1 TB/s, from the last-level cache in part), one
// row 3 to 4: the launch and three trips to memory.
template <typename T>
__global__ void __launch_bounds__(kThreads)
gather_kernel(const T *__restrict__ logits, RowBins *__restrict__ rows, u64 *__restrict__ list, int64_t M, int32_t V, Order<T> order)
{
    const int64_t m = row_of_block();
    if (m >= M) return;
    __shared__ uint32_t found, base;
    const int tid = threadIdx.x;
    const CutBins c = rows[m].cuts;
    const float top = rows[m].top, per_bin = rows[m].per_bin;
    Eight e;
    e.load(logits + m * V, (int32_t)blockIdx.x * kSlice + tid * 8, V);
    if (tid == 0) found = 0;
    if (!c.any()) return;
    lds_barrier();
    // the bins as ranges of marks, both ends among them (integers, as the bins were made from: from 2^24 on float32 has no odd ones)
    const int top_mark = top_mark_of(top, per_bin);
    uint32_t hits = 0;
    auto mark_hits = [&](int first_bin, int last_bin) {
        const int from = last_bin >= kBins - 1 ? INT32_MIN : top_mark - start_of(last_bin + 1) + 1, to = first_bin == 0 ? INT32_MAX : top_mark - start_of(first_bin);
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            const int mark = mark_of(e.x[j], per_bin);
            hits |= (uint32_t)(mark >= from && mark <= to) << j;
        }
    };
    e.settle();
    if (c.p_first >= 0) mark_hits(c.p_first, c.p_last);
    if (c.k_bin >= 0) mark_hits(c.k_bin, c.k_bin);
    if (c.min_first >= 0) mark_hits(c.min_first, c.min_last);
    uint32_t at = 0;
    if (hits) {
#pragma unroll
        for (int j = 0; j < 8; ++j) hits &= counts(e.x[j]) ? ~0u : ~(1u << j);
        at = atomicAdd(&found, (uint32_t)__popc(hits));
    }
    lds_barrier();
    if (tid == 0) base = found ? atomicAdd(&rows[m].listed, found) : 0;
    lds_barrier();
    at += base;
    if (hits) {
#pragma unroll
        for (int j = 0; j < 8; ++j)
            if (hits >> j & 1) {
                if (at < (uint32_t)kList) list[m * kList + at] = order.place(e.x[j], e.start + j);
                ++at;
            }
    }
}

// What is kept of a row, for the kernel that writes the distribution.
struct RowCut {
    double inv_sum;
    float above;                                                     // larger logits are kept, and equal ones up to this token
    int32_t token;
    float most;
    int32_t state;                                                   // 0: nothing is left of the row, 1: something is, -1: its settings are not known
};

// ---- the cut, and the draws: one workgroup to a row
// Bound by what follows one another.  One row of 50280, top-p, one child, 11 us: the row's sums 2.1, units of the tokens 0.7, the cut 3.6, sums of the chunks
// 1.8, the child 2.3.  A further child costs 2.2 (its chunk 0.8, the chunk's tokens 0.5, their weights and sums 0.6, the rest 0.3), a cut of
// another kind 2.2.  96 rows of three children 18, 128 rows of 131071 18.  (A part of a range found by all 16 wavefronts in place of one: 0.7 us
// slower; prefix sums of four wavefronts share a SIMD's issue.)
constexpr int kFew = 64;                                             // places that a wavefront looks through
constexpr int kFine = 1024;                                          // parts that a range of places is cut into

// (parts in a row stand one further apart every 16: a lane has 16 of them)
__device__ __forceinline__ int padded(int part) { return part + (part >> 4); }

struct RowShared {
    u64 place[kList], units[kList];
    RowBins bins;
    ChunkScale scale[kMaxChunks];
    u64 fine_mass[kFine + kFine / 16];
    uint32_t fine_number[kFine + kFine / 16];
    u64 chunk_mass[kMaxChunks];                                      // kept, relative to the chunk's largest
    u64 wave_part[kWideWaves];
    float part[kWideWaves];
    u64 drawn[8];
    float u[8];
    u64 few[kFew], few_mass[kFew];
    u64 lo, hi, need, before, cut, found, sum;
    uint32_t n_few, n;
    int32_t chunk;                                                   // of the next child (-1: nothing is left, -2: the rest is to be weighed anew)
    double inv_sum;
};

// prefix sums over the workgroup, without the thread's own; the whole sum in *total.  FREE: nobody reads parts any more.
template <bool FREE> __device__ __forceinline__ u64 wide_prefix(u64 v, u64 *parts, u64 *total)
{
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const u64 mine = wave_prefix(v);
    if (!FREE) lds_barrier();
    if (lane == 63) parts[wave] = mine;
    lds_barrier();
    const u64 waves = wave_prefix(lane < kWideWaves ? parts[lane] : 0);
    *total = lane_of(waves, kWideWaves - 1);
    const int before = __builtin_amdgcn_readfirstlane(wave - 1);
    return (before >= 0 ? lane_of(waves, before) : 0) + mine - v;
}

template <typename T> struct Row {
    const T *x;
    int32_t V;
    float top, per_bin;
    int top_mark, scale;
    Weights weights;
    Order<T> order;
    const ChunkScale *chunks;
    // units of a token relative to its chunk's largest logit, and to the row's
    __device__ __forceinline__ u64 own_units(float v, int32_t token) const { return weights.units(v, chunks[token / kSlice].most, scale); }
    __device__ __forceinline__ u64 units(float v, int32_t token) const { return scaled(own_units(v, token), chunks[token / kSlice].factor); }
    __device__ __forceinline__ int bin(float v) const { return bin_of(mark_of(v, per_bin), top_mark); }
    // f(logit, token) for every token that counts, a thread's share of them
    template <typename F> __device__ __forceinline__ void each(F f) const
    {
#pragma unroll 1
        for (int32_t v0 = threadIdx.x; v0 < V; v0 += kWide * 8) {
            float v[8];
#pragma unroll
            for (int i = 0; i < 8; ++i) v[i] = ld_io(x, min(v0 + i * kWide, V - 1));
#pragma unroll 1
            for (int i = 0; i < 8; ++i) {                            // (rolled up: seldom run, and long)
                const float one = v[0];
#pragma unroll
                for (int j = 0; j < 7; ++j) v[j] = v[j + 1];
                if (v0 + i * kWide < V && counts(one)) f(one, v0 + i * kWide);
            }
        }
    }
};

// Tokens of the bins with cuts: in LDS, or where there are too many for that the row itself.
struct Held {
    const u64 *place, *units;
    int n;
    __device__ __forceinline__ uint32_t number() const { return (uint32_t)n; }
    template <typename F> __device__ __forceinline__ void each(F f) const
    {
#pragma unroll 1
        for (int i = threadIdx.x; i < n; i += kWide) f(place[i], units[i]);
    }
};
template <typename T> struct Scanned {
    const Row<T> &row;
    CutBins bins;
    __device__ __forceinline__ uint32_t number() const { return kFew + 1; }
    template <typename F> __device__ __forceinline__ void each(F f) const
    {
        row.each([&](float v, int32_t token) {
            if (bins.has(row.bin(v))) f(row.order.place(v, token), row.units(v, token));
        });
    }
};

// The place in bins first .. last at which the sum of units (BY_NUMBER: the number of tokens), largest first, reaches `need` (at least one; the last
// place of the bins where it does not, by a rounding of the sums), and the units up to it.  A range of places is cut into 1024 parts until a wavefront
// can look through what is left; it halves ten times a turn, so that any bin, one of nothing but ties too, is through after a few (one, most often).
// `n`: how many tokens there are where they are these bins' only, and known.
template <bool BY_NUMBER, typename T, typename Tokens>
__device__ __forceinline__ u64 reach(RowShared &s, const Row<T> &row, const Tokens &tokens, int first, int last, uint32_t n, u64 need, u64 *units)
{
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    // (a neighbourhood of the bins' borders: what is in it of others is left out by its bin)
    const int above = row.top_mark - start_of(first) + 1, from = row.top_mark - start_of(last + 1) + 1;
    const float upper = (float)above / row.per_bin, lower = (float)from / row.per_bin, around = 0x1p-120f / row.per_bin;
    const float high = first == 0 ? row.top : fminf(upper + fabsf(upper) * 0x1p-20f + around, row.top), low = lower - fabsf(lower) * 0x1p-20f - around;
    const bool open = last == kBins - 1 || from <= (int)-kEndMark || !(low > -INFINITY);
    u64 hi = row.order.place(high, 0) | (((u64)1 << row.order.bits) - 1), lo = open ? 0 : row.order.place(low, 0) >> row.order.bits << row.order.bits;
    auto in_bins = [&](u64 place) {
        const int b = row.bin(row.order.logit(place));
        return b >= first && b <= last;
    };
    lds_barrier();
    if (tid == 0) s.need = need, s.before = 0, s.cut = 0, s.found = 0, s.n_few = 0;
#pragma unroll 1
    for (int turn = 0; n > kFew && turn < 8; ++turn) {               // (lo < hi: places differ)
        const int width = 64 - __clzll(hi - lo), shift = width > 10 ? width - 10 : 0;
        s.fine_mass[padded(tid)] = 0, s.fine_number[padded(tid)] = 0;
        lds_barrier();
        tokens.each([&](u64 place, u64 w) {
            if (place < lo || place > hi || !in_bins(place)) return;
            const int at = padded((int)((hi - place) >> shift));
            atomicAdd(&s.fine_mass[at], w);
            atomicAdd(&s.fine_number[at], 1u);
        });
        lds_barrier();
        if (wave == 0) {
            // the lane whose 16 parts reach what is needed, then of those the part
            const u64 wanted = s.need;
            u64 mass = 0, number = 0;
#pragma unroll 4
            for (int i = 0; i < 16; ++i) mass += s.fine_mass[padded(lane * 16 + i)], number += s.fine_number[padded(lane * 16 + i)];
            auto choose = [&](u64 mass_before, u64 number_before, u64 *mass_ahead, u64 *number_ahead) {
                const u64 mass_to = mass_before + wave_prefix(mass), number_to = number_before + wave_prefix(number);
                const uint64_t there = __ballot(number > 0 && (BY_NUMBER ? number_to : mass_to) >= wanted), some = __ballot(number > 0);
                const int at = there ? __builtin_ctzll(there) : some ? 63 - __builtin_clzll(some) : 0;
                *mass_ahead = lane_of(mass_to - mass, at), *number_ahead = lane_of(number_to - number, at);
                return at;
            };
            u64 mass_ahead, number_ahead;
            const int first = 16 * choose(0, 0, &mass_ahead, &number_ahead);
            mass = lane < 16 ? s.fine_mass[padded(first + lane)] : 0, number = lane < 16 ? s.fine_number[padded(first + lane)] : 0;
            const int at = choose(mass_ahead, number_ahead, &mass_ahead, &number_ahead);
            if (lane == 0) {
                const u64 before = BY_NUMBER ? number_ahead : mass_ahead;
                s.need = wanted > before ? wanted - before : 1;
                s.before += mass_ahead;
                s.hi = hi - ((u64)(first + at) << shift);
                const u64 span = ((u64)1 << shift) - 1;
                s.lo = s.hi - lo > span ? s.hi - span : lo;
                s.n = s.fine_number[padded(first + at)];
            }
        }
        lds_barrier();
        lo = s.lo, hi = s.hi, n = s.n;
    }
    lds_barrier();
    tokens.each([&](u64 place, u64 w) {
        if (place < lo || place > hi || !in_bins(place)) return;
        const uint32_t at = atomicAdd(&s.n_few, 1u);
        if (at < kFew) s.few[at] = place, s.few_mass[at] = w;
    });
    lds_barrier();
    if (wave == 0) {
        const int few = __builtin_amdgcn_readfirstlane((int)min(s.n_few, (uint32_t)kFew));
        const u64 place = lane < few ? s.few[lane] : 0, mine = lane < few ? s.few_mass[lane] : 0;
        u64 number_before = 0, mass_before = 0;
#pragma unroll 1
        for (int i = 0; i < few; ++i) {
            const u64 other = lane_of(place, i), its = lane_of(mine, i);
            number_before += other > place, mass_before += other > place ? its : 0;
        }
        const u64 before = BY_NUMBER ? number_before : mass_before, own = BY_NUMBER ? 1 : mine;
        const bool last = number_before + 1 == (u64)few;
        if (lane < few && before < s.need && (s.need <= before + own || last)) {
            s.cut = place;
            s.found = s.before + mass_before + mine;
        }
    }
    lds_barrier();
    *units = s.found;
    return s.cut;
}

// A place that a row is cut at, and its bin: bins before it are kept whole, of it the places from the cut on.
struct Cut {
    u64 place;
    int bin;
};

// The cut of a row: min-p's, then top-k's, then top-p's.  What is kept of the cut's bin goes to its chunks.
template <typename T, typename Tokens> __device__ __forceinline__ Cut cut_of(RowShared &s, const Settings &r, const CutBins &c, const Row<T> &row, const Tokens &tokens)
{
    const int tid = threadIdx.x;
    auto bin_of_place = [&](u64 place) { return row.bin(row.order.logit(place)); };
    Cut cut{0, kBins};
    u64 sum = s.bins.mass[kBins - 1], number = s.bins.number[kBins - 1];
    if (c.min_first >= 0) {
        lds_barrier();
        if (tid == 0) s.lo = ~(u64)0, s.sum = 0, s.n = 0;
        lds_barrier();
        u64 lowest = ~(u64)0, mass = 0;
        uint32_t n = 0;
        tokens.each([&](u64 place, u64 w) {
            const int b = bin_of_place(place);
            if (b < c.min_first || b > c.min_last || !(row.weights.of(row.order.logit(place), row.top) >= (double)r.min_p)) return;
            lowest = min(lowest, place), mass += w, ++n;
        });
        // (of a wavefront first: a thousand atomics on one address took three microseconds)
        const uint64_t any = __ballot(n > 0);
        if (any) {
            const u64 top = ~lowest;
            const uint32_t high = wave_max((uint32_t)(top >> 32)), low = wave_max((uint32_t)(top >> 32) == high ? (uint32_t)top : 0);
            mass = wave_sum(mass), n = (uint32_t)wave_sum((u64)n);
            if ((tid & 63) == 0) atomicMin(&s.lo, ~((u64)high << 32 | low)), atomicAdd(&s.sum, mass), atomicAdd(&s.n, n);
        }
        lds_barrier();
        sum = ahead_of(s.bins.mass, c.min_first) + s.sum, number = ahead_of(s.bins.number, c.min_first) + s.n;
        cut.place = s.lo, cut.bin = bin_of_place(s.lo);
        if (s.n == 0) cut.place = ((u64)row.order.key(row.order.place(c.min_above, 0)) + 1) << row.order.bits, cut.bin = c.min_first;   // all of the bins before, nothing of these
    }
    u64 inside;
    if (r.top_k > 0 && (u64)r.top_k < number) {
        const bool alone = c.min_first < 0 && c.p_first < 0;
        const u64 place = reach<true>(s, row, tokens, c.k_bin, c.k_bin, alone ? tokens.number() : kFew + 1, (u64)r.top_k - ahead_of(s.bins.number, c.k_bin), &inside);
        if (place > cut.place) cut.place = place, cut.bin = c.k_bin, sum = ahead_of(s.bins.mass, c.k_bin) + inside;   // (a cut is one of the list's places)
    }
    if (r.top_p < 1.0f) {
        const u64 need = share_of(sum, r.top_p), before = ahead_of(s.bins.mass, c.p_first);
        const bool alone = c.min_first < 0 && c.k_bin < 0;
        const u64 place = reach<false>(s, row, tokens, c.p_first, c.p_last, alone ? tokens.number() : kFew + 1, need > before ? need - before : 1, &inside);
        if (place > cut.place) cut.place = place, cut.bin = row.bin(row.order.logit(place));
    }
    return cut;
}

// The units of every chunk ahead of the bin of the cut, and with them what is kept of that bin.
template <typename T, typename Tokens>
__device__ __forceinline__ void chunk_sums(RowShared &s, const Chunks &from, int64_t m, int chunks, const Cut &cut, const Row<T> &row, const Tokens &tokens)
{
    lds_barrier();
    for (int i = threadIdx.x; i < chunks; i += kWide) {
        const int shift = s.scale[i].shift, b = cut.bin == kBins ? kBins - 1 : chunk_bin(start_of(cut.bin), shift);
        s.chunk_mass[i] = shift < kNoChunk && b >= 0 ? from.mass[(m * chunks + i) * kBins + b] : 0;
    }
    lds_barrier();
    if (cut.bin < kBins)
        tokens.each([&](u64 place, u64) {
            const float v = row.order.logit(place);
            const int32_t token = row.order.token(place);
            if (place >= cut.place && row.bin(v) == cut.bin) atomicAdd(&s.chunk_mass[token / kSlice], row.own_units(v, token));
        });
    lds_barrier();
}

// Where the bins with cuts have more tokens than the list: the same by reading the row for every step, one CU to a row.  Flat rows of large vocabularies
// come here, and long ties: 131071 normally distributed logits, divided by T, with a deviation of 0.6 under a top-p of 0.8 709 us a call (with 1.3,
// whose list is long enough, 29), 128 such rows 830 (75), 128 rows of 50280 with 0.2 393 (0.4: 50); a row of one value 1.0 ms of 50280, 2.6 of
// 131071; 2^21 logits with 2.5 6.2 ms (4.0: 0.1).  (Not inlined: the other rows do not fetch it.)
template <typename T>
__device__ __attribute__((noinline)) Cut scan_cut(RowShared &s, const Settings &r, const CutBins &c, const Row<T> &row, const Chunks &from, int64_t m, int chunks)
{
    const Scanned<T> tokens{row, c};
    const Cut cut = cut_of(s, r, c, row, tokens);
    chunk_sums(s, from, m, chunks, cut, row, tokens);
    return cut;
}

// Where next to nothing is left beside what was drawn, units are too coarse for it: the sums of the chunks with drawn tokens again, relative to the
// largest that is left there, and all chunks' against the largest that is left anywhere.  (A chunk whose largest has no weight beside the row's has
// none here.)
template <typename T>
__device__ __attribute__((noinline)) void sums_of_the_rest(RowShared &s, const Row<T> &row, u64 cut, int drawn, float top, int chunks)
{
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    auto most_of_all = [&](float v) {
        v = wave_max(v);
        lds_barrier();
        if (lane == 0) s.part[wave] = v;
        lds_barrier();
        return wave_max(s.part[lane & (kWideWaves - 1)]);
    };
#pragma unroll 1
    for (int d = 0; d < drawn; ++d) {
        if (!s.drawn[d]) continue;
        const int chunk = row.order.token(s.drawn[d]) / kSlice, first = chunk * kSlice + 2 * tid;
        float v[2], most = -INFINITY;
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            v[i] = ld_io(row.x, min(first + i, row.V - 1));
            const u64 place = row.order.place(v[i], first + i);
            bool open = first + i < row.V && counts(v[i]) && place >= cut;
            for (int e = 0; e < drawn; ++e) open = open && place != s.drawn[e];
            v[i] = open ? v[i] : -INFINITY;
            most = fmaxf(most, v[i]);
        }
        most = most_of_all(most);
        u64 sum = 0, all;
#pragma unroll
        for (int i = 0; i < 2; ++i) sum += counts(v[i]) ? row.weights.units(v[i], most, row.scale) : 0;
        wide_prefix<false>(sum, s.wave_part, &all);
        if (tid == 0) s.chunk_mass[chunk] = all, s.scale[chunk].most = most;
    }
    lds_barrier();
    const float mine = tid < chunks && s.chunk_mass[tid] > 0 && row.weights.of(s.scale[tid].most, top) > 0.0 ? s.scale[tid].most : -INFINITY;
    const float most = most_of_all(mine);
    if (tid < chunks) s.scale[tid].factor = counts(mine) ? row.weights.of(mine, most) : 0.0;
    lds_barrier();
}

template <typename T>
__global__ void __launch_bounds__(kWide)
draw_kernel(const T *__restrict__ logits, Chunks from, const RowBins *__restrict__ rows, const ChunkScale *__restrict__ scales, const u64 *__restrict__ list,
            RowCut *__restrict__ cuts, SampleArgs a, int scale, int chunks, Order<T> order)
{
    __shared__ RowShared s;
    const int64_t m = blockIdx.x;
    const int tid = threadIdx.x;
    const uint32_t n = rows[m].listed;
    const float top = rows[m].top;
    const CutBins c = rows[m].cuts;
    if (tid < kBins) s.bins.mass[tid] = rows[m].mass[tid], s.bins.number[tid] = rows[m].number[tid];
    if (tid < chunks) s.scale[tid] = scales[m * chunks + tid];
    if (tid == 0) s.inv_sum = 0.0;
    if (tid < 8) s.drawn[tid] = 0, s.u[tid] = tid < a.k ? a.u[m * a.k + tid] : 0.0f;
    const u64 first_place = tid < (int)n && tid < kList ? list[m * kList + tid] : 0;
    const Settings r = settings_of(a, m);
    lds_barrier();
    Row<T> row{logits + m * a.V, (int32_t)a.V, top, r.per_bin, top_mark_of(top, r.per_bin), scale, r.weights, order, s.scale};
    const bool some = r.known && counts(top);

    Cut cut{0, kBins};
    if (some) {
        Held held{s.place, s.units, 0};
        if (c.any()) {
            if (n <= kList) {
                held.n = (int)n;
#pragma unroll 1
                for (int i = tid; i < (int)n; i += kWide) {
                    const u64 place = i == tid ? first_place : list[m * kList + i];
                    s.place[i] = place, s.units[i] = row.units(order.logit(place), order.token(place));
                }
                cut = cut_of(s, r, c, row, held);
            } else {
                const Row<T> row_there = row;                        // (copies: what the call takes by address stays out of registers)
                const Settings r_there = r;
                const CutBins c_there = c;
                cut = scan_cut(s, r_there, c_there, row_there, from, m, chunks);
            }
        }
        if (n <= kList || cut.bin == kBins) chunk_sums(s, from, m, chunks, cut, row, held);
    }

    // ---- the draws: the chunk by one wavefront (by all of them, alike, it took 0.3 us longer: they share the SIMDs' issue), the token by all
    const int per = (chunks + 63) / 64, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);   // chunks to a lane
    auto choose = [&](int j, bool weighed_anew) {
        auto mass_of = [&](int i) { return i < chunks ? scaled(s.chunk_mass[i], s.scale[i].factor) : 0; };
        u64 mine = 0;
#pragma unroll 1
        for (int i = 0; i < per; ++i) mine += mass_of(lane * per + i);
        const u64 to = wave_prefix(mine), left = lane_of(to, 63);
        if (j == 0) s.inv_sum = 1.0 / __builtin_ldexp((double)left, -scale);
        // (that the last of what is kept was drawn, with nothing left, says that all of it was)
        bool out = left == 0 && cut.place != 0;
        for (int d = 0, is = 0; out && d < j; ++d) is |= s.drawn[d] == cut.place, out = d + 1 < j || is;
        if (j > 0 && !weighed_anew && left < (r.top_k > 0 && r.top_k <= 1024 ? (u64)1 << 30 : (u64)1 << 39) && !out) {
            s.chunk = -2;
            return;
        }
        if (left == 0) {
            s.chunk = -1;
            return;
        }
        const float u = s.u[j];
        const u64 f = !(u > 0.0f) ? 0 : u >= 1.0f ? ~(u64)0 : (u64)((double)u * 18446744073709551616.0);
        const u64 bound = __umul64hi(left, f);                       // the sum that is to be passed
        int chunk = __builtin_ctzll(__ballot(to > bound));
        u64 ahead = lane_of(to - mine, chunk);
        if (per > 1) {
            const u64 one = lane < per ? mass_of(chunk * per + lane) : 0, to_one = ahead + wave_prefix(one);
            const int at = __builtin_ctzll(__ballot(to_one > bound));
            chunk = chunk * per + at, ahead = lane_of(to_one - one, at);
        }
        s.chunk = chunk;
        s.need = min((u64)((double)(bound - ahead) / s.scale[chunk].factor), s.chunk_mass[chunk] - 1);
    };
#pragma unroll 1
    for (int j = 0; some && j < a.k; ++j) {
        if (wave == 0) choose(j, false);
        lds_barrier();
        if (s.chunk == -2) {
            const Row<T> row_there = row;
            sums_of_the_rest(s, row_there, cut.place, j, top, chunks);
            if (wave == 0) choose(j, true);
            lds_barrier();
        }
        const int chunk = s.chunk;
        if (chunk < 0) break;                                        // (for good)
        const u64 inside = s.need;
        const int32_t first = chunk * kSlice + 2 * tid;
        const float most = s.scale[chunk].most;
        float v[2];
        u64 w[2], sum = 0, all;
#pragma unroll
        for (int i = 0; i < 2; ++i) v[i] = ld_io(row.x, min(first + i, row.V - 1));
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            const u64 p = order.place(v[i], first + i);
            w[i] = first + i < row.V && counts(v[i]) && p >= cut.place ? row.weights.units(v[i], most, scale) : 0;
        }
        for (int d = 0; d < j; ++d) {
            const int32_t token = s.drawn[d] ? order.token(s.drawn[d]) : -1;
#pragma unroll
            for (int i = 0; i < 2; ++i) w[i] = first + i == token ? 0 : w[i];
        }
#pragma unroll
        for (int i = 0; i < 2; ++i) sum += w[i];
        u64 start = wide_prefix<true>(sum, s.wave_part, &all);       // (of the chunks' sums nothing is read by then)
        if (start <= inside && inside < start + sum) {               // one thread
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                if (start <= inside && inside < start + w[i]) s.drawn[j] = order.place(v[i], first + i), s.chunk_mass[chunk] -= w[i];
                start += w[i];
            }
        }
        lds_barrier();
    }
    // a wavefront to a child
    if (const int j = wave; j < a.k) {
        const u64 place = s.drawn[j];
        const int64_t out = m * a.k + j;
        const int32_t token = place ? order.token(place) : -1;
        if (lane == 0) {
            a.idx[out] = token;
            a.prob[out] = place ? (float)(row.weights.of(order.logit(place), top) * s.inv_sum) : 0.0f;
        }
        if (a.path_out)
            for (int64_t t = lane; t <= a.path_len; t += 64) a.path_out[out * (a.path_len + 1) + t] = t < a.path_len ? a.path[m * a.path_len + t] : token;
    }
    if (tid == 0 && a.dist) {
        const bool all = cut.place == 0;
        cuts[m] = RowCut{s.inv_sum, all ? -INFINITY : order.logit(cut.place), all ? -1 : order.token(cut.place), top, !r.known ? -1 : some ? 1 : 0};
    }
}

// ---- the distribution: a workgroup to a chunk
// Bound by memory: 128 rows of 131071 float32 logits 21.5 us (134 MB read and written: 6.2 TB/s, logits from the last-level cache in part).
template <typename T>
__global__ void __launch_bounds__(kThreads)
dist_kernel(const T *__restrict__ logits, const RowCut *__restrict__ cuts, float *__restrict__ dist, SampleArgs a)
{
    const int64_t m = row_of_block();
    if (m >= a.M) return;
    const int32_t V = (int32_t)a.V, v0 = (int32_t)blockIdx.x * kSlice + (int32_t)threadIdx.x * 8;
    Eight e;
    e.load(logits + m * V, v0, V);
    const Settings r = settings_of(a, m);
    const RowCut c = cuts[m];
    float q[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        q[i] = c.state < 0 ? __int_as_float(0x7fc00000) : 0.0f;
        if (c.state > 0 && (e.x[i] > c.above || (e.x[i] == c.above && e.start + i <= c.token))) q[i] = (float)(r.weights.of(e.x[i], c.most) * c.inv_sum);
    }
    float *to = dist + m * V;
    if (v0 + 8 <= V) {
        store8(to + v0, q);
    } else if (v0 < V) {
        const int first = V >= 8 ? v0 - e.start : 0, end = V >= 8 ? 8 : V;
#pragma unroll
        for (int i = 0; i < 8; ++i)
            if (i >= first && i < end) to[e.start + i] = q[i];
    }
}

int64_t chunks_of(int64_t V) { return (V + kSlice - 1) / kSlice; }

struct Places {                                                      // of the parts of the workspace, in bytes
    size_t mass, number, rows, scales, cuts, list, most, all;
};
Places places_of(int64_t M, int64_t V)
{
    const size_t chunks = (size_t)(M * chunks_of(V));
    auto up = [](size_t n) { return (n + 15) / 16 * 16; };
    Places p;
    p.mass = 0;
    p.number = p.mass + chunks * kBins * sizeof(u64);
    p.rows = p.number + chunks * kBins * sizeof(uint32_t);
    p.scales = p.rows + up((size_t)M * sizeof(RowBins));
    p.cuts = p.scales + chunks * sizeof(ChunkScale);
    p.list = p.cuts + up((size_t)M * sizeof(RowCut));
    p.most = p.list + (size_t)M * kList * sizeof(u64);
    p.all = p.most + up(chunks * sizeof(float));
    return p;
}

template <typename T> hipError_t launch(const T *logits, unsigned char *ws, const SampleArgs &a, hipStream_t stream)
{
    const Places p = places_of(a.M, a.V);
    const int64_t chunks = chunks_of(a.V);
    const unsigned rows_y = (unsigned)(a.M < kRowsY ? a.M : kRowsY), rows_z = (unsigned)((a.M + kRowsY - 1) / kRowsY);
    const dim3 grid((unsigned)chunks, rows_y, rows_z);
    const Chunks c{reinterpret_cast<u64 *>(ws + p.mass), reinterpret_cast<uint32_t *>(ws + p.number), reinterpret_cast<float *>(ws + p.most)};
    RowBins *rows = reinterpret_cast<RowBins *>(ws + p.rows);
    ChunkScale *scales = reinterpret_cast<ChunkScale *>(ws + p.scales);
    u64 *list = reinterpret_cast<u64 *>(ws + p.list);
    RowCut *cuts = reinterpret_cast<RowCut *>(ws + p.cuts);
    int bits = 0;
    while ((int64_t)1 << bits < a.V) ++bits;
    const int scale = bits < 12 ? 51 : 63 - bits;
    const Order<T> order{bits};
    bins_kernel<T><<<grid, kThreads, 0, stream>>>(logits, c, a, scale);
    plan_kernel<T><<<(unsigned)a.M, kWide, 0, stream>>>(c, rows, scales, a, (int)chunks);
    gather_kernel<T><<<grid, kThreads, 0, stream>>>(logits, rows, list, a.M, (int32_t)a.V, order);
    draw_kernel<T><<<(unsigned)a.M, kWide, 0, stream>>>(logits, c, rows, scales, list, cuts, a, scale, (int)chunks, order);
    if (a.dist) dist_kernel<T><<<grid, kThreads, 0, stream>>>(logits, cuts, a.dist, a);
    return hipGetLastError();
}

}  // namespace

// (a launch has fewer than 2^32 threads, and the kernel of a row a thread for each of its chunks)
bool sample_fits(int64_t M, int64_t V)
{
    return V <= (int64_t)kSlice * kMaxChunks && M <= (0xffffffff / kWide) && M <= (0xffffffff / kThreads) / (V > 0 ? chunks_of(V) : 1);
}

size_t sample_workspace_bytes(int64_t M, int64_t V) { return places_of(M, V).all; }

hipError_t launch_sample(const void *logits, void *ws, const SampleArgs &a, int io, hipStream_t stream)
{
    unsigned char *w = static_cast<unsigned char *>(ws);
    return io == kIoBf16 ? launch(static_cast<const bf16_t *>(logits), w, a, stream) : launch(static_cast<const float *>(logits), w, a, stream);
}

}  // namespace mamba
