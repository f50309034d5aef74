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
// (47 for 50280 tokens).  Integer sums do not depend on their order: neither on how a row is cut over workgroups nor on which of them is first.
#include "device_math.h"
#include "launch.h"
#include "logit_rows.h"

namespace mamba {
namespace {

typedef unsigned long long u64;

constexpr int kThreads = 256;                                        // of the kernels that have a slice of a row
constexpr int kSlice = kThreads * 8;
constexpr int kMaxSlices = 1024;
constexpr int kBins = 64;                                            // of a row's weights, each half an octave
constexpr int kWide = 1024, kWideWaves = kWide / 64;                 // threads of the kernel that has a row

// What a row is drawn by, as it is known ahead of its logits.
struct Settings {
    double inv_T;
    float per_bin;                                                   // bins to a unit of logits
    float min_p, top_p;
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
    const bool greedy = r.known && T == 0.0f, drawn = r.known && !greedy;   // the first of the largest; a row that is not known is not looked at
    r.inv_T = drawn ? 1.0 / (double)T : 1.0;
    r.per_bin = fminf((float)(r.inv_T * 2.8853900817779268), 1e30f); // 2 / ln 2: half octaves
    r.min_p = drawn ? fminf(min_p, 1.0f) : greedy ? 1.0f : 0.0f;
    r.top_p = drawn ? top_p : 1.0f;
    r.top_k = greedy ? 1 : drawn && top_k > 0 ? top_k : 0;
    return r;
}

// Tokens in order: a larger number is ahead.  Logits order as signed integers (-0 as +0), ties by the lower index.
__device__ __forceinline__ uint32_t key_of(float x)
{
    const int32_t b = __float_as_int(x + 0.0f);
    return (uint32_t)(b ^ ((b >> 31) & 0x7fffffff)) ^ 0x80000000u;
}
__device__ __forceinline__ float value_of(uint32_t key)
{
    const int32_t b = (int32_t)(key ^ 0x80000000u);
    return __int_as_float(b ^ ((b >> 31) & 0x7fffffff));
}
__device__ __forceinline__ u64 place_of(float x, int32_t token) { return (u64)key_of(x) << 32 | (uint32_t)~token; }
__device__ __forceinline__ float logit_of(u64 place) { return value_of((uint32_t)(place >> 32)); }
__device__ __forceinline__ int32_t token_of(u64 place) { return (int32_t)~(uint32_t)place; }

__device__ __forceinline__ bool counts(float x) { return x > -INFINITY; }   // (no NaN, which is as -inf)

// e^v for v <= 0: 2^n e^z, |z| <= ln 2 / 2, e^z by its Taylor series, whose next term is below 2^-57.  Written out, every operation one rounding:
// kernels that add up the same weights come to the same units.
__device__ __forceinline__ double exp_of(double v)
{
#pragma clang fp contract(off)
    const double n = __builtin_rint(fmax(v, -800.0) * 1.4426950408889634074);
    double z = __builtin_fma(n, -0x1.62e42fefa39efp-1, fmax(v, -800.0));      // ln 2 in two parts
    z = __builtin_fma(n, -0x1.abc9e3b39803fp-56, z);
    double e = 1.0 / 6227020800.0;
    constexpr double kInverse[13] = {1.0, 1.0, 1.0 / 2, 1.0 / 6, 1.0 / 24, 1.0 / 120, 1.0 / 720, 1.0 / 5040, 1.0 / 40320, 1.0 / 362880, 1.0 / 3628800,
                                     1.0 / 39916800, 1.0 / 479001600};
#pragma unroll
    for (int i = 12; i >= 0; --i) e = __builtin_fma(e, z, kInverse[i]);
    return __builtin_ldexp(e, (int)n);
}

// weight of x relative to `most`, the largest logit (or the largest that is left)
__device__ __forceinline__ double weight_of(float x, float most, double inv_T)
{
#pragma clang fp contract(off)
    if (x == most) return 1.0;
    const double e = ((double)x - (double)most) * inv_T;
    return e == e ? exp_of(e) : 0.0;                                 // (an infinite logit leaves the others nothing)
}
__device__ __forceinline__ u64 units_of(double w, double one) { return (u64)(w * one + 0.5); }
__device__ __forceinline__ int bin_of(float x, float most, float per_bin)
{
    const float d = (most - x) * per_bin;
    return (int)fminf(d == d ? d : 0.0f, (float)(kBins - 1));
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
#pragma unroll
        for (int i = 0; i < 8; ++i) valid &= counts(x[i]) ? ~0u : ~(1u << i);
    }
    __device__ __forceinline__ bool has(int i) const { return valid >> i & 1; }
};

__device__ __forceinline__ float wave_max(float v)
{
#pragma unroll
    for (int d = 32; d; d >>= 1) v = fmaxf(v, __shfl_xor(v, d));
    return v;
}
__device__ __forceinline__ u64 wave_sum(u64 v)
{
#pragma unroll
    for (int d = 32; d; d >>= 1) v += __shfl_xor(v, d);
    return v;
}
__device__ __forceinline__ u64 wave_prefix(u64 v, int lane)          // with the lane's own
{
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) {
        const u64 o = __shfl_up(v, d);
        v += lane >= d ? o : 0;
    }
    return v;
}

// ---- the largest logit of every slice
template <typename T>
__global__ void __launch_bounds__(kThreads) most_kernel(const T *__restrict__ logits, float *__restrict__ most, int64_t M, int32_t V)
{
    const int64_t m = row_of_block();
    if (m >= M) return;
    Eight e;
    e.load(logits + m * V, (int32_t)blockIdx.x * kSlice + (int32_t)threadIdx.x * 8, V);
    float v = -INFINITY;
#pragma unroll
    for (int i = 0; i < 8; ++i) v = e.has(i) ? fmaxf(v, e.x[i]) : v;
    __shared__ float part[kThreads / 64];
    v = wave_max(v);
    if ((threadIdx.x & 63) == 0) part[threadIdx.x >> 6] = v;
    __syncthreads();
    if (threadIdx.x == 0) most[m * gridDim.x + blockIdx.x] = fmaxf(fmaxf(part[0], part[1]), fmaxf(part[2], part[3]));
}

template <int THREADS> __device__ __forceinline__ float row_most(const float *most, int slices, float *part)
{
    float v = -INFINITY;
    for (int s = threadIdx.x; s < slices; s += THREADS) v = fmaxf(v, most[s]);
    v = wave_max(v);
    if ((threadIdx.x & 63) == 0) part[threadIdx.x >> 6] = v;
    __syncthreads();
    v = part[0];
#pragma unroll
    for (int w = 1; w < THREADS / 64; ++w) v = fmaxf(v, part[w]);
    return v;
}

// ---- weights of every slice by bins: their sum and their number
template <typename T>
__global__ void __launch_bounds__(kThreads)
bins_kernel(const T *__restrict__ logits, const float *__restrict__ most, u64 *__restrict__ mass, uint32_t *__restrict__ number, SampleArgs a, double one)
{
    const int64_t m = row_of_block(), slices = gridDim.x;
    if (m >= a.M) return;
    __shared__ float part[kThreads / 64];
    __shared__ u64 bin_mass[kBins];
    __shared__ uint32_t bin_number[kBins];
    const int tid = threadIdx.x;
    Eight e;
    e.load(logits + m * a.V, (int32_t)blockIdx.x * kSlice + tid * 8, (int32_t)a.V);
    const Settings r = settings_of(a, m);
    if (tid < kBins) bin_mass[tid] = 0, bin_number[tid] = 0;
    const float top = row_most<kThreads>(most + m * slices, (int)slices, part);
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        if (!e.has(i)) continue;
        const double w = weight_of(e.x[i], top, r.inv_T);
        if (!(w >= (double)r.min_p)) continue;
        const int b = bin_of(e.x[i], top, r.per_bin);
        atomicAdd(&bin_mass[b], units_of(w, one));
        atomicAdd(&bin_number[b], 1u);
    }
    __syncthreads();
    if (tid < kBins) {
        const int64_t at = (m * slices + blockIdx.x) * kBins + tid;
        mass[at] = bin_mass[tid];
        number[at] = bin_number[tid];
    }
}

// What is kept of a row, for the kernel that writes the distribution.
struct RowCut {
    u64 cut;                                                         // places from here on are kept
    double inv_sum;
    float most;
    int32_t state;                                                   // 0: nothing is left of the row, 1: something is, -1: its settings are not known
};

// ---- the cut, and the draws: one workgroup to a row
constexpr int kList = 4096;                                          // places that LDS holds
constexpr int kFew = 64;                                             // places that a wavefront looks through
constexpr int kFine = 1024;                                          // parts that a range of places is cut into

struct RowShared {
    u64 list[kList];
    u64 fine_mass[kFine];
    u64 slice_mass[kMaxSlices];
    u64 bin_mass[kBins], bin_part[kWideWaves][kBins];
    u64 wave_part[2][kWideWaves];
    u64 drawn[8];
    u64 few[kFew];
    u64 lo, hi, need, before, cut, found;
    uint32_t fine_number[kFine], bin_number[kBins], number_part[kWideWaves][kBins];
    uint32_t wave_number[2][kWideWaves];
    uint32_t n_list, n_few, n;
    int32_t bin;
    float part[kWideWaves];
};

// prefix sums over the workgroup, without the thread's own; the whole sum in *total
__device__ __forceinline__ u64 wide_prefix(u64 v, u64 *parts, u64 *total)
{
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const u64 mine = wave_prefix(v, lane);
    __syncthreads();                                                 // (the last use of parts is over)
    if (lane == 63) parts[wave] = mine;
    __syncthreads();
    u64 before = 0, all = 0;
#pragma unroll
    for (int w = 0; w < kWideWaves; ++w) {
        before += w < wave ? parts[w] : 0;
        all += parts[w];
    }
    *total = all;
    return before + mine - v;
}

template <typename T> struct Row {
    const T *x;
    int32_t V;
    float most, per_bin;
    double inv_T, one;
    float min_p;
    __device__ __forceinline__ double weight(float v) const { return weight_of(v, most, inv_T); }
    __device__ __forceinline__ u64 units(float v) const { return units_of(weight(v), one); }
    __device__ __forceinline__ int bin(float v) const { return bin_of(v, most, per_bin); }
    // f(logit, token) for every token that counts, a thread's share of them
    template <typename F> __device__ __forceinline__ void each(F f) const
    {
        for (int32_t v0 = threadIdx.x * 8; v0 < V; v0 += kWide * 8) {
            Eight e;
            e.load(x, v0, V);
#pragma unroll
            for (int i = 0; i < 8; ++i)
                if (e.has(i)) f(e.x[i], e.start + i);
        }
    }
    // the same for those of a bin that are heavy enough
    template <typename F> __device__ __forceinline__ void each_of_bin(int b, F f) const
    {
        each([&](float v, int32_t token) {
            if (bin(v) == b && (min_p <= 0.0f || weight(v) >= (double)min_p)) f(place_of(v, token));
        });
    }
};

// The place in bin b at which the sum of weights (BY_NUMBER: the number of tokens), largest first, reaches `need` (at least one), and the
// units up to it.  A range of places is cut into 1024 parts until a wavefront can look through what is left; it halves ten times a turn, so
// that any row, one of nothing but ties too, is through after seven.
template <bool BY_NUMBER, typename T> __device__ __forceinline__ u64 reach(RowShared &s, const Row<T> &row, int b, u64 need, u64 *units)
{
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    __syncthreads();
    if (tid == 0) s.n_list = 0, s.lo = ~(u64)0, s.hi = 0, s.need = need, s.before = 0;
    __syncthreads();
    u64 lo = ~(u64)0, hi = 0;
    row.each_of_bin(b, [&](u64 place) {
        lo = min(lo, place), hi = max(hi, place);
        const uint32_t at = atomicAdd(&s.n_list, 1u);
        if (at < kList) s.list[at] = place;
    });
    if (hi) atomicMin(&s.lo, lo), atomicMax(&s.hi, hi);
    __syncthreads();
    uint32_t n = s.n_list;
    bool listed = n <= kList;
    auto each_left = [&](u64 from, u64 to, auto f) {
        if (listed) {
            for (uint32_t i = tid; i < s.n_list; i += kWide)
                if (s.list[i] >= from && s.list[i] <= to) f(s.list[i]);
        } else {
            row.each_of_bin(b, [&](u64 place) {
                if (place >= from && place <= to) f(place);
            });
        }
    };
    lo = s.lo, hi = s.hi;
    for (int turn = 0; n > kFew && turn < 8; ++turn) {               // (lo < hi: places differ)
        const int width = 64 - __clzll(hi - lo), shift = width > 10 ? width - 10 : 0;
        for (int i = tid; i < kFine; i += kWide) s.fine_mass[i] = 0, s.fine_number[i] = 0;
        __syncthreads();
        each_left(lo, hi, [&](u64 place) {
            const int at = (int)((hi - place) >> shift);
            atomicAdd(&s.fine_mass[at], row.units(logit_of(place)));
            atomicAdd(&s.fine_number[at], 1u);
        });
        __syncthreads();
        const u64 mine_mass = s.fine_mass[tid], mine_number = s.fine_number[tid];
        u64 all;
        const u64 mass_before = wide_prefix(mine_mass, s.wave_part[0], &all), number_before = wide_prefix(mine_number, s.wave_part[1], &all);
        const u64 before = BY_NUMBER ? number_before : mass_before, mine = BY_NUMBER ? mine_number : mine_mass;
        const u64 wanted = s.need;
        __syncthreads();
        if (before < wanted && wanted <= before + mine) {            // one thread
            s.need = wanted - before;
            s.before += mass_before;
            s.hi = hi - ((u64)tid << shift);
            const u64 span = ((u64)1 << shift) - 1;
            s.lo = s.hi - lo > span ? s.hi - span : lo;
            s.n = (uint32_t)mine_number;
        }
        __syncthreads();
        lo = s.lo, hi = s.hi, n = s.n;
        if (!listed && n <= kList) {
            if (tid == 0) s.n_list = 0;
            __syncthreads();
            row.each_of_bin(b, [&](u64 place) {
                if (place >= lo && place <= hi) s.list[atomicAdd(&s.n_list, 1u)] = place;
            });
            listed = true;
            __syncthreads();
        }
    }
    if (tid == 0) s.n_few = 0;
    __syncthreads();
    each_left(lo, hi, [&](u64 place) {
        const uint32_t at = atomicAdd(&s.n_few, 1u);
        if (at < kFew) s.few[at] = place;
    });
    __syncthreads();
    if (wave == 0) {
        const u64 place = lane < (int)n ? s.few[lane] : 0;
        const u64 mine = lane < (int)n ? row.units(logit_of(place)) : 0;
        u64 number_before = 0, mass_before = 0;
        for (uint32_t i = 0; i < min(n, (uint32_t)kFew); ++i) {
            const u64 other = s.few[i], theirs = __shfl(mine, (int)i);
            if (other > place) ++number_before, mass_before += theirs;
        }
        const u64 before = BY_NUMBER ? number_before : mass_before, own = BY_NUMBER ? 1 : mine;
        if (lane < (int)n && before < s.need && s.need <= before + own) {
            s.cut = place;
            s.found = s.before + mass_before + mine;
        }
    }
    __syncthreads();
    *units = s.found;
    return s.cut;
}

// bin in which the prefix sums of v, one bin to a lane, reach need; what is before it in *before
__device__ __forceinline__ int reaching_bin(u64 v, u64 need, int lane, u64 *before)
{
    const u64 to = wave_prefix(v, lane), from = to - v;
    const int b = __builtin_ctzll(__ballot(from < need && need <= to) | (u64)1 << 63);
    *before = __shfl(from, b);
    return b;
}

// need = v p rounded up, at least one, exactly: p has 24 bits
__device__ __forceinline__ u64 share_of(u64 v, float p)
{
    if (!(p > 0.0f)) return 1;
    const double scaled = (double)p * 18446744073709551616.0;        // 2^64, p < 1
    const u64 f = (u64)scaled, high = __umul64hi(v, f);
    return max(high + (v * f != 0), (u64)1);
}

template <typename T>
__global__ void __launch_bounds__(kWide)
draw_kernel(const T *__restrict__ logits, const float *__restrict__ most, const u64 *__restrict__ mass, const uint32_t *__restrict__ number,
            RowCut *__restrict__ cuts, SampleArgs a, double one, int slices)
{
    __shared__ RowShared s;
    const int64_t m = blockIdx.x;
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const Settings r = settings_of(a, m);
    const float top = row_most<kWide>(most + m * slices, slices, s.part);
    mass += m * slices * kBins, number += m * slices * kBins;
    Row<T> row{logits + m * a.V, (int32_t)a.V, top, r.per_bin, r.inv_T, one, r.min_p};

    u64 sum = 0, cut = 0;
    int cut_bin = kBins;                                             // bins before this one are kept whole
    const bool some = r.known && counts(top);
    if (some) {
        // ---- the row's bins
        {
            u64 v = 0;
            uint32_t n = 0;
            for (int i = wave; i < slices; i += kWideWaves) v += mass[(int64_t)i * kBins + lane], n += number[(int64_t)i * kBins + lane];
            s.bin_part[wave][lane] = v, s.number_part[wave][lane] = n;
        }
        __syncthreads();
        u64 bin_mass = 0, bin_number = 0;                            // of bin `lane`, in every wavefront
#pragma unroll
        for (int w = 0; w < kWideWaves; ++w) bin_mass += s.bin_part[w][lane], bin_number += s.number_part[w][lane];
        sum = wave_sum(bin_mass);
        const u64 all = wave_sum(bin_number);
        // ---- the cut
        u64 before, inside;
        if (r.top_k > 0 && (u64)r.top_k < all) {
            cut_bin = reaching_bin(bin_number, (u64)r.top_k, lane, &before);
            cut = reach<true>(s, row, cut_bin, (u64)r.top_k - before, &inside);
            sum = wave_sum(lane < cut_bin ? bin_mass : 0) + inside;
        }
        if (r.top_p < 1.0f) {
            const u64 need = share_of(sum, r.top_p);
            cut_bin = reaching_bin(bin_mass, need, lane, &before);
            cut = reach<false>(s, row, cut_bin, need - before, &inside);
            sum = wave_sum(lane < cut_bin ? bin_mass : 0) + inside;
        }
        // ---- what is kept of every slice
        __syncthreads();
        for (int i = wave; i < slices; i += kWideWaves) {
            const u64 v = wave_sum(lane < cut_bin ? mass[(int64_t)i * kBins + lane] : 0);
            if (lane == 0) s.slice_mass[i] = v;
        }
        __syncthreads();
        if (cut_bin < kBins)
            row.each_of_bin(cut_bin, [&](u64 place) {
                if (place >= cut) atomicAdd(&s.slice_mass[token_of(place) / kSlice], row.units(logit_of(place)));
            });
        __syncthreads();
    }
    const double inv_sum = 1.0 / ((double)sum / one);
    if (tid == 0 && a.dist) cuts[m] = RowCut{cut, inv_sum, top, !r.known ? -1 : some ? 1 : 0};

    // ---- the draws
    // (with a weight: one below float64's range, or beside an infinite logit, is none)
    auto open = [&](float v, u64 place, int drawn) {
        const double w = weight_of(v, top, r.inv_T);
        bool is = place >= cut && w >= (double)r.min_p && w > 0.0;
        for (int i = 0; i < drawn; ++i) is = is && place != s.drawn[i];
        return is;
    };
    u64 left = sum;
    for (int j = 0; j < a.k; ++j) {
        // Where next to nothing is left beside what was drawn, units are too coarse for it: again, relative to the largest that is left.
        if (some && j > 0 && left < (u64)1 << 39) {
            u64 best = 0;
            row.each([&](float v, int32_t token) {
                const u64 place = place_of(v, token);
                if (place > best && open(v, place, j)) best = place;
            });
            __syncthreads();
            if (tid == 0) s.hi = 0;
            for (int i = tid; i < slices; i += kWide) s.slice_mass[i] = 0;
            __syncthreads();
            if (best) atomicMax(&s.hi, best);
            __syncthreads();
            best = s.hi;
            left = 0;
            if (best) {
                row.most = logit_of(best);
                u64 mine = 0;
                row.each([&](float v, int32_t token) {
                    if (!open(v, place_of(v, token), j)) return;
                    const u64 w = row.units(v);
                    mine += w;
                    atomicAdd(&s.slice_mass[token / kSlice], w);
                });
                wide_prefix(mine, s.wave_part[0], &left);
            }
        }
        u64 place = 0;
        if (left > 0) {                                              // (the same for all threads)
            const float u = a.u[m * a.k + j];
            const u64 f = !(u > 0.0f) ? 0 : u >= 1.0f ? ~(u64)0 : (u64)((double)u * 18446744073709551616.0);
            const u64 bound = __umul64hi(left, f);                   // the sum that is to be passed
            u64 all;
            const u64 mine = tid < slices ? s.slice_mass[tid] : 0, from = wide_prefix(mine, s.wave_part[0], &all);
            if (from <= bound && bound < from + mine) s.bin = tid, s.need = bound - from;
            if (tid == 0) s.drawn[j] = 0, s.found = 0;
            __syncthreads();
            const int slice = s.bin;
            const u64 inside = s.need;
            u64 w[2], p[2];
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                const int32_t token = slice * kSlice + 2 * tid + i;
                const float v = token < row.V ? ld_io(row.x, token) : -INFINITY;
                p[i] = place_of(v, token);
                w[i] = counts(v) && open(v, p[i], j) ? row.units(v) : 0;
            }
            const u64 at = wide_prefix(w[0] + w[1], s.wave_part[1], &all);
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                const u64 start = at + (i ? w[0] : 0);
                if (start <= inside && inside < start + w[i]) {
                    s.drawn[j] = p[i];
                    s.found = w[i];
                    s.slice_mass[slice] -= w[i];
                }
            }
            __syncthreads();
            place = s.drawn[j];
            left -= s.found;
        }
        const int64_t out = m * a.k + j;
        const int32_t token = place ? token_of(place) : -1;
        if (tid == 0) {
            a.idx[out] = token;
            a.prob[out] = place ? (float)(weight_of(logit_of(place), top, r.inv_T) * inv_sum) : 0.0f;
            if (!place) s.drawn[j] = 0;
        }
        if (a.path_out)
            for (int64_t t = tid; t <= a.path_len; t += kWide)
                a.path_out[out * (a.path_len + 1) + t] = t < a.path_len ? a.path[m * a.path_len + t] : token;
        __syncthreads();
    }
}

// ---- the distribution
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
        const double w = weight_of(e.x[i], c.most, r.inv_T);
        const bool kept = c.state > 0 && counts(e.x[i]) && place_of(e.x[i], e.start + i) >= c.cut && w >= (double)r.min_p;
        q[i] = c.state < 0 ? __int_as_float(0x7fc00000) : kept ? (float)(w * c.inv_sum) : 0.0f;
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

int64_t slices_of(int64_t V) { return (V + kSlice - 1) / kSlice; }

struct Places {                                                      // of the parts of the workspace, in bytes
    size_t mass, number, most, cuts, all;
};
Places places_of(int64_t M, int64_t V)
{
    const size_t slices = (size_t)(M * slices_of(V));
    Places p;
    p.mass = 0;
    p.number = p.mass + slices * kBins * sizeof(u64);
    p.cuts = p.number + slices * kBins * sizeof(uint32_t);
    p.most = p.cuts + (size_t)M * sizeof(RowCut);
    p.all = p.most + (slices * sizeof(float) + 15) / 16 * 16;
    return p;
}

template <typename T> hipError_t launch(const T *logits, unsigned char *ws, const SampleArgs &a, hipStream_t stream)
{
    const int64_t slices = slices_of(a.V);
    const dim3 grid((unsigned)slices, (unsigned)(a.M < kRowsY ? a.M : kRowsY), (unsigned)((a.M + kRowsY - 1) / kRowsY));
    const Places p = places_of(a.M, a.V);
    u64 *mass = reinterpret_cast<u64 *>(ws + p.mass);
    uint32_t *number = reinterpret_cast<uint32_t *>(ws + p.number);
    RowCut *cuts = reinterpret_cast<RowCut *>(ws + p.cuts);
    float *most = reinterpret_cast<float *>(ws + p.most);
    int bits = 0;
    while ((int64_t)1 << bits < a.V) ++bits;
    const double one = (double)((u64)1 << (63 - bits));
    most_kernel<T><<<grid, kThreads, 0, stream>>>(logits, most, a.M, (int32_t)a.V);
    bins_kernel<T><<<grid, kThreads, 0, stream>>>(logits, most, mass, number, a, one);
    draw_kernel<T><<<(unsigned)a.M, kWide, 0, stream>>>(logits, most, mass, number, cuts, a, one, (int)slices);
    if (a.dist) dist_kernel<T><<<grid, kThreads, 0, stream>>>(logits, cuts, a.dist, a);
    return hipGetLastError();
}

}  // namespace

// (a launch has fewer than 2^32 threads, and the kernel of a row a thread for each of its slices)
bool sample_fits(int64_t M, int64_t V)
{
    return V <= (int64_t)kSlice * kMaxSlices && M <= (0xffffffff / kWide) && M <= (0xffffffff / kThreads) / (V > 0 ? slices_of(V) : 1);
}

size_t sample_workspace_bytes(int64_t M, int64_t V) { return places_of(M, V).all; }

hipError_t launch_sample(const void *logits, void *ws, const SampleArgs &a, int io, hipStream_t stream)
{
    unsigned char *w = static_cast<unsigned char *>(ws);
    return io == kIoBf16 ? launch(static_cast<const bf16_t *>(logits), w, a, stream) : launch(static_cast<const float *>(logits), w, a, stream);
}

}  // namespace mamba
