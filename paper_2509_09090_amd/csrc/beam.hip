// Beam search: the best continuations of several beams over the vocabulary, and the reordering of a cache in 8 bits that follows.
//
// A token's total is s + (l - log sum exp l), the beam's score and its logarithm of a probability.  Within a beam totals order as the
// logits do, so the best k of a beam are found on halves, and only they get a total, in binary64.  The order of two beams' totals depends on
// their sums of exponentials, whose terms are binary32's.  A term 2^x of the largest is off by 0.9 |x| 2^-24 of itself for the roundings of x and of log2 e (in
// parts, as sums are brought below larger logits: those add up to x), 2 units for its power, 3 for a sum of eight, 2 for each of at most 10 powers that bring it
// below a larger one: (0.9 |x| + 25) 2^-24.  Terms with |x| > 14 are at most 2^(14 - |x|) of their slab's sum (slabs are joined in binary64),
// so a sum is off by no more than 38 x 2^-24 of itself.  Most terms are near their own thread's largest, where the rounding is below a unit: flat tails of 2^20
// logits, 3 to 14 below a largest one in each slab, are off by 1.6 units at most.
#include <algorithm>

#include "common.h"

namespace sqap {

typedef unsigned v4u __attribute__((ext_vector_type(4)));
typedef unsigned v4u_any __attribute__((ext_vector_type(4), aligned(2)));
typedef unsigned v2u __attribute__((ext_vector_type(2)));
typedef unsigned long long u64;

constexpr int kBeamT = 256, kBeamWaves = kBeamT / 64, kBeamMost = kBeamMostOutputs;
constexpr int kRankedAtMost = 192;                                     // of a list
constexpr unsigned kMinusInf = 0x03ffu;                               // key of minus infinity, the lowest there is
constexpr float kLog2e = 1.44269502f;

// Keys of halves that are neither NaN nor minus zero: integers that order as the halves do.
__device__ __forceinline__ unsigned key_of(unsigned h) { return h & 0x8000u ? ~h & 0xffffu : h | 0x8000u; }
__device__ __forceinline__ unsigned half_of(unsigned key) { return key & 0x8000u ? key & 0x7fffu : ~key & 0xffffu; }
__device__ __forceinline__ float value_of(unsigned key) { return __half2float(__ushort_as_half((unsigned short)half_of(key))); }

// Eight logits: NaN becomes minus infinity, minus zero zero.
__device__ __forceinline__ v4u clean(v4u v)
{
    union { v4u u; v2h h[4]; } x;
    x.u = v;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const v2h zero = {(_Float16)0.f, (_Float16)0.f}, least = {(_Float16)-INFINITY, (_Float16)-INFINITY};
        x.h[i] = __builtin_elementwise_max(x.h[i] + zero, least);
    }
    return x.u;
}
constexpr unsigned kTwoMinusInf = 0xfc00fc00u;
// Eight halves without the first n, minus infinity behind them.
__device__ __forceinline__ v4u without_first(v4u v, int n)
{
    if (n >= 8) return v4u{kTwoMinusInf, kTwoMinusInf, kTwoMinusInf, kTwoMinusInf};
    if (n & 4) v = v4u{v[2], v[3], kTwoMinusInf, kTwoMinusInf};
    if (n & 2) v = v4u{v[1], v[2], v[3], kTwoMinusInf};
    if (n & 1) v = v4u{v[0] >> 16 | v[1] << 16, v[1] >> 16 | v[2] << 16, v[2] >> 16 | v[3] << 16, v[3] >> 16 | kTwoMinusInf << 16};
    return v;
}
__device__ __forceinline__ unsigned half_at(const v4u &v, int e) { return e & 1 ? v[e >> 1] >> 16 : v[e >> 1] & 0xffffu; }
__device__ __forceinline__ unsigned largest_of(const v4u &v)         // of the eight: minus infinity where all are NaN, no minus zero
{
    union { v4u u; v2h h[4]; } x;
    x.u = v;
    const v2h zero = {(_Float16)0.f, (_Float16)0.f};
    const v2h m = __builtin_elementwise_max(__builtin_elementwise_max(x.h[0], x.h[1]), __builtin_elementwise_max(x.h[2], x.h[3])) + zero;
    union { _Float16 h; unsigned short u; } y;
    y.h = __builtin_elementwise_max(__builtin_elementwise_max(m[0], m[1]), (_Float16)-INFINITY);
    return y.u;
}

// Exponentials of logits below a largest one, `top`, are 2^(l log2 e - c) with c = top log2 e rounded: one mixed-precision multiply-add (of half I of
// h) and the power.  Sums of them are kept below c; what its rounding makes of them is put right once (below_top).
template <int I>
__device__ __forceinline__ float power_of(const v2h h, float c)
{
    float r;
    if (I == 0) asm("v_fma_mix_f32 %0, %1, %2, -%3 op_sel_hi:[1,0,0]" : "=v"(r) : "v"(h), "s"(kLog2e), "v"(c));
    else asm("v_fma_mix_f32 %0, %1, %2, -%3 op_sel:[1,0,0] op_sel_hi:[1,0,0]" : "=v"(r) : "v"(h), "s"(kLog2e), "v"(c));
    return __builtin_amdgcn_exp2f(r);
}
__device__ __forceinline__ float eight_powers(const v4u &v, float c)
{
    union { v4u u; v2h h[4]; } x;
    x.u = v;
    float e[8];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        e[2 * i] = power_of<0>(x.h[i], c);
        e[2 * i + 1] = power_of<1>(x.h[i], c);
    }
    return ((e[0] + e[1]) + (e[2] + e[3])) + ((e[4] + e[5]) + (e[6] + e[7]));
}
__device__ __forceinline__ bool usual(float top) { return fabsf(top) <= 65504.f; }         // neither infinite nor nothing at all
__device__ __forceinline__ float below(float from, float to) { return __builtin_amdgcn_exp2f(from * kLog2e - to * kLog2e); }
__device__ __forceinline__ double below_top(double sum, float top)
{
    return usual(top) ? sum + sum * (((double)(top * kLog2e) - (double)top * (double)kLog2e) * 0.69314718055994531) : sum;
}

// How many of the workgroup's 256 values in LDS are at least `from` (all wavefronts ask the same: four values to a lane).
__device__ __forceinline__ int at_least(const v4u &mine, unsigned from)
{
    return __popcll(__ballot(mine[0] >= from)) + __popcll(__ballot(mine[1] >= from)) + __popcll(__ballot(mine[2] >= from)) + __popcll(__ballot(mine[3] >= from));
}

struct BeamRow {
    double sum;                                                       // of exp(l - top); top infinite: how many are
    float top;                                                        // largest logit
};
struct BeamArgs {
    const __half *logits;
    int64_t ld;
    int batch, beams, vocab, k, slabs;
    const float *scores;
    const int32_t *done;
    int32_t eos;
    BeamRow *rows;                                                    // [batch * beams][slabs]
    v2u *best;                                                        // [batch * beams][slabs][k]: key, token; key 0: none
    int32_t *parent, *token;
    float *score;
    int32_t *done_out;
};

// One workgroup per row and slab of 2048 PIECES logits, which it holds in registers.  The largest of each piece of eight, with the piece's place
// below it, is a number of its own; at least k pieces are not below the k-th largest of the threads' largest, and the slab's
// best k lie in those: any other piece has k logits before its own.  They go to LDS, a thread takes one of their logits each, and those that reach the
// smallest of these maxima are listed and ranked.  128 rows of 128001 (32.8 MB) in 14.4 us, 2.3 TB/s: a slab's start and loads (6.2
// of the 14.4, by themselves), one exponential per logit (3.1), a search over 16 bits, listing and ranking (5) follow one another, and the 1024 workgroups, four to a
// compute unit, are all there at once (81 registers and 27.7 KB leave five), so that all load, then all compute; rows of one wavefront each, without barriers, 16.3.  4 rows of 32000 in 4.8 us: latency.
template <int PIECES>
__global__ __launch_bounds__(kBeamT) void beam_rows_kernel(const BeamArgs a)
{
    constexpr int MOST = kBeamMost * PIECES;                          // pieces of the k threads that reach the bound
    __shared__ unsigned place[MOST], pieces, listed;
    __shared__ __attribute__((aligned(16))) unsigned tops[kBeamT], list[MOST * 8];
    __shared__ v4u piece[MOST];
    __shared__ float wave_top[kBeamWaves];
    __shared__ double wave_sum_[kBeamWaves];
    const int t = threadIdx.x, l = t & 63, wave = t >> 6, slab = blockIdx.x % a.slabs;
    const int64_t row = blockIdx.x / a.slabs;
    if (a.done && a.done[row] != 0) return;
    const int first = slab * (kBeamT * 8 * PIECES);
    const __half *from = a.logits + row * a.ld;
    // (a piece over the end is read as the row's last eight and put right below: nothing waits before all of them have been asked for)
    v4u v[PIECES];
    if (a.vocab >= 8) {
#pragma unroll
        for (int p = 0; p < PIECES; ++p) v[p] = *reinterpret_cast<const v4u_any *>(from + min(first + (p * kBeamT + t) * 8, a.vocab - 8));
    } else {
        v[0] = v4u{kTwoMinusInf, kTwoMinusInf, kTwoMinusInf, kTwoMinusInf};
        if (t == 0)
            for (int e = a.vocab - 1; e >= 0; --e) v[0] = v4u{v[0][0] << 16 | __half_as_ushort(from[e]), v[0][0] >> 16 | v[0][1] << 16,
                                                             v[0][1] >> 16 | v[0][2] << 16, v[0][2] >> 16 | v[0][3] << 16};
#pragma unroll
        for (int p = 1; p < PIECES; ++p) v[p] = v4u{kTwoMinusInf, kTwoMinusInf, kTwoMinusInf, kTwoMinusInf};
    }
    if (t == 0) pieces = 0, listed = 0;
    // piece by piece as they arrive: the largest, and the sum of exponentials below the thread's largest so far (eight of them in binary32, those
    // sums in binary64: beside one large term many small ones count)
    unsigned mine = 0, keys[PIECES];
    float top = -INFINITY;
    double sum = 0.0;
#pragma unroll
    for (int p = 0; p < PIECES; ++p) {
        const int over = first + (p * kBeamT + t) * 8 + 8 - a.vocab;
        if (over > 0 && a.vocab >= 8) v[p] = without_first(v[p], over);
        const unsigned largest = largest_of(v[p]);
        keys[p] = key_of(largest) << 11 | (2047 - (p * kBeamT + t));
        mine = max(mine, keys[p]);
        const float here = __half2float(__ushort_as_half((unsigned short)largest));
        if (here > top) {
            sum = usual(here) ? sum * (double)below(top, here) : 0.0;
            top = here;
        }
        if (usual(top)) sum += (double)eight_powers(v[p], top * kLog2e);
    }
    if (sum != sum || top > 65504.f) {                                // NaN, or infinite logits: those are counted
        sum = 0.0;
#pragma unroll
        for (int p = 0; p < PIECES; ++p) {
            const v4u x = clean(v[p]);
            if (usual(top)) sum += (double)eight_powers(x, top * kLog2e);
            else
#pragma unroll
                for (int e = 0; e < 8; ++e) sum += half_at(x, e) == 0x7c00u ? 1.0 : 0.0;
        }
    }
    tops[t] = mine;
    const float most = wavefront_max(top);
    const double part = wave_sum(top == most ? sum : usual(most) ? sum * (double)below(top, most) : 0.0);
    if (l == 0) wave_top[wave] = most, wave_sum_[wave] = part;
    __syncthreads();
    // a number that k of the threads' largest reach, and no other: bits from the highest on, until the count is right
    const v4u four = *reinterpret_cast<const v4u *>(tops + 4 * l);
    unsigned reach = 0;
    for (int bit = 26; bit >= 0; --bit) {
        const unsigned next = reach | 1u << bit;
        const int n = at_least(four, next);
        if (n >= a.k) reach = next;
        if (n == a.k) break;
    }
    if (mine >= reach) {
#pragma unroll
        for (int p = 0; p < PIECES; ++p)
            if (keys[p] >= reach) {
                const unsigned at = atomicAdd(&pieces, 1u);
                piece[at] = clean(v[p]);
                place[at] = p * kBeamT + t;
            }
    }
    __syncthreads();
    const unsigned least = max(reach >> 11, kMinusInf + 1);
    for (int i = t; i < 8 * (int)pieces; i += kBeamT) {
        const unsigned key = key_of(reinterpret_cast<const unsigned short *>(&piece[i >> 3])[i & 7]);
        if (key >= least) list[atomicAdd(&listed, 1u)] = key << 14 | (16383 - (place[i >> 3] * 8 + (i & 7)));
    }
    __syncthreads();
    int n = (int)listed;
    const unsigned *ranked = list;
    if (n > kRankedAtMost && n <= 8 * 64) {
        // nearly as many outputs as pieces: the k-th largest of the list first, as above, and only those that reach it are ranked (46 x 31 rows of 427
        // logits with 62 outputs 48 us, so 17; the ranking of some hundred is shorter)
        unsigned x[8], bound = 0;
#pragma unroll
        for (int i = 0; i < 8; ++i) x[i] = l + 64 * i < n ? list[l + 64 * i] : 0;
        for (int bit = 29; bit >= 0; --bit) {
            const unsigned next = bound | 1u << bit;
            int count = 0;
#pragma unroll
            for (int i = 0; i < 8; ++i) count += __popcll(__ballot(x[i] >= next));
            if (count >= a.k) bound = next;
            if (count == a.k) break;
        }
        if (t == 0) pieces = 0;
        __syncthreads();
        for (int i = t; i < n; i += kBeamT)
            if (list[i] >= bound) tops[atomicAdd(&pieces, 1u)] = list[i];
        __syncthreads();
        n = (int)pieces;
        ranked = tops;
    }
    v2u *best = a.best + (row * a.slabs + slab) * a.k;
    for (int i = t; i < n; i += kBeamT) {
        const unsigned own = ranked[i];
        int rank = 0;
        for (int j = 0; j < n; j += 8) {
            const v4u x = *reinterpret_cast<const v4u *>(ranked + j), y = *reinterpret_cast<const v4u *>(ranked + j + 4);
#pragma unroll
            for (int e = 0; e < 4; ++e) rank += (j + e < n && x[e] > own ? 1 : 0) + (j + 4 + e < n && y[e] > own ? 1 : 0);
        }
        if (rank < a.k) best[rank] = v2u{own >> 14, (unsigned)first + 16383 - (own & 16383)};
    }
    for (int i = n + t; i < a.k; i += kBeamT) best[i] = v2u{0, 0};
    if (t == 0) {
        float whole = wave_top[0];
        for (int w = 1; w < kBeamWaves; ++w) whole = fmaxf(whole, wave_top[w]);
        double all = 0.0;
        for (int w = 0; w < kBeamWaves; ++w)
            if (wave_top[w] == whole) all += wave_sum_[w];
            else if (usual(whole)) all += wave_sum_[w] * (double)below(wave_top[w], whole);
        a.rows[row * a.slabs + slab] = BeamRow{below_top(all, whole), whole};
    }
}

// What orders candidates: the total as an integer that orders as binary64 does, then the lower beam, the higher logit, the lower token.  No
// two candidates have the same of both; total 0: none.
struct Candidate {
    u64 total, tie;
};
__device__ __forceinline__ bool before(const Candidate &x, const Candidate &y) { return x.total > y.total || (x.total == y.total && x.tie > y.tie); }
__device__ __forceinline__ u64 total_key(double v)
{
    if (!(v > -INFINITY)) return 0;
    const u64 b = (u64)__double_as_longlong(v + 0.0);                 // (minus zero becomes zero)
    return b >> 63 ? ~b : b | 1ull << 63;
}
__device__ __forceinline__ double total_of(u64 key) { return __longlong_as_double((long long)(key >> 63 ? key & ~(1ull << 63) : ~key)); }
constexpr int kTieBeam = 36, kTieKey = 20;                            // (tokens have 20 bits, keys 16)

// One workgroup per batch element: the rows' sums from their slabs', then the best k of all their candidates, as in beam_rows_kernel: the best of each of 256
// groups of threads, a number that k of those reach, the few candidates that reach it ranked.  6.3 us for 4 beams of 16 slabs with 4 each, 7.6 for 8 beams of 8 slabs
// with 16: three waits for memory and a search over 64 bits, on one compute unit.
constexpr int kSurvivors = 2048, kGroups = 256;
template <int T>
__global__ __launch_bounds__(T) void beam_select_kernel(const BeamArgs a)
{
    constexpr int WAVES = T / 64, KEPT = 8;                           // candidates that a thread keeps; of more, it works out the others again
    __shared__ Candidate tops[kGroups], list[kSurvivors];
    __shared__ float top[kBeamMost];
    __shared__ double log_sum[kBeamMost], score[kBeamMost];
    __shared__ int ended[kBeamMost], listed, counts[WAVES];
    const int t = threadIdx.x, l = t & 63, wave = t >> 6, each = a.slabs * a.k, all = a.beams * each;
    const int64_t b = blockIdx.x, row0 = b * a.beams;
    if (t == 0) listed = 0;
    v2u words[KEPT];
#pragma unroll
    for (int i = 0; i < KEPT; ++i) words[i] = a.best[row0 * each + min(t + i * T, all - 1)];
    // rows' sums: eight lanes each
    for (int r0 = 0; r0 < a.beams; r0 += T / 8) {
        const int r = r0 + t / 8, i0 = t % 8;
        if (r >= a.beams) break;                                      // (all eight lanes)
        const bool done = a.done && a.done[row0 + r] != 0;
        const double own = (double)a.scores[row0 + r];
        const BeamRow *rows = a.rows + (row0 + r) * a.slabs;
        float m = -INFINITY;
        double sum = 0.0;
        if (!done) {
            for (int i = i0; i < a.slabs; i += 8) {                   // (the larger of two: the other's terms below it)
                const BeamRow x = rows[i];
                const float both = fmaxf(m, x.top);
                if (usual(both)) sum = x.top == both ? x.sum + sum * exp((double)m - (double)both) : sum + x.sum * exp((double)x.top - (double)both);
                else if (both > 0.f) sum = (m == both ? sum : 0.0) + (x.top == both ? x.sum : 0.0);
                m = both;
            }
        }
#pragma unroll
        for (int d = 4; d > 0; d >>= 1) {
            const float other = __shfl_xor(m, d), both = fmaxf(m, other);
            const double more = __shfl_xor(sum, d);
            const float low = fminf(m, other);
            if (usual(both)) {
                const double f = low == both ? 1.0 : exp((double)low - (double)both);
                sum = (m == both ? sum : sum * f) + (other == both ? more : more * f);
            } else if (both > 0.f) {
                sum = (m == both ? sum : 0.0) + (other == both ? more : 0.0);
            }
            m = both;
        }
        if (i0 == 0) {
            top[r] = m;
            log_sum[r] = done ? 0.0 : log(sum);
            score[r] = own;
            ended[r] = done;
        }
    }
    __syncthreads();
    auto candidate_of = [&](int c, v2u have) {
        const int r = c / each, i = c - r * each;
        Candidate x = {0, 0};
        if (ended[r]) {
            if (i == 0) x.total = total_key(score[r]), x.tie = (u64)(kBeamMost - 1 - r) << kTieBeam | (unsigned)((1 << kTieKey) - 1 - a.eos);
            return x;
        }
        if (have[0] == 0) return x;
        const float v = value_of(have[0]), m = top[r];
        if (!usual(m) && v != m) return x;                   // (beside infinite logits the others have no probability)
        x.total = total_key(score[r] + ((v == m ? 0.0 : (double)v - (double)m) - log_sum[r]));
        x.tie = (u64)(kBeamMost - 1 - r) << kTieBeam | (u64)have[0] << kTieKey | ((1u << kTieKey) - 1 - have[1]);
        return x;
    };
    Candidate kept[KEPT], mine = {0, 0};
#pragma unroll
    for (int i = 0; i < KEPT; ++i) {
        kept[i] = t + i * T < all ? candidate_of(t + i * T, words[i]) : Candidate{0, 0};
        if (before(kept[i], mine)) mine = kept[i];
    }
    auto others = [&](auto enter) {                                   // four asked for at a time
        for (int c0 = t + KEPT * T; c0 < all; c0 += 4 * T) {
            v2u w[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) w[i] = a.best[row0 * each + min(c0 + i * T, all - 1)];
#pragma unroll
            for (int i = 0; i < 4; ++i)
                if (c0 + i * T < all) enter(candidate_of(c0 + i * T, w[i]));
        }
    };
    others([&](const Candidate &x) {
        if (before(x, mine)) mine = x;
    });
#pragma unroll
    for (int d = 1; d < T / kGroups; d <<= 1) {
        const Candidate x = {(u64)__shfl_xor((unsigned long long)mine.total, d), (u64)__shfl_xor((unsigned long long)mine.tie, d)};
        if (before(x, mine)) mine = x;
    }
    if (t % (T / kGroups) == 0) tops[t / (T / kGroups)] = mine;
    __syncthreads();
    // (all wavefronts the same: the best of four groups to a lane)
    Candidate four[4], reach = {0, 0};
#pragma unroll
    for (int i = 0; i < 4; ++i) four[i] = tops[4 * l + i];
    // the highest number, bit by bit, that k of them reach, or one that exactly k do: of totals, then where those are equal of the ties
    auto search = [&](auto by_total, auto by_both) {
        for (int bit = 63; bit >= 0; --bit) {
            const u64 next = reach.total | 1ull << bit;
            const int n = by_total(next);
            if (n >= a.k) reach.total = next;
            if (n == a.k) return;
        }
        for (int bit = kTieBeam + 5; bit >= 0; --bit) {
            const Candidate next = {reach.total, reach.tie | 1ull << bit};
            const int n = by_both(next);
            if (n >= a.k) reach = next;
            if (n == a.k) return;
        }
    };
    search(
        [&](u64 from) {
            int n = 0;
#pragma unroll
            for (int i = 0; i < 4; ++i) n += __popcll(__ballot(four[i].total >= from));
            return n;
        },
        [&](const Candidate &from) {
            int n = 0;
#pragma unroll
            for (int i = 0; i < 4; ++i) n += __popcll(__ballot(!before(from, four[i])));
            return n;
        });
    auto list_them = [&] {
        if (before(reach, mine)) return;
        auto enter = [&](const Candidate &x) {
            if (x.total == 0 || before(reach, x)) return;
            const int at = atomicAdd(&listed, 1);
            if (at < kSurvivors) list[at] = x;
        };
#pragma unroll
        for (int i = 0; i < KEPT; ++i) enter(kept[i]);
        others(enter);
    };
    list_them();
    __syncthreads();
    if (listed > kSurvivors) {                                        // many of few threads: count all of them instead
        reach = Candidate{0, 0};
        auto count = [&](const Candidate &from) {
            int n = 0;
            if (!before(from, mine)) {
#pragma unroll
                for (int i = 0; i < KEPT; ++i) n += before(from, kept[i]) ? 0 : 1;
                others([&](const Candidate &x) { n += before(from, x) ? 0 : 1; });
            }
#pragma unroll
            for (int i = 32; i > 0; i >>= 1) n += __shfl_xor(n, i);
            __syncthreads();
            if (l == 0) counts[wave] = n;
            __syncthreads();
            n = 0;
            for (int w = 0; w < WAVES; ++w) n += counts[w];
            return n;
        };
        search([&](u64 from) { return count(Candidate{from, 0}); }, count);
        if (t == 0) listed = 0;
        __syncthreads();
        list_them();
        __syncthreads();
    }
    const int n = min(listed, kSurvivors);
    int32_t *parent = a.parent + b * a.k, *token = a.token + b * a.k, *done_out = a.done_out ? a.done_out + b * a.k : nullptr;
    float *out = a.score + b * a.k;
    for (int i = t; i < n; i += T) {
        const Candidate own = list[i];
        int rank = 0;
        for (int j = 0; j < n; ++j) rank += before(list[j], own) ? 1 : 0;
        if (rank >= a.k) continue;
        const int r = kBeamMost - 1 - (int)(own.tie >> kTieBeam), of = (1 << kTieKey) - 1 - (int)(own.tie & ((1u << kTieKey) - 1));
        parent[rank] = r;
        token[rank] = of;
        out[rank] = (float)total_of(own.total);
        if (done_out) done_out[rank] = ended[r] || of == a.eos ? 1 : 0;
    }
    if (n >= a.k) return;
    // Fewer than k with a probability, all of them listed: the others follow in the order of their places, at most k + n of which have to be looked at.
    static_assert(2 * kBeamMost <= T, "a place for each thread");
    const int64_t places = (int64_t)a.beams * a.vocab;
    bool is_listed = t >= places;
    int behind = t;                                                   // places in front that are not listed
    for (int j = 0; j < n; ++j) {
        const int64_t place = (int64_t)(kBeamMost - 1 - (int)(list[j].tie >> kTieBeam)) * a.vocab + ((1 << kTieKey) - 1 - (int)(list[j].tie & ((1u << kTieKey) - 1)));
        is_listed = is_listed || place == t;
        behind -= place < t ? 1 : 0;
    }
    if (!is_listed && n + behind < a.k) {
        const int r = t / a.vocab, of = t % a.vocab;
        parent[n + behind] = r;
        token[n + behind] = of;
        out[n + behind] = -INFINITY;
        if (done_out) done_out[n + behind] = ended[r] || of == a.eos ? 1 : 0;
    }
    if (t < a.k && t >= places) {
        parent[t] = token[t] = -1;
        out[t] = -INFINITY;
        if (done_out) done_out[t] = 0;
    }
}

// Slabs as large as leave the device its workgroups, and no larger than a row.
static int beam_pieces(int64_t rows, int vocab)
{
    for (int pieces = 8; pieces > 1; pieces /= 2)
        if (vocab > kBeamT * 4 * pieces && rows * ((vocab + kBeamT * 8 * pieces - 1) / (kBeamT * 8 * pieces)) >= 256) return pieces;
    return vocab > 64 * kBeamT * 8 ? 8 : 1;
}
static int beam_slabs(int64_t rows, int vocab)
{
    const int slab = kBeamT * 8 * beam_pieces(rows, vocab);
    return (vocab + slab - 1) / slab;
}

size_t beam_workspace_bytes(int batch, int beams, int vocab, int k)
{
    const int64_t rows = (int64_t)batch * beams;
    return (size_t)rows * beam_slabs(rows, vocab) * ((size_t)k * sizeof(v2u) + sizeof(BeamRow));
}

sqap_status launch_beam_select(const __half *logits, int64_t ld, int batch, int beams, int vocab, const float *scores, const int32_t *done, int32_t eos,
                               int k, int32_t *parent, int32_t *token, float *score, int32_t *done_out, void *workspace, hipStream_t st)
{
    const int64_t rows = (int64_t)batch * beams;
    const int pieces = beam_pieces(rows, vocab), slabs = beam_slabs(rows, vocab);
    BeamRow *const sums = static_cast<BeamRow *>(workspace);
    const BeamArgs a = {logits, ld, batch, beams, vocab, k, slabs, scores, done, eos, sums, reinterpret_cast<v2u *>(sums + rows * slabs), parent, token, score, done_out};
    const dim3 grid((unsigned)(rows * slabs)), block(kBeamT);
    switch (pieces) {
    case 8: hipLaunchKernelGGL(beam_rows_kernel<8>, grid, block, 0, st, a); break;
    case 4: hipLaunchKernelGGL(beam_rows_kernel<4>, grid, block, 0, st, a); break;
    case 2: hipLaunchKernelGGL(beam_rows_kernel<2>, grid, block, 0, st, a); break;
    default: hipLaunchKernelGGL(beam_rows_kernel<1>, grid, block, 0, st, a); break;
    }
    SQAP_HIP_CHECK(hipGetLastError());
    // (up to 2048 candidates: 4 beams of 32000 10.4 us, with 1024 threads 11.7; 26908 of them, 31 beams with 62 outputs: 106 us and 35)
    if (beams * slabs * k <= 2048) hipLaunchKernelGGL(beam_select_kernel<256>, dim3(batch), dim3(256), 0, st, a);
    else hipLaunchKernelGGL(beam_select_kernel<1024>, dim3(batch), dim3(1024), 0, st, a);
    SQAP_HIP_CHECK(hipGetLastError());
    return SQAP_OK;
}

// ---------------------------------------------------------------- reordering of a cache

// What sequence i of a group takes over: its parent and the parent's length, for the lane of number i; `moves` for those that change.
struct Parents {
    int parent, length;
    u64 moves;
};
__device__ __forceinline__ Parents parents_of(const int32_t *parents, const int32_t *lengths, int64_t first, int width, int capacity)
{
    const int l = threadIdx.x & 63;
    Parents p = {l, 0, 0};
    if (l < width) {
        const int of = parents[first + l];
        if (of >= 0 && of < width) p.parent = of;
        p.length = lengths[first + p.parent];
    }
    p.moves = __ballot(l < width && p.parent != l && p.length > 0 && p.length <= capacity);
    return p;
}

// The lane's piece of every sequence that takes over something, from the I-th on: all of them are read (on the way down) before the first is written
// (on the way back), so that in place is no matter.  base: of the group's first sequence, the others `pitch` bytes apart; `takes` says by a
// sequence's length whether this lane has anything of it.  (An array of pieces is made one wide register, copied at each of them.)
template <int I, int WIDTH, typename V, typename Takes>
__device__ __forceinline__ void move_pieces(char *base, int64_t pitch, unsigned offset, const Parents &p, u64 &moves, Takes takes)
{
    V piece;
    if (moves >> I & 1) {
        const char *from = base + __builtin_amdgcn_readlane(p.parent, I) * pitch;
        if (takes(__builtin_amdgcn_readlane(p.length, I))) piece = *reinterpret_cast<const V *>(from + offset);
    }
    if constexpr (I + 1 < WIDTH) move_pieces<I + 1, WIDTH, V>(base, pitch, offset, p, moves, takes);
    else asm volatile("" : "+s"(moves));                              // (no path of its own for each set of sequences)
    if (moves >> I & 1) {
        char *to = base + I * pitch;
        if (takes(__builtin_amdgcn_readlane(p.length, I))) *reinterpret_cast<V *>(to + offset) = piece;
    }
}

// One workgroup per group, key head and 256 pieces of a block (of all sequences of the group at once), of the unfinished block's rows, or of
// the scales; V: a piece.  All of a group's sequences are read before any is written, so it works in place; who takes over nothing new moves nothing.  64
// sequences of 8 key heads, up to 2000 positions, 217 MB of reads and writes together: 46 us on data that no cache holds, 4.7 TB/s of the 5.06 that a copy reaches;
// 4 sequences of 32 heads, up to 70 positions, 3.9: latency.
template <int D, int WIDTH, typename V>
__global__ __launch_bounds__(256) void cache8_reorder_kernel(const Cache8View cache, const int32_t *__restrict__ parents, int width,
                                                             const int32_t *__restrict__ lengths, int32_t *__restrict__ lengths_out, int block_groups)
{
    constexpr int BYTES = 2 * kCache8Block * D, SPLIT = BYTES / (256 * (int)sizeof(V)), TAIL_SPLIT = 2 * SPLIT;
    const int t = threadIdx.x, h = blockIdx.y;
    const int64_t first = (int64_t)blockIdx.z * width, heads = cache.kv_heads, head = first * heads + h;
    const Parents p = parents_of(parents, lengths, first, width, cache.blocks * kCache8Block);
    if (lengths_out && h == 0 && blockIdx.x == 0 && t < width) lengths_out[first + t] = p.length;
    if ((int)blockIdx.x < block_groups) {
#pragma unroll 1
        for (int x = blockIdx.x;; x += block_groups) {
            const int block = x / SPLIT;
            u64 moves = __ballot(p.moves >> (t & 63) & 1 && block < p.length / kCache8Block);
            if (moves == 0) break;                                    // (nor any block behind it)
            move_pieces<0, WIDTH, V>(reinterpret_cast<char *>(cache.codes) + (head * cache.blocks + block) * BYTES, heads * cache.blocks * BYTES,
                                     (unsigned)(x % SPLIT * 256 + t) * (unsigned)sizeof(V), p, moves, [](int) { return true; });
        }
        return;
    }
    const int x = (int)blockIdx.x - block_groups;
    if (x < TAIL_SPLIT) {
        const unsigned offset = (unsigned)(x * 256 + t) * (unsigned)sizeof(V);
        const int row = (int)(offset / (2 * D)) % kCache8Block;
        u64 moves = __ballot(p.moves >> (t & 63) & 1 && p.length % kCache8Block > 0);
        move_pieces<0, WIDTH, V>(reinterpret_cast<char *>(cache.tail) + head * 2 * BYTES, heads * 2 * BYTES, offset, p, moves,
                                 [&](int n) { return row < n % kCache8Block; });
        return;
    }
#pragma unroll 1
    for (int from = 0;; from += 256) {                                // (a wavefront has 64 scales: the longest decides whether there are any)
        const int block = from + t;
        u64 moves = __ballot(p.moves >> (t & 63) & 1 && from + (t & ~63) < p.length / kCache8Block);
        if (__syncthreads_or(moves != 0) == 0) break;
        move_pieces<0, WIDTH, v2u>(reinterpret_cast<char *>(cache.scales) + head * cache.blocks * 8, heads * cache.blocks * 8, (unsigned)block * 8u, p, moves,
                                   [&](int n) { return block < n / kCache8Block; });
    }
}

template <int D, int WIDTH, typename V>
static void launch_reorder(const Cache8View &cache, const int32_t *parents, int width, const int32_t *lengths, int longest, int32_t *lengths_out, hipStream_t st)
{
    constexpr int SPLIT = 2 * kCache8Block * D / (int)sizeof(V) / 256;
    const int blocks = std::min(longest / kCache8Block, cache.blocks);         // (no cache holds more: groups without a block cost a launch 0.4 ns each)
    const int block_groups = (int)std::min<int64_t>(std::max<int64_t>(1, (int64_t)blocks * SPLIT), 65536);
    const dim3 grid(block_groups + 2 * SPLIT + 1, cache.kv_heads, cache.batch / width);
    hipLaunchKernelGGL((cache8_reorder_kernel<D, WIDTH, V>), grid, dim3(256), 0, st, cache, parents, width, lengths, lengths_out, block_groups);
}

template <int D>
static void launch_reorder_d(const Cache8View &cache, const int32_t *parents, int width, const int32_t *lengths, int longest, int32_t *lengths_out, hipStream_t st)
{
    if (width <= 4) launch_reorder<D, 4, v4u>(cache, parents, width, lengths, longest, lengths_out, st);
    else if (width <= 8) launch_reorder<D, 8, v4u>(cache, parents, width, lengths, longest, lengths_out, st);
    else if (width <= 16) launch_reorder<D, 16, v4u>(cache, parents, width, lengths, longest, lengths_out, st);
    else if (width <= 32) launch_reorder<D, 32, v4u>(cache, parents, width, lengths, longest, lengths_out, st);
    else launch_reorder<D, 64, v2u>(cache, parents, width, lengths, longest, lengths_out, st);
}

sqap_status launch_cache8_reorder(const Cache8View &cache, int d, const int32_t *parents, int width, const int32_t *lengths, int longest,
                                  int32_t *lengths_out, hipStream_t st)
{
    if (d == 64) launch_reorder_d<64>(cache, parents, width, lengths, longest, lengths_out, st);
    else launch_reorder_d<128>(cache, parents, width, lengths, longest, lengths_out, st);
    SQAP_HIP_CHECK(hipGetLastError());
    return SQAP_OK;
}

}  // namespace sqap
