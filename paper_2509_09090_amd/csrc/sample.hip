// Sampling of the next token from half-precision logits: temperature, the k most likely, the smallest set that holds a share p of the
// mass, a least share of the most likely one's probability, then the inverse of the cumulated masses in index order at a given number.
//
// A token's mass is a function of its logit alone, 2^40 exp((l - max) / T) rounded to an integer: sums of masses are exact, so that
// no order of addition shows, and every cut is a cut between two keys (a half as an integer that orders as the half does) plus a number
// of tokens of the key at the cut, lowest indices first.
#include <algorithm>

#include "common.h"

namespace sqap {

typedef unsigned v4u __attribute__((ext_vector_type(4)));
typedef unsigned v4u_any __attribute__((ext_vector_type(4), aligned(2)));
typedef _Float16 v2h __attribute__((ext_vector_type(2)));
typedef unsigned long long u64;

constexpr int kSampleT = 1024, kSampleWaves = kSampleT / 64, kSlab = 64 * 8;
constexpr int kSampleCached = 32768;                                  // logits that are kept in LDS
constexpr int kBins = 4096;                                           // of 16 keys each
constexpr int kFlat = 4;                                              // (see its use)
constexpr int kTieShift = 52;                                         // a slab's ties above its mass, which has 50 bits at most
constexpr unsigned kKeyMinusInf = 0x03ffu;                            // the lowest key there is

// Keys of halves that are neither NaN nor minus zero (see `clean`): integers that order as the halves do.
__device__ __forceinline__ unsigned key_of(unsigned h) { return h & 0x8000u ? ~h & 0xffffu : h | 0x8000u; }
__device__ __forceinline__ unsigned half_of(unsigned key) { return key & 0x8000u ? key & 0x7fffu : ~key & 0xffffu; }
__device__ __forceinline__ float value_of(unsigned key)
{
    return __half2float(__ushort_as_half((unsigned short)half_of(key)));
}

__device__ __forceinline__ unsigned bin_of(unsigned key) { return kBins - 1 - (key >> 4); }

// exp2((value - top) * per_nat) in units of 2^-40, a whole number in binary64 (whose multiply-adds run at binary32's rate, and no instruction
// of binary32's exponential comes near what a vocabulary of equal shares needs: borders 2^-17 of the mass apart).  The difference is exact; the
// power of two of its fraction, at most a half, is the Taylor series to the eighth power, off by less than 2^-32.  A top that is infinite
// is taken for a large number, and everything else to be far below.
struct Mass {
    static constexpr float kCap = 131072.f;
    double top, per_nat;
    __device__ __forceinline__ void set(float top_, double per_nat_)
    {
        top = fminf(top_, kCap);
        per_nat = top_ > kCap ? 1e30 : per_nat_;
    }
    __device__ __forceinline__ double units(float value) const
    {
        const double p = ((double)__builtin_amdgcn_fmed3f(value, -kCap, kCap) - top) * per_nat, n = rint(p), x = p - n;
        double e = 1.3215486790144305e-06;                            // ln(2)^8 / 8!
        e = fma(e, x, 1.5252733804059838e-05);
        e = fma(e, x, 1.5403530393381606e-04);
        e = fma(e, x, 1.3333558146428441e-03);
        e = fma(e, x, 9.618129107628477e-03);
        e = fma(e, x, 5.5504108664821576e-02);
        e = fma(e, x, 2.402265069591007e-01);
        e = fma(e, x, 6.931471805599453e-01);
        e = fma(e, x, 1.0);
        return rint(ldexp(e, max((int)n, -1000) + 40));               // (the conversion saturates)
    }
    static __device__ __forceinline__ u64 of(double w)                // (whole, below 2^52)
    {
        return (u64)__double_as_longlong(w + 4503599627370496.0) & 0xfffffffffffffull;
    }
    __device__ __forceinline__ u64 operator()(float value) const { return of(units(value)); }
};

// Inclusive sums over the lanes: inside rows of 16 by shifts, then the rows' last lanes are added to the rows behind.
template <int CTRL, int ROWS>
__device__ __forceinline__ u64 dpp_add(u64 v)
{
    const unsigned lo = (unsigned)__builtin_amdgcn_update_dpp(0, (int)(unsigned)v, CTRL, ROWS, 0xf, false);
    const unsigned hi = (unsigned)__builtin_amdgcn_update_dpp(0, (int)(unsigned)(v >> 32), CTRL, ROWS, 0xf, false);
    return v + ((u64)hi << 32 | lo);
}
__device__ __forceinline__ u64 wave_scan(u64 v)
{
    v = dpp_add<0x111, 0xf>(v);
    v = dpp_add<0x112, 0xf>(v);
    v = dpp_add<0x114, 0xf>(v);
    v = dpp_add<0x118, 0xf>(v);
    v = dpp_add<0x142, 0xa>(v);
    return dpp_add<0x143, 0xc>(v);
}
__device__ __forceinline__ u64 row_scan(u64 v)                      // inside rows of 16 only
{
    v = dpp_add<0x111, 0xf>(v);
    v = dpp_add<0x112, 0xf>(v);
    v = dpp_add<0x114, 0xf>(v);
    return dpp_add<0x118, 0xf>(v);
}
__device__ __forceinline__ u64 lane_value(u64 v, int l)
{
    return (u64)(unsigned)__builtin_amdgcn_readlane((int)(unsigned)v, l) | (u64)(unsigned)__builtin_amdgcn_readlane((int)(unsigned)(v >> 32), l) << 32;
}
template <int CTRL, int ROWS>
__device__ __forceinline__ unsigned dpp_add(unsigned v)
{
    return v + (unsigned)__builtin_amdgcn_update_dpp(0, (int)v, CTRL, ROWS, 0xf, false);
}
__device__ __forceinline__ unsigned wave_scan(unsigned v)
{
    v = dpp_add<0x111, 0xf>(v);
    v = dpp_add<0x112, 0xf>(v);
    v = dpp_add<0x114, 0xf>(v);
    v = dpp_add<0x118, 0xf>(v);
    v = dpp_add<0x142, 0xa>(v);
    return dpp_add<0x143, 0xc>(v);
}
__device__ __forceinline__ unsigned wave_total(unsigned v) { return (unsigned)__builtin_amdgcn_readlane((int)wave_scan(v), 63); }

struct SampleArgs {
    const __half *logits;
    int64_t ld;
    int vocab, slabs;                    // slabs of 512 logits
    const float *temperature, *top_p, *min_p, *uniform;
    const int32_t *top_k;
    int32_t *token;
    float *prob;
};

// kListed: candidates that are kept; the row itself takes the place of two thirds of them where it is kept too
template <bool CACHED>
struct alignas(16) SampleLds {
    static constexpr int kListed = CACHED ? 8192 : 24576;
    v4u last[64];                        // the last slab, with minus infinity behind its end
    u64 bins[kBins];                     // masses or counts by key / 16, the largest first
    u64 keys[16];                        // counts of one bin's
    u64 wave_sum[kSampleWaves];
    u64 before;
    unsigned ties_before;
    unsigned wave_max[kSampleWaves];
    int found;
    unsigned listed;
    unsigned list[kListed];              // key, and above it the slab
};

// One workgroup per row; a wavefront has every 16th slab of 512 logits, eight to a lane.  CACHED: the row is kept in LDS
// after the first pass; otherwise it is read again where it is needed, four slabs ahead.
// What bounds it is the instructions of one compute unit: some 28 for each token where all of them count (128001 of them: 30 us, where
// the largest alone is found in 6), and the 16 wavefronts' share in every step that is not about the row, so that each step stands here once
// and has few barriers.  First a bound is found below which nothing can stay: for top-k the k-th largest of the threads' maxima, for top-p alone
// the point where the maxima of the lanes' eight have the mass that is asked for (the total has to be known first), for min-p its
// own.  One pass collects the logits from there on in LDS in no order (all that follows is sums of integers), and the cut is found
// among those, for top-k by counts and for top-p by masses: a histogram of 4096 bins, and of the 16 keys of the bin that holds the cut.  The masses
// that stay are added up by slab, and the drawn token's slab alone is looked at again.  Where more stay than LDS has room for,
// the passes go over the row.  A row of 32000: the largest 3.6 us, no filter 12.9, top-k 40 11.7, top-p 0.9 19.0, all three 17.0; of 128001:
// 6.4, 36.8, 20.0, 54.6, 28.0, and 114 where the 97 in 100 that stay are tens of thousands.  (Full passes throughout, with the
// histogram of every token and masses in binary32: 28 and 99 us for all three and for top-p.)
template <bool CACHED>
__global__ __launch_bounds__(kSampleT) void sample_kernel(const SampleArgs a)
{
    extern __shared__ __attribute__((aligned(16))) uint8_t raw_lds[];
    using Lds = SampleLds<CACHED>;
    constexpr int kListed = Lds::kListed;
    Lds &lds = *reinterpret_cast<Lds *>(raw_lds);
    v4u *cached = reinterpret_cast<v4u *>(raw_lds + sizeof(Lds));
    u64 *slab_sum = reinterpret_cast<u64 *>(raw_lds + sizeof(Lds) + (CACHED ? (size_t)a.slabs * kSlab * 2 : 0));
    const int b = blockIdx.x, t = threadIdx.x, l = t & 63, wave = __builtin_amdgcn_readfirstlane(t >> 6);
    const unsigned short *row = reinterpret_cast<const unsigned short *>(a.logits + (int64_t)b * a.ld);
    const int slabs = a.slabs, last = slabs - 1;
    const float temperature = a.temperature ? a.temperature[b] : 1.f, p_given = a.top_p ? a.top_p[b] : 1.f, m_given = a.min_p ? a.min_p[b] : 0.f;
    const float u = a.uniform[b];
    const int k_given = a.top_k ? a.top_k[b] : 0;
    // a lane's logits of a slab other than the last (of the last but one where there is none; nothing where there is but one)
    auto fetch = [&](int s) {
        v4u v = {0, 0, 0, 0};
        if (last > 0) v = *reinterpret_cast<const v4u_any *>(row + min(s, last - 1) * kSlab + l * 8);
        return v;
    };
    // minus infinity in the place of NaN, zero in that of minus zero
    auto clean = [](v4u v) {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            union { unsigned u; v2h h; } x = {v[i]};
            const v2h zero = {(_Float16)0.f, (_Float16)0.f}, least = {(_Float16)-INFINITY, (_Float16)-INFINITY};
            x.h = __builtin_elementwise_max(x.h + zero, least);
            v[i] = x.u;
        }
        return v;
    };
    auto half_at = [](const v4u &v, int e) {
        const unsigned lo = e & 2 ? v[1] : v[0], hi = e & 2 ? v[3] : v[2];
        return (e & 4 ? hi : lo) >> (16 * (e & 1)) & 0xffffu;
    };
    auto float_of = [](unsigned h) { return __half2float(__ushort_as_half((unsigned short)h)); };
    auto largest = [](const v4u &v) {
        union { unsigned u; v2h h; } x[4] = {{v[0]}, {v[1]}, {v[2]}, {v[3]}};
        const v2h m = __builtin_elementwise_max(__builtin_elementwise_max(x[0].h, x[1].h), __builtin_elementwise_max(x[2].h, x[3].h));
        return fmaxf((float)m[0], (float)m[1]);
    };
    auto key_of_value = [](float value) { return key_of(__half_as_ushort(__float2half_rn(value))); };
    // body(slab, logits) over this wavefront's slabs; `ahead` runs after the first loads
    auto each_loaded = [&](auto ahead, auto body) {
        v4u v0 = fetch(wave), v1 = fetch(wave + kSampleWaves), v2 = fetch(wave + 2 * kSampleWaves), v3 = fetch(wave + 3 * kSampleWaves);
        ahead();
        for (int s = wave; s < slabs; s += kSampleWaves) {
            v4u now = v0;
            v0 = v1;
            v1 = v2;
            v2 = v3;
            v3 = fetch(s + 4 * kSampleWaves);
            if (s == last) now = lds.last[l];
            body(s, clean(now));
        }
    };
    auto each_slab = [&](auto body) {
        if constexpr (CACHED) {
            for (int s = wave; s < slabs; s += kSampleWaves) body(s, cached[s * 64 + l]);
        } else {
            each_loaded([] {}, body);
        }
    };
    // (all three are values of halves)
    auto any_between = [](const v4u &v, float low, float high) {
        const v2h l2 = {(_Float16)low, (_Float16)low}, h2 = {(_Float16)high, (_Float16)high};
        typedef unsigned short v2s __attribute__((ext_vector_type(2)));
        v2s outside = {0, 0};
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            union { unsigned u; v2h h; v2s s; } x = {v[i]}, y;
            y.h = __builtin_elementwise_min(__builtin_elementwise_max(x.h, l2), h2);
            x.u ^= y.u;
            outside += __builtin_elementwise_min(x.s, v2s{1, 1});
        }
        return outside[0] + outside[1] < 8;
    };
    // which of a lane's eight are `least` or more
    auto from_bits = [&](const v4u &v, float least) {
        unsigned bits = 0;
#pragma unroll
        for (int e = 0; e < 8; ++e) bits |= float_of(half_at(v, e)) >= least ? 1u << e : 0u;
        return bits;
    };
    bool listed = false;
    unsigned n_listed = 0;
    // The sum of the threads in front, and of all.  (A barrier lies between the last reads of wave_sum and this.)
    auto block_scan = [&](u64 v, u64 &front) {
        const u64 cum = wave_scan(v);
        if (l == 63) lds.wave_sum[wave] = cum;
        __syncthreads();
        const u64 waves = row_scan(lds.wave_sum[l & (kSampleWaves - 1)]);
        front = cum - v + (wave ? lane_value(waves, wave - 1) : 0);
        return lane_value(waves, kSampleWaves - 1);
    };
    // From the largest key down, the first bin whose inclusive sum reaches `target` (>= 1), and the sum before it; -1: none.  Bins and keys are
    // zeroes again.
    auto first_bin = [&](u64 target) {
        __syncthreads();
        u64 of[4], sum = 0, at;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            sum += of[i] = lds.bins[4 * t + i];
            lds.bins[4 * t + i] = 0;
        }
        if (t < 16) lds.keys[t] = 0;
        const u64 all = block_scan(sum, at);
        if (at < target && at + sum >= target) {
            int i = 0;
#pragma unroll
            for (int x = 0; x < 3; ++x)
                if (i == x && at + of[x] < target) at += of[x], ++i;
            lds.found = kBins - 1 - (4 * t + i);
            lds.before = at;
        }
        __syncthreads();
        return all >= target ? lds.found : -1;
    };

    // ---- the largest logit, and each thread's
    float mine = -INFINITY;
    int mine_at = wave;
    each_loaded(
        [&] {
            if (t < kSlab) reinterpret_cast<unsigned short *>(lds.last)[t] = last * kSlab + t < a.vocab ? row[last * kSlab + t] : 0xfc00;
            if (t == 0) lds.found = a.vocab, lds.listed = 0;
#pragma unroll
            for (int i = 0; i < 4; ++i) lds.bins[4 * t + i] = 0;
            for (int s = t; s < slabs; s += kSampleT) slab_sum[s] = 0;
            __syncthreads();
        },
        [&](int s, const v4u &v) {
            if constexpr (CACHED) cached[s * 64 + l] = v;
            const float m = largest(v);
            mine_at = m > mine ? s : mine_at;
            mine = fmaxf(mine, m);
        });
    unsigned top_key = key_of_value(mine);
    top_key = max(top_key, dpp_move<kDppXor1>(top_key));
    top_key = max(top_key, dpp_move<kDppXor2>(top_key));
    top_key = max(top_key, dpp_move<kDppHalfMirror>(top_key));
    top_key = max(top_key, dpp_move<kDppMirror>(top_key));
    top_key = max(max((unsigned)__builtin_amdgcn_readlane((int)top_key, 0), (unsigned)__builtin_amdgcn_readlane((int)top_key, 16)),
                  max((unsigned)__builtin_amdgcn_readlane((int)top_key, 32), (unsigned)__builtin_amdgcn_readlane((int)top_key, 48)));
    if (l == 0) lds.wave_max[wave] = top_key;
    __syncthreads();
    top_key = lds.wave_max[l & (kSampleWaves - 1)];
    top_key = max(top_key, dpp_move<kDppXor1>(top_key));
    top_key = max(top_key, dpp_move<kDppXor2>(top_key));
    top_key = max(top_key, dpp_move<kDppHalfMirror>(top_key));
    top_key = (unsigned)__builtin_amdgcn_readfirstlane((int)max(top_key, dpp_move<kDppMirror>(top_key)));
    if (top_key <= kKeyMinusInf) {                                    // nothing can be drawn
        if (t == 0) {
            a.token[b] = -1;
            if (a.prob) a.prob[b] = 0.f;
        }
        return;
    }
    const float top = value_of(top_key);
    if (!(temperature > 0.f)) {                                       // the most likely one
        if (mine == top) {
            const v4u v = clean(mine_at == last ? lds.last[l] : fetch(mine_at));
            atomicMin(&lds.found, mine_at * kSlab + l * 8 + (int)__builtin_ctz(from_bits(v, top)));
        }
        __syncthreads();
        if (t == 0) {
            a.token[b] = lds.found;
            if (a.prob) a.prob[b] = 1.f;
        }
        return;
    }
    const double per_nat = 1.4426950408889634074 / (double)temperature;
    Mass mass;
    mass.set(top, per_nat);

    const float lowest = value_of(kKeyMinusInf + 1);                  // (minus infinity never stays)
    const int k = k_given > 0 && k_given < a.vocab ? k_given : 0;     // 0: all
    const bool by_mass = !(p_given >= 1.f);
    // min-p: the lowest value whose mass is enough, the top's at the latest: of 2^16 keys, 64 at a time
    float min_value = lowest;
    if (m_given > 0.f) {
        const double enough = (double)fminf(m_given, 1.f) * 1099511627776.0;
        int below = 0;                                                // (the lowest key of all has no mass)
#pragma unroll 1
        for (int step = 1024; step; step >>= step == 1 ? 1 : step == 16 ? 4 : 6) {
            const int key = below + step * (l + 1);
            const u64 is = __ballot(key >= (int)top_key || (key > (int)kKeyMinusInf && mass.units(value_of((unsigned)key)) >= enough));
            below += is ? step * (int)__builtin_ctzll(is) : step * 64;
        }
        min_value = fmaxf(lowest, value_of((unsigned)min(below + 1, (int)top_key)));
    }

    // the cut: keys above it stay, and `cut_count` of its own key, of which there are `cut_has`
    unsigned cut = 0;
    u64 cut_count = ~0ull, cut_has = 0, total = 0, front;
    u64 tie_mass = 0;
    bool some = false;                                                // (only some of the cut's key stay: they have to be told apart)
    float from = lowest;
    const bool plain = !k && !by_mass && !(m_given > 0.f);
    // masses of the row from `from` on, except for those of `tie_half`: by slab in `slab_sum`, with the number of ties; kMaxima: each eight's
    // maximum by its key; kAll: each by its key (or each as one).  The lane's sum is returned.
    enum { kNone, kMaxima, kAll };
    const std::integral_constant<int, kNone> no_bins;
    const std::integral_constant<int, kMaxima> maxima;
    const std::integral_constant<int, kAll> all_bins;
    auto masses = [&](auto bins_c, unsigned tie_half, bool counting) {
        constexpr int BINS = decltype(bins_c)::value;
        u64 mine = 0;
        const float above = tie_half < 0x10000u ? value_of(key_of(tie_half) + 1) : from;
        each_slab([&](int s, const v4u &v) {
            u64 sum = 0;
            unsigned ties = 0;
            const float m = largest(v);
            if (__any(m >= from)) {
                double w[8], eight = 0.0;                             // (exact)
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    const float value = float_of(half_at(v, e));
                    w[e] = BINS == kAll && counting ? 1099511627776.0 : mass.units(value);
                    w[e] = value >= above ? w[e] : 0.0;
                    eight += w[e];
                }
                if constexpr (BINS == kAll) {                         // (behind the last of them: a branch in between would part their chains)
                    __builtin_amdgcn_sched_barrier(0);
#pragma unroll
                    for (int e = 0; e < 8; ++e)
                        if (w[e] > 0.0) atomicAdd(&lds.bins[bin_of(key_of(half_at(v, e)))], mass.of(w[e]));
                }
                if (tie_half < 0x10000u) {
#pragma unroll
                    for (int e = 0; e < 8; ++e) ties += half_at(v, e) == tie_half ? 1 : 0;
                }
                sum = mass.of(eight);                                 // 43 bits; 20 of them and the rest on their own
                mine += sum;
                sum = ((u64)wave_total((unsigned)(sum >> 20)) << 20) + wave_total((unsigned)sum & 0xfffffu);
                if (tie_half < 0x10000u) ties = wave_total(ties);
                if constexpr (BINS == kMaxima) {
                    const u64 w = mass(m);
                    if (w) atomicAdd(&lds.bins[bin_of(key_of_value(m))], w);
                }
            }
            if (l == 0) slab_sum[s] = sum + ((u64)ties << kTieShift);
        });
        return mine;
    };
    constexpr unsigned kNoHalf = 0x10000u;
    // Top-p alone, where the threads' maxima are several times the largest: more tokens are likely to stay than LDS has room for, and the first
    // pass over the masses leaves the histogram of them all, instead of that of the eights' maxima and a second pass (rows of 128001 of which
    // tens of thousands stay: 107 to 114 us, 141 without; where few stay all the same, 17 us more).
    const bool flat = by_mass && !k && block_scan(mass(mine), front) > (u64)kFlat << 40;
    int bin = -1;
    for (bool final = plain;; final = true) {
        // ---- what stays, by slab; the first time (top-p alone) all
        if (final || (by_mass && !k)) {
            if (listed) {
                for (unsigned i = t; i < n_listed; i += kSampleT) {
                    const unsigned key = lds.list[i] & 0xffffu;
                    const u64 add = some && key == cut ? 1ull << kTieShift : mass(value_of(key));
                    if (add && value_of(key) >= from) atomicAdd(&slab_sum[lds.list[i] >> 16], add);
                }
            } else if (final) {
                masses(no_bins, some ? half_of(cut) : kNoHalf, false);
            } else if (flat) {
                masses(all_bins, kNoHalf, false);
            } else {
                masses(maxima, kNoHalf, false);
            }
            __syncthreads();
        }
        if (final) break;

        // ---- the bound
        u64 target = (u64)k;
        if (k && k <= kSampleT) {
            if (mine > -INFINITY) atomicAdd(&lds.bins[bin_of(key_of_value(mine))], 1ull);
        } else if (by_mass && !k) {
            u64 two = 0;
#pragma unroll
            for (int i = 0; i < 2; ++i)
                if (2 * t + i < slabs) {
                    two += slab_sum[2 * t + i];
                    slab_sum[2 * t + i] = 0;                          // (what is on the list is added to them)
                }
            total = block_scan(two, front);
            target = min(total, max(1ull, p_given > 0.f ? (u64)ceil((double)p_given * (double)total) : 1ull));
        }
        if (by_mass || k) {
            bin = first_bin(target);
            if (bin > (int)(kKeyMinusInf >> 4)) from = value_of((unsigned)bin << 4);
        } else {
            from = min_value;
        }
        // ---- what is not below it
        if (k <= kListed && (from > lowest || a.vocab <= kListed)) {
            bool room = true;
            each_slab([&](int s, const v4u &v) {
                unsigned bits = room && largest(v) >= from ? from_bits(v, from) : 0;
                if (__any(bits != 0)) {
                    const unsigned n = __builtin_popcount(bits), upto = wave_scan(n), of_all = (unsigned)__builtin_amdgcn_readlane((int)upto, 63);
                    unsigned first = 0;
                    if (l == 0) first = atomicAdd(&lds.listed, of_all);
                    first = (unsigned)__builtin_amdgcn_readfirstlane((int)first);
                    room = first + of_all <= kListed;
                    unsigned at = first + upto - n;
                    for (; room && bits; bits &= bits - 1, ++at) lds.list[at] = key_of(half_at(v, __builtin_ctz(bits))) | (unsigned)s << 16;
                }
            });
            __syncthreads();
            n_listed = lds.listed;
            listed = n_listed <= kListed;
        }
        // ---- the cut, for top-k by counts and then for top-p by masses
#pragma unroll 1
        for (int round = k ? 0 : 1; round < (by_mass ? 2 : 1); ++round) {
            const bool counting = round == 0;
            u64 kept = 0;
            if (flat) {
                // (the bound's bin is the cut's)
            } else if (listed) {
                for (unsigned i = t; i < n_listed; i += kSampleT) {
                    const unsigned key = lds.list[i] & 0xffffu;
                    const u64 w = value_of(key) < from || (cut && key == cut) ? 0 : counting ? 1 : mass(value_of(key));
                    kept += w;
                    if (w) atomicAdd(&lds.bins[bin_of(key)], w);
                }
            } else {
                kept = masses(all_bins, cut ? half_of(cut) : kNoHalf, counting);
            }
            if (!counting && k) {
                const u64 ties = cut ? cut_count * mass(value_of(cut)) : 0;
                if (t == 0 && ties) atomicAdd(&lds.bins[bin_of(cut)], ties);
                total = block_scan(kept, front) + ties;
                target = min(total, max(1ull, p_given > 0.f ? (u64)ceil((double)p_given * (double)total) : 1ull));
            }
            if (counting && !listed) target <<= 40;
            if (!flat) bin = first_bin(target);
            if (bin < 0) continue;                                    // (fewer tokens than k can be drawn: all of them stay)
            const u64 rest = counting && !listed ? (target - lds.before) >> 40 : target - lds.before;
            const float low = bin > (int)(kKeyMinusInf >> 4) ? fmaxf(from, value_of((unsigned)bin << 4)) : from;
            const unsigned key0 = (unsigned)bin << 4;
            const float high = value_of(min(key0 + 15u, top_key));
            if (listed) {
                for (unsigned i = t; i < n_listed; i += kSampleT) {
                    const unsigned key = lds.list[i] & 0xffffu;
                    if (key - key0 < 16u && value_of(key) >= low) atomicAdd(&lds.keys[key & 15], 1ull);
                }
            } else {
                each_slab([&](int, const v4u &v) {
                    unsigned bits = 0;
                    if (largest(v) >= low && any_between(v, low, high)) {
#pragma unroll
                        for (int e = 0; e < 8; ++e) bits |= key_of(half_at(v, e)) - key0 < 16u ? 1u << e : 0u;
                    }
                    for (; bits; bits &= bits - 1) {
                        const unsigned h = half_at(v, __builtin_ctz(bits));
                        if (float_of(h) >= low) atomicAdd(&lds.keys[key_of(h) & 15], 1ull);
                    }
                });
            }
            __syncthreads();
            // (a lane per key, the largest first)
            const unsigned key = (unsigned)bin << 4 | (15u - (l & 15));
            const u64 has = l < 16 && key >= cut ? lds.keys[key & 15] : 0, n = cut && key == cut ? min(has, cut_count) : has;
            const u64 w = counting ? 1 : mass(value_of(key)), cum = wave_scan(n * w);
            const int at = __builtin_ctzll(__ballot(n * w > 0 && cum >= rest) | 1ull << 63) & 15;
            const u64 left = rest - lane_value(cum - n * w, at), each = max(1ull, lane_value(w, at));
            u64 count = (u64)((double)left / (double)each);
            if (count * each < left) ++count;
            cut = (unsigned)__builtin_amdgcn_readlane((int)key, at);
            cut_count = max(1ull, count);
            cut_has = lane_value(has, at);
            from = value_of(cut);
        }
        some = cut && cut_count < cut_has && from >= min_value;       // (below min-p's value none of them stays)
        tie_mass = some ? mass(from) : 0;
        from = fmaxf(from, min_value);
    }

    // ---- the slab of the drawn token: each thread has two
    u64 of[2], ties[2] = {0, 0}, ties_front = 0;
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        const u64 both = 2 * t + i < slabs ? slab_sum[2 * t + i] : 0;
        of[i] = both & ((1ull << kTieShift) - 1);
        ties[i] = both >> kTieShift;
    }
    if (some) {
        block_scan(ties[0] + ties[1], ties_front);
        __syncthreads();
        u64 in_front = ties_front;
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            if (in_front < cut_count) of[i] += min(ties[i], cut_count - in_front) * tie_mass;
            in_front += ties[i];
        }
    }
    const u64 all = block_scan(of[0] + of[1], front);
    u64 target = u > 0.f ? (u64)((double)fminf(u, 1.f) * (double)all) : 0;
    target = min(target, all - 1) + 1;
    if (front < target && front + of[0] + of[1] >= target) {
        const int i = front + of[0] < target ? 1 : 0;
        lds.found = 2 * t + i;
        lds.before = front + (i ? of[0] : 0);
        lds.ties_before = (unsigned)(ties_front + (i ? ties[0] : 0));
    }
    __syncthreads();
    if (wave) return;
    const int s = lds.found;
    const v4u v = CACHED ? cached[s * 64 + l] : clean(s == last ? lds.last[l] : fetch(s));
    u64 rank = 0;
    if (some) {
        unsigned n = 0;
#pragma unroll
        for (int e = 0; e < 8; ++e) n += key_of(half_at(v, e)) == cut ? 1 : 0;
        rank = lds.ties_before + wave_scan(n) - n;
    }
    u64 w[8], lane_mass = 0;
#pragma unroll
    for (int e = 0; e < 8; ++e) {
        const unsigned h = half_at(v, e);
        const bool stays = float_of(h) >= from && !(some && key_of(h) == cut && rank++ >= cut_count);
        w[e] = stays ? mass(float_of(h)) : 0;
        lane_mass += w[e];
    }
    const u64 cum = wave_scan(lane_mass), before = lds.before;
    const u64 reached = __ballot(before + cum >= target);
    if (reached == 0 || l != __builtin_ctzll(reached)) return;
    u64 at = before + cum - lane_mass, chosen = 0;
    int e = 0;
#pragma unroll
    for (int x = 0; x < 8; ++x)
        if (e == x) {
            chosen = w[x];
            if (x < 7 && at + w[x] < target) at += w[x], ++e;
        }
    a.token[b] = s * kSlab + l * 8 + e;
    if (a.prob) a.prob[b] = (float)((double)chosen / (double)all);
}

sqap_status launch_sample(const __half *logits, int64_t ld, int batch, int vocab, const float *temperature, const int32_t *top_k,
                          const float *top_p, const float *min_p, const float *uniform, int32_t *token, float *prob, hipStream_t st)
{
    const int slabs = (vocab + kSlab - 1) / kSlab;
    const bool cached = vocab <= kSampleCached;
    const size_t lds = (size_t)slabs * sizeof(u64) + (cached ? sizeof(SampleLds<true>) + (size_t)slabs * kSlab * 2 : sizeof(SampleLds<false>));
    static std::atomic<bool> ready[kMaxDeviceSlots];
    if (!ready[device_slot()].load(std::memory_order_relaxed)) {
        constexpr int most_cached = sizeof(SampleLds<true>) + kSampleCached * 2 + kSampleCached / kSlab * sizeof(u64);
        constexpr int most = sizeof(SampleLds<false>) + kSampleMaxVocab / kSlab * sizeof(u64);
        static_assert(most_cached <= 163840 && most <= 163840, "a compute unit's LDS");
        SQAP_HIP_CHECK(hipFuncSetAttribute(reinterpret_cast<const void *>(sample_kernel<true>), hipFuncAttributeMaxDynamicSharedMemorySize, most_cached));
        SQAP_HIP_CHECK(hipFuncSetAttribute(reinterpret_cast<const void *>(sample_kernel<false>), hipFuncAttributeMaxDynamicSharedMemorySize, most));
        ready[device_slot()].store(true, std::memory_order_relaxed);
    }
    for (int64_t first = 0; first < batch; first += most_workgroups(kSampleT)) {
        const auto at = [&](auto *p) { return p ? p + first : p; };
        const SampleArgs a = {logits + first * ld, ld, vocab, slabs, at(temperature), at(top_p), at(min_p), at(uniform), at(top_k), at(token), at(prob)};
        const dim3 grid((unsigned)std::min(most_workgroups(kSampleT), batch - first)), block(kSampleT);
        if (cached) hipLaunchKernelGGL(sample_kernel<true>, grid, block, lds, st, a);
        else hipLaunchKernelGGL(sample_kernel<false>, grid, block, lds, st, a);
        SQAP_HIP_CHECK(hipGetLastError());
    }
    return SQAP_OK;
}

}  // namespace sqap
