// Sampling of the next token from half-precision logits: temperature, the k most likely, the smallest set that holds a share p of the
// mass, a least share of the most likely one's probability, then the inverse of the cumulated masses in index order at a given number.
//
// A token's mass is a function of its logit alone, 2^40 exp((l - max) / T) rounded down to an integer: sums of masses are exact, so that
// no order of addition shows, and every cut is a cut between two keys (a half as an integer that orders as the half does) plus a number
// of tokens of the key at the cut, lowest indices first.
#include <algorithm>

#include "common.h"

namespace sqap {

typedef unsigned v4u __attribute__((ext_vector_type(4)));
typedef unsigned v4u_any __attribute__((ext_vector_type(4), aligned(2)));
typedef unsigned long long u64;

constexpr int kSampleT = 1024, kSampleWaves = kSampleT / 64, kSampleCopies = 8;
constexpr int kSampleMaxSlabs = kSampleMaxVocab / (8 * kSampleT);
constexpr unsigned kKeyMinusInf = 0x03ffu;                            // keys up to here: minus infinity, and 0 for NaN
constexpr double kMassOne = 1099511627776.0;                          // 2^40

__device__ __forceinline__ unsigned key_of(unsigned h)
{
    const unsigned m = h & 0x7fffu;
    if (m == 0) return 0x8000u;                                       // the two zeros are equal
    if (m > 0x7c00u) return 0u;                                       // NaN is below every number
    return h & 0x8000u ? ~h & 0xffffu : h | 0x8000u;
}
__device__ __forceinline__ float value_of(unsigned key)
{
    return __half2float(__ushort_as_half((unsigned short)(key & 0x8000u ? key & 0x7fffu : ~key & 0xffffu)));
}

// The exponent in two parts (x times a binary64 factor as two binary32 ones), so that a mass is off by 2^-22 or so however far the logit is
// from the largest.
struct Mass {
    unsigned top;
    float top_value, hi, lo;
    __device__ __forceinline__ u64 operator()(unsigned key) const
    {
        if (key == top) return 1ull << 40;
        const float x = value_of(key) - top_value, p = x * hi;
        if (key <= kKeyMinusInf || !(p > -41.f)) return 0;
        const float rest = fmaf(x, lo, fmaf(x, hi, -p));
        const float w = exp2f(p) * fmaf(rest, 0.6931471805599453f, 1.f);
        const float a = floorf(w * 1048576.f);
        return ((u64)(unsigned)a << 20) + (u64)(unsigned)((w * 1048576.f - a) * 1048576.f);
    }
};

__device__ __forceinline__ u64 shfl_up64(u64 v, int by) { return (u64)__shfl_up((long long)v, by); }

// Inclusive sums over the lanes.
__device__ __forceinline__ u64 wave_scan(u64 v)
{
    const int l = threadIdx.x & 63;
#pragma unroll
    for (int by = 1; by < 64; by <<= 1) {
        const u64 o = shfl_up64(v, by);
        if (l >= by) v += o;
    }
    return v;
}

// By one whole wavefront: the first of n values whose inclusive sum reaches `target` (>= 1; there is one), and the sum before it.
__device__ __forceinline__ int first_reaching(const u64 *values, int n, u64 target, u64 &before)
{
    const int l = threadIdx.x & 63, per = (n + 63) / 64;
    u64 mine = 0;
    for (int i = 0; i < per; ++i)
        if (l * per + i < n) mine += values[l * per + i];
    const u64 sum = wave_scan(mine);
    const u64 reached = __ballot(sum >= target);
    const int lane = reached ? __builtin_ctzll(reached) : 63;
    u64 cum = (u64)__shfl((long long)(sum - mine), lane);
    int at = lane * per;
    for (; at < n - 1 && cum + values[at] < target; ++at) cum += values[at];
    before = cum;
    return at;
}

struct SampleArgs {
    const __half *logits;
    int64_t ld;
    int vocab;
    const float *temperature, *top_p, *min_p, *uniform;
    const int32_t *top_k;
    int32_t *token;
    float *prob;
};

struct SampleLds {
    u64 mass[256], bins[256 * kSampleCopies];
    unsigned count[256 * kSampleCopies];
    u64 count64[256];
    u64 table[kSampleMaxSlabs * kSampleWaves];
    unsigned ties[kSampleMaxSlabs * kSampleWaves];
    unsigned wave_top[kSampleWaves];
    int found;
    unsigned cut_key;
    u64 cut_count, cut_mass, cut_total, before;
};

// One workgroup per row.  PIECES > 0: the row is kept in registers, 8 neighbouring logits per piece; 0: it is read again for every pass.
template <int PIECES>
__global__ __launch_bounds__(kSampleT) void sample_kernel(const SampleArgs a)
{
    extern __shared__ __attribute__((aligned(16))) uint8_t raw_lds[];
    SampleLds &lds = *reinterpret_cast<SampleLds *>(raw_lds);
    const int b = blockIdx.x, t = threadIdx.x, l = t & 63, wave = t >> 6;
    const unsigned short *row = reinterpret_cast<const unsigned short *>(a.logits + (int64_t)b * a.ld);
    const int slabs = PIECES ? PIECES : (a.vocab + 8 * kSampleT - 1) / (8 * kSampleT);
    auto load = [&](int i) {
        const int at = (i * kSampleT + t) * 8;
        v4u v = {0x7e007e00u, 0x7e007e00u, 0x7e007e00u, 0x7e007e00u};  // past the end: NaN
        if (at + 8 <= a.vocab) {
            v = *reinterpret_cast<const v4u_any *>(row + at);
        } else {
            for (int e = 0; e < 8 && at + e < a.vocab; ++e) {
                const unsigned shift = 16 * (e & 1);
                v[e >> 1] = (v[e >> 1] & ~(0xffffu << shift)) | (unsigned)row[at + e] << shift;
            }
        }
        return v;
    };
    v4u held[PIECES ? PIECES : 1];
    if (PIECES)
#pragma unroll
        for (int i = 0; i < PIECES; ++i) held[i] = load(i);
    // body(key, slab, element) over this thread's logits, slab by slab
    auto each = [&](auto body) {
        if constexpr (PIECES > 0) {
#pragma unroll
            for (int i = 0; i < PIECES; ++i)
#pragma unroll
                for (int e = 0; e < 8; ++e) body(key_of(held[i][e >> 1] >> (16 * (e & 1)) & 0xffffu), i, e);
        } else {
            for (int i = 0; i < slabs; ++i) {
                const v4u v = load(i);
#pragma unroll
                for (int e = 0; e < 8; ++e) body(key_of(v[e >> 1] >> (16 * (e & 1)) & 0xffffu), i, e);
            }
        }
    };

    unsigned top = 0;
    each([&](unsigned key, int, int) { top = max(top, key); });
    for (int by = 32; by > 0; by >>= 1) top = max(top, (unsigned)__shfl_xor((int)top, by));
    if (l == 0) lds.wave_top[wave] = top;
    if (t == 0) lds.found = a.vocab;
    __syncthreads();
    for (int w = 0; w < kSampleWaves; ++w) top = max(top, lds.wave_top[w]);
    if (top <= kKeyMinusInf) {                                        // nothing can be drawn
        if (t == 0) {
            a.token[b] = -1;
            if (a.prob) a.prob[b] = 0.f;
        }
        return;
    }
    const float temperature = a.temperature ? a.temperature[b] : 1.f;
    if (!(temperature > 0.f)) {                                       // the most likely one
        int first = a.vocab;
        each([&](unsigned key, int i, int e) {
            if (key == top) first = min(first, (i * kSampleT + t) * 8 + e);
        });
        if (first < a.vocab) atomicMin(&lds.found, first);
        __syncthreads();
        if (t == 0) {
            a.token[b] = lds.found;
            if (a.prob) a.prob[b] = 1.f;
        }
        return;
    }
    Mass mass;
    mass.top = top;
    mass.top_value = value_of(top);
    const double per_nat = 1.4426950408889634074 / (double)temperature;
    mass.hi = (float)per_nat;
    mass.lo = (float)(per_nat - (double)mass.hi);

    const int k_given = a.top_k ? a.top_k[b] : 0;
    const int k = k_given > 0 && k_given < a.vocab ? k_given : 0;     // 0: all
    const float p_given = a.top_p ? a.top_p[b] : 1.f;
    const bool by_mass = !(p_given >= 1.f);
    const float m_given = a.min_p ? a.min_p[b] : 0.f;
    const u64 least = m_given > 0.f ? (u64)ceil(fmin((double)m_given, 1.0) * kMassOne) : 0;

    // the cut: keys above it stay, and `cut_count` of its own key
    unsigned cut = 0;
    u64 cut_count = ~0ull;
    if (k || by_mass) {
        auto clear = [&] {
            for (int i = t; i < 256 * kSampleCopies; i += kSampleT) {
                lds.bins[i] = 0;
                lds.count[i] = 0;
            }
            __syncthreads();
        };
        // values from the largest key down; copies added
        auto gather = [&](bool masses) {
            __syncthreads();
            if (t < 256) {
                u64 m = 0, c = 0;
                for (int x = 0; x < kSampleCopies; ++x) {
                    if (masses) m += lds.bins[(255 - t) * kSampleCopies + x];
                    c += lds.count[(255 - t) * kSampleCopies + x];
                }
                if (masses) lds.mass[t] = m;
                lds.count64[t] = c;
            }
            __syncthreads();
        };
        // counts of the 256 keys of one bin
        auto keys_of_bin = [&](unsigned bin) {
            clear();
            each([&](unsigned key, int, int) {
                if (key >> 8 == bin) atomicAdd(&lds.count[(key & 255) * kSampleCopies + (t & (kSampleCopies - 1))], 1u);
            });
            gather(false);
        };
        clear();
        each([&](unsigned key, int, int) {
            if (key > kKeyMinusInf) {
                const int at = (key >> 8) * kSampleCopies + (t & (kSampleCopies - 1));
                if (k) atomicAdd(&lds.count[at], 1u);
                if (by_mass) {
                    const u64 w = mass(key);
                    if (w) atomicAdd(&lds.bins[at], w);
                }
            }
        });
        gather(true);
        int bin_k = -1;                                               // (places from the top, as gather() leaves them)
        if (k) {
            if (wave == 0) {
                u64 all = 0;
                for (int i = l; i < 256; i += 64) all += lds.count64[i];
                all = wave_scan(all);
                all = (u64)__shfl((long long)all, 63);
                u64 before = 0;
                const int at = all >= (u64)k ? first_reaching(lds.count64, 256, (u64)k, before) : -1;
                if (l == 0) {
                    lds.found = at;
                    lds.before = before;
                }
            }
            __syncthreads();
            bin_k = lds.found;
            if (bin_k >= 0) {
                const u64 rest = (u64)k - lds.before;
                keys_of_bin(255 - bin_k);
                if (wave == 0) {
                    u64 before;
                    const int at = first_reaching(lds.count64, 256, rest, before);
                    if (l == 0) {
                        lds.cut_key = (unsigned)(255 - bin_k) << 8 | (unsigned)(255 - at);
                        lds.cut_count = rest - before;
                    }
                }
                __syncthreads();
                cut = lds.cut_key;
                cut_count = lds.cut_count;
            }
        }
        if (by_mass) {
            __syncthreads();
            // the bin of the k-th key holds what stays of it
            if (bin_k >= 0) {
                if (wave == 0) {
                    u64 m = 0;
                    for (int i = l; i < 256; i += 64) {
                        const unsigned key = (unsigned)(255 - bin_k) << 8 | (unsigned)(255 - i);
                        if (key >= cut) m += (key == cut ? cut_count : lds.count64[i]) * mass(key);
                    }
                    m = wave_scan(m);
                    if (l == 63) lds.mass[bin_k] = m;
                }
                if (t > bin_k && t < 256) lds.mass[t] = 0;
                __syncthreads();
            }
            if (wave == 0) {
                u64 all = 0;
                for (int i = l; i < 256; i += 64) all += lds.mass[i];
                all = wave_scan(all);
                all = (u64)__shfl((long long)all, 63);
                const double share = p_given > 0.f ? ceil((double)p_given * (double)all) : 1.0;
                const u64 target = min(all, max(1ull, (u64)share));
                u64 before;
                const int at = first_reaching(lds.mass, 256, target, before);
                if (l == 0) {
                    lds.found = at;
                    lds.before = before;
                    lds.cut_total = target;
                }
            }
            __syncthreads();
            const int bin = lds.found;
            const u64 rest = lds.cut_total - lds.before;
            if (bin != bin_k) keys_of_bin(255 - bin);
            __syncthreads();
            if (t < 256) {
                const unsigned key = (unsigned)(255 - bin) << 8 | (unsigned)(255 - t);
                lds.mass[t] = key < cut ? 0 : (key == cut && bin == bin_k ? cut_count : lds.count64[t]) * (key > kKeyMinusInf ? mass(key) : 0);
            }
            __syncthreads();
            if (wave == 0) {
                u64 before;
                const int at = first_reaching(lds.mass, 256, rest, before);
                if (l == 0) {
                    const unsigned key = (unsigned)(255 - bin) << 8 | (unsigned)(255 - at);
                    const u64 w = max(1ull, mass(key));
                    lds.cut_key = key;
                    lds.cut_count = (rest - before + w - 1) / w;
                }
            }
            __syncthreads();
            cut = lds.cut_key;
            cut_count = lds.cut_count;
        }

    }

    // how many tokens of the cut's key lie before each slab of each wavefront
    const bool count_ties = cut_count != ~0ull;
    const int entries = slabs * kSampleWaves;
    if (count_ties) {
        auto slab_done = [&](int i, unsigned n) {
            for (int by = 32; by > 0; by >>= 1) n += (unsigned)__shfl_xor((int)n, by);
            if (l == 0) lds.ties[i * kSampleWaves + wave] = n;
        };
        unsigned n = 0;
        each([&](unsigned key, int i, int e) {
            n = (e == 0 ? 0 : n) + (key == cut ? 1 : 0);
            if (e == 7) slab_done(i, n);
        });
        __syncthreads();
        if (wave == 0) {
            const int per = (entries + 63) / 64;
            u64 mine = 0;
            for (int i = 0; i < per; ++i)
                if (l * per + i < entries) mine += lds.ties[l * per + i];
            u64 cum = wave_scan(mine) - mine;
            for (int i = 0; i < per; ++i)
                if (l * per + i < entries) {
                    const unsigned n_here = lds.ties[l * per + i];
                    lds.ties[l * per + i] = (unsigned)cum;
                    cum += n_here;
                }
        }
        __syncthreads();
    }
    // masses of what stays, by slab and wavefront
    unsigned before_ties = 0;
    auto kept = [&](unsigned key, int i, int e, unsigned own_ties) -> u64 {
        // own_ties: this lane's tokens of the cut's key in this slab
        if (e == 0 && count_ties) {
            u64 n = own_ties;
            before_ties = lds.ties[i * kSampleWaves + wave] + (unsigned)(wave_scan(n) - n);
        }
        if (key < cut || key <= kKeyMinusInf) return 0;
        if (count_ties && key == cut && (u64)before_ties++ >= cut_count) return 0;
        const u64 w = mass(key);
        return w >= least ? w : 0;
    };
    auto slab_mass = [&](const v4u &v, int i, u64 (&w)[8]) {
        unsigned ties = 0;
        if (count_ties)
#pragma unroll
            for (int e = 0; e < 8; ++e) ties += key_of(v[e >> 1] >> (16 * (e & 1)) & 0xffffu) == cut ? 1 : 0;
        u64 sum = 0;
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            w[e] = kept(key_of(v[e >> 1] >> (16 * (e & 1)) & 0xffffu), i, e, ties);
            sum += w[e];
        }
        return sum;
    };
    u64 w[8];
    auto total_of = [&](const v4u &v, int i) {
        const u64 sum = wave_scan(slab_mass(v, i, w));
        if (l == 63) lds.table[i * kSampleWaves + wave] = sum;
    };
    if constexpr (PIECES > 0) {
#pragma unroll
        for (int i = 0; i < PIECES; ++i) total_of(held[i], i);
    } else {
        for (int i = 0; i < slabs; ++i) total_of(load(i), i);
    }
    __syncthreads();
    if (wave == 0) {
        u64 all = 0;
        for (int i = l; i < entries; i += 64) all += lds.table[i];
        all = wave_scan(all);
        all = (u64)__shfl((long long)all, 63);
        const float u = a.uniform[b];
        u64 target = u > 0.f ? (u64)((double)fminf(u, 1.f) * (double)all) : 0;
        target = min(target, all - 1) + 1;
        u64 before;
        const int at = first_reaching(lds.table, entries, target, before);
        if (l == 0) {
            lds.found = at;
            lds.before = target - before;
            lds.cut_total = all;
        }
    }
    __syncthreads();
    const int slab = lds.found / kSampleWaves;
    if (wave != lds.found % kSampleWaves) return;
    const u64 sum = slab_mass(load(slab), slab, w);
    const u64 cum = wave_scan(sum), target = lds.before;
    const u64 reached = __ballot(cum >= target);
    if (l != __builtin_ctzll(reached)) return;
    u64 at = cum - sum;
    int e = 0;
    for (; e < 7 && at + w[e] < target; ++e) at += w[e];
    u64 chosen = 0;
#pragma unroll
    for (int i = 0; i < 8; ++i) chosen = i == e ? w[i] : chosen;
    a.token[b] = (slab * kSampleT + t) * 8 + e;
    if (a.prob) a.prob[b] = (float)((double)chosen / (double)lds.cut_total);
}

sqap_status launch_sample(const __half *logits, int64_t ld, int batch, int vocab, const float *temperature, const int32_t *top_k,
                          const float *top_p, const float *min_p, const float *uniform, int32_t *token, float *prob, hipStream_t st)
{
    const SampleArgs a = {logits, ld, vocab, temperature, top_p, min_p, uniform, top_k, token, prob};
    static std::atomic<bool> ready[kMaxDeviceSlots];
    const int pieces = (vocab + 8 * kSampleT - 1) / (8 * kSampleT);
    if (!ready[device_slot()].load(std::memory_order_relaxed)) {
        for (const void *f : {reinterpret_cast<const void *>(sample_kernel<1>), reinterpret_cast<const void *>(sample_kernel<4>), reinterpret_cast<const void *>(sample_kernel<0>)})
            SQAP_HIP_CHECK(hipFuncSetAttribute(f, hipFuncAttributeMaxDynamicSharedMemorySize, sizeof(SampleLds)));
        ready[device_slot()].store(true, std::memory_order_relaxed);
    }
    const dim3 grid(batch), block(kSampleT);
    if (pieces <= 1) hipLaunchKernelGGL(sample_kernel<1>, grid, block, sizeof(SampleLds), st, a);
    else if (pieces <= 4) hipLaunchKernelGGL(sample_kernel<4>, grid, block, sizeof(SampleLds), st, a);
    else hipLaunchKernelGGL(sample_kernel<0>, grid, block, sizeof(SampleLds), st, a);
    SQAP_HIP_CHECK(hipGetLastError());
    return SQAP_OK;
}

}  // namespace sqap
