// A key/value cache held in 8 bits, and attention over it.
//
// 64 positions of a key head are a block: codes in -127 .. 127 with one binary32 scale for its keys and one for its values.  A block gets
// its codes once, when its last row arrives; until then its rows stay as they are, in half precision (`tail`), so that what the cache
// holds does not depend on how many rows came with a call, and no code is rounded twice.
// Codes are exact as halves (integers below 2^11), and so are their products with halves in binary32: attention runs on the half
// precision matrix instructions with the scales outside (the keys' on the scores, the values' on the probabilities).
//
// Codes lie in the order in which the lanes of a 16x16x32 matrix instruction hold them (lane l: row r = l % 16, group g = l / 16):
//   keys    [4 tiles of 16 positions][d / 64][lane][16]   position 16 T + r, columns 64 c + 16 g + 0 .. 15
//   values  [d / 16][lane][16]                            column 16 t + r; byte 8 s + 4 q + i: position 32 s + 16 q + 4 g + i
// The values' order of positions is that of the lanes' scores, so that probabilities enter the second product where they were computed.
#include <algorithm>

#include "common.h"
#include "decode_attn.h"

namespace sqap {

typedef _Float16 v8h __attribute__((ext_vector_type(8)));
typedef _Float16 v4h __attribute__((ext_vector_type(4)));
typedef _Float16 v2h __attribute__((ext_vector_type(2)));
typedef float v4f __attribute__((ext_vector_type(4)));
typedef float v16f __attribute__((ext_vector_type(16)));
typedef int v4i __attribute__((ext_vector_type(4)));
typedef unsigned v2u __attribute__((ext_vector_type(2)));
typedef unsigned long long u64;

constexpr int kBlock = kCache8Block;
constexpr float kLog2e = 1.4426950408889634f;

// ---------------------------------------------------------------- pieces

template <int D>
__device__ __forceinline__ int8_t *block_codes(const Cache8View &c, int64_t head, int block, int values)
{
    return c.codes + ((head * c.blocks + block) * 2 + values) * (kBlock * D);
}

// Four codes as halves: the byte with its sign flipped behind 0x64 is 1024 + (code + 128), from which 1152 is taken.
__device__ __forceinline__ v4h halves_of(int w)
{
    const unsigned u = (unsigned)w ^ 0x80808080u;
    union { unsigned u[2]; v2h h[2]; } x;
    x.u[0] = __builtin_amdgcn_perm(0x64646464u, u, 0x04010400u);
    x.u[1] = __builtin_amdgcn_perm(0x64646464u, u, 0x04030402u);
    const v2h bias = {(_Float16)1152.f, (_Float16)1152.f};
    const v2h a = x.h[0] - bias, b = x.h[1] - bias;
    return v4h{a[0], a[1], b[0], b[1]};
}
__device__ __forceinline__ v8h halves_of(int lo, int hi)
{
    const v4h a = halves_of(lo), b = halves_of(hi);
    return v8h{a[0], a[1], a[2], a[3], b[0], b[1], b[2], b[3]};
}

// The code of x: 127 x / amax to the nearest, halfway cases to even.  127 x is exact; the quotient with its remainder put right is exact
// wherever it is representable, as every halfway case is, and a quotient that is not halfway is 2^-12 or more away from that.
struct Steps {
    float amax, reciprocal;
};
__device__ __forceinline__ Steps steps_of(float amax) { return {amax, amax > 0.f ? 1.0f / amax : 0.f}; }
__device__ __forceinline__ int code_of(float x, const Steps &s)
{
    const float n = 127.0f * x, q = n * s.reciprocal;
    return (int)rintf(fmaf(fmaf(-q, s.amax, n), s.reciprocal, q));
}
// largest magnitude of a half, as its bits: infinities and NaN are above all numbers
__device__ __forceinline__ unsigned magnitude(__half h) { return __half_as_ushort(h) & 0x7fffu; }
__device__ __forceinline__ bool finite_bits(unsigned m) { return m < 0x7c00u; }
__device__ __forceinline__ float scale_of(unsigned m) { return finite_bits(m) ? __half2float(__ushort_as_half((unsigned short)m)) / 127.0f : NAN; }

__device__ __forceinline__ unsigned wavefront_umax(unsigned v)
{
    v = max(v, dpp_move<kDppXor1>(v));
    v = max(v, dpp_move<kDppXor2>(v));
    v = max(v, dpp_move<kDppHalfMirror>(v));
    v = max(v, dpp_move<kDppMirror>(v));
    return max(max((unsigned)__builtin_amdgcn_readlane((int)v, 0), (unsigned)__builtin_amdgcn_readlane((int)v, 16)),
               max((unsigned)__builtin_amdgcn_readlane((int)v, 32), (unsigned)__builtin_amdgcn_readlane((int)v, 48)));
}

// half-split rotation of one pair, as rope_kernel does it
__device__ __forceinline__ void rotate_pair(__half lo, __half hi, double cs, double sn, __half &out_lo, __half &out_hi)
{
    const double a = (double)__half2float(lo), b = (double)__half2float(hi);
    out_lo = __float2half_rn((float)(a * cs - b * sn));
    out_hi = __float2half_rn((float)(b * cs + a * sn));
}

// Sine and cosine of an angle below some 2^50, in binary64: the nearest multiple of pi / 2 is taken off in two parts of 53 bits (each
// product exact inside its multiply-add), what is left is at most pi / 4, where the Taylor series to the 15th and 16th power are off by
// less than half a unit of the last place of the larger one.  Without branches, so that a thread's pairs run side by side: a quarter of the
// instructions of the library's, which also serves angles beyond.
__constant__ const double kSeries[15] = {-1.0 / 1307674368000.0, 1.0 / 20922789888000.0, 1.0 / 6227020800.0, -1.0 / 87178291200.0, -1.0 / 39916800.0,
                                         1.0 / 479001600.0, 1.0 / 362880.0, -1.0 / 3628800.0, -1.0 / 5040.0, 1.0 / 40320.0, 1.0 / 120.0,
                                         -1.0 / 720.0, -1.0 / 6.0, 1.0 / 24.0, -0.5};
__device__ __forceinline__ void sincos_of(double a, double &sn, double &cs)
{
    const double n = rint(a * 0.63661977236758134308);
    double r = fma(-n, 1.5707963267948965580, a);
    r = fma(-n, 6.1232339957367658860e-17, r);
    const double z = r * r;
    double s = kSeries[0], c = kSeries[1];
#pragma unroll
    for (int i = 2; i < 14; i += 2) {
        s = fma(s, z, kSeries[i]);
        c = fma(c, z, kSeries[i + 1]);
    }
    c = fma(c, z, kSeries[14]);
    s = fma(s * z, r, r);
    c = fma(c, z, 1.0);
    const int q = (int)fma(-4.0, floor(0.25 * n), n);                 // (n itself may be beyond an integer)
    const double x = q & 1 ? c : s, y = q & 1 ? s : c;
    sn = q & 2 ? -x : x;
    cs = (q + 1) & 2 ? -y : y;
}

// Where a sequence's new rows lie: [row, row + n) of the fused rows, or nothing (n = 0) where the arrays do not describe one.
struct Span {
    int row, n, past;
    bool fits;                  // in the cache
};
__device__ __forceinline__ Span span_of(const int32_t *starts, const int32_t *past, int b, int rows, int max_new, int capacity)
{
    Span s = {starts[b], 0, past[b], false};
    const int end = starts[b + 1];
    if (s.past >= 0 && s.row >= 0 && end >= s.row && end <= rows) s.n = end - s.row;
    s.fits = s.n > 0 && s.n <= max_new && s.past <= capacity - s.n;
    return s;
}

// ---------------------------------------------------------------- append

// Where the code of column x and place `at` (of 64) lies in the values' half of a block; in LDS the four 16-byte pieces of a column are moved
// round by its column's eights, so that the threads of a row, 8 columns apart, write to different banks.
__device__ __forceinline__ int value_at(int s) { return ((s >> 2) & 3) << 4 | (s >> 5) << 3 | ((s >> 4) & 1) << 2 | (s & 3); }
__device__ __forceinline__ int value_byte(int x, int at) { return x * 64 + ((at >> 4) + (x >> 3) & 3) * 16 + (at & 15); }
__device__ __forceinline__ int value_piece(int u) { const int x = (u >> 6) * 16 + (u & 15); return x * 64 + (((u >> 4) & 3) + (x >> 3) & 3) * 16; }

constexpr int kAppendGroups = 512, kAppendSplit = 96, kAppendValues = 256;
// One workgroup per sequence, `share` key heads and block that the new rows touch (the first and the last of them together: the one reads
// the tail that the other writes).  The block's angles are evaluated once, into LDS.  Then, head by head: keys, D / 16 threads per position with 8
// pairs of columns (i, i + D / 2) each; the same threads turn the query heads that share the key head, and take the value row, whose codes
// pass through LDS to their order.
template <int D>
__global__ __launch_bounds__(4 * D, 2) void cache8_append_kernel(const __half *__restrict__ QKV, int64_t ld, const int32_t *__restrict__ starts,
                                                                 const int32_t *__restrict__ pos, const int32_t *__restrict__ past, int rows, int max_new,
                                                                 int H, int share, int split, const Cache8View cache, __half *__restrict__ Q_out, int64_t ldq,
                                                                 const RopeFreq freq)
{
    constexpr int P = 8, HALF = D / 2, SUBS = HALF / P, T = 4 * D, WAVES = T / 64;
    extern __shared__ __attribute__((aligned(16))) uint8_t lds[];
    double2 *angles = reinterpret_cast<double2 *>(lds);               // [64][HALF], pair i of a position at i ^ (i / 8) % 8: no two lanes on one bank
    int8_t *turned = reinterpret_cast<int8_t *>(angles + kBlock * HALF);          // the values' codes, 64 D
    unsigned *tops = reinterpret_cast<unsigned *>(turned + kBlock * D);           // [2][keys, values][WAVES]
    const int b = blockIdx.z, t = threadIdx.x, wave = t >> 6;
    const Span sp = span_of(starts, past, b, rows, max_new, cache.blocks * kBlock);
    if (!sp.fits) return;
    const int end = sp.past + sp.n, first = sp.past / kBlock, last = (end - 1) / kBlock, G = H / cache.kv_heads;
    // what this workgroup does of its heads: 1 keys, 2 values, 4 queries; one of three alone, values or the others, or all
    const int groups = (cache.kv_heads + share - 1) / share, group = blockIdx.y % groups, role = blockIdx.y / groups, does = split == 3 ? 1 << role : split == 2 ? 5 - 3 * role : 7;
    const int head0 = group * share, heads = min(share, cache.kv_heads - head0);
    int block = first + (int)blockIdx.x;
    const bool keys = does & 1, values = does & 2, queries = Q_out && (does & 4);
    const bool joined = (keys || values) && sp.past % kBlock != 0 && last > first;       // the tail is read by the first block and written by the last
    if (block > last || (joined && blockIdx.x > 0 && block == last)) return;
    if (!keys && !values && !queries) return;
    struct Row {
        v4i lo, hi;                                                   // eight halves each
    };
    const int slot = t / SUBS, sub = t % SUBS;
    auto load_row = [&](const __half *from, Row &x) {                 // columns 8 sub .. and HALF + 8 sub ..
        x.lo = *reinterpret_cast<const v4i *>(from + sub * P);
        x.hi = *reinterpret_cast<const v4i *>(from + HALF + sub * P);
    };
    auto store_row = [&](__half *to, const Row &x) {
        *reinterpret_cast<v4i *>(to + sub * P) = x.lo;
        *reinterpret_cast<v4i *>(to + HALF + sub * P) = x.hi;
    };
    auto half_at = [](const v4i &x, int i) { return __ushort_as_half((unsigned short)((unsigned)x[i >> 1] >> (16 * (i & 1)))); };
    auto turn_row = [&](Row &x) {
#pragma unroll
        for (int w = 0; w < 4; ++w) {
            unsigned lo = 0, hi = 0;
#pragma unroll
            for (int e = 0; e < 2; ++e) {
                const double2 a = angles[slot * HALF + ((sub * P + 2 * w + e) ^ sub)];
                __half y, z;
                rotate_pair(half_at(x.lo, 2 * w + e), half_at(x.hi, 2 * w + e), a.x, a.y, y, z);
                lo |= (unsigned)__half_as_ushort(y) << (16 * e);
                hi |= (unsigned)__half_as_ushort(z) << (16 * e);
            }
            x.lo[w] = (int)lo;
            x.hi[w] = (int)hi;
            __builtin_amdgcn_sched_barrier(0);                        // two pairs side by side: eight would need another wavefront's registers
        }
    };
    for (int turn = 0;; ++turn) {
        const bool full = (block + 1) * kBlock <= end;
        const int p = block * kBlock + slot;
        const bool is_new = p >= sp.past && p < end;
        const int at = sp.row + (is_new ? p - sp.past : 0);
        const __half *row = QKV + (int64_t)at * ld;
        if (turn > 0) __syncthreads();                                // (the angles of the first block have been read)
        auto fetch_rows = [&](int h, Row &key, Row &value, Row &query) {
            const int64_t tail = ((int64_t)b * cache.kv_heads + h) * 2 * kBlock * D + slot * D;
            if (keys) load_row(is_new ? row + (int64_t)(H + h) * D : cache.tail + tail, key);        // (an absent row is read and dropped)
            if (values) load_row(is_new ? row + (int64_t)(H + cache.kv_heads + h) * D : cache.tail + tail + kBlock * D, value);
            if (queries && is_new) load_row(row + (int64_t)h * G * D, query);
        };
        Row key = {v4i{0, 0, 0, 0}, v4i{0, 0, 0, 0}}, value = key, query = key;
        fetch_rows(head0, key, value, query);                         // (before the angles are worked out)
        if (keys || queries) {
            constexpr int EACH = kBlock * HALF / T, STEP = T / HALF;  // positions of a thread, STEP apart, all with one frequency
            const int i = t % HALF, s0 = t / HALF;
            const double f = freq.f[i];
            int at_pos[EACH];
#pragma unroll
            for (int k = 0; k < EACH; ++k) {
                const int q = block * kBlock + s0 + k * STEP - sp.past;
                at_pos[k] = pos[sp.row + min(max(q, 0), sp.n - 1)];
            }
#pragma unroll 2
            for (int k = 0; k < EACH; ++k) {
                const int s = s0 + k * STEP;
                double2 a;
                sincos_of((double)at_pos[k] * f, a.y, a.x);
                angles[s * HALF + (i ^ ((i >> 3) & 7))] = a;
            }
        }
        for (int hh = 0; hh < heads; ++hh) {
            const int h = head0 + hh;
            const int64_t head = (int64_t)b * cache.kv_heads + h;
            __half *tail_k = cache.tail + head * 2 * kBlock * D, *tail_v = tail_k + kBlock * D;
            if (hh > 0) fetch_rows(h, key, value, query);
            const bool turns = queries && is_new;
            if (hh == 0) __syncthreads();                             // the angles are there
            if (is_new) {
                if (keys) turn_row(key);
                if (turns) {
                    __half *to = Q_out + (int64_t)at * ldq + (int64_t)h * G * D;
                    for (int j = 0; j < G; ++j) {
                        Row next = query;
                        if (j + 1 < G) load_row(row + (int64_t)(h * G + j + 1) * D, next);
                        turn_row(query);
                        store_row(to + (int64_t)j * D, query);
                        query = next;
                    }
                }
            }
            if (!keys && !values) continue;
            unsigned top_k = 0, top_v = 0;
            if (full) {
#pragma unroll
                for (int i = 0; i < P; ++i) top_k = max(top_k, max(magnitude(half_at(key.lo, i)), magnitude(half_at(key.hi, i))));
#pragma unroll
                for (int i = 0; i < P; ++i) top_v = max(top_v, max(magnitude(half_at(value.lo, i)), magnitude(half_at(value.hi, i))));
                top_k = wavefront_umax(top_k);
                top_v = wavefront_umax(top_v);
                if ((t & 63) == 0) {
                    tops[(hh & 1) * 2 * WAVES + wave] = top_k;
                    tops[(hh & 1) * 2 * WAVES + WAVES + wave] = top_v;
                }
            }
            __syncthreads();                                          // (and nobody reads this head's tail any more)
            if (full) {
#pragma unroll
                for (int w = 0; w < WAVES; ++w) {
                    top_k = max(top_k, tops[(hh & 1) * 2 * WAVES + w]);
                    top_v = max(top_v, tops[(hh & 1) * 2 * WAVES + WAVES + w]);
                }
                const bool ok_k = finite_bits(top_k), ok_v = finite_bits(top_v);
                const Steps sk = steps_of(__half2float(__ushort_as_half((unsigned short)top_k))), sv = steps_of(__half2float(__ushort_as_half((unsigned short)top_v)));
                int8_t *kc = block_codes<D>(cache, head, block, 0), *vc = block_codes<D>(cache, head, block, 1);
                auto store = [&](int column, const v4i &x) {          // half a piece of 16 columns
                    unsigned w[2] = {0u, 0u};
#pragma unroll
                    for (int i = 0; i < 8; ++i) w[i >> 2] |= (unsigned)(ok_k ? code_of(__half2float(half_at(x, i)), sk) & 255 : 0) << (8 * (i & 3));
                    int8_t *to = kc + ((((slot >> 4) * (D / 64) + (column >> 6)) * 64 + ((column >> 4) & 3) * 16 + (slot & 15)) * 16 + (column & 15));
                    *reinterpret_cast<v2u *>(to) = v2u{w[0], w[1]};
                };
                if (keys) {
                    store(sub * P, key.lo);
                    store(HALF + sub * P, key.hi);
                    if (t == 0) cache.scales[(head * cache.blocks + block) * 2] = scale_of(top_k);
                }
                if (!values) continue;
                // values: a byte for each of this thread's columns to its place in the block, then whole pieces out
#pragma unroll
                for (int i = 0; i < P; ++i) {
                    const int x = sub * P + i, at_slot = value_at(slot);
                    turned[value_byte(x, at_slot)] = (int8_t)(ok_v ? code_of(__half2float(half_at(value.lo, i)), sv) : 0);
                    turned[value_byte(HALF + x, at_slot)] = (int8_t)(ok_v ? code_of(__half2float(half_at(value.hi, i)), sv) : 0);
                }
                __syncthreads();
                if (t < kBlock * D / 16) reinterpret_cast<v4i *>(vc)[t] = *reinterpret_cast<const v4i *>(turned + value_piece(t));
                if (t == 0) cache.scales[(head * cache.blocks + block) * 2 + 1] = scale_of(top_v);
            } else if (is_new) {
                if (keys) store_row(tail_k + slot * D, key);
                if (values) store_row(tail_v + slot * D, value);
            }
        }
        if (!joined || blockIdx.x > 0 || block == last) return;
        block = last;
    }
}

// ---------------------------------------------------------------- reading back

template <int D>
__global__ __launch_bounds__(256) void cache8_read_kernel(const Cache8View cache, const int32_t *__restrict__ lengths, int first, int count, int from,
                                                          __half *__restrict__ out, int64_t ld)
{
    // One workgroup per position (of those from the from-th on); a thread per two columns of a head, whose codes it gathers byte by byte.  A call to
    // look at a cache, not one of a step: 1500 positions of 32 heads of 128 24 us, 100003 of 8 heads 323 (1.9 TB/s of codes and halves).
    const int j = from + (int)blockIdx.x, b = blockIdx.y, p = first + j, n = lengths[b];
    __half *row = out + ((int64_t)b * count + j) * ld;
    for (int u = threadIdx.x; u < cache.kv_heads * D; u += 256) {
        const int which = u >= cache.kv_heads * D / 2, w = (u - which * (cache.kv_heads * D / 2)) * 2, h = w / D, c = w % D;
        const int64_t head = (int64_t)b * cache.kv_heads + h;
        __half v[2] = {__half(0.f), __half(0.f)};
        if (p < n && n <= cache.blocks * kBlock) {
            const int s = p % kBlock, block = p / kBlock;
            if (block == n / kBlock) {
                const __half *from = cache.tail + ((head * 2 + which) * kBlock + s) * D + c;
                v[0] = from[0];
                v[1] = from[1];
            } else {
                const float scale = cache.scales[(head * cache.blocks + block) * 2 + which];
                const int8_t *codes = block_codes<D>(cache, head, block, which);
#pragma unroll
                for (int e = 0; e < 2; ++e) {
                    const int x = c + e;
                    const int at = which ? ((x >> 4) * 64 + ((s >> 2) & 3) * 16 + (x & 15)) * 16 + (s >> 5) * 8 + ((s >> 4) & 1) * 4 + (s & 3)
                                         : (((s >> 4) * (D / 64) + (x >> 6)) * 64 + ((x >> 4) & 3) * 16 + (s & 15)) * 16 + (x & 15);
                    v[e] = __float2half_rn((float)codes[at] * scale);
                }
            }
        }
        __half *to = row + (int64_t)which * cache.kv_heads * D + w;
        to[0] = v[0];
        to[1] = v[1];
    }
}

// ---------------------------------------------------------------- attention of many rows

// What both attentions keep of the values' scales: sums of values are held in units of `unit`, the scale of the block that last changed
// it.  A block whose scale is above it or below 2^-8 of it makes the sums change units; others enter through their probabilities,
// which then stay in the range that a half resolves.
struct Unit {
    float unit = 0.f;
    // factor for the block's probabilities; `change` is what the sums so far have to be multiplied with (1: nothing)
    __device__ __forceinline__ float enter(float scale, float &change)
    {
        change = 1.f;
        if (!(scale > 0.f)) return 1.f;                               // no values but zeros, or NaN: the sums stay as they are
        if (scale > unit || scale < unit * 0.00390625f) {
            change = unit / scale;
            unit = scale;
        }
        return scale * __builtin_amdgcn_rcpf(unit);                   // (a unit of the last place or two: as much as any of the sums' roundings)
    }
};

// The maximum is the rounded product of a score and the keys' scale, the scores that are taken from it enter by a multiply-add, unrounded, which
// also takes in the maximum and the probabilities' factor as one number.  From here on (in units of ln 2) either rounding could be worth more than a
// probability has room for: the scores are rounded as well, and the maximum is taken from them before anything else.
constexpr float kLargeScore = 1048576.f;
// The maximum lags behind by up to this: with 32 rows to a wavefront some row has a new one in most blocks, and the sums are 64 registers.
constexpr float kRaiseBy = 6.f;
// Probabilities (and so all sums of them) are 2^9 times as large: below 2^15 with the lag, and what is below the smallest half is below 2^-33 of
// the largest, so that many of them together are not missing from the sums of values that they are divided out of.
constexpr float kLift = 9.f;
// A probability enters the second product as the sum of two halves, which together hold it to 2^-22 of itself: what one half leaves out (2.0e-4 of
// the outputs' norm) is as much as the rounding of the outputs.
__device__ __forceinline__ void two_halves(float a, float b, v2h &high, v2h &low)
{
    high = v2h{(_Float16)a, (_Float16)b};
    low = v2h{(_Float16)remainder_of<0>(high, a), (_Float16)remainder_of<1>(high, b)};
}

// NaN for workgroup `number`'s rows of a sequence that does not fit: of as many tiles as there are of its longest
template <int D>
__device__ __forceinline__ void nan_rows(__half *O, int64_t ldo, int first, int64_t n_rows, int G, int kh, int number, int tiles, int per_tile)
{
    for (int64_t tile = (int64_t)number * per_tile; tile < n_rows; tile += (int64_t)tiles * per_tile)
        for (int u = threadIdx.x; u < per_tile * D; u += blockDim.x) {
            const int64_t row = tile + u / D;
            if (row < n_rows) O[(first + row / G) * ldo + (kh * G + row % G) * D + u % D] = __ushort_as_half(0x7e00);
        }
}

// Rows are (query, head) pairs of the heads that share a key head, query first, 32 to a wavefront and WAVES wavefronts to a workgroup, so
// that a block of keys and values is taken from memory and made halves once for all of them.  Everything is transposed (scores:
// positions x rows), as in attention.hip: probabilities are the second product's operand where they were computed.
// What bounds it is the vector ALU beside the matrix cores, 355 instructions to 48 matrix instructions per wavefront and block, a tenth of them
// exponentials: 1500, 1115 and 1446 rows of 32 heads over 8 behind 2000, 1994 and 420 positions in some 270 us, 0.52 PFLOP/s (a library product of
// halves reaches 1.24); with probabilities of one half, 32 matrix instructions and 305 others, it was 230, and the outputs 2.0e-4 of their norm
// further off.  (Then the next block's scores multiplied between this one's probabilities, in the same wavefront: 335 us, the registers do not suffice.)
// A block's p = 2^(s - m) times its factor is one exponential, of s sk + (log2 factor - m); the sum of the probabilities is put right by the
// factor once per block.  The hardware's exponential, logarithm and reciprocal are off by a unit of the last place of binary32 or so each, which is
// less than the rounding of the scores and of the sums.
template <int D, int WAVES>
__global__ __launch_bounds__(64 * WAVES, 2) void cache8_attention_kernel(const __half *__restrict__ Q, int64_t ldq, const int32_t *__restrict__ starts,
                                                                         const int32_t *__restrict__ past, int rows, int max_new, int H,
                                                                         const Cache8View cache, __half *__restrict__ O, int64_t ldo, int tiles)
{
    constexpr int T = 64 * WAVES, TILE = 32 * WAVES, NP = D / 16, CT = D / 32, BUF = 2 * kBlock * D * 2, COUNT = kBlock * D / 16;
    constexpr int PIECES = (COUNT + T - 1) / T;
    extern __shared__ __attribute__((aligned(16))) uint8_t lds[];     // two buffers: keys [2][NP] KiB, values [CT][4] KiB
    __shared__ int not_finite;
    // a key head's tiles behind one L2 (workgroup b runs on XCD b % 8) where the heads fill all of them; the longest first
    const int pairs = cache.kv_heads * cache.batch, id = blockIdx.x;
    int pair, number;
    if (pairs % 8 == 0) {
        pair = (id & 7) + 8 * ((id >> 3) % (pairs / 8));
        number = (id >> 3) / (pairs / 8);
    } else {
        pair = id % pairs;
        number = id / pairs;
    }
    const int b = pair / cache.kv_heads, kh = pair % cache.kv_heads;
    const int t = threadIdx.x, l = t & 63, wave = t >> 6, c = l & 31, h = l >> 5;
    const Span sp = span_of(starts, past, b, rows, max_new, cache.blocks * kBlock);
    const int G = H / cache.kv_heads;
    if (!sp.fits) {                                                   // (of more than max_new rows too: all of them)
        nan_rows<D>(O, ldo, sp.row, (int64_t)sp.n * G, G, kh, number, tiles, TILE);
        return;
    }
    const int n_rows = sp.n * G, tile = (tiles - 1 - number) * TILE;  // (the launch keeps max_new * G in 32 bits)
    if (tile >= n_rows) return;
    const int mine = tile + wave * 32 + c;
    const int mine_in = min(mine, n_rows - 1);
    const int query = mine_in / G, head = kh * G + mine_in % G;
    if (t == 0) not_finite = 0;
    const int end = sp.past + sp.n, sees = sp.past + query;           // last position that this lane's row sees
    const int tile_last = sp.past + (min(tile + TILE, n_rows) - 1) / G, n_blocks = tile_last / kBlock + 1;
    const int64_t kv_head = (int64_t)b * cache.kv_heads + kh;
    const __half *tail_k = cache.tail + kv_head * 2 * kBlock * D, *tail_v = tail_k + kBlock * D;
    const float *scales = cache.scales + kv_head * cache.blocks * 2;
    const int tail_block = end / kBlock, tail_rows = end % kBlock;

    v8h qf[NP];
#pragma unroll
    for (int m = 0; m < NP; ++m)
        qf[m] = *reinterpret_cast<const v8h *>(Q + (int64_t)(sp.row + query) * ldq + (int64_t)head * D + 16 * m + 8 * h);

    v4i kraw[PIECES], vraw[PIECES];
    auto fetch = [&](int j) {
        if (j >= n_blocks || j == tail_block) return;
        const v4i *k = reinterpret_cast<const v4i *>(block_codes<D>(cache, kv_head, j, 0)), *v = reinterpret_cast<const v4i *>(block_codes<D>(cache, kv_head, j, 1));
#pragma unroll
        for (int i = 0; i < PIECES; ++i) {
            const int u = t + T * i;
            if (COUNT % T != 0 && u >= COUNT) break;
            kraw[i] = k[u];
            vraw[i] = v[u];
        }
    };
    auto keep = [&](int j) {
        if (j >= n_blocks) return;
        uint8_t *kt = lds + (j & 1) * BUF, *vt = kt + kBlock * D * 2;
        if (j != tail_block) {
#pragma unroll
            for (int i = 0; i < PIECES; ++i) {
                const int u = t + T * i, r = u & 15, g = (u >> 4) & 3, x = u >> 6;
                if (COUNT % T != 0 && u >= COUNT) break;
                // keys: piece x = (T, c): position 16 T + r, columns 64 c + 16 g ..
                const int tk = x / (D / 64), m = (x % (D / 64)) * 4 + g, row = 16 * (tk & 1) + r;
                uint8_t *to = kt + (((tk >> 1) * NP + m) * 64 + row) * 16;
                *reinterpret_cast<v8h *>(to) = halves_of(kraw[i][0], kraw[i][1]);
                *reinterpret_cast<v8h *>(to + 512) = halves_of(kraw[i][2], kraw[i][3]);
                // values: piece x: column 16 x + r, four positions per word
                const int col = 16 * x + r;
                uint8_t *vo = vt + ((col >> 5) * 4 * 64 + (g & 1) * 32 + (col & 31)) * 16 + (g >> 1) * 8;
#pragma unroll
                for (int n = 0; n < 4; ++n) *reinterpret_cast<v4h *>(vo + n * 1024) = halves_of(vraw[i][n]);
            }
            return;
        }
        bool odd = false;
        for (int u = t; u < kBlock * D / 8; u += T) {
            const int s = u / (D / 8), x = (u % (D / 8)) * 8;
            v8h k = {}, v = {};
            if (s < tail_rows) {
                k = *reinterpret_cast<const v8h *>(tail_k + s * D + x);
                v = *reinterpret_cast<const v8h *>(tail_v + s * D + x);
            }
            *reinterpret_cast<v8h *>(kt + (((s >> 5) * NP + (x >> 4)) * 64 + ((x >> 3) & 1) * 32 + (s & 31)) * 16) = k;
            const int n = s >> 4, o = s & 15;                         // 8 q + 4 h + i of its sixteen positions
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                const int col = x + e;
                _Float16 w = v[e];
                if (!(__builtin_fabsf((float)w) <= 65504.f)) {        // comes back at the end, to the rows that see it
                    w = (_Float16)0.f;
                    odd = true;
                }
                *reinterpret_cast<_Float16 *>(vt + (((col >> 5) * 4 + n) * 64 + ((o >> 2) & 1) * 32 + (col & 31)) * 16 + (o >> 3) * 8 + (o & 3) * 2) = w;
            }
        }
        if (odd) not_finite = 1;
    };

    v16f ot[CT];
#pragma unroll
    for (int ct = 0; ct < CT; ++ct)
#pragma unroll
        for (int i = 0; i < 16; ++i) ot[ct][i] = 0.f;
    float mrun = -INFINITY, lrun = 0.f;
    Unit unit;
    const float per_d = kLog2e / sqrtf((float)D);
    const int wave_last = sp.past + min(tile + wave * 32 + 31, n_rows - 1) / G, wave_first = sp.past + min(tile + wave * 32, n_rows - 1) / G;
    __syncthreads();
    fetch(0);
    keep(0);
    float2 sc = {0.f, 0.f};
    if (tail_block != 0) sc = *reinterpret_cast<const float2 *>(scales);
    for (int j = 0; j < n_blocks; ++j) {
        fetch(j + 1);
        // (keys that are all zeros: the scores are, times anything but zero, which would make NaN of a masked one)
        const float sk = j == tail_block || sc.x == 0.f ? per_d : sc.x * per_d, sv = j == tail_block ? 1.f : sc.y;
        if (j + 1 < n_blocks && j + 1 != tail_block) sc = *reinterpret_cast<const float2 *>(scales + 2 * (j + 1));
        lds_barrier();
        if (j * kBlock <= wave_last) {
            const uint8_t *kt = lds + (j & 1) * BUF + l * 16, *vt = kt + kBlock * D * 2;
            v16f s[2];
            __builtin_amdgcn_s_setprio(1);                            // (before the other workgroup's exponentials: 3 in 100; not for the values' products)
#pragma unroll
            for (int tt = 0; tt < 2; ++tt) {
#pragma unroll
                for (int i = 0; i < 16; ++i) s[tt][i] = 0.f;
#pragma unroll
                for (int m = 0; m < NP; ++m)
                    s[tt] = __builtin_amdgcn_mfma_f32_32x32x16_f16(*reinterpret_cast<const v8h *>(kt + (tt * NP + m) * 1024), qf[m], s[tt], 0, 0, 0);
            }
            __builtin_amdgcn_s_setprio(0);
            if ((j + 1) * kBlock - 1 > wave_first) {                  // some row does not see some position
                const int last = sees - j * kBlock - 4 * h;
#pragma unroll
                for (int tt = 0; tt < 2; ++tt)
#pragma unroll
                    for (int i = 0; i < 16; ++i)
                        if (32 * tt + 8 * (i >> 2) + (i & 3) > last) s[tt][i] = -INFINITY;
            }
            float top = -INFINITY;
#pragma unroll
            for (int tt = 0; tt < 2; ++tt)
#pragma unroll
                for (int i = 0; i < 16; ++i) top = fmaxf(top, s[tt][i]);
            top = fmaxf(top, __shfl_xor(top, 32));
            if (top > -INFINITY) top *= sk;                           // (nothing seen: it stays, whatever the scale)
            float change;
            const float factor = unit.enter(sv, change);
            if (top - mrun > kRaiseBy) {                              // (a row that sees nothing of the block keeps its maximum)
                const float raise = exp2f(mrun - top);
                change *= raise;
                lrun *= raise;
                mrun = top;
            }
            if (__any(change != 1.f)) {
#pragma unroll
                for (int ct = 0; ct < CT; ++ct)
#pragma unroll
                    for (int i = 0; i < 16; ++i) ot[ct][i] *= change;
            }
            float by = sk, from = __log2f(factor) + kLift;
            const bool bad = !(sk >= 0.f && sv >= 0.f);               // keys or values that are NaN as a whole: for the rows that see any of them
            if (bad || __any(fabsf(top) > kLargeScore && top > -INFINITY)) {        // (a masked score times NaN would be NaN, too)
#pragma unroll
                for (int tt = 0; tt < 2; ++tt)
#pragma unroll
                    for (int i = 0; i < 16; ++i) {
                        float w = bad ? NAN : s[tt][i] * sk;
                        asm volatile("" : "+v"(w));                   // (rounded)
                        s[tt][i] = s[tt][i] == -INFINITY ? -INFINITY : w - mrun;
                    }
                by = 1.f;
            } else {
                from -= mrun;
            }
            float sum = 0.f;
#pragma unroll
            for (int n = 0; n < 4; ++n) {                             // 16 positions at a time: all at once would not leave the registers
                v8h p, rest, v[CT];
#pragma unroll
                for (int i = 0; i < 8; i += 2) {
                    const float s0 = s[n >> 1][(n & 1) * 8 + i], s1 = s[n >> 1][(n & 1) * 8 + i + 1];
                    const float e0 = __builtin_amdgcn_exp2f(fmaf(s0, by, from)), e1 = __builtin_amdgcn_exp2f(fmaf(s1, by, from));
                    sum += e0;
                    sum += e1;
                    v2h high, low;
                    two_halves(e0, e1, high, low);
                    p[i] = high[0];
                    p[i + 1] = high[1];
                    rest[i] = low[0];
                    rest[i + 1] = low[1];
                }
#pragma unroll
                for (int ct = 0; ct < CT; ++ct) v[ct] = *reinterpret_cast<const v8h *>(vt + (ct * 4 + n) * 1024);
#pragma unroll
                for (int ct = 0; ct < CT; ++ct) ot[ct] = __builtin_amdgcn_mfma_f32_32x32x16_f16(v[ct], p, ot[ct], 0, 0, 0);
#pragma unroll
                for (int ct = 0; ct < CT; ++ct) ot[ct] = __builtin_amdgcn_mfma_f32_32x32x16_f16(v[ct], rest, ot[ct], 0, 0, 0);
            }
            lrun += sum * __builtin_amdgcn_rcpf(factor);
        }
        keep(j + 1);
    }
    lrun += __shfl_xor(lrun, 32);
    const float norm = unit.unit / lrun;
    const bool odd = tile_last / kBlock == tail_block && not_finite;
    if (mine >= n_rows) return;
    __half *to = O + (int64_t)(sp.row + query) * ldo + (int64_t)head * D;
#pragma unroll
    for (int ct = 0; ct < CT; ++ct)
#pragma unroll
        for (int a = 0; a < 4; ++a) {
            const int col = 32 * ct + 8 * a + 4 * h;
            union { __half h[4]; v2u v; } u;
#pragma unroll
            for (int i = 0; i < 4; ++i) u.h[i] = __float2half_rn(ot[ct][4 * a + i] * norm);
            *reinterpret_cast<v2u *>(to + col) = u.v;
        }
    if (odd) {                                                        // infinities and NaN among the tail's values that this row sees
#pragma unroll 1
        for (int x = 0; x < D / 2; ++x) {
            const int col = (x >> 2) * 8 + 4 * h + (x & 3);
            float o = __half2float(to[col]);
#pragma unroll 1
            for (int s = 0; s <= sees - tail_block * kBlock; ++s) {
                const float v = __half2float(tail_v[s * D + col]);
                if (!(fabsf(v) <= 65504.f)) o += v;
            }
            to[col] = __float2half_rn(o);
        }
    }
}

// ---------------------------------------------------------------- 16 rows and a block of their own to a wavefront

// Sums of a wavefront's blocks: row l % 16, columns 16 i + 4 (l / 16) ...
template <int D>
struct WaveSums {
    v4f o[D / 16];
    float m = -INFINITY, l = 0.f;
    Unit unit;
    __device__ __forceinline__ WaveSums()
    {
#pragma unroll
        for (int i = 0; i < D / 16; ++i) o[i] = v4f{0.f, 0.f, 0.f, 0.f};
    }
    // key(T, m), value(i, n): operands of the products; `then` runs when the keys have been used; `ends`: this lane's row sees the first
    // `sees` + 1 positions of the block only.
    template <typename Key, typename Value, typename Then>
    __device__ __forceinline__ void add(const v8h (&q)[D / 32], float sk, float sv, bool ends, int sees, Key key, Value value, Then then)
    {
        const int g = (threadIdx.x & 63) >> 4;
        v4f s[4];
#pragma unroll
        for (int T4 = 0; T4 < 4; ++T4) s[T4] = v4f{0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int T4 = 0; T4 < 4; ++T4)
#pragma unroll
            for (int m = 0; m < D / 32; ++m) s[T4] = __builtin_amdgcn_mfma_f32_16x16x32_f16(key(T4, m), q[m], s[T4], 0, 0, 0);
        const float per_d = kLog2e / sqrtf((float)D);
        sk = sk == 0.f ? per_d : sk * per_d;                          // (keys that are all zeros: as in cache8_attention_kernel)
        then();
        if (ends) {
#pragma unroll
            for (int T4 = 0; T4 < 4; ++T4)
#pragma unroll
                for (int i = 0; i < 4; ++i)
                    if (16 * T4 + 4 * g + i > sees) s[T4][i] = -INFINITY;
        }
        float top = -INFINITY;
#pragma unroll
        for (int T4 = 0; T4 < 4; ++T4)
#pragma unroll
            for (int i = 0; i < 4; ++i) top = fmaxf(top, s[T4][i]);
        top = fmaxf(top, __shfl_xor(top, 16));
        top = fmaxf(top, __shfl_xor(top, 32));
        if (top > -INFINITY) top *= sk;
        float change;
        const float factor = unit.enter(sv, change);
        if (top - m > kRaiseBy) {
            const float raise = exp2f(m - top);
            change *= raise;
            l *= raise;
            m = top;
        }
        if (__any(change != 1.f)) {
#pragma unroll
            for (int i = 0; i < D / 16; ++i) o[i] *= change;
        }
        // (no score above minus infinity so far: nothing is added, other wavefronts' blocks may have some)
        const float taken = m == -INFINITY ? 0.f : m;
        float by = sk, from = __log2f(factor) + kLift;
        const bool bad = !(sk >= 0.f && sv >= 0.f);                   // (NaN as a whole: as in cache8_attention_kernel)
        if (bad || __any(fabsf(top) > kLargeScore && top > -INFINITY)) {
#pragma unroll
            for (int T4 = 0; T4 < 4; ++T4)
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    float w = bad ? NAN : s[T4][i] * sk;
                    asm volatile("" : "+v"(w));                       // (rounded)
                    s[T4][i] = s[T4][i] == -INFINITY ? -INFINITY : w - taken;
                }
            by = 1.f;
        } else {
            from -= taken;
        }
        float sum = 0.f;
#pragma unroll
        for (int n = 0; n < 2; ++n) {
            v8h p, rest;
#pragma unroll
            for (int i = 0; i < 8; i += 2) {
                const float s0 = s[2 * n + (i >> 2)][i & 3], s1 = s[2 * n + (i >> 2)][(i & 3) + 1];
                const float e0 = __builtin_amdgcn_exp2f(fmaf(s0, by, from)), e1 = __builtin_amdgcn_exp2f(fmaf(s1, by, from));
                sum += e0;
                sum += e1;
                v2h high, low;
                two_halves(e0, e1, high, low);
                p[i] = high[0];
                p[i + 1] = high[1];
                rest[i] = low[0];
                rest[i + 1] = low[1];
            }
#pragma unroll
            for (int i = 0; i < D / 16; ++i) {
                const v8h v = value(i, n);
                o[i] = __builtin_amdgcn_mfma_f32_16x16x32_f16(v, p, o[i], 0, 0, 0);
                o[i] = __builtin_amdgcn_mfma_f32_16x16x32_f16(v, rest, o[i], 0, 0, 0);
            }
        }
        l += sum * __builtin_amdgcn_rcpf(factor);
    }
};

// slot of position s in the values' order: 8 of each 32 per lane group; and where column x has it: its eights are moved round by the column's,
// so that the threads of a row, 8 columns apart, write to different banks
__device__ __forceinline__ int value_slot(int s) { return (s & 32) | ((s >> 2) & 3) << 3 | ((s >> 4) & 1) << 2 | (s & 3); }
__device__ __forceinline__ int value_place(int x, int at) { return ((at + (x & ~7)) & 56) | (at & 7); }

// Few rows: tiles of 16 (query, head) pairs, and the blocks dealt to the workgroup's wavefronts, each of which takes keys and values to its own
// registers as the decode call does (heads of 128 take all 256 registers; an address lies in memory and is read once a block).
constexpr int kFewRowsWaves = 8;
template <int D>
struct FewRowsLds {
    __attribute__((aligned(16))) union {
        struct {
            unsigned short k[kBlock][D + 8];     // as in DecodeLds
            unsigned short v[D][kBlock + 8];
        } tail;
        float o[kFewRowsWaves][16][D + 4];
    } u;
    float m[kFewRowsWaves][16], l[kFewRowsWaves][16];
    int not_finite;
};
template <int D>
__global__ __launch_bounds__(64 * kFewRowsWaves, 2) void cache8_few_rows_kernel(const __half *__restrict__ Q, int64_t ldq, const int32_t *__restrict__ starts,
                                                                                const int32_t *__restrict__ past, int rows, int max_new, int H,
                                                                                const Cache8View cache, __half *__restrict__ O, int64_t ldo, int tiles)
{
    constexpr int C = D / 64, DT = D / 16, T = 64 * kFewRowsWaves;
    extern __shared__ __attribute__((aligned(16))) uint8_t raw_lds[];
    FewRowsLds<D> &lds = *reinterpret_cast<FewRowsLds<D> *>(raw_lds);
    const int pairs = cache.kv_heads * cache.batch, id = blockIdx.x;
    int pair, number;
    if (pairs % 8 == 0) {                                             // (as in cache8_attention_kernel)
        pair = (id & 7) + 8 * ((id >> 3) % (pairs / 8));
        number = (id >> 3) / (pairs / 8);
    } else {
        pair = id % pairs;
        number = id / pairs;
    }
    const int b = pair / cache.kv_heads, kh = pair % cache.kv_heads;
    const int t = threadIdx.x, l = t & 63, wave = __builtin_amdgcn_readfirstlane(t >> 6), r = l & 15, g = l >> 4;
    const Span sp = span_of(starts, past, b, rows, max_new, cache.blocks * kBlock);
    const int G = H / cache.kv_heads;
    if (!sp.fits) {
        nan_rows<D>(O, ldo, sp.row, (int64_t)sp.n * G, G, kh, number, tiles, 16);
        return;
    }
    const int n_rows = sp.n * G, tile = (tiles - 1 - number) * 16;
    if (tile >= n_rows) return;
    const int mine = min(tile + r, n_rows - 1), query = mine / G, first_query = tile / G;
    const int end = sp.past + sp.n, sees = sp.past + query, first_sees = sp.past + first_query;
    const int n_blocks = (sp.past + (min(tile + 16, n_rows) - 1) / G) / kBlock + 1, tail_block = end / kBlock, tail_rows = end % kBlock;
    const int64_t head = (int64_t)b * cache.kv_heads + kh;
    const __half *tail_k = cache.tail + head * 2 * kBlock * D, *tail_v = tail_k + kBlock * D;
    v4i kraw[4 * C], vraw[DT];
    float2 sc = {0.f, 0.f};
    auto fetch_keys = [&](int j) {
        if (j >= n_blocks || j == tail_block) return;
        sc = reinterpret_cast<const float2 *>(cache.scales)[head * cache.blocks + j];
        const v4i *k = reinterpret_cast<const v4i *>(block_codes<D>(cache, head, j, 0)) + l;
#pragma unroll
        for (int i = 0; i < 4 * C; ++i) kraw[i] = k[i * 64];
    };
    auto fetch_values = [&](int j) {
        if (j >= n_blocks || j == tail_block) return;
        const v4i *v = reinterpret_cast<const v4i *>(block_codes<D>(cache, head, j, 1)) + l;
#pragma unroll
        for (int i = 0; i < DT; ++i) vraw[i] = v[i * 64];
    };
    fetch_keys(wave);
    fetch_values(wave);
    v8h q[2 * C];
    const __half *from = Q + (int64_t)(sp.row + query) * ldq + (int64_t)(kh * G + mine - query * G) * D;
#pragma unroll
    for (int m = 0; m < 2 * C; ++m) q[m] = *reinterpret_cast<const v8h *>(from + 64 * (m >> 1) + 16 * g + 8 * (m & 1));
    const bool has_tail = n_blocks - 1 == tail_block;
    if (has_tail) {
        if (t == 0) lds.not_finite = 0;
        __syncthreads();
        bool odd = false;
        for (int u = t; u < kBlock * D / 8; u += T) {
            const int s = u / (D / 8), x = (u % (D / 8)) * 8, at = value_slot(s);
            v4i k = {0, 0, 0, 0}, v = k;
            if (s < tail_rows) {
                k = *reinterpret_cast<const v4i *>(tail_k + s * D + x);
                v = *reinterpret_cast<const v4i *>(tail_v + s * D + x);
            }
            *reinterpret_cast<v4i *>(&lds.u.tail.k[s][x]) = k;
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                unsigned short w = (unsigned short)((unsigned)v[e >> 1] >> (16 * (e & 1)));
                if ((w & 0x7fffu) >= 0x7c00u) w = 0, odd = true;      // comes back at the end, to the rows that see it
                lds.u.tail.v[x + e][value_place(x, at)] = w;
            }
        }
        if (odd) lds.not_finite = 1;
        __syncthreads();
    }
    WaveSums<D> sums;
    for (int j = wave; j < n_blocks; j += kFewRowsWaves) {
        const bool ends = (j + 1) * kBlock - 1 > first_sees;
        const int last = sees - j * kBlock;
        if (j != tail_block) {
            const float2 scale = sc;
            sums.add(
                q, scale.x, scale.y, ends, last,
                [&](int T4, int m) {
                    const v4i w = kraw[T4 * C + (m >> 1)];
                    return (m & 1) ? halves_of(w[2], w[3]) : halves_of(w[0], w[1]);
                },
                [&](int i, int n) { return halves_of(vraw[i][2 * n], vraw[i][2 * n + 1]); }, [&] { fetch_keys(j + kFewRowsWaves); });
            fetch_values(j + kFewRowsWaves);
        } else {
            sums.add(
                q, 1.f, 1.f, true, min(last, tail_rows - 1),
                [&](int T4, int m) { return *reinterpret_cast<const v8h *>(&lds.u.tail.k[16 * T4 + r][64 * (m >> 1) + 16 * g + 8 * (m & 1)]); },
                [&](int i, int n) { return *reinterpret_cast<const v8h *>(&lds.u.tail.v[16 * i + r][value_place(16 * i + r, 32 * n + 8 * g)]); }, [] {});
        }
    }
    sums.l += __shfl_xor(sums.l, 16);
    sums.l += __shfl_xor(sums.l, 32);
    const bool odd = has_tail && lds.not_finite;
    __syncthreads();                                                  // the tail's rows have been read
    const int waves = min(n_blocks, kFewRowsWaves);
    if (wave < waves) {
#pragma unroll
        for (int i = 0; i < DT; ++i) *reinterpret_cast<v4f *>(&lds.u.o[wave][r][16 * i + 4 * g]) = sums.o[i] * sums.unit.unit;
        if (g == 0) {
            lds.m[wave][r] = sums.m;
            lds.l[wave][r] = sums.l;
        }
    }
    __syncthreads();
    const int row = t / (D / 4), col = t % (D / 4) * 4;               // four columns of a row
    if (row >= 16 || tile + row >= n_rows) return;
    const int of = (tile + row) / G;
    float top = -INFINITY, sum = 0.f;
    for (int w = 0; w < waves; ++w) top = fmaxf(top, lds.m[w][row]);
    v4f o = {0.f, 0.f, 0.f, 0.f};
    for (int w = 0; w < waves; ++w) {
        const float f = exp2f(lds.m[w][row] - top);
        sum += f * lds.l[w][row];
        o += f * *reinterpret_cast<const v4f *>(&lds.u.o[w][row][col]);
    }
    const float norm = 1.f / sum;
    union { __half h[4]; v2u v; } out;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        float x = o[i] * norm;
        if (odd) {                                                    // infinities and NaN among the tail's values that this row sees
            x = __half2float(__float2half_rn(x));
#pragma unroll 1
            for (int s = 0; s <= sp.past + of - tail_block * kBlock; ++s) {
                const float v = __half2float(tail_v[s * D + col + i]);
                if (!(fabsf(v) <= 65504.f)) x += v;
            }
        }
        out.h[i] = __float2half_rn(x);
    }
    *reinterpret_cast<v2u *>(O + (int64_t)(sp.row + of) * ldo + (int64_t)(kh * G + tile + row - of * G) * D + col) = out.v;
}

// ---------------------------------------------------------------- attention of one row per sequence

// One workgroup per sequence, key head, up to 16 of the query heads that share it, and share of the sequence's blocks; a block is one
// wavefront's.  The workgroup whose share ends with the last block appends the new row there.  Where there are several shares, each leaves
// its sums in the workspace and the workgroup that arrives last adds them in their order.  Codes are read once, whole pieces to a lane, a block
// ahead: 100003 positions of 8 key heads in 51 us, 4.0 TB/s of the 6.0 that reading alone reaches; what is missing is the start (the new row's
// angles, the unfinished block) and the joining of 64 shares per head, which 64 positions alone show to be 7 us.
constexpr int kDecodeWaves = 4, kMaxShares = 128;
struct DecodeArgs {
    const __half *QKV;
    int64_t ld;
    const int32_t *pos, *past;
    int H, G, chunks, shares, per_share;                      // shares of the longest sequence, and its blocks in each
    Cache8View cache;
    __half *O;
    int64_t ldo;
    unsigned *counters;
    float *partials;
    RopeFreq freq;
};

template <int D>
struct DecodeLds {
    __attribute__((aligned(16))) _Float16 q[16][D];
    __attribute__((aligned(16))) union {
        struct {
            unsigned short k[kBlock][D + 8];     // rows of the last block
            unsigned short v[D][kBlock + 8];     // its values, transposed, positions in the order of the codes (value_place)
        } tail;
        float o[kDecodeWaves][16][D + 4];        // the wavefronts' sums
    } u;
    double cs[D / 2], sn[D / 2];
    __half knew[D], vnew[D];
    float m[kDecodeWaves][16], l[kDecodeWaves][16];
    unsigned top[2][kDecodeWaves];
    int odd[D];                                  // what is not finite among a column's values in the tail: 1 infinity, 2 minus infinity, 4 NaN
    int arrived;
};

template <int D>
__global__ __launch_bounds__(64 * kDecodeWaves, 2) void cache8_decode_kernel(const DecodeArgs a)
{
    constexpr int HALF = D / 2, C = D / 64, T = 64 * kDecodeWaves, DT = D / 16;
    __shared__ DecodeLds<D> lds;
    const Cache8View &cache = a.cache;
    const int share = blockIdx.x, kh = blockIdx.y / a.chunks, chunk = blockIdx.y % a.chunks, b = blockIdx.z;
    const int t = threadIdx.x, l = t & 63, wave = __builtin_amdgcn_readfirstlane(t >> 6), r = l & 15, g = l >> 4;
    const int first_head = kh * a.G + chunk * 16, heads = min(16, a.G - chunk * 16);
    const int past = a.past[b];
    if (past < 0) return;
    const __half *row = a.QKV + (int64_t)b * a.ld;
    __half *out = a.O + (int64_t)b * a.ldo + (int64_t)first_head * D;
    if (past >= cache.blocks * kBlock) {                              // no room: nothing is appended, and the outputs say so
        if (share == 0)
            for (int i = t; i < heads * D; i += T) out[i] = __ushort_as_half(0x7e00);
        return;
    }
    const int last = past / kBlock, slot = past % kBlock;
    const int per_share = max(a.per_share, (last + a.shares) / a.shares), active = (last + per_share) / per_share;
    const int begin = share * per_share, stop = min(begin + per_share, last + 1);
    if (begin > last) return;
    const bool has_last = stop == last + 1;
    const int64_t head = (int64_t)b * cache.kv_heads + kh;
    __half *tail_k = cache.tail + head * 2 * kBlock * D, *tail_v = tail_k + kBlock * D;

    // everything that does not wait for the rotation is asked for first: this wavefront's first block, the unfinished block's rows
    v4i kraw[4 * C], vraw[DT];
    auto fetch_keys = [&](int j) {
        if (j >= stop || j == last) return;
        const v4i *k = reinterpret_cast<const v4i *>(block_codes<D>(cache, head, j, 0)) + l;
#pragma unroll
        for (int i = 0; i < 4 * C; ++i) kraw[i] = k[i * 64];
    };
    auto fetch_values = [&](int j) {
        if (j >= stop || j == last) return;
        const v4i *v = reinterpret_cast<const v4i *>(block_codes<D>(cache, head, j, 1)) + l;
#pragma unroll
        for (int i = 0; i < DT; ++i) vraw[i] = v[i * 64];
    };
    const float2 *scales = reinterpret_cast<const float2 *>(cache.scales + head * cache.blocks * 2);
    float2 sc = {0.f, 0.f};
    auto fetch_scales = [&](int j) {
        if (j < stop && j != last) sc = scales[j];
    };
    __half qnew[16 * HALF / T][2];
#pragma unroll
    for (int i = 0; i < 16 * HALF / T; ++i) {
        const int u = t + i * T;
        if (u >= heads * HALF) break;
        const __half *q = row + (int64_t)(first_head + u / HALF) * D + u % HALF;
        qnew[i][0] = q[0];
        qnew[i][1] = q[HALF];
    }
    const double angle = t < HALF ? (double)a.pos[b] * a.freq.f[t] : 0.0;
    __half knew[2] = {}, vnew[2] = {};
    if (has_last && t < HALF) {
        const __half *k = row + (int64_t)(a.H + kh) * D, *v = row + (int64_t)(a.H + cache.kv_heads + kh) * D;
        knew[0] = k[t], knew[1] = k[t + HALF];
        vnew[0] = v[t], vnew[1] = v[t + HALF];
    }
    constexpr int UNITS = kBlock * D / 8 / T;                         // 8 columns of a row of the tail each
    v4i tk[UNITS], tv[UNITS];
    if (has_last) {
#pragma unroll
        for (int i = 0; i < UNITS; ++i) {
            const int u = t + i * T, s = u / (D / 8), x = (u % (D / 8)) * 8;
            tk[i] = tv[i] = v4i{0, 0, 0, 0};
            if (s < slot) {
                tk[i] = *reinterpret_cast<const v4i *>(tail_k + s * D + x);
                tv[i] = *reinterpret_cast<const v4i *>(tail_v + s * D + x);
            }
        }
    }
    fetch_scales(begin + wave);
    fetch_keys(begin + wave);
    fetch_values(begin + wave);

    if (t < HALF) sincos_of(angle, lds.sn[t], lds.cs[t]);
    if (t < D) lds.odd[t] = 0;
    __syncthreads();
#pragma unroll
    for (int k = 0; k < 16 * HALF / T; ++k) {
        const int u = t + k * T, j = u / HALF, i = u % HALF;
        if (u >= heads * HALF) break;
        __half x, y;
        rotate_pair(qnew[k][0], qnew[k][1], lds.cs[i], lds.sn[i], x, y);
        lds.q[j][i] = (_Float16)__half2float(x);
        lds.q[j][i + HALF] = (_Float16)__half2float(y);
    }
    if (has_last && t < HALF) {
        rotate_pair(knew[0], knew[1], lds.cs[t], lds.sn[t], lds.knew[t], lds.knew[t + HALF]);
        lds.vnew[t] = vnew[0];
        lds.vnew[t + HALF] = vnew[1];
    }
    __syncthreads();
    float tail_sk = 1.f, tail_sv = 1.f;
    if (has_last) {
        const bool full = slot == kBlock - 1;
        unsigned top_k = 0, top_v = 0;
        // (times the low half of a probability, zero or negative as often as not, an infinity would be NaN: it is added at the end)
        auto set_aside = [&](int x, __half v, int at) {
            const float w = __half2float(v);
            const bool odd = !finite_bits(magnitude(v));
            if (odd) atomicOr(&lds.odd[x], w > 0.f ? 1 : w < 0.f ? 2 : 4);
            lds.u.tail.v[x][value_place(x, at)] = odd ? 0 : __half_as_ushort(v);
        };
#pragma unroll
        for (int i = 0; i < UNITS; ++i) {
            const int u = t + i * T, s = u / (D / 8), x = (u % (D / 8)) * 8, at = value_slot(s);
            *reinterpret_cast<v4i *>(&lds.u.tail.k[s][x]) = tk[i];
            unsigned mk = 0, mv = 0;
#pragma unroll
            for (int w = 0; w < 4; ++w) {
                mk = max(mk, max((unsigned)tk[i][w] & 0x7fffu, (unsigned)tk[i][w] >> 16 & 0x7fffu));
                mv = max(mv, max((unsigned)tv[i][w] & 0x7fffu, (unsigned)tv[i][w] >> 16 & 0x7fffu));
            }
            top_k = max(top_k, mk);
            top_v = max(top_v, mv);
            if (!full && !finite_bits(mv)) {
#pragma unroll 1
                for (int e = 0; e < 8; ++e) set_aside(x + e, reinterpret_cast<const __half *>(tail_v + s * D + x)[e], at);
            } else {
#pragma unroll
                for (int e = 0; e < 8; ++e) lds.u.tail.v[x + e][value_place(x, at)] = (unsigned short)((unsigned)tv[i][e >> 1] >> (16 * (e & 1)));
            }
        }
        __syncthreads();
        if (t < D) {                                                  // the new row
            lds.u.tail.k[slot][t] = __half_as_ushort(lds.knew[t]);
            if (full) lds.u.tail.v[t][value_place(t, value_slot(slot))] = __half_as_ushort(lds.vnew[t]);
            else set_aside(t, lds.vnew[t], value_slot(slot));
            top_k = max(top_k, magnitude(lds.knew[t]));
            top_v = max(top_v, magnitude(lds.vnew[t]));
        }
        if (full) {
            top_k = wavefront_umax(top_k);
            top_v = wavefront_umax(top_v);
            if (l == 0) lds.top[0][wave] = top_k, lds.top[1][wave] = top_v;
            __syncthreads();
#pragma unroll
            for (int w = 0; w < kDecodeWaves; ++w) top_k = max(top_k, lds.top[0][w]), top_v = max(top_v, lds.top[1][w]);
            tail_sk = scale_of(top_k);
            tail_sv = scale_of(top_v);
            const bool ok_k = finite_bits(top_k), ok_v = finite_bits(top_v);
            const Steps sk = steps_of(__half2float(__ushort_as_half((unsigned short)top_k))), sv = steps_of(__half2float(__ushort_as_half((unsigned short)top_v)));
            int *kc = reinterpret_cast<int *>(block_codes<D>(cache, head, last, 0)), *vc = reinterpret_cast<int *>(block_codes<D>(cache, head, last, 1));
            // words of four codes, in the order of the cache; the rows in LDS become their codes
            for (int u = t; u < kBlock * D / 4; u += T) {
                const int e4 = u & 3, lane = (u >> 2) & 63, x = u >> 8, lr = lane & 15, lg = lane >> 4;
                unsigned short *k = &lds.u.tail.k[(x / C) * 16 + lr][(x % C) * 64 + lg * 16 + e4 * 4];
                unsigned short *v = &lds.u.tail.v[x * 16 + lr][value_place(x * 16 + lr, (e4 >> 1) * 32 + lg * 8 + (e4 & 1) * 4)];
                int wk = 0, wv = 0;
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const int ck = ok_k ? code_of(__half2float(__ushort_as_half(k[e])), sk) : 0, cv = ok_v ? code_of(__half2float(__ushort_as_half(v[e])), sv) : 0;
                    k[e] = __half_as_ushort(__float2half_rn((float)ck));
                    v[e] = __half_as_ushort(__float2half_rn((float)cv));
                    wk |= (ck & 255) << (8 * e);
                    wv |= (cv & 255) << (8 * e);
                }
                if (chunk == 0) {
                    kc[u] = wk;
                    vc[u] = wv;
                }
            }
            if (chunk == 0 && t == 0) {
                float *to = cache.scales + (head * cache.blocks + last) * 2;
                to[0] = tail_sk;
                to[1] = tail_sv;
            }
        } else if (chunk == 0 && t < D) {
            tail_k[slot * D + t] = lds.knew[t];
            tail_v[slot * D + t] = lds.vnew[t];
        }
        __syncthreads();
    }

    // queries: column r of the products; columns past the heads repeat the last head
    v8h qf[2 * C];
#pragma unroll
    for (int m = 0; m < 2 * C; ++m) qf[m] = *reinterpret_cast<const v8h *>(&lds.q[min(r, heads - 1)][64 * (m >> 1) + 16 * g + 8 * (m & 1)]);
    WaveSums<D> own;
    int j = begin + wave;
    for (; j < stop && j < last; j += kDecodeWaves) {
        const float2 scale = sc;
        own.add(
            qf, scale.x, scale.y, false, 0,
            [&](int T4, int m) {
                const v4i w = kraw[T4 * C + (m >> 1)];
                return (m & 1) ? halves_of(w[2], w[3]) : halves_of(w[0], w[1]);
            },
            [&](int i, int n) { return halves_of(vraw[i][2 * n], vraw[i][2 * n + 1]); },
            [&] {
                fetch_scales(j + kDecodeWaves);
                fetch_keys(j + kDecodeWaves);                         // (into the registers that have just become free)
            });
        fetch_values(j + kDecodeWaves);
    }
    if (j < stop)
        own.add(
            qf, tail_sk, tail_sv, true, slot,
            [&](int T4, int m) { return *reinterpret_cast<const v8h *>(&lds.u.tail.k[16 * T4 + r][64 * (m >> 1) + 16 * g + 8 * (m & 1)]); },
            [&](int i, int n) { return *reinterpret_cast<const v8h *>(&lds.u.tail.v[16 * i + r][value_place(16 * i + r, 32 * n + 8 * g)]); }, [] {});
    own.l += __shfl_xor(own.l, 16);
    own.l += __shfl_xor(own.l, 32);
    __syncthreads();                                                  // the last block's rows have been read
#pragma unroll
    for (int i = 0; i < DT; ++i)
#pragma unroll
        for (int e = 0; e < 4; ++e) lds.u.o[wave][r][16 * i + 4 * g + e] = own.o[i][e] * own.unit.unit;
    if (g == 0) {
        lds.m[wave][r] = own.m;
        lds.l[wave][r] = own.l;
    }
    __syncthreads();
    // the wavefronts' sums in one
    const int64_t item = (int64_t)b * gridDim.y + blockIdx.y;
    const int per_item = heads_of_partial(a.G) * (D + 2);
    float *mine = a.partials + (item * a.shares + share) * per_item;
    auto merged = [&](int j, int i, float &top, float &sum) {
        top = -INFINITY;
#pragma unroll
        for (int w = 0; w < kDecodeWaves; ++w) top = fmaxf(top, lds.m[w][j]);
        // (no score above minus infinity: the share has nothing to add to the others; where there are none the softmax is 0 / 0)
        const float from = top == -INFINITY && active > 1 ? 0.f : top;
        sum = 0.f;
        float o = 0.f;
#pragma unroll
        for (int w = 0; w < kDecodeWaves; ++w) {
            if (begin + w >= stop) break;                             // a wavefront without a block
            const float f = exp2f(lds.m[w][j] - from);
            sum += f * lds.l[w][j];
            o += f * lds.u.o[w][j][i];
        }
        const int odd = lds.odd[i];
        if (odd) o = odd == 1 ? o + INFINITY : odd == 2 ? o - INFINITY : NAN;
        return o;
    };
    if (active == 1) {
        for (int u = t; u < heads * D; u += T) {
            float top, sum;
            const float o = merged(u / D, u % D, top, sum);
            out[u] = __float2half_rn(o / sum);
        }
        return;
    }
    for (int u = t; u < heads * D; u += T) {
        float top, sum;
        const float o = merged(u / D, u % D, top, sum);
        __hip_atomic_store(mine + u, o, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
        if (u % D == 0) {
            __hip_atomic_store(mine + heads * D + u / D, top, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
            __hip_atomic_store(mine + heads * D + heads + u / D, sum, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
        }
    }
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");                  // this wavefront's stores have arrived before the workgroup does
    __syncthreads();
    if (t == 0) lds.arrived = (int)__hip_atomic_fetch_add(a.counters + item, 1u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    __syncthreads();
    if (lds.arrived != active - 1) return;
    if (t == 0) __hip_atomic_store(a.counters + item, 0u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);      // the next call starts from zero again
    // The shares' sums in one: their maxima and sums first, a factor for each share and head, then the outputs, two columns per load, the
    // shares dealt to as many groups of threads as there are.
    const float *all = a.partials + item * a.shares * per_item;
    float *factor = &lds.u.o[0][0][0];                                // [share][head]
    __syncthreads();
    for (int u = t; u < active * heads; u += T) factor[u] = __hip_atomic_load(all + (int64_t)(u / heads) * per_item + heads * D + u % heads, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    __syncthreads();
    if (t < heads) {
        float top = -INFINITY;
        for (int w = 0; w < active; ++w) top = fmaxf(top, factor[w * heads + t]);
        lds.m[0][t] = top;
    }
    __syncthreads();
    for (int u = t; u < active * heads; u += T) factor[u] = exp2f(factor[u] - lds.m[0][u % heads]);
    float *sums = factor + kMaxShares * 16;                           // [share][head]
    for (int u = t; u < active * heads; u += T)
        sums[u] = __hip_atomic_load(all + (int64_t)(u / heads) * per_item + heads * D + heads + u % heads, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    __syncthreads();
    if (t < heads) {
        float sum = 0.f;
        for (int w = 0; w < active; ++w) sum += factor[w * heads + t] * sums[w * heads + t];
        lds.l[0][t] = 1.f / sum;
    }
    const int pairs = heads * (D / 2), groups = max(1, T / pairs);
    float2 *parts = reinterpret_cast<float2 *>(sums);                 // [group][pair], over the sums that have been added
    for (int u0 = 0; u0 < pairs; u0 += T) {
        const int u = u0 + t % (pairs < T ? pairs : T), group = pairs < T ? t / pairs : 0;
        float2 o = {0.f, 0.f};
        if (u < pairs && group < groups) {
            const int j = u / (D / 2);
#pragma unroll 8
            for (int w = group; w < active; w += groups) {
                const u64 raw = __hip_atomic_load(reinterpret_cast<const u64 *>(all + (int64_t)w * per_item) + u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
                const float f = factor[w * heads + j], x = __uint_as_float((unsigned)raw), y = __uint_as_float((unsigned)(raw >> 32));
                o.x += fabsf(x) < INFINITY ? f * x : x;               // (an infinite value stays one however small the share's weight)
                o.y += fabsf(y) < INFINITY ? f * y : y;
            }
        }
        if (groups > 1) {
            __syncthreads();
            if (u < pairs && group > 0 && group < groups) parts[(group - 1) * pairs + u] = o;
            __syncthreads();
            if (u < pairs && group == 0)
                for (int w = 0; w < groups - 1; ++w) o.x += parts[w * pairs + u].x, o.y += parts[w * pairs + u].y;
        } else if (u0 == 0) {
            __syncthreads();
        }
        if (u < pairs && group == 0) {
            const float norm = lds.l[0][u / (D / 2)];
            out[2 * u] = __float2half_rn(o.x * norm);
            out[2 * u + 1] = __float2half_rn(o.y * norm);
        }
    }
}

// ---------------------------------------------------------------- launches

template <int D>
static sqap_status launch_append_d(const __half *QKV, int64_t ld, const int32_t *starts, const int32_t *pos, const int32_t *past, int rows, int max_new,
                                   int H, double base, const Cache8View &cache, __half *Q_out, int64_t ldq, hipStream_t st)
{
    constexpr int LDS = kBlock * D / 2 * 16 + kBlock * D + 4 * 4 * D / 64 * 4;
    static std::atomic<bool> ready[kMaxDeviceSlots];
    if (LDS > 65536 && !ready[device_slot()].load(std::memory_order_relaxed)) {
        SQAP_HIP_CHECK(hipFuncSetAttribute(reinterpret_cast<const void *>(cache8_append_kernel<D>), hipFuncAttributeMaxDynamicSharedMemorySize, LDS));
        ready[device_slot()].store(true, std::memory_order_relaxed);
    }
    const int columns = (max_new + kBlock - 2) / kBlock + 1;          // blocks that the longest sequence touches, at most
    // heads that share a workgroup's angles: as many as leave the device its workgroups.  Where there are
    // few, keys, values and queries have workgroups of their own: each is a chain of its own, but keys and queries work out the same
    // angles (148 rows of 8 key and 32 query heads, 32 of them: 15.3 us together, 10.3 apart; 512 of 8, 72: 8.7 and 7.2; 148 of 32, 128: 8.9 and 9.5).
    // With some more, values alone are apart (148 rows of 32 heads: 8.1 us; 900 of 8, 128: 11.6 together and 10.7; but three prompts, 600: 29.6 and 32.7).
    // Angles for more than one head: 2000 rows of 32 heads 25.0 us with 512 workgroups, 35.5 with 256, 27.8 with 1024.
    const int64_t items = (int64_t)columns * cache.batch * cache.kv_heads;
    const int share = (int)std::max<int64_t>(1, std::min<int64_t>(cache.kv_heads, items / kAppendGroups));
    const int split = items <= kAppendSplit ? 3 : items <= kAppendValues ? 2 : 1;
    hipLaunchKernelGGL(cache8_append_kernel<D>, dim3(columns, (cache.kv_heads + share - 1) / share * split, cache.batch), dim3(4 * D), LDS, st, QKV, ld,
                       starts, pos, past, rows, max_new, H, share, split, cache, Q_out, ldq, rope_frequencies(D, base));
    SQAP_HIP_CHECK(hipGetLastError());
    return SQAP_OK;
}

sqap_status launch_cache8_append(const __half *QKV, int64_t ld, const int32_t *starts, const int32_t *pos, const int32_t *past, int rows, int max_new,
                                 int H, double base, const Cache8View &cache, int d, __half *Q_out, int64_t ldq, hipStream_t st)
{
    return d == 64 ? launch_append_d<64>(QKV, ld, starts, pos, past, rows, max_new, H, base, cache, Q_out, ldq, st)
                   : launch_append_d<128>(QKV, ld, starts, pos, past, rows, max_new, H, base, cache, Q_out, ldq, st);
}

sqap_status launch_cache8_read(const Cache8View &cache, int d, const int32_t *lengths, int first, int count, __half *out, int64_t ld, hipStream_t st)
{
    for (int64_t from = 0; from < count; from += most_workgroups(256)) {
        const dim3 grid((unsigned)std::min(most_workgroups(256), count - from), cache.batch);
        if (d == 64) hipLaunchKernelGGL(cache8_read_kernel<64>, grid, dim3(256), 0, st, cache, lengths, first, count, (int)from, out, ld);
        else hipLaunchKernelGGL(cache8_read_kernel<128>, grid, dim3(256), 0, st, cache, lengths, first, count, (int)from, out, ld);
        SQAP_HIP_CHECK(hipGetLastError());
    }
    return SQAP_OK;
}

// Tiles of 16 rows, whose blocks are dealt to eight wavefronts, where there would be few tiles of 128: 148 rows of 32 heads (64 of those) take
// 9.0 us so and 11.0 otherwise, 512 of 8 heads (32) 8.0 and 19.0, 20 of 32 heads over 8 behind 2000 (8) 18 and 62, 1500 of 8 behind 2000
// (96) 67 and 103, 300 of 32 heads (96) 13.9 and 15.1; but 500 of 32 (128) 23.7 and 21.3, 1000 of 32 over 8 (256) 56 and 37.
constexpr int kFewTiles = 96;

template <int D>
static sqap_status launch_attention_d(const __half *Q, int64_t ldq, const int32_t *starts, const int32_t *past, int rows, int max_new, int H,
                                      const Cache8View &cache, __half *O, int64_t ldo, hipStream_t st)
{
    constexpr int WAVES = 4, LDS = 2 * 2 * kBlock * D * 2;
    static std::atomic<bool> ready[kMaxDeviceSlots];
    if (!ready[device_slot()].load(std::memory_order_relaxed)) {
        SQAP_HIP_CHECK(hipFuncSetAttribute(reinterpret_cast<const void *>(cache8_attention_kernel<D, WAVES>), hipFuncAttributeMaxDynamicSharedMemorySize, LDS));
        SQAP_HIP_CHECK(hipFuncSetAttribute(reinterpret_cast<const void *>(cache8_few_rows_kernel<D>), hipFuncAttributeMaxDynamicSharedMemorySize,
                                           (int)sizeof(FewRowsLds<D>)));
        ready[device_slot()].store(true, std::memory_order_relaxed);
    }
    const auto tiles_of = [&](int per_tile) { return std::max<int64_t>(1, ((int64_t)max_new * (H / cache.kv_heads) + per_tile - 1) / per_tile); };
    const int64_t pairs = (int64_t)cache.kv_heads * cache.batch;
    const bool few = tiles_of(32 * WAVES) * pairs <= kFewTiles;
    const int64_t tiles = tiles_of(few ? 16 : 32 * WAVES), items = tiles * pairs;
    if (few)
        hipLaunchKernelGGL(cache8_few_rows_kernel<D>, dim3((unsigned)items), dim3(64 * kFewRowsWaves), sizeof(FewRowsLds<D>), st, Q, ldq, starts, past, rows,
                           max_new, H, cache, O, ldo, (int)tiles);
    else
        hipLaunchKernelGGL((cache8_attention_kernel<D, WAVES>), dim3((unsigned)items), dim3(64 * WAVES), LDS, st, Q, ldq, starts, past, rows, max_new, H,
                           cache, O, ldo, (int)tiles);
    SQAP_HIP_CHECK(hipGetLastError());
    return SQAP_OK;
}

sqap_status launch_cache8_attention(const __half *Q, int64_t ldq, const int32_t *starts, const int32_t *past, int rows, int max_new, int H,
                                    const Cache8View &cache, int d, __half *O, int64_t ldo, hipStream_t st)
{
    return d == 64 ? launch_attention_d<64>(Q, ldq, starts, past, rows, max_new, H, cache, O, ldo, st)
                   : launch_attention_d<128>(Q, ldq, starts, past, rows, max_new, H, cache, O, ldo, st);
}

// Shares of a sequence.  One up to eight blocks: a wavefront's second block costs 1.5 us, joining 2.5.  Beyond, shares of four blocks while
// there are few (1500 positions of 32 heads: 11.4 us, shares of eight 12.4), of eight at least once there are eight (4000: 14.0, of four
// 16.6); and no more than two workgroups per compute unit in all, which is what their registers leave room for (100k positions of 8 key
// heads: 52 us with 512 workgroups, 66 with 768).
constexpr int kDecodeGroups = 512;
static int blocks_of(int positions) { return positions / kBlock + (positions % kBlock != 0); }      // (of any number up to 2^31 - 1)
static int decode_shares(int batch, int H, int kv_heads, int longest)
{
    const int chunks = (H / kv_heads + 15) / 16, blocks = blocks_of(longest);
    const int64_t items = (int64_t)batch * kv_heads * chunks;
    const int wanted = blocks <= 8 ? 1 : std::max((blocks + 7) / 8, std::min(8, (blocks + 3) / 4));
    return (int)std::max<int64_t>(1, std::min<int64_t>({wanted, kDecodeGroups / items, kMaxShares}));
}

// Counters in front, one for each sequence, key head and 16 of its query heads; where there is more than one share, that is 256 of them at
// most.  The room for them is the same whatever the sizes: no call's sums lie where another's counters are.
constexpr size_t kCounterBytes = 16384;
static_assert(kCounterBytes >= kDecodeGroups / 2 * sizeof(unsigned), "a counter for each item that is shared");

size_t cache8_workspace_bytes(int batch, int H, int kv_heads, int d, int longest)
{
    const int shares = decode_shares(batch, H, kv_heads, longest), G = H / kv_heads;
    if (shares == 1) return 0;
    const size_t items = (size_t)batch * kv_heads * ((G + 15) / 16);
    return kCounterBytes + items * shares * heads_of_partial(G) * (d + 2) * 4;
}

sqap_status launch_cache8_decode(const __half *QKV, int64_t ld, const int32_t *pos, const int32_t *past, int H, double base, const Cache8View &cache,
                                 int d, int longest, __half *O, int64_t ldo, void *workspace, hipStream_t st)
{
    DecodeArgs a = {};
    a.QKV = QKV;
    a.ld = ld;
    a.pos = pos;
    a.past = past;
    a.H = H;
    a.G = H / cache.kv_heads;
    a.chunks = (a.G + 15) / 16;
    a.shares = decode_shares(cache.batch, H, cache.kv_heads, longest);
    a.per_share = (blocks_of(longest) + a.shares - 1) / a.shares;
    a.cache = cache;
    a.O = O;
    a.ldo = ldo;
    a.counters = static_cast<unsigned *>(workspace);
    a.partials = reinterpret_cast<float *>(static_cast<char *>(workspace) + kCounterBytes);
    a.freq = rope_frequencies(d, base);
    const dim3 grid(a.shares, cache.kv_heads * a.chunks, cache.batch);
    if (d == 64) hipLaunchKernelGGL(cache8_decode_kernel<64>, grid, dim3(64 * kDecodeWaves), 0, st, a);
    else hipLaunchKernelGGL(cache8_decode_kernel<128>, grid, dim3(64 * kDecodeWaves), 0, st, a);
    SQAP_HIP_CHECK(hipGetLastError());
    return SQAP_OK;
}

}  // namespace sqap
