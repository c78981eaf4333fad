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

// ---------------------------------------------------------------- attention in parts

// Attention behind a shared prefix is worked out in parts: of the rows of a whole group over shares of the prefix, and of each sequence's
// rows over its own positions.  A part leaves, for each row and head, the sum of the values times p = 2^(s - m + kLift), the maximum m
// (in units of ln 2) and the sum of the p; cache8_join_kernel puts them together.
enum class Part { Whole, Own, Prefix };
struct Parts {
    float *o;                   // [part][row][head][D]
    float2 *ml;                 // [part][row][head]
    int64_t pairs;              // rows times heads
    int prefix_shares;          // the parts in front; own ones behind them
    int width;                  // sequences that share a prefix
    const int32_t *length;      // of the prefixes, [groups]
};

// The rows of a group: [row, row + n), nothing where they are not within the fused rows or more than have been announced.
struct GroupRows {
    int row, n;
};
__device__ __forceinline__ GroupRows group_rows(const int32_t *starts, int group, int width, int rows, int max_new)
{
    if (!starts) return {group * width, width};
    GroupRows r = {starts[group * width], 0};
    const int end = starts[(group + 1) * width];
    if (r.row >= 0 && end >= r.row && end <= rows && (int64_t)(end - r.row) <= (int64_t)width * max_new) r.n = end - r.row;
    return r;
}

// The blocks of a prefix that a share has: [first, end); `active` shares have any.
struct PrefixShare {
    int first, end, active;
};
__device__ __forceinline__ PrefixShare prefix_share(int length, int capacity, int shares, int share)
{
    if (length <= 0 || length > capacity) return {0, 0, 0};
    const int blocks = (length + kBlock - 1) / kBlock, each = (blocks + shares - 1) / shares;
    return {min(share * each, blocks), min((share + 1) * each, blocks), (blocks + each - 1) / each};
}

// Whether a sequence's rows lie within its group's.  Where starts are not in order they may be another group's, and the sequence is skipped: a part of it
// would lie where that group's own is.
__device__ __forceinline__ bool in_its_group(const int32_t *starts, int b, int width, const Span &sp)
{
    const int first = b / width * width;
    return sp.row >= starts[first] && sp.row + sp.n <= starts[first + width];
}

// A sequence behind a prefix: `rows` says whether it has any that count, `fits` whether they are worked out (their outputs are NaN otherwise).
struct Member {
    Span sp;
    bool rows, fits;
    int length;
};
__device__ __forceinline__ Member member_of(const int32_t *starts, const int32_t *past, int b, int rows, int max_new, int capacity, int prefix_capacity, const Parts &parts)
{
    const int group = b / parts.width;
    Member m = {Span{b, 1, past[b], true}, true, true, parts.length[group]};
    if (starts) {
        m.sp = span_of(starts, past, b, rows, max_new, capacity);
        m.rows = m.sp.n > 0 && in_its_group(starts, b, parts.width, m.sp);
        m.fits = m.sp.fits && group_rows(starts, group, parts.width, rows, max_new).n > 0;
    } else {
        m.rows = m.sp.past >= 0;
        m.fits = m.sp.past < capacity;
    }
    m.fits = m.fits && m.length >= 0 && m.length <= prefix_capacity;
    return m;
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

// A block of keys and values in LDS, as halves in the order of the products' operands: keys [2][D / 16] KiB, values [D / 32][4] KiB.  kraw, vraw: the
// pieces of a thread of T, as the cache has them.
template <int D, int T>
__device__ __forceinline__ void keep_codes(uint8_t *kt, const v4i *kraw, const v4i *vraw)
{
    constexpr int NP = D / 16, COUNT = kBlock * D / 16, PIECES = (COUNT + T - 1) / T;
    uint8_t *vt = kt + kBlock * D * 2;
    const int t = threadIdx.x;
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
}
// The same of an unfinished block; says whether there are values among this thread's that are not finite (they come back at the end, to the rows
// that see them).
template <int D, int T>
__device__ __forceinline__ bool keep_tail(uint8_t *kt, const __half *tail_k, const __half *tail_v, int tail_rows)
{
    constexpr int NP = D / 16;
    uint8_t *vt = kt + kBlock * D * 2;
    bool odd = false;
    for (int u = threadIdx.x; u < kBlock * D / 8; u += T) {
        const int s = u / (D / 8), x = (u % (D / 8)) * 8;
        v8h k = {}, v = {};
        if (s < tail_rows) {
            k = *reinterpret_cast<const v8h *>(tail_k + s * D + x);
            v = *reinterpret_cast<const v8h *>(tail_v + s * D + x);
        }
        *reinterpret_cast<v8h *>(kt + (((s >> 5) * NP + (x >> 4)) * 64 + ((x >> 3) & 1) * 32 + (s & 31)) * 16) = k;
        const int n = s >> 4, o = s & 15;                             // 8 q + 4 h + i of its sixteen positions
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            const int col = x + e;
            _Float16 w = v[e];
            if (!(__builtin_fabsf((float)w) <= 65504.f)) {
                w = (_Float16)0.f;
                odd = true;
            }
            *reinterpret_cast<_Float16 *>(vt + (((col >> 5) * 4 + n) * 64 + ((o >> 2) & 1) * 32 + (col & 31)) * 16 + (o >> 3) * 8 + (o & 3) * 2) = w;
        }
    }
    return odd;
}

// Sums of a wavefront's 32 rows: row l % 32, columns 32 ct + 8 a + 4 (l / 32) ...  ALONE: all that the rows see passes through here, so that a row without
// a score above minus infinity is 0 / 0; otherwise it adds nothing to what others have.
template <int D, bool ALONE>
struct TileSums {
    static constexpr int NP = D / 16, CT = D / 32;
    v16f ot[CT];
    float mrun = -INFINITY, lrun = 0.f;
    Unit unit;
    __device__ __forceinline__ TileSums()
    {
#pragma unroll
        for (int ct = 0; ct < CT; ++ct)
#pragma unroll
            for (int i = 0; i < 16; ++i) ot[ct][i] = 0.f;
    }
    // kt: a block in LDS; sk: the keys' scale times log2(e) / sqrt(d); masked: some row does not see some position, this lane's sees 0 .. last.
    __device__ __forceinline__ void add(const uint8_t *kt, const v8h (&qf)[NP], float sk, float sv, bool masked, int last)
    {
        const int l = threadIdx.x & 63, h = l >> 5;
        const uint8_t *vt = kt + kBlock * D * 2 + l * 16;
        kt += l * 16;
        v16f s[2];
        __builtin_amdgcn_s_setprio(1);                                // (before the other workgroup's exponentials: 3 in 100; not for the values' products)
#pragma unroll
        for (int tt = 0; tt < 2; ++tt)
#pragma unroll
            for (int i = 0; i < 16; ++i) s[tt][i] = 0.f;
        // the two halves of the block in turn, keys AHEAD products before they enter (left to itself the compiler reads one and waits for it)
        constexpr int AHEAD = 4;
        v8h k[AHEAD];
#pragma unroll
        for (int i = 0; i < AHEAD; ++i) k[i] = *reinterpret_cast<const v8h *>(kt + ((i & 1) * NP + (i >> 1)) * 1024);
        __builtin_amdgcn_sched_group_barrier(0x100, AHEAD, 0);
#pragma unroll
        for (int i = 0; i < 2 * NP; ++i) {
            s[i & 1] = __builtin_amdgcn_mfma_f32_32x32x16_f16(k[i % AHEAD], qf[i >> 1], s[i & 1], 0, 0, 0);
            __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);
            if (i + AHEAD < 2 * NP) {
                k[i % AHEAD] = *reinterpret_cast<const v8h *>(kt + (((i + AHEAD) & 1) * NP + ((i + AHEAD) >> 1)) * 1024);
                __builtin_amdgcn_sched_group_barrier(0x100, 1, 0);
            }
        }
        __builtin_amdgcn_s_setprio(0);
        if (masked) {
            last -= 4 * h;
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
        if (top > -INFINITY) top *= sk;                               // (nothing seen: it stays, whatever the scale)
        float change;
        const float factor = unit.enter(sv, change);
        if (top - mrun > kRaiseBy) {                                  // (a row that sees nothing of the block keeps its maximum)
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
        const float taken = !ALONE && mrun == -INFINITY ? 0.f : mrun;
        float by = sk, from = __log2f(factor) + kLift;
        const bool bad = !(sk >= 0.f && sv >= 0.f);                   // keys or values that are NaN as a whole: for the rows that see any of them
        if (bad || __any(fabsf(top) > kLargeScore && top > -INFINITY)) {            // (a masked score times NaN would be NaN, too)
#pragma unroll
            for (int tt = 0; tt < 2; ++tt)
#pragma unroll
                for (int i = 0; i < 16; ++i) {
                    float w = bad ? NAN : s[tt][i] * sk;
                    asm volatile("" : "+v"(w));                       // (rounded)
                    s[tt][i] = s[tt][i] == -INFINITY ? -INFINITY : w - taken;
                }
            by = 1.f;
        } else {
            from -= taken;
        }
        float sum = 0.f;
        v8h p[2], rest[2], v[2][CT];
        auto values = [&](int n) {
#pragma unroll
            for (int ct = 0; ct < CT; ++ct) v[n & 1][ct] = *reinterpret_cast<const v8h *>(vt + (ct * 4 + n) * 1024);
        };
        auto powers = [&](int n) {
#pragma unroll
            for (int i = 0; i < 8; i += 2) {
                const float s0 = s[n >> 1][(n & 1) * 8 + i], s1 = s[n >> 1][(n & 1) * 8 + i + 1];
                const float e0 = __builtin_amdgcn_exp2f(fmaf(s0, by, from)), e1 = __builtin_amdgcn_exp2f(fmaf(s1, by, from));
                sum += e0;
                sum += e1;
                v2h high, low;
                two_halves(e0, e1, high, low);
                p[n & 1][i] = high[0];
                p[n & 1][i + 1] = high[1];
                rest[n & 1][i] = low[0];
                rest[n & 1][i + 1] = low[1];
            }
        };
        values(0);
        __builtin_amdgcn_sched_barrier(0);
        powers(0);
#pragma unroll
        for (int n = 0; n < 4; ++n) {
            if (n < 3) values(n + 1);
            __builtin_amdgcn_sched_barrier(0);
#pragma unroll
            for (int ct = 0; ct < CT; ++ct) ot[ct] = __builtin_amdgcn_mfma_f32_32x32x16_f16(v[n & 1][ct], p[n & 1], ot[ct], 0, 0, 0);
#pragma unroll
            for (int ct = 0; ct < CT; ++ct) ot[ct] = __builtin_amdgcn_mfma_f32_32x32x16_f16(v[n & 1][ct], rest[n & 1], ot[ct], 0, 0, 0);
            if (n < 3) powers(n + 1);
            __builtin_amdgcn_sched_barrier(0);
        }
        lrun += sum * __builtin_amdgcn_rcpf(factor);
    }
    // a row's sums in units of one; the row, divided by its sum
    __device__ __forceinline__ void write_part(float2 *ml, float *o) const
    {
        const int h = (threadIdx.x & 63) >> 5;
        if (h == 0) *ml = {mrun, lrun};
#pragma unroll
        for (int ct = 0; ct < CT; ++ct)
#pragma unroll
            for (int a = 0; a < 4; ++a) {
                v4f x;
#pragma unroll
                for (int i = 0; i < 4; ++i) x[i] = ot[ct][4 * a + i] * unit.unit;
                *reinterpret_cast<v4f *>(o + 32 * ct + 8 * a + 4 * h) = x;
            }
    }
    __device__ __forceinline__ void write_rows(__half *to) const
    {
        const int h = (threadIdx.x & 63) >> 5;
        const float norm = unit.unit / lrun;
#pragma unroll
        for (int ct = 0; ct < CT; ++ct)
#pragma unroll
            for (int a = 0; a < 4; ++a) {
                union { __half h[4]; v2u v; } u;
#pragma unroll
                for (int i = 0; i < 4; ++i) u.h[i] = __float2half_rn(ot[ct][4 * a + i] * norm);
                *reinterpret_cast<v2u *>(to + 32 * ct + 8 * a + 4 * h) = u.v;
            }
    }
};
// infinities and NaN among the first `seen` rows of an unfinished block's values, to what a lane has written of its row
template <int D, typename X, typename Get, typename Set>
__device__ __forceinline__ void add_odd(X *to, const __half *tail_v, int seen, Get get, Set set)
{
    const int h = (threadIdx.x & 63) >> 5;
#pragma unroll 1
    for (int x = 0; x < D / 2; ++x) {
        const int col = (x >> 2) * 8 + 4 * h + (x & 3);
        float o = get(to[col]);
#pragma unroll 1
        for (int s = 0; s < seen; ++s) {
            const float v = __half2float(tail_v[s * D + col]);
            if (!(fabsf(v) <= 65504.f)) o += v;
        }
        to[col] = set(o);
    }
}
template <int D>
__device__ __forceinline__ void add_odd(float *to, const __half *tail_v, int seen)
{
    add_odd<D>(to, tail_v, seen, [](float x) { return x; }, [](float x) { return x; });
}
template <int D>
__device__ __forceinline__ void add_odd(__half *to, const __half *tail_v, int seen)
{
    add_odd<D>(to, tail_v, seen, [](__half x) { return __half2float(x); }, [](float x) { return __float2half_rn(x); });
}

// Rows are (query, head) pairs of the heads that share a key head, query first, 32 to a wavefront and WAVES wavefronts to a workgroup, so
// that a block of keys and values is taken from memory and made halves once for all of them.  Everything is transposed (scores:
// positions x rows), as in attention.hip: probabilities are the second product's operand where they were computed.
// What bounds it is the vector ALU beside the matrix cores, 357 instructions to 48 matrix instructions per wavefront and block, a tenth of them
// exponentials: 1500, 1115 and 1446 rows of 32 heads over 8 behind 2000, 1994 and 420 positions in some 285 us, 0.49 PFLOP/s (a library product of
// halves reaches 1.24; keys read from LDS ahead of their products took 8 us off).  With probabilities of one half, 32 matrix instructions and 305 others, it
// took 40 us less, and the outputs were 2.0e-4 of their norm further off.  (Then the next block's scores multiplied between this one's probabilities, in the same wavefront: 335 us, the registers do not suffice.)
// A block's p = 2^(s - m) times its factor is one exponential, of s sk + (log2 factor - m); the sum of the probabilities is put right by the
// factor once per block.  The hardware's exponential, logarithm and reciprocal are off by a unit of the last place of binary32 or so each, which is
// less than the rounding of the scores and of the sums.
// As a part of the attention behind a shared prefix (Part::Prefix) the rows are a group's, all of them see the whole of `cache`, the prefixes,
// and a workgroup has a share of its blocks.
template <int D, int WAVES, Part PART>
__global__ __launch_bounds__(64 * WAVES, 2) void cache8_attention_kernel(const __half *__restrict__ Q, int64_t ldq, const int32_t *__restrict__ starts,
                                                                         const int32_t *__restrict__ past, int rows, int max_new, int H,
                                                                         const Cache8View cache, __half *__restrict__ O, int64_t ldo, int tiles,
                                                                         const Parts parts)
{
    constexpr int T = 64 * WAVES, TILE = 32 * WAVES, NP = D / 16, BUF = 2 * kBlock * D * 2, COUNT = kBlock * D / 16;
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
    const int G = H / cache.kv_heads;
    Span sp;
    int n_rows, tile, part = parts.prefix_shares;
    PrefixShare share = {0, 0, 0};
    if constexpr (PART == Part::Prefix) {
        const GroupRows r = group_rows(starts, b, parts.width, rows, max_new);
        part = number / tiles;
        sp = {r.row, r.n, parts.length[b], true};
        share = prefix_share(sp.past, cache.blocks * kBlock, parts.prefix_shares, part);
        if (share.first >= share.end) return;
        tile = number % tiles * TILE;
    } else {
        sp = span_of(starts, past, b, rows, max_new, cache.blocks * kBlock);
        if (!sp.fits) {                                               // (of more than max_new rows too: all of them)
            if constexpr (PART == Part::Whole) nan_rows<D>(O, ldo, sp.row, (int64_t)sp.n * G, G, kh, number, tiles, TILE);
            return;
        }
        if (PART == Part::Own && !in_its_group(starts, b, parts.width, sp)) return;
        tile = (tiles - 1 - number) * TILE;
    }
    n_rows = sp.n * G;                                                // (the launch keeps max_new * G in 32 bits)
    if (tile >= n_rows) return;
    const int mine = tile + wave * 32 + c;
    const int mine_in = min(mine, n_rows - 1);
    const int query = mine_in / G, head = kh * G + mine_in % G;
    if (t == 0) not_finite = 0;
    // the positions that the cache holds, the last one that this lane's row sees, and that a row of the tile does
    const int end = PART == Part::Prefix ? sp.past : sp.past + sp.n, sees = PART == Part::Prefix ? sp.past - 1 : sp.past + query;
    const int tile_last = PART == Part::Prefix ? sp.past - 1 : sp.past + (min(tile + TILE, n_rows) - 1) / G;
    const int j_first = PART == Part::Prefix ? share.first : 0, n_blocks = PART == Part::Prefix ? share.end : tile_last / kBlock + 1;
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
        uint8_t *kt = lds + (j & 1) * BUF;
        if (j != tail_block) keep_codes<D, T>(kt, kraw, vraw);
        else if (keep_tail<D, T>(kt, tail_k, tail_v, tail_rows)) not_finite = 1;
    };

    TileSums<D, PART == Part::Whole> sums;
    const float per_d = kLog2e / sqrtf((float)D);
    const int wave_last = PART == Part::Prefix ? tile_last : sp.past + min(tile + wave * 32 + 31, n_rows - 1) / G;
    const int wave_first = PART == Part::Prefix ? tile_last : sp.past + min(tile + wave * 32, n_rows - 1) / G;
    __syncthreads();
    fetch(j_first);
    keep(j_first);
    float2 sc = {0.f, 0.f};
    if (tail_block != j_first) sc = *reinterpret_cast<const float2 *>(scales + 2 * j_first);
    for (int j = j_first; j < n_blocks; ++j) {
        fetch(j + 1);
        // (keys that are all zeros: the scores are, times anything but zero, which would make NaN of a masked one)
        const float sk = j == tail_block || sc.x == 0.f ? per_d : sc.x * per_d, sv = j == tail_block ? 1.f : sc.y;
        if (j + 1 < n_blocks && j + 1 != tail_block) sc = *reinterpret_cast<const float2 *>(scales + 2 * (j + 1));
        lds_barrier();
        if (j * kBlock <= wave_last) sums.add(lds + (j & 1) * BUF, qf, sk, sv, (j + 1) * kBlock - 1 > wave_first, sees - j * kBlock);
        keep(j + 1);
    }
    sums.lrun += __shfl_xor(sums.lrun, 32);
    const bool odd = n_blocks - 1 == tail_block && not_finite;
    if (mine >= n_rows) return;
    if constexpr (PART != Part::Whole) {
        const int64_t pair = part * parts.pairs + (int64_t)(sp.row + query) * H + head;
        sums.write_part(parts.ml + pair, parts.o + pair * D);
        if (odd) add_odd<D>(parts.o + pair * D, tail_v, sees - tail_block * kBlock + 1);
        return;
    }
    __half *to = O + (int64_t)(sp.row + query) * ldo + (int64_t)head * D;
    sums.write_rows(to);
    if (odd) add_odd<D>(to, tail_v, sees - tail_block * kBlock + 1);
}

// ---------------------------------------------------------------- long prompts behind prefixes

// Many rows to a sequence: tiles of 128 of one sequence pass over its prefix's blocks and then their own, and the blocks of all tiles together are
// dealt out evenly, so that no compute unit ends early (2675 rows of 32 heads over 8 behind prefixes of 6000 and 2900, append and joining
// included: 449 us, with the prefix and own positions in parts of whole tiles 527; 430 since keys are read ahead).  A tile inside a workgroup's range is finished there; of one over its ends, the workgroups leave their sums,
// one at the beginning and one at the end of each range, and cache8_long_join_kernel adds them.  Ranges are counted in tiles as long as their
// sequence's longest (a tile's real blocks, fewer where its rows see less, are parted in the same proportion).
// Of those 430 append is 20 and joining 15; 2250 rows behind 2000 take 189 with append (26) and joining (15).  Matrix cores are busy for 43 in 100 cycles, 8.3
// vector instructions stand beside each of theirs, and the clock falls as more of both are issued (2.11 to 1.99 GHz: the power limit).
constexpr int kLongBatch = 1024, kLongParts = 32, kLongLeast = 4, kLongTiles = 64, kLongWork = 16000;
struct LongSlot {                // what a workgroup's first range belongs to, where it is the rest of a tile
    int b, kh, tile, first, count;       // the workgroup that begins the tile, how many have a share of it; count 0: none, or not its second
    int pad[3];
};
struct LongArgs {
    const __half *Q;
    int64_t ldq;
    const int32_t *starts, *past;
    int rows, max_new, H;
    Cache8View cache, prefix;
    Parts parts;                 // (width and lengths)
    __half *O;
    int64_t ldo;
    LongSlot *slots;             // [workgroups]
    float2 *ml;                  // [workgroups][beginning, end][128]
    float *o;                    // [workgroups][beginning, end][128][D]
};
// (read from LDS, but the same in all lanes: into scalar registers)
__device__ __forceinline__ int uniform(int x) { return __builtin_amdgcn_readfirstlane(x); }
__device__ __forceinline__ int64_t uniform(int64_t x)
{
    return (int64_t)((u64)(unsigned)__builtin_amdgcn_readfirstlane((int)x) | (u64)(unsigned)__builtin_amdgcn_readfirstlane((int)(x >> 32)) << 32);
}
__device__ __forceinline__ int blocks_up(int positions) { return (positions + kBlock - 1) / kBlock; }

template <int D>
__global__ __launch_bounds__(256, 2) void cache8_long_kernel(const LongArgs a)
{
    constexpr int T = 256, TILE = 128, NP = D / 16, BUF = 2 * kBlock * D * 2, COUNT = kBlock * D / 16, PIECES = (COUNT + T - 1) / T;
    extern __shared__ __attribute__((aligned(16))) uint8_t lds[];     // two buffers
    __shared__ int64_t before[kLongBatch + 1];                        // blocks of the tiles of one key head in front of each sequence
    __shared__ int64_t wave_sum_[4];
    __shared__ int wave_most[4], not_finite[2];
    const Cache8View &cache = a.cache, &prefix = a.prefix;
    const int t = threadIdx.x, l = t & 63, wave = uniform(t >> 6), c = l & 31, h = l >> 5, G = a.H / cache.kv_heads, batch = cache.batch;
    const int groups = gridDim.x, w = (int)(blockIdx.x & 7) * (groups / 8) + (int)(blockIdx.x >> 3);      // neighbours behind one L2
    auto member = [&](int b) { return member_of(a.starts, a.past, b, a.rows, a.max_new, cache.blocks * kBlock, prefix.blocks * kBlock, a.parts); };
    auto tiles_of = [&](const Member &m) { return (m.sp.n * G + TILE - 1) / TILE; };      // (the launch keeps max_new * G in 32 bits)
    auto blocks_of_tile = [&](const Member &m) { return blocks_up(m.length) + blocks_up(m.sp.past + m.sp.n); };
    {
        constexpr int EACH = kLongBatch / T;
        int64_t mine[EACH], sum = 0;
        int most = 0;
#pragma unroll
        for (int i = 0; i < EACH; ++i) {
            const int b = t * EACH + i;
            mine[i] = sum;
            if (b >= batch) continue;
            const Member m = member(b);
            if (m.rows && m.fits) {
                sum += (int64_t)tiles_of(m) * blocks_of_tile(m);
                most = max(most, blocks_of_tile(m));
            }
        }
        int64_t upto = sum;
#pragma unroll
        for (int i = 1; i < 64; i <<= 1) {
            const int64_t x = __shfl_up(upto, i);
            if (l >= i) upto += x;
            most = max(most, __shfl_xor(most, i));
        }
        if (l == 63) wave_sum_[wave] = upto, wave_most[wave] = most;
        __syncthreads();
        upto -= sum;
        for (int i = 0; i < wave; ++i) upto += wave_sum_[i];
#pragma unroll
        for (int i = 0; i < EACH; ++i) before[t * EACH + i] = upto + mine[i];
        if (t == T - 1) before[kLongBatch] = upto + sum;
        __syncthreads();
    }
    const int64_t of_head = uniform(before[kLongBatch]), total = of_head * cache.kv_heads;
    const int most = uniform(max(max(wave_most[0], wave_most[1]), max(wave_most[2], wave_most[3])));
    const int64_t range = max(max((total + groups - 1) / groups, (int64_t)(most + kLongParts - 1) / kLongParts), (int64_t)kLongLeast);
    for (int b = w; b < batch; b += groups) {                         // sequences that do not fit
        const Member m = member(b);
        if (!m.rows || m.fits) continue;
        for (int64_t u = t; u < (int64_t)m.sp.n * a.H * D; u += T) a.O[(m.sp.row + u / (a.H * D)) * a.ldo + u % (a.H * D)] = __ushort_as_half(0x7e00);
    }
    LongSlot slot = {0, 0, 0, 0, 0, {0, 0, 0}};
    const int64_t stop = min((w + 1) * range, total);
    const float per_d = kLog2e / sqrtf((float)D);
    for (int64_t u = w * range; u < stop;) {
        const int kh = (int)(u / of_head);
        const int64_t at = u % of_head;
        int b = 0;
        for (int step = kLongBatch / 2; step > 0; step /= 2)
            if (before[b + step] <= at) b += step;
        b = uniform(b);                                               // (the last that begins there: those without tiles lie before it)
        const Member m = member(b);
        const Span &sp = m.sp;
        const int64_t in_sequence = at - uniform(before[b]);
        const int nominal = blocks_of_tile(m), tile_number = (int)(in_sequence / nominal), from = (int)(in_sequence - (int64_t)tile_number * nominal);
        const int upto = (int)min((int64_t)nominal, from + (stop - u));
        const int64_t tile_start = u - from;
        u += upto - from;
        const int n_rows = sp.n * G, tile = tile_number * TILE, tile_last = sp.past + (min(tile + TILE, n_rows) - 1) / G;
        const int of_prefix = blocks_up(m.length), n_blocks = of_prefix + tile_last / kBlock + 1;
        const int first = (int)((int64_t)from * n_blocks / nominal), end = (int)((int64_t)upto * n_blocks / nominal);
        const int mine = tile + wave * 32 + c, mine_in = min(mine, n_rows - 1), query = mine_in / G, head = kh * G + mine_in % G;
        const int sees = sp.past + query, wave_last = sp.past + min(tile + wave * 32 + 31, n_rows - 1) / G, wave_first = sp.past + min(tile + wave * 32, n_rows - 1) / G;
        const int64_t prefix_head = (int64_t)(b / a.parts.width) * prefix.kv_heads + kh, own_head = (int64_t)b * cache.kv_heads + kh;
        const __half *prefix_tail = prefix.tail + prefix_head * 2 * kBlock * D, *own_tail = cache.tail + own_head * 2 * kBlock * D;
        const int prefix_rest = m.length % kBlock, own_unfinished = of_prefix + (sp.past + sp.n) / kBlock, own_rest = (sp.past + sp.n) % kBlock;
        auto unfinished = [&](int j) { return j == own_unfinished || (j == of_prefix - 1 && prefix_rest > 0); };
        v8h qf[NP];
#pragma unroll
        for (int i = 0; i < NP; ++i) qf[i] = *reinterpret_cast<const v8h *>(a.Q + (int64_t)(sp.row + query) * a.ldq + (int64_t)head * D + 16 * i + 8 * h);
        v4i kraw[PIECES], vraw[PIECES];
        float2 sc = {0.f, 0.f};
        auto fetch = [&](int j) {
            if (j >= end || unfinished(j)) return;
            const bool in_prefix = j < of_prefix;
            const int8_t *codes = in_prefix ? block_codes<D>(prefix, prefix_head, j, 0) : block_codes<D>(cache, own_head, j - of_prefix, 0);
            const v4i *k = reinterpret_cast<const v4i *>(codes), *v = reinterpret_cast<const v4i *>(codes + kBlock * D);
#pragma unroll
            for (int i = 0; i < PIECES; ++i) {
                const int x = t + T * i;
                if (COUNT % T != 0 && x >= COUNT) break;
                kraw[i] = k[x];
                vraw[i] = v[x];
            }
        };
        auto scale_of_block = [&](int j) {
            if (j >= end || unfinished(j)) return;
            sc = *reinterpret_cast<const float2 *>(j < of_prefix ? prefix.scales + (prefix_head * prefix.blocks + j) * 2 : cache.scales + (own_head * cache.blocks + j - of_prefix) * 2);
        };
        auto keep = [&](int j) {
            if (j >= end) return;
            uint8_t *kt = lds + (j & 1) * BUF;
            if (!unfinished(j)) {
                keep_codes<D, T>(kt, kraw, vraw);
                return;
            }
            const bool in_prefix = j < of_prefix;
            const __half *tail = in_prefix ? prefix_tail : own_tail;
            if (keep_tail<D, T>(kt, tail, tail + kBlock * D, in_prefix ? prefix_rest : own_rest)) not_finite[in_prefix ? 0 : 1] = 1;
        };
        TileSums<D, false> sums;
        __syncthreads();                                              // (the tile before has been read, and its flags)
        if (t < 2) not_finite[t] = 0;
        __syncthreads();
        fetch(first);
        keep(first);
        scale_of_block(first);
        for (int j = first; j < end; ++j) {
            fetch(j + 1);
            const bool as_it_is = unfinished(j);
            const float sk = as_it_is || sc.x == 0.f ? per_d : sc.x * per_d, sv = as_it_is ? 1.f : sc.y;
            scale_of_block(j + 1);
            lds_barrier();
            const int at_own = (j - of_prefix) * kBlock;              // (the prefix: all of its positions)
            if (at_own <= wave_last)
                sums.add(lds + (j & 1) * BUF, qf, sk, sv, at_own < 0 ? as_it_is : at_own + kBlock - 1 > wave_first, at_own < 0 ? prefix_rest - 1 : sees - at_own);
            keep(j + 1);
        }
        sums.lrun += __shfl_xor(sums.lrun, 32);
        __syncthreads();
        const bool odd_prefix = not_finite[0], odd_own = not_finite[1];      // (of blocks in this range)
        const bool whole = from == 0 && upto == nominal;
        if (from > 0) {
            const int begun = (int)(tile_start / range), ended = (int)((tile_start + nominal - 1) / range);
            if (begun == w - 1) slot = {b, kh, tile, begun, ended - begun + 1, {0, 0, 0}};
        }
        if (mine >= n_rows) continue;
        const int odd_rows = odd_own ? sees - (own_unfinished - of_prefix) * kBlock + 1 : 0;
        if (whole) {
            __half *to = a.O + (int64_t)(sp.row + query) * a.ldo + (int64_t)head * D;
            sums.write_rows(to);
            if (odd_prefix) add_odd<D>(to, prefix_tail + kBlock * D, prefix_rest);
            if (odd_own) add_odd<D>(to, own_tail + kBlock * D, odd_rows);
        } else {
            const int64_t place = ((int64_t)w * 2 + (from > 0 ? 0 : 1)) * TILE + wave * 32 + c;
            sums.write_part(a.ml + place, a.o + place * D);
            if (odd_prefix) add_odd<D>(a.o + place * D, prefix_tail + kBlock * D, prefix_rest);
            if (odd_own) add_odd<D>(a.o + place * D, own_tail + kBlock * D, odd_rows);
        }
    }
    if (t == 0) a.slots[w] = slot;
}

// The shares of a tile that begins in one workgroup's range and ends in another's: two workgroups for each boundary that is a tile's first.
// 15 us for some 500 boundaries: two shares of 66 KB each, 67 MB in all, just written.
template <int D>
__global__ __launch_bounds__(256) void cache8_long_join_kernel(const LongArgs a)
{
    constexpr int LANES = D / 4, EACH = 256 / LANES, ROWS = 64;
    const int w = blockIdx.y, t = threadIdx.x, lane = t % LANES, G = a.H / a.cache.kv_heads;
    const LongSlot slot = a.slots[w];
    if (slot.count == 0) return;
    const Span sp = span_of(a.starts, a.past, slot.b, a.rows, a.max_new, a.cache.blocks * kBlock);
    auto place_of = [&](int i, int row) { return ((int64_t)(slot.first + i) * 2 + (i == 0 ? 1 : 0)) * 128 + row; };
    // (all of a thread's rows side by side: a share costs one wait for memory)
    constexpr int ROUNDS = ROWS / EACH;
    const int row0 = (int)blockIdx.x * ROWS + t / LANES;
    float top[ROUNDS], sum[ROUNDS];
    v4f o[ROUNDS];
#pragma unroll
    for (int k = 0; k < ROUNDS; ++k) top[k] = -INFINITY, sum[k] = 0.f, o[k] = v4f{0.f, 0.f, 0.f, 0.f};
    for (int i = 0; i < slot.count; ++i) {
        const float2 *ml = a.ml + place_of(i, row0);
#pragma unroll
        for (int k = 0; k < ROUNDS; ++k) top[k] = fmaxf(top[k], ml[k * EACH].x);         // (rows behind the last hold what they like)
    }
    for (int i = 0; i < slot.count; ++i) {
        const int64_t place = place_of(i, row0);
        float2 ml[ROUNDS];
        v4f x[ROUNDS];
#pragma unroll
        for (int k = 0; k < ROUNDS; ++k) {
            ml[k] = a.ml[place + k * EACH];
            x[k] = *reinterpret_cast<const v4f *>(a.o + (place + k * EACH) * D + lane * 4);
        }
#pragma unroll
        for (int k = 0; k < ROUNDS; ++k) {
            const float f = exp2f(ml[k].x - top[k]);                  // (no score above minus infinity anywhere: 0 / 0)
            sum[k] += f * ml[k].y;
#pragma unroll
            for (int e = 0; e < 4; ++e) o[k][e] += fabsf(x[k][e]) < INFINITY ? f * x[k][e] : x[k][e];        // (an infinite value stays one however small its weight)
        }
    }
#pragma unroll
    for (int k = 0; k < ROUNDS; ++k) {
        const int pair = slot.tile + row0 + k * EACH;
        if (pair >= sp.n * G) break;
        const float norm = 1.f / sum[k];
        union { __half h[4]; v2u v; } out;
#pragma unroll
        for (int e = 0; e < 4; ++e) out.h[e] = __float2half_rn(o[k][e] * norm);
        *reinterpret_cast<v2u *>(a.O + (int64_t)(sp.row + pair / G) * a.ldo + (int64_t)(slot.kh * G + pair % G) * D + lane * 4) = out.v;
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
template <int D, Part PART>
__global__ __launch_bounds__(64 * kFewRowsWaves, 2) void cache8_few_rows_kernel(const __half *__restrict__ Q, int64_t ldq, const int32_t *__restrict__ starts,
                                                                                const int32_t *__restrict__ past, int rows, int max_new, int H,
                                                                                const Cache8View cache, __half *__restrict__ O, int64_t ldo, int tiles,
                                                                                const Parts parts)
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
        if constexpr (PART == Part::Whole) nan_rows<D>(O, ldo, sp.row, (int64_t)sp.n * G, G, kh, number, tiles, 16);
        return;
    }
    if (PART == Part::Own && !in_its_group(starts, b, parts.width, sp)) return;
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
    const float taken = PART != Part::Whole && top == -INFINITY ? 0.f : top;
    v4f o = {0.f, 0.f, 0.f, 0.f};
    for (int w = 0; w < waves; ++w) {
        const float f = exp2f(lds.m[w][row] - taken);
        sum += f * lds.l[w][row];
        o += f * *reinterpret_cast<const v4f *>(&lds.u.o[w][row][col]);
    }
    if constexpr (PART != Part::Whole) {
        const int64_t pair = parts.prefix_shares * parts.pairs + (int64_t)(sp.row + of) * H + kh * G + tile + row - of * G;
        if (odd) {                                                    // (as below)
#pragma unroll
            for (int i = 0; i < 4; ++i)
#pragma unroll 1
                for (int s = 0; s <= sp.past + of - tail_block * kBlock; ++s) {
                    const float v = __half2float(tail_v[s * D + col + i]);
                    if (!(fabsf(v) <= 65504.f)) o[i] += v;
                }
        }
        if (col == 0) parts.ml[pair] = {top, sum};
        *reinterpret_cast<v4f *>(parts.o + pair * D + col) = o;
        return;
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

// Few rows behind a prefix that is not long: the same over the prefix's blocks and the sequence's own, which are dealt out together; no parts.  8 x up to 20 rows of
// 12 heads of 64 behind 148 positions in 5 to 7 us, latency: lengths, codes and queries, a product, the joining of the wavefronts.  Part::Own: own positions alone, as a part.
template <int D, int WAVES, int TAILS>
struct ShortLds {
    __attribute__((aligned(16))) union {
        unsigned short v[TAILS][D][kBlock + 8];  // unfinished values: of the prefix (where it takes part), of the sequence
        float o[WAVES][16][D + 4];
    } u;
    float m[WAVES][16], l[WAVES][16];
    int not_finite[2];
};
struct ShortArgs {
    const __half *Q;
    int64_t ldq;
    const int32_t *starts, *past;
    int rows, max_new, H;
    Cache8View cache, prefix;
    Parts parts;                 // (width and lengths)
    __half *O;
    int64_t ldo;
    int tiles;
};
template <int D, int WAVES, Part PART>
__global__ __launch_bounds__(64 * WAVES, D == 64 ? 4 : 2) void cache8_short_kernel(const ShortArgs a)
{
    constexpr int C = D / 64, DT = D / 16, T = 64 * WAVES, OF_TAIL = kBlock / 4 * D / 8, TAILS = PART == Part::Own ? 1 : 2, UNITS = (TAILS * OF_TAIL + T - 1) / T;
    extern __shared__ __attribute__((aligned(16))) uint8_t raw_lds[];
    using Lds = ShortLds<D, WAVES, TAILS>;
    Lds &lds = *reinterpret_cast<Lds *>(raw_lds);
    const Cache8View &cache = a.cache, &prefix = a.prefix;
    const int pairs = cache.kv_heads * cache.batch, id = blockIdx.x, pair = id % pairs, number = id / pairs;
    const int b = pair / cache.kv_heads, kh = pair % cache.kv_heads, group = PART == Part::Own ? 0 : b / a.parts.width;
    const int t = threadIdx.x, l = t & 63, wave = __builtin_amdgcn_readfirstlane(t >> 6), r = l & 15, g = l >> 4, G = a.H / cache.kv_heads;
    Member member;
    if constexpr (PART == Part::Own) {
        const Span own = span_of(a.starts, a.past, b, a.rows, a.max_new, cache.blocks * kBlock);
        member = {own, own.n > 0 && in_its_group(a.starts, b, a.parts.width, own), own.fits, 0};
    } else {
        member = member_of(a.starts, a.past, b, a.rows, a.max_new, cache.blocks * kBlock, prefix.blocks * kBlock, a.parts);
    }
    if (!member.rows) return;
    const Span &sp = member.sp;
    if (!member.fits) {
        if constexpr (PART == Part::Whole) nan_rows<D>(a.O, a.ldo, sp.row, (int64_t)sp.n * G, G, kh, number, a.tiles, 16);
        return;
    }
    const int n_rows = sp.n * G, tile = (a.tiles - 1 - number) * 16;
    if (tile >= n_rows) return;
    const int mine = min(tile + r, n_rows - 1), query = mine / G, first_sees = sp.past + tile / G, sees = sp.past + query;
    const int last = sp.past + (min(tile + 16, n_rows) - 1) / G, end = sp.past + sp.n;
    // finished blocks of the prefix, then own ones that some row sees; then the unfinished ones
    const int of_prefix = member.length / kBlock, finished = of_prefix + min(last / kBlock + 1, end / kBlock);
    const int prefix_rest = member.length % kBlock, own_rest = last / kBlock == end / kBlock ? end % kBlock : 0;
    auto rest = [&](int x) { return PART != Part::Own && x == 0 ? prefix_rest : own_rest; };
    const int64_t heads[2] = {(int64_t)group * prefix.kv_heads + kh, (int64_t)b * cache.kv_heads + kh};
    const __half *const prefix_tail = prefix.tail + heads[0] * 2 * kBlock * D, *const own_tail = cache.tail + heads[1] * 2 * kBlock * D;
    auto tail = [&](int x) { return PART != Part::Own && x == 0 ? prefix_tail : own_tail; };
    v4i kraw[4 * C], vraw[DT];
    float2 sc = {0.f, 0.f};
    auto codes_of = [&](int j, int values) {
        return reinterpret_cast<const v4i *>(PART != Part::Own && j < of_prefix ? block_codes<D>(prefix, heads[0], j, values) : block_codes<D>(cache, heads[1], j - of_prefix, values)) + l;
    };
    auto fetch_keys = [&](int j) {
        if (j >= finished) return;
        sc = *reinterpret_cast<const float2 *>(PART != Part::Own && j < of_prefix ? prefix.scales + (heads[0] * prefix.blocks + j) * 2 : cache.scales + (heads[1] * cache.blocks + j - of_prefix) * 2);
        const v4i *k = codes_of(j, 0);
#pragma unroll
        for (int i = 0; i < 4 * C; ++i) kraw[i] = k[i * 64];
    };
    auto fetch_values = [&](int j) {
        if (j >= finished) return;
        const v4i *v = codes_of(j, 1);
#pragma unroll
        for (int i = 0; i < DT; ++i) vraw[i] = v[i * 64];
    };
    // unfinished values, 4 positions of 8 columns at a time
    v4i tv[UNITS][4];
#pragma unroll
    for (int i = 0; i < UNITS; ++i) {
        const int u = t + i * T, x = u / OF_TAIL + 2 - TAILS, s = u % OF_TAIL / (D / 8) * 4, col = u % (D / 8) * 8;
#pragma unroll
        for (int p = 0; p < 4; ++p) {
            tv[i][p] = v4i{0, 0, 0, 0};
            if (x < 2 && s + p < rest(x)) tv[i][p] = *reinterpret_cast<const v4i *>(tail(x) + (kBlock + s + p) * D + col);
        }
    }
    fetch_keys(wave);
    fetch_values(wave);
    v8h q[2 * C];
    const __half *from = a.Q + (int64_t)(sp.row + query) * a.ldq + (int64_t)(kh * G + mine - query * G) * D;
#pragma unroll
    for (int m = 0; m < 2 * C; ++m) q[m] = *reinterpret_cast<const v8h *>(from + 64 * (m >> 1) + 16 * g + 8 * (m & 1));
    if (t < 2) lds.not_finite[t] = 0;
    __syncthreads();
#pragma unroll
    for (int i = 0; i < UNITS; ++i) {
        const int u = t + i * T, x = u / OF_TAIL + 2 - TAILS, s = u % OF_TAIL / (D / 8) * 4, col = u % (D / 8) * 8, at = value_slot(s);
        if (x >= 2 || rest(x) == 0) continue;
        if (s >= rest(x)) {                                           // (252 sequences of 64 heads, 4 rows behind 30 positions: 66.5 us; with these among the others 71.5)
#pragma unroll
            for (int e = 0; e < 8; ++e) *reinterpret_cast<v2u *>(&lds.u.v[x - 2 + TAILS][col + e][value_place(col + e, at)]) = v2u{0, 0};
            continue;
        }
        bool odd = false;
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            unsigned w[4];
#pragma unroll
            for (int p = 0; p < 4; ++p) {
                w[p] = (unsigned)tv[i][p][e >> 1] >> (16 * (e & 1)) & 0xffffu;
                if ((w[p] & 0x7fffu) >= 0x7c00u) w[p] = 0, odd = true;      // comes back at the end, to the rows that see it
            }
            *reinterpret_cast<v2u *>(&lds.u.v[x - 2 + TAILS][col + e][value_place(col + e, at)]) = v2u{w[0] | w[1] << 16, w[2] | w[3] << 16};
        }
        if (odd) lds.not_finite[x] = 1;
    }
    __syncthreads();
    WaveSums<D> sums;
    int j = wave;
    for (; j < finished; j += WAVES) {
        const float2 scale = sc;
        const int at_own = (j - of_prefix) * kBlock;
        sums.add(
            q, scale.x, scale.y, at_own >= 0 && at_own + kBlock - 1 > first_sees, sees - at_own,
            [&](int T4, int m) {
                const v4i w = kraw[T4 * C + (m >> 1)];
                return (m & 1) ? halves_of(w[2], w[3]) : halves_of(w[0], w[1]);
            },
            [&](int i, int n) { return halves_of(vraw[i][2 * n], vraw[i][2 * n + 1]); }, [&] { fetch_keys(j + WAVES); });
        fetch_values(j + WAVES);
    }
    j -= finished;                                                    // the unfinished ones go to the wavefronts whose turn it is
    int which = prefix_rest > 0 ? 0 : 1, left = (prefix_rest > 0) + (own_rest > 0);
    if (j == 1 && left == 2) which = 1;
    if (j < left) {
        const __half *keys = tail(which);
        sums.add(
            q, 1.f, 1.f, true, which == 0 ? prefix_rest - 1 : min(sees - end / kBlock * kBlock, own_rest - 1),
            [&](int T4, int m) { return *reinterpret_cast<const v8h *>(keys + min(16 * T4 + r, rest(which) - 1) * D + 64 * (m >> 1) + 16 * g + 8 * (m & 1)); },
            [&](int i, int n) { return *reinterpret_cast<const v8h *>(&lds.u.v[which - 2 + TAILS][16 * i + r][value_place(16 * i + r, 32 * n + 8 * g)]); }, [] {});
    }
    sums.l += __shfl_xor(sums.l, 16);
    sums.l += __shfl_xor(sums.l, 32);
    __syncthreads();                                                  // the tails' rows have been read
#pragma unroll
    for (int i = 0; i < DT; ++i) *reinterpret_cast<v4f *>(&lds.u.o[wave][r][16 * i + 4 * g]) = sums.o[i] * sums.unit.unit;
    if (g == 0) {
        lds.m[wave][r] = sums.m;
        lds.l[wave][r] = sums.l;
    }
    __syncthreads();
    const int waves = min(finished + left, WAVES), col = t % (D / 4) * 4;          // four columns of a row
    for (int row = t / (D / 4); row < 16 && tile + row < n_rows; row += T / (D / 4)) {
        const int of = (tile + row) / G;
        float top = -INFINITY, sum = 0.f;
        for (int w = 0; w < waves; ++w) top = fmaxf(top, lds.m[w][row]);
        const float taken = PART == Part::Own && top == -INFINITY ? 0.f : top;
        v4f o = {0.f, 0.f, 0.f, 0.f};
        for (int w = 0; w < waves; ++w) {
            const float f = exp2f(lds.m[w][row] - taken);
            sum += f * lds.l[w][row];
            o += f * *reinterpret_cast<const v4f *>(&lds.u.o[w][row][col]);
        }
        if constexpr (PART == Part::Own) {
            const int64_t place = a.parts.prefix_shares * a.parts.pairs + (int64_t)(sp.row + of) * a.H + kh * G + tile + row - of * G;
            if (lds.not_finite[1]) {                                  // (as below)
#pragma unroll
                for (int i = 0; i < 4; ++i)
#pragma unroll 1
                    for (int s = 0; s <= sp.past + of - end / kBlock * kBlock; ++s) {
                        const float v = __half2float(own_tail[kBlock * D + s * D + col + i]);
                        if (!(fabsf(v) <= 65504.f)) o[i] += v;
                    }
            }
            if (col == 0) a.parts.ml[place] = {top, sum};
            *reinterpret_cast<v4f *>(a.parts.o + place * D + col) = o;
            continue;
        }
        const float norm = 1.f / sum;
        union { __half h[4]; v2u v; } out;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            float y = o[i] * norm;
#pragma unroll 1
            for (int x = 0; x < 2; ++x) {
                if (!lds.not_finite[x]) continue;                         // infinities and NaN among a tail's values that this row sees
                y = __half2float(__float2half_rn(y));
                const int seen = x == 0 ? prefix_rest : sp.past + of - end / kBlock * kBlock + 1;
#pragma unroll 1
                for (int s = 0; s < seen; ++s) {
                    const float v = __half2float(tail(x)[kBlock * D + s * D + col + i]);
                    if (!(fabsf(v) <= 65504.f)) y += v;
                }
            }
            out.h[i] = __float2half_rn(y);
        }
        *reinterpret_cast<v2u *>(a.O + (int64_t)(sp.row + of) * a.ldo + (int64_t)(kh * G + tile + row - of * G) * D + col) = out.v;
    }
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
    // behind a shared prefix
    Cache8View prefix;
    int prefix_tiles;                                         // of a group and key head, 16 rows each
    Parts parts;
    __half *q_out;                                            // receives the rotated queries, [batch][H D], where not null
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

// 16 (row, head) pairs of a group and key head over a share of the group's prefix, whose blocks are dealt to the wavefronts as in the decode
// kernel.  ROTATE: Q are the fused rows of the decode call, rotated here.
struct PrefixTile {
    const __half *Q;
    int64_t ld;
    const int32_t *starts, *pos;
    int rows, max_new, H;
};
template <int D, bool ROTATE>
__device__ __forceinline__ void prefix_tile(DecodeLds<D> &lds, const PrefixTile &a, const Cache8View &prefix, const Parts &parts, const RopeFreq &freq,
                                            int group, int kh, int tile, int share)
{
    constexpr int HALF = D / 2, C = D / 64, T = 64 * kDecodeWaves, DT = D / 16;
    const int t = threadIdx.x, l = t & 63, wave = __builtin_amdgcn_readfirstlane(t >> 6), r = l & 15, g = l >> 4, G = a.H / prefix.kv_heads;
    const GroupRows rows = group_rows(a.starts, group, parts.width, a.rows, a.max_new);
    const int length = parts.length[group], pair0 = tile * 16, pairs = min(16, rows.n * G - pair0);
    const PrefixShare own = prefix_share(length, prefix.blocks * kBlock, parts.prefix_shares, share);
    if (pairs <= 0 || own.first >= own.end) return;
    const int64_t head = (int64_t)group * prefix.kv_heads + kh;
    const int tail_block = length / kBlock, tail_rows = length % kBlock;
    const bool has_tail = own.end - 1 == tail_block;
    const __half *tail_k = prefix.tail + head * 2 * kBlock * D, *tail_v = tail_k + kBlock * D;
    v4i kraw[4 * C], vraw[DT];
    float2 sc = {0.f, 0.f};
    auto fetch_keys = [&](int j) {
        if (j >= own.end || j == tail_block) return;
        sc = reinterpret_cast<const float2 *>(prefix.scales)[head * prefix.blocks + j];
        const v4i *k = reinterpret_cast<const v4i *>(block_codes<D>(prefix, head, j, 0)) + l;
#pragma unroll
        for (int i = 0; i < 4 * C; ++i) kraw[i] = k[i * 64];
    };
    auto fetch_values = [&](int j) {
        if (j >= own.end || j == tail_block) return;
        const v4i *v = reinterpret_cast<const v4i *>(block_codes<D>(prefix, head, j, 1)) + l;
#pragma unroll
        for (int i = 0; i < DT; ++i) vraw[i] = v[i * 64];
    };
    constexpr int UNITS = kBlock * D / 8 / T;                         // 8 columns of a row of the tail each
    v4i tk[UNITS], tv[UNITS];
    if (has_tail) {
#pragma unroll
        for (int i = 0; i < UNITS; ++i) {
            const int u = t + i * T, s = u / (D / 8), x = (u % (D / 8)) * 8;
            tk[i] = tv[i] = v4i{0, 0, 0, 0};
            if (s < tail_rows) {
                tk[i] = *reinterpret_cast<const v4i *>(tail_k + s * D + x);
                tv[i] = *reinterpret_cast<const v4i *>(tail_v + s * D + x);
            }
        }
    }
    fetch_keys(own.first + wave);
    fetch_values(own.first + wave);
    v8h qf[2 * C];
    auto query = [&](int pair) { return a.Q + (int64_t)(rows.row + (pair0 + pair) / G) * a.ld + (int64_t)(kh * G + (pair0 + pair) % G) * D; };
    if constexpr (ROTATE) {
        __half q[16 * HALF / T][2];
#pragma unroll
        for (int i = 0; i < 16 * HALF / T; ++i) {
            const int u = t + i * T;
            const __half *from = query(min(u / HALF, pairs - 1)) + u % HALF;
            q[i][0] = from[0];
            q[i][1] = from[HALF];
        }
        // angles of the tile's rows, once for the heads of each
        double2 *angles = reinterpret_cast<double2 *>(&lds.u);        // [row][HALF]
        static_assert(sizeof(lds.u) >= 16 * HALF * sizeof(double2), "angles of sixteen rows");
        const int first = pair0 / G, count = (pair0 + pairs - 1) / G - first + 1;
        for (int u = t; u < count * HALF; u += T) {
            double2 x;
            sincos_of((double)a.pos[rows.row + first + u / HALF] * freq.f[u % HALF], x.y, x.x);
            angles[u] = x;
        }
        __syncthreads();
#pragma unroll
        for (int i = 0; i < 16 * HALF / T; ++i) {
            const int u = t + i * T, pair = u / HALF, x = u % HALF;
            const double2 w = angles[((pair0 + min(pair, pairs - 1)) / G - first) * HALF + x];
            __half lo, hi;
            rotate_pair(q[i][0], q[i][1], w.x, w.y, lo, hi);
            lds.q[pair][x] = (_Float16)__half2float(lo);
            lds.q[pair][x + HALF] = (_Float16)__half2float(hi);
        }
        __syncthreads();
#pragma unroll
        for (int m = 0; m < 2 * C; ++m) qf[m] = *reinterpret_cast<const v8h *>(&lds.q[r][64 * (m >> 1) + 16 * g + 8 * (m & 1)]);
    } else {
        const __half *from = query(min(r, pairs - 1));
#pragma unroll
        for (int m = 0; m < 2 * C; ++m) qf[m] = *reinterpret_cast<const v8h *>(from + 64 * (m >> 1) + 16 * g + 8 * (m & 1));
    }
    if (has_tail) {
        if (t == 0) lds.arrived = 0;                                  // values that are not finite: come back at the end
        __syncthreads();
        bool odd = false;
#pragma unroll
        for (int i = 0; i < UNITS; ++i) {
            const int u = t + i * T, s = u / (D / 8), x = (u % (D / 8)) * 8, at = value_slot(s);
            *reinterpret_cast<v4i *>(&lds.u.tail.k[s][x]) = tk[i];
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                unsigned short w = (unsigned short)((unsigned)tv[i][e >> 1] >> (16 * (e & 1)));
                if ((w & 0x7fffu) >= 0x7c00u) w = 0, odd = true;
                lds.u.tail.v[x + e][value_place(x, at)] = w;
            }
        }
        if (odd) lds.arrived = 1;
        __syncthreads();
    }
    WaveSums<D> sums;
    int j = own.first + wave;
    for (; j < own.end && j < tail_block; j += kDecodeWaves) {        // (the unfinished block behind the loop: inside it would cost 85 registers)
        const float2 scale = sc;
        sums.add(
            qf, scale.x, scale.y, false, 0,
            [&](int T4, int m) {
                const v4i w = kraw[T4 * C + (m >> 1)];
                return (m & 1) ? halves_of(w[2], w[3]) : halves_of(w[0], w[1]);
            },
            [&](int i, int n) { return halves_of(vraw[i][2 * n], vraw[i][2 * n + 1]); }, [&] { fetch_keys(j + kDecodeWaves); });
        fetch_values(j + kDecodeWaves);
    }
    if (j < own.end)
        sums.add(
            qf, 1.f, 1.f, true, tail_rows - 1,
            [&](int T4, int m) { return *reinterpret_cast<const v8h *>(&lds.u.tail.k[16 * T4 + r][64 * (m >> 1) + 16 * g + 8 * (m & 1)]); },
            [&](int i, int n) { return *reinterpret_cast<const v8h *>(&lds.u.tail.v[16 * i + r][value_place(16 * i + r, 32 * n + 8 * g)]); }, [] {});
    sums.l += __shfl_xor(sums.l, 16);
    sums.l += __shfl_xor(sums.l, 32);
    const bool odd = has_tail && lds.arrived;
    __syncthreads();                                                  // the tail's rows have been read
    const int waves = min(own.end - own.first, kDecodeWaves);
    if (wave < waves) {
#pragma unroll
        for (int i = 0; i < DT; ++i) *reinterpret_cast<v4f *>(&lds.u.o[wave][r][16 * i + 4 * g]) = sums.o[i] * sums.unit.unit;
        if (g == 0) {
            lds.m[wave][r] = sums.m;
            lds.l[wave][r] = sums.l;
        }
    }
    __syncthreads();
    for (int u = t; u < pairs * (D / 4); u += T) {
        const int pair = u / (D / 4), col = u % (D / 4) * 4;
        float top = -INFINITY, sum = 0.f;
        for (int w = 0; w < waves; ++w) top = fmaxf(top, lds.m[w][pair]);
        const float taken = top == -INFINITY ? 0.f : top;             // (no score above it: nothing is added to the other parts)
        v4f o = {0.f, 0.f, 0.f, 0.f};
        for (int w = 0; w < waves; ++w) {
            const float f = exp2f(lds.m[w][pair] - taken);
            sum += f * lds.l[w][pair];
            o += f * *reinterpret_cast<const v4f *>(&lds.u.o[w][pair][col]);
        }
        if (odd) {
#pragma unroll
            for (int i = 0; i < 4; ++i)
#pragma unroll 1
                for (int s = 0; s < tail_rows; ++s) {
                    const float v = __half2float(tail_v[s * D + col + i]);
                    if (!(fabsf(v) <= 65504.f)) o[i] += v;
                }
        }
        const int64_t at = share * parts.pairs + (int64_t)(rows.row + (pair0 + pair) / G) * a.H + kh * G + (pair0 + pair) % G;
        if (col == 0) parts.ml[at] = {top, sum};
        *reinterpret_cast<v4f *>(parts.o + at * D + col) = o;
    }
}
template <int D>
__global__ __launch_bounds__(64 * kDecodeWaves, 2) void cache8_prefix_kernel(const PrefixTile a, const Cache8View prefix, const Parts parts, int tiles)
{
    __shared__ DecodeLds<D> lds;
    prefix_tile<D, false>(lds, a, prefix, parts, RopeFreq{}, blockIdx.z / tiles, blockIdx.y, blockIdx.z % tiles, blockIdx.x);
}

// SHARED: the own positions of sequences that share a prefix, and in the workgroups in front of them (where there are any) the prefix; all of them leave parts.
// Three workgroups to a compute unit (4 x 32 rows of 32 heads over 8 behind 1000 positions 26 us, with two 32).
template <int D, bool SHARED>
__global__ __launch_bounds__(64 * kDecodeWaves, SHARED ? 3 : 2) void cache8_decode_kernel(const DecodeArgs a)
{
    constexpr int HALF = D / 2, C = D / 64, T = 64 * kDecodeWaves, DT = D / 16;
    __shared__ DecodeLds<D> lds;
    const Cache8View &cache = a.cache;
    int share = blockIdx.x, kh = blockIdx.y / a.chunks, chunk = blockIdx.y % a.chunks, b = blockIdx.z;
    if constexpr (SHARED) {                                           // (in one dimension: a workgroup without work takes 9 ns to come and go)
        int id = blockIdx.x;
        const int items = a.prefix.batch * cache.kv_heads * a.parts.prefix_shares, behind = items * a.prefix_tiles;
        if (id < behind) {                                            // tiles of one share behind one L2 where the shares fill all of them
            const int item = id % items;
            prefix_tile<D, true>(lds, PrefixTile{a.QKV, a.ld, nullptr, a.pos, cache.batch, 1, a.H}, a.prefix, a.parts, a.freq,
                                 item / a.parts.prefix_shares / cache.kv_heads, item / a.parts.prefix_shares % cache.kv_heads, id / items, item % a.parts.prefix_shares);
            return;
        }
        id -= behind;
        share = id % a.shares;
        id /= a.shares;
        chunk = id % a.chunks;
        kh = id / a.chunks % cache.kv_heads;
        b = id / a.chunks / cache.kv_heads;
    }
    const int t = threadIdx.x, l = t & 63, wave = __builtin_amdgcn_readfirstlane(t >> 6), r = l & 15, g = l >> 4;
    const int first_head = kh * a.G + chunk * 16, heads = min(16, a.G - chunk * 16);
    const int past = a.past[b];
    if (past < 0) return;
    const __half *row = a.QKV + (int64_t)b * a.ld;
    __half *out = a.O + (int64_t)b * a.ldo + (int64_t)first_head * D;
    if (past >= cache.blocks * kBlock) {                              // no room: nothing is appended, and the outputs say so
        if (SHARED) return;                                           // (cache8_join_kernel sees to that)
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
    // values of the rows that are missing: zero, sixteen bytes at a time (242 sequences of 32 heads, a first own row behind 17 positions: 63 us, with zeros
    // taken through the transposition below 73)
    if (has_last && slot < kBlock - 1)
#pragma unroll
        for (int i = 0; i < D * kBlock / 8 / T; ++i) *reinterpret_cast<v4i *>(&lds.u.tail.v[(t + i * T) / 8][(t + i * T) % 8 * 8]) = v4i{0, 0, 0, 0};
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
    if (SHARED && a.q_out && begin == 0)
        for (int u = t; u < heads * (D / 8); u += T)
            *reinterpret_cast<v8h *>(a.q_out + ((int64_t)b * a.H + first_head) * D + u * 8) = *reinterpret_cast<const v8h *>(&lds.q[0][0] + u * 8);
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
            if (s >= slot) break;                                     // (keys behind the new row: scores that are masked)
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
    if (begin + wave < stop) {
#pragma unroll
        for (int i = 0; i < DT; ++i)
#pragma unroll
            for (int e = 0; e < 4; ++e) lds.u.o[wave][r][16 * i + 4 * g + e] = own.o[i][e] * own.unit.unit;
    }
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
        const float from = top == -INFINITY && (SHARED || active > 1) ? 0.f : top;
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
    if constexpr (SHARED) {
        const int64_t pair = (a.parts.prefix_shares + share) * a.parts.pairs + (int64_t)b * a.H + first_head;
        for (int u = t; u < heads * D; u += T) {
            float top, sum;
            a.parts.o[pair * D + u] = merged(u / D, u % D, top, sum);
            if (u % D == 0) a.parts.ml[pair + u / D] = {top, sum};
        }
        return;
    }
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

// ---------------------------------------------------------------- the parts in one

// The parts of a (row, head) pair: D / 4 lanes with four columns each; the lanes share out the parts' maxima and sums first.  SPLIT groups of such
// lanes deal out a pair's parts, where there are many.  One workgroup per sequence and 1024 / D / SPLIT of its pairs.
constexpr int kMostParts = 128;                                       // of a pair
struct JoinArgs {
    const int32_t *starts, *past;                             // starts null: one row per sequence
    int rows, max_new, H, capacity, prefix_capacity;
    int own_shares, own_each;                                 // as in DecodeArgs; one share where there are prompts
    Parts parts;
    __half *O;
    int64_t ldo;
};
template <int D, int SPLIT>
__global__ __launch_bounds__(256) void cache8_join_kernel(const JoinArgs a)
{
    constexpr int LANES = D / 4, EACH = 256 / LANES / SPLIT, KEPT = kMostParts / LANES;
    __shared__ __attribute__((aligned(16))) float sums[SPLIT > 1 ? SPLIT * EACH * D : 4];
    const int b = blockIdx.y, t = threadIdx.x, lane = t % LANES;
    const Member member = member_of(a.starts, a.past, b, a.rows, a.max_new, a.capacity, a.prefix_capacity, a.parts);
    if (!member.rows) return;
    const Span &sp = member.sp;
    const bool fits = member.fits;
    const PrefixShare prefix = prefix_share(member.length, a.prefix_capacity, a.parts.prefix_shares, 0);
    const int last = sp.past / kBlock, own_each = max(a.own_each, (last + a.own_shares) / a.own_shares);
    const int own = a.starts ? 1 : (last + own_each) / own_each, all = prefix.active + own;
    auto part_of = [&](int i) { return i < prefix.active ? i : a.parts.prefix_shares + i - prefix.active; };
    const int64_t pairs = (int64_t)sp.n * a.H;
    const int turn = SPLIT > 1 ? t / LANES / EACH : 0;                // the groups of a pair take every SPLIT-th four parts
    for (int64_t p0 = (int64_t)blockIdx.x * EACH; p0 < pairs; p0 += (int64_t)gridDim.x * EACH) {
        const int64_t p = p0 + t / LANES % EACH;
        if (SPLIT == 1 && p >= pairs) break;                          // (otherwise a workgroup has one round, and its last pairs may be none)
        const bool is_pair = p < pairs;
        const int64_t row = sp.row + p / a.H, head = p % a.H, at = row * a.H + head;
        __half *to = a.O + row * a.ldo + head * D + lane * 4;
        union { __half h[4]; v2u v; } out;
        if (!fits) {
            out.v = v2u{0x7e007e00u, 0x7e007e00u};
            if (is_pair && turn == 0) *reinterpret_cast<v2u *>(to) = out.v;
            continue;
        }
        float2 ml[KEPT];
        float top = -INFINITY, sum = 0.f;
#pragma unroll
        for (int k = 0; k < KEPT; ++k) {
            const int i = k * LANES + lane;
            ml[k] = float2{-INFINITY, 0.f};
            if (i < all && is_pair) ml[k] = a.parts.ml[part_of(i) * a.parts.pairs + at];
            top = fmaxf(top, ml[k].x);
        }
#pragma unroll
        for (int i = LANES / 2; i > 0; i >>= 1) top = fmaxf(top, __shfl_xor(top, i));
#pragma unroll
        for (int k = 0; k < KEPT; ++k) {
            ml[k].x = k * LANES + lane < all ? exp2f(ml[k].x - top) : 0.f;             // (no score above minus infinity anywhere: 0 / 0)
            sum += k * LANES + lane < all ? ml[k].x * ml[k].y : 0.f;
        }
#pragma unroll
        for (int i = LANES / 2; i > 0; i >>= 1) sum += __shfl_xor(sum, i);
        v4f o = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int k = 0; k < KEPT; ++k) {
            const int n = min(all - k * LANES, LANES);
            for (int i0 = 4 * turn; i0 < n && is_pair; i0 += 4 * SPLIT) {                       // four of them asked for at a time (the last one again where there are fewer, for nothing)
                v4f x[4];
                float f[4];
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const int of = min(i0 + i, n - 1);
                    f[i] = i0 + i < n ? __shfl(ml[k].x, of, LANES) : 0.f;
                    x[i] = *reinterpret_cast<const v4f *>(a.parts.o + (part_of(k * LANES + of) * a.parts.pairs + at) * D + lane * 4);
                }
#pragma unroll
                for (int i = 0; i < 4; ++i)
#pragma unroll
                    for (int e = 0; e < 4; ++e) o[e] += fabsf(x[i][e]) < INFINITY ? f[i] * x[i][e] : x[i][e];      // (an infinite value stays one however small its weight)
            }
        }
        if constexpr (SPLIT > 1) {
            *reinterpret_cast<v4f *>(sums + t * 4) = o;               // [group of a pair][pair][column]
            __syncthreads();
            if (turn > 0 || !is_pair) return;
            for (int x = 1; x < SPLIT; ++x) o += *reinterpret_cast<const v4f *>(sums + t * 4 + x * EACH * D);
        }
        const float norm = 1.f / sum;
#pragma unroll
        for (int e = 0; e < 4; ++e) out.h[e] = __float2half_rn(o[e] * norm);
        *reinterpret_cast<v2u *>(to) = out.v;
        if (SPLIT > 1) return;
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

template <int D, int WAVES, Part PART>
static sqap_status launch_short(const ShortArgs &a, hipStream_t st)
{
    constexpr int LDS = sizeof(ShortLds<D, WAVES, PART == Part::Own ? 1 : 2>);
    static std::atomic<bool> ready[kMaxDeviceSlots];
    if (!ready[device_slot()].load(std::memory_order_relaxed)) {
        SQAP_HIP_CHECK(hipFuncSetAttribute(reinterpret_cast<const void *>(cache8_short_kernel<D, WAVES, PART>), hipFuncAttributeMaxDynamicSharedMemorySize, LDS));
        ready[device_slot()].store(true, std::memory_order_relaxed);
    }
    hipLaunchKernelGGL((cache8_short_kernel<D, WAVES, PART>), dim3((unsigned)a.tiles * a.cache.kv_heads * a.cache.batch), dim3(64 * WAVES), LDS, st, a);
    SQAP_HIP_CHECK(hipGetLastError());
    return SQAP_OK;
}

// Tiles of 16 rows, whose blocks are dealt to eight wavefronts, where there would be few tiles of 128: 148 rows of 32 heads (64 of those) take
// 9.0 us so and 11.0 otherwise, 512 of 8 heads (32) 8.0 and 19.0, 20 of 32 heads over 8 behind 2000 (8) 18 and 62, 1500 of 8 behind 2000
// (96) 67 and 103, 300 of 32 heads (96) 13.9 and 15.1; but 500 of 32 (128) 23.7 and 21.3, 1000 of 32 over 8 (256) 56 and 37.
constexpr int kFewTiles = 96;
// Parts of many sequences with up to 32 rows each: cache8_short_kernel, whose two wavefronts and two workgroups' LDS leave four to a CU, in place of tiles of
// 128 that are almost empty (512 x 2 rows of 32 heads over 8, prefix and join included, 85 us and 119; 700 x 2 of 12 heads of 64 53 and 89).
constexpr int kShortTiles = 512, kOwnTiles = 2;

template <int D, Part PART>
static sqap_status launch_attention_d(const __half *Q, int64_t ldq, const int32_t *starts, const int32_t *past, int rows, int max_new, int H,
                                      const Cache8View &cache, __half *O, int64_t ldo, const Parts &parts, hipStream_t st)
{
    constexpr int WAVES = 4, LDS = 2 * 2 * kBlock * D * 2;
    static std::atomic<bool> ready[kMaxDeviceSlots];
    if (!ready[device_slot()].load(std::memory_order_relaxed)) {
        SQAP_HIP_CHECK(hipFuncSetAttribute(reinterpret_cast<const void *>(cache8_attention_kernel<D, WAVES, PART>), hipFuncAttributeMaxDynamicSharedMemorySize, LDS));
        SQAP_HIP_CHECK(hipFuncSetAttribute(reinterpret_cast<const void *>(cache8_few_rows_kernel<D, PART>), hipFuncAttributeMaxDynamicSharedMemorySize,
                                           (int)sizeof(FewRowsLds<D>)));
        ready[device_slot()].store(true, std::memory_order_relaxed);
    }
    const auto tiles_of = [&](int per_tile) { return std::max<int64_t>(1, ((int64_t)max_new * (H / cache.kv_heads) + per_tile - 1) / per_tile); };
    const int64_t pairs = (int64_t)cache.kv_heads * cache.batch;
    const bool few = tiles_of(32 * WAVES) * pairs <= kFewTiles;
    const int64_t tiles = tiles_of(few ? 16 : 32 * WAVES), items = tiles * pairs;
    if constexpr (PART == Part::Own) {
        if (tiles_of(16) * pairs > kShortTiles && tiles_of(16) <= kOwnTiles)
            return launch_short<D, 2, Part::Own>(ShortArgs{Q, ldq, starts, past, rows, max_new, H, cache, cache, parts, nullptr, 0, (int)tiles_of(16)}, st);
    }
    if (few)
        hipLaunchKernelGGL((cache8_few_rows_kernel<D, PART>), dim3((unsigned)items), dim3(64 * kFewRowsWaves), sizeof(FewRowsLds<D>), st, Q, ldq, starts, past, rows,
                           max_new, H, cache, O, ldo, (int)tiles, parts);
    else
        hipLaunchKernelGGL((cache8_attention_kernel<D, WAVES, PART>), dim3((unsigned)items), dim3(64 * WAVES), LDS, st, Q, ldq, starts, past, rows, max_new, H,
                           cache, O, ldo, (int)tiles, parts);
    SQAP_HIP_CHECK(hipGetLastError());
    return SQAP_OK;
}

sqap_status launch_cache8_attention(const __half *Q, int64_t ldq, const int32_t *starts, const int32_t *past, int rows, int max_new, int H,
                                    const Cache8View &cache, int d, __half *O, int64_t ldo, hipStream_t st)
{
    return d == 64 ? launch_attention_d<64, Part::Whole>(Q, ldq, starts, past, rows, max_new, H, cache, O, ldo, Parts{}, st)
                   : launch_attention_d<128, Part::Whole>(Q, ldq, starts, past, rows, max_new, H, cache, O, ldo, Parts{}, st);
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
    if (d == 64) hipLaunchKernelGGL((cache8_decode_kernel<64, false>), grid, dim3(64 * kDecodeWaves), 0, st, a);
    else hipLaunchKernelGGL((cache8_decode_kernel<128, false>), grid, dim3(64 * kDecodeWaves), 0, st, a);
    SQAP_HIP_CHECK(hipGetLastError());
    return SQAP_OK;
}

// ---- behind a shared prefix

// How the prefixes are dealt out: shares of two blocks to a wavefront (64 rows of 32 heads over 8 behind 1000 positions 16.3 us, with one 20.4), of one up
// to 8 blocks.  Up to 64 pairs to a group and key head: tiles of 16, blocks dealt to the wavefronts; up to 256 of them, too, where all tiles together
// have no more than 20000 blocks: the tiles of 128 want two launches more (32 rows of 32 heads over 8 behind 1000 positions 14 and 27 us,
// behind 20000 45 and 48, behind 100003 187 and 128; 64 behind 1000 23 and 29).
// Prompts of few rows: tiles of 16 that pass over prefix and own positions by themselves.  Up to 512 tiles, which the device holds at once, with eight
// wavefronts, while they are up to 12000 blocks in all (16 x 10 rows of 32 heads over 8 behind 1000 positions, 6144: 25 us, in parts 30; behind 4000 54
// and 39) and prefixes up to 48 blocks long, or 256 tiles (10 rows behind 1000 positions 13 and 20, behind 4000 27 and 24).  More tiles with two wavefronts,
// four to a CU (128 x 4 rows of 32 heads over 8 behind 100 positions 16.5 us, with eight 27), where they repeat the prefixes' blocks no more than 20 times
// as often as full tiles of 16 over one block would (256 x 4 rows behind 500 positions, 8 times: 42 us, in parts 59; behind 1000, 16: 57 and 63; 243 x 7 of 12
// heads behind 798, 30: 61 and 52; 512 x 2 behind 600, 20: 92 and 64, behind 2000, 64: 208 and 86).
constexpr int kShortBlocks = 12000, kShortPrefix = 48, kShortRepeats = 20;
constexpr int kFewPairs = 64, kFewPairsAtMost = 256, kFewBlocks = 20000, kPrefixGroups = 512, kMostPrefixShares = 64;
struct SharedPlan {
    bool together, direct;       // long prompts: cache8_long_kernel; short ones: cache8_short_kernel,
    int waves;                   // with so many wavefronts
    int groups;                  // its workgroups
    bool few;
    int64_t tiles;               // of a group and key head
    int shares, own_shares;
    int64_t pairs;               // rows times heads
    size_t q, ml, o, bytes;      // where they are in the workspace
};
static SharedPlan shared_plan(bool prompt, int batch, int groups, int H, int kv_heads, int d, int rows, int max_new, int own_shares, int longest_prefix)
{
    SharedPlan p = {};
    const int64_t of_group = std::min<int64_t>((int64_t)(batch / groups) * max_new, rows) * (H / kv_heads);
    const int blocks = std::max(1, blocks_of(longest_prefix));
    p.few = of_group <= kFewPairs || (of_group <= kFewPairsAtMost && (of_group + 15) / 16 * groups * kv_heads * blocks <= kFewBlocks);
    p.tiles = std::max<int64_t>(1, (of_group + (p.few ? 15 : 127)) / (p.few ? 16 : 128));
    const int64_t items = p.tiles * groups * kv_heads;
    p.shares = (int)std::max<int64_t>(1, std::min<int64_t>({p.few && blocks > 8 ? (blocks + 7) / 8 : (blocks + 3) / 4, kPrefixGroups / items, kMostPrefixShares}));
    p.own_shares = own_shares;
    p.pairs = (int64_t)rows * H;
    const auto up = [](size_t n) { return (n + 15) / 16 * 16; };
    const int64_t tiles = ((int64_t)std::max(1, max_new) * (H / kv_heads) + 15) / 16 * kv_heads * batch;          // of 16
    // rows that fill three quarters of a tile of 128 on average, 64 of those (128 rows of 32 heads over 8, 32 tiles, behind 2000 positions 47 us and 20
    // otherwise, behind 20000 110 and 91; 64 tiles behind 2000 46 and 45; 330 behind 6000 194 and 279), and more than a start's worth of work: the kernel
    // takes 36 us at the least (8 x 148 rows behind 100 positions, 7104 blocks of tiles of 16: 47 us and 33; 300 behind 1000, 11400: 46 and 37; 16 x 100
    // behind 200, 16000: 49 and 46; 8 x 148 behind 500, 23680: 49 and 49; 8 x 300 behind 100, 24000: 56 and 65)
    p.together = max_new > 1 && batch <= kLongBatch && (int64_t)rows * (H / kv_heads) >= (int64_t)batch * 96 && (int64_t)rows * H >= 128 * kLongTiles &&
                 tiles * (blocks + (max_new + 127) / 128) > kLongWork;
    if (p.together) {
        p.groups = std::max(8, device_cu_count() * 2 / 8 * 8);
        p.ml = kCounterBytes + (size_t)p.groups * sizeof(LongSlot);
        p.o = p.ml + (size_t)p.groups * 256 * sizeof(float2);
        p.bytes = p.o + (size_t)p.groups * 256 * d * sizeof(float);
        return p;
    }
    p.waves = tiles <= kShortTiles ? kFewRowsWaves : 2;
    // (no rows announced: NaN for those there are)
    p.direct = prompt && (max_new == 0 || (tiles <= kShortTiles ? tiles * blocks <= kShortBlocks && (blocks <= kShortPrefix || tiles >= 256)
                                                                : tiles <= most_workgroups(256) && tiles * 16 * blocks < kShortRepeats * (int64_t)rows * H));
    if (p.direct) return p;                                           // (no workspace)
    p.q = kCounterBytes;                                              // (left alone, for calls that want it zero)
    p.ml = p.q + (max_new == 1 ? up((size_t)p.pairs * d * 2) : 0);
    p.o = p.ml + up((size_t)(p.shares + own_shares) * p.pairs * sizeof(float2));
    p.bytes = p.o + (size_t)(p.shares + own_shares) * p.pairs * d * sizeof(float);
    return p;
}
static int own_shares_of(int batch, int H, int kv_heads, int longest)
{
    return std::min(decode_shares(batch, H, kv_heads, longest), kMostParts - kMostPrefixShares);
}

size_t cache8_shared_workspace_bytes(bool prompt, int batch, int groups, int H, int kv_heads, int d, int rows, int max_new, int longest, int longest_prefix)
{
    return shared_plan(prompt, batch, groups, H, kv_heads, d, rows, max_new, prompt ? 1 : own_shares_of(batch, H, kv_heads, longest), longest_prefix).bytes;
}

template <int D>
static sqap_status launch_prefix(const SharedPlan &plan, const PrefixTile &a, const Cache8View &prefix, const Parts &parts, hipStream_t st)
{
    if (plan.few) {
        hipLaunchKernelGGL(cache8_prefix_kernel<D>, dim3(plan.shares, prefix.kv_heads, (unsigned)(prefix.batch * plan.tiles)), dim3(64 * kDecodeWaves), 0, st, a, prefix,
                           parts, (int)plan.tiles);
    } else {
        constexpr int WAVES = 4, LDS = 2 * 2 * kBlock * D * 2;
        static std::atomic<bool> ready[kMaxDeviceSlots];
        if (!ready[device_slot()].load(std::memory_order_relaxed)) {
            SQAP_HIP_CHECK(hipFuncSetAttribute(reinterpret_cast<const void *>(cache8_attention_kernel<D, WAVES, Part::Prefix>),
                                               hipFuncAttributeMaxDynamicSharedMemorySize, LDS));
            ready[device_slot()].store(true, std::memory_order_relaxed);
        }
        const int64_t items = plan.tiles * plan.shares * prefix.kv_heads * prefix.batch;
        hipLaunchKernelGGL((cache8_attention_kernel<D, WAVES, Part::Prefix>), dim3((unsigned)items), dim3(64 * WAVES), LDS, st, a.Q, a.ld, a.starts, nullptr, a.rows,
                           a.max_new, a.H, prefix, nullptr, 0, (int)plan.tiles, parts);
    }
    SQAP_HIP_CHECK(hipGetLastError());
    return SQAP_OK;
}

// Four groups of lanes to a pair where there are more than eight parts and the pairs alone would leave the device half empty.
template <int D>
static sqap_status launch_join(const JoinArgs &a, int batch, hipStream_t st)
{
    constexpr int EACH = 1024 / D, SPLIT = 4;
    const int64_t pairs = (int64_t)std::max(1, a.max_new) * a.H, groups = (pairs + EACH - 1) / EACH;
    if (a.max_new == 1 && a.parts.prefix_shares > 8 && groups * batch < 1024)
        hipLaunchKernelGGL((cache8_join_kernel<D, SPLIT>), dim3((unsigned)((pairs + EACH / SPLIT - 1) / (EACH / SPLIT)), batch), dim3(256), 0, st, a);
    else
        hipLaunchKernelGGL((cache8_join_kernel<D, 1>), dim3((unsigned)std::min<int64_t>(groups, 1 << 16), batch), dim3(256), 0, st, a);
    SQAP_HIP_CHECK(hipGetLastError());
    return SQAP_OK;
}

template <int D>
static sqap_status launch_shared_d(const __half *Q, int64_t ldq, const int32_t *starts, const int32_t *past, int rows, int max_new, int H, const Cache8View &cache,
                                   const Cache8View &prefix, const int32_t *length, int longest_prefix, __half *O, int64_t ldo, char *workspace, hipStream_t st)
{
    const SharedPlan plan = shared_plan(true, cache.batch, prefix.batch, H, cache.kv_heads, D, rows, max_new, 1, longest_prefix);
    if (plan.together) {
        constexpr int LDS = 2 * 2 * kBlock * D * 2;
        static std::atomic<bool> ready[kMaxDeviceSlots];
        if (!ready[device_slot()].load(std::memory_order_relaxed)) {
            SQAP_HIP_CHECK(hipFuncSetAttribute(reinterpret_cast<const void *>(cache8_long_kernel<D>), hipFuncAttributeMaxDynamicSharedMemorySize, LDS));
            ready[device_slot()].store(true, std::memory_order_relaxed);
        }
        const LongArgs a = {Q, ldq, starts, past, rows, max_new, H, cache, prefix, Parts{nullptr, nullptr, 0, 0, cache.batch / prefix.batch, length}, O, ldo,
                            reinterpret_cast<LongSlot *>(workspace + kCounterBytes), reinterpret_cast<float2 *>(workspace + plan.ml),
                            reinterpret_cast<float *>(workspace + plan.o)};
        hipLaunchKernelGGL(cache8_long_kernel<D>, dim3(plan.groups), dim3(256), LDS, st, a);
        SQAP_HIP_CHECK(hipGetLastError());
        hipLaunchKernelGGL(cache8_long_join_kernel<D>, dim3(2, plan.groups), dim3(256), 0, st, a);
        SQAP_HIP_CHECK(hipGetLastError());
        return SQAP_OK;
    }
    if (plan.direct) {
        const int tiles = std::max(1, (max_new * (H / cache.kv_heads) + 15) / 16);
        const ShortArgs a = {Q, ldq, starts, past, rows, max_new, H, cache, prefix, Parts{nullptr, nullptr, 0, 0, cache.batch / prefix.batch, length}, O, ldo, tiles};
        return plan.waves == 2 ? launch_short<D, 2, Part::Whole>(a, st) : launch_short<D, kFewRowsWaves, Part::Whole>(a, st);
    }
    const Parts parts = {reinterpret_cast<float *>(workspace + plan.o), reinterpret_cast<float2 *>(workspace + plan.ml), plan.pairs, plan.shares,
                         cache.batch / prefix.batch, length};
    sqap_status s = launch_prefix<D>(plan, PrefixTile{Q, ldq, starts, nullptr, rows, max_new, H}, prefix, parts, st);
    if (s == SQAP_OK) s = launch_attention_d<D, Part::Own>(Q, ldq, starts, past, rows, max_new, H, cache, nullptr, 0, parts, st);
    if (s != SQAP_OK) return s;
    return launch_join<D>(JoinArgs{starts, past, rows, max_new, H, cache.blocks * kBlock, prefix.blocks * kBlock, 1, 1, parts, O, ldo}, cache.batch, st);
}

sqap_status launch_cache8_shared(const __half *Q, int64_t ldq, const int32_t *starts, const int32_t *past, int rows, int max_new, int H, const Cache8View &cache,
                                 const Cache8View &prefix, const int32_t *length, int longest_prefix, int d, __half *O, int64_t ldo, void *workspace, hipStream_t st)
{
    char *const ws = static_cast<char *>(workspace);
    return d == 64 ? launch_shared_d<64>(Q, ldq, starts, past, rows, max_new, H, cache, prefix, length, longest_prefix, O, ldo, ws, st)
                   : launch_shared_d<128>(Q, ldq, starts, past, rows, max_new, H, cache, prefix, length, longest_prefix, O, ldo, ws, st);
}

template <int D>
static sqap_status launch_shared_decode_d(DecodeArgs a, const int32_t *length, int longest_prefix, char *workspace, hipStream_t st)
{
    const Cache8View &cache = a.cache, &prefix = a.prefix;
    const SharedPlan plan = shared_plan(false, cache.batch, prefix.batch, a.H, cache.kv_heads, D, cache.batch, 1, a.shares, longest_prefix);
    a.parts = {reinterpret_cast<float *>(workspace + plan.o), reinterpret_cast<float2 *>(workspace + plan.ml), plan.pairs, plan.shares, cache.batch / prefix.batch, length};
    a.prefix_tiles = plan.few ? (int)plan.tiles : 0;
    a.q_out = plan.few ? nullptr : reinterpret_cast<__half *>(workspace + plan.q);
    const int64_t items = (int64_t)prefix.batch * a.prefix_tiles * cache.kv_heads * plan.shares + (int64_t)a.shares * cache.kv_heads * a.chunks * cache.batch;
    hipLaunchKernelGGL((cache8_decode_kernel<D, true>), dim3((unsigned)items), dim3(64 * kDecodeWaves), 0, st, a);
    SQAP_HIP_CHECK(hipGetLastError());
    if (!plan.few) {
        const sqap_status s = launch_prefix<D>(plan, PrefixTile{a.q_out, (int64_t)a.H * D, nullptr, nullptr, cache.batch, 1, a.H}, prefix, a.parts, st);
        if (s != SQAP_OK) return s;
    }
    return launch_join<D>(JoinArgs{nullptr, a.past, cache.batch, 1, a.H, cache.blocks * kBlock, prefix.blocks * kBlock, a.shares, a.per_share, a.parts, a.O, a.ldo},
                          cache.batch, st);
}

sqap_status launch_cache8_shared_decode(const __half *QKV, int64_t ld, const int32_t *pos, const int32_t *past, int H, double base, const Cache8View &cache,
                                        const Cache8View &prefix, const int32_t *length, int d, int longest, int longest_prefix, __half *O, int64_t ldo,
                                        void *workspace, hipStream_t st)
{
    DecodeArgs a = {};
    a.QKV = QKV;
    a.ld = ld;
    a.pos = pos;
    a.past = past;
    a.H = H;
    a.G = H / cache.kv_heads;
    a.chunks = (a.G + 15) / 16;
    a.shares = own_shares_of(cache.batch, H, cache.kv_heads, longest);
    a.per_share = (blocks_of(longest) + a.shares - 1) / a.shares;
    a.cache = cache;
    a.prefix = prefix;
    a.O = O;
    a.ldo = ldo;
    a.freq = rope_frequencies(d, base);
    char *const ws = static_cast<char *>(workspace);
    return d == 64 ? launch_shared_decode_d<64>(a, length, longest_prefix, ws, st) : launch_shared_decode_d<128>(a, length, longest_prefix, ws, st);
}

}  // namespace sqap
