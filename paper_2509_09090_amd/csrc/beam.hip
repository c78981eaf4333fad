// Beam search: the best continuations of several beams over the vocabulary, and the reordering of a cache in 8 bits that follows.
//
// A token's total is s + (l - log sum exp l), the beam's score and its logarithm of a probability.  Within a beam totals order as the
// logits do, so the best k of a beam are found on halves, and only they get a total, in binary64: two of them that differ do so by far
// more than the sums of exponentials are off by.
#include <algorithm>

#include "common.h"

namespace sqap {

typedef unsigned v4u __attribute__((ext_vector_type(4)));
typedef unsigned v4u_any __attribute__((ext_vector_type(4), aligned(2)));
typedef unsigned v2u __attribute__((ext_vector_type(2)));
typedef unsigned long long u64;

constexpr int kBeamT = 256, kBeamWaves = kBeamT / 64, kBeamMost = kBeamMostOutputs;
constexpr unsigned kMinusInf = 0x03ffu;                               // key of minus infinity, the lowest there is
constexpr float kLog2eHigh = 1.44269502f, kLog2eLow = 1.92596299e-8f; // log2(e) as the sum of two

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
__device__ __forceinline__ unsigned half_at(const v4u &v, int e) { return e & 1 ? v[e >> 1] >> 16 : v[e >> 1] & 0xffffu; }
__device__ __forceinline__ float float_at(const v4u &v, int e) { return __half2float(__ushort_as_half((unsigned short)half_at(v, e))); }
__device__ __forceinline__ unsigned largest_of(const v4u &v)         // key of the largest of the eight
{
    union { v4u u; v2h h[4]; } x;
    x.u = v;
    const v2h m = __builtin_elementwise_max(__builtin_elementwise_max(x.h[0], x.h[1]), __builtin_elementwise_max(x.h[2], x.h[3]));
    union { v2h h; unsigned u; } y;
    y.h = m;
    return max(key_of(y.u & 0xffffu), key_of(y.u >> 16));
}

// exp(value - top), of a difference below zero
__device__ __forceinline__ float exp_of(float value, float top)
{
    const float d = value - top;
    return __builtin_amdgcn_exp2f(fmaf(d, kLog2eHigh, d * kLog2eLow));
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
// best k lie in those: any other piece has k logits before its own.  Of their logits those that reach the smallest of these maxima are listed and ranked.
template <int PIECES>
__global__ __launch_bounds__(kBeamT) void beam_rows_kernel(const BeamArgs a)
{
    constexpr int LISTED = kBeamMost * PIECES * 8;
    __shared__ unsigned tops[kBeamT], list[LISTED], listed;
    __shared__ float wave_top[kBeamWaves];
    __shared__ double wave_sum_[kBeamWaves];
    const int t = threadIdx.x, l = t & 63, wave = t >> 6, slab = blockIdx.x % a.slabs;
    const int64_t row = blockIdx.x / a.slabs;
    if (a.done && a.done[row] != 0) return;
    const int first = slab * (kBeamT * 8 * PIECES);
    const __half *from = a.logits + row * a.ld;
    v4u v[PIECES];
#pragma unroll
    for (int p = 0; p < PIECES; ++p) {
        const int at = first + (p * kBeamT + t) * 8;
        v[p] = v4u{0xfc00fc00u, 0xfc00fc00u, 0xfc00fc00u, 0xfc00fc00u};
        if (at + 8 <= a.vocab) v[p] = *reinterpret_cast<const v4u_any *>(from + at);
        else {
#pragma unroll
            for (int e = 0; e < 8; ++e)
                if (at + e < a.vocab) {
                    const unsigned h = __half_as_ushort(from[at + e]);
                    v[p][e >> 1] = e & 1 ? (v[p][e >> 1] & 0xffffu) | h << 16 : (v[p][e >> 1] & 0xffff0000u) | h;
                }
        }
    }
    if (t == 0) listed = 0;
    unsigned mine = 0, keys[PIECES];
#pragma unroll
    for (int p = 0; p < PIECES; ++p) {
        v[p] = clean(v[p]);
        keys[p] = largest_of(v[p]) << 11 | (2047 - (p * kBeamT + t));
        mine = max(mine, keys[p]);
    }
    tops[t] = mine;
    // the sum of exponentials, of each thread below its own largest logit
    const float top = value_of(mine >> 11);
    // (eight of them in binary32, those sums in binary64: beside one large term many small ones count)
    double sum = 0.0;
    if (fabsf(top) <= 65504.f) {
#pragma unroll
        for (int p = 0; p < PIECES; ++p) {
            float x[8];
#pragma unroll
            for (int e = 0; e < 8; ++e) x[e] = exp_of(float_at(v[p], e), top);
            sum += (double)(((x[0] + x[1]) + (x[2] + x[3])) + ((x[4] + x[5]) + (x[6] + x[7])));
        }
    } else if (top > 0.f) {
#pragma unroll
        for (int p = 0; p < PIECES; ++p)
#pragma unroll
            for (int e = 0; e < 8; ++e) sum += half_at(v[p], e) == 0x7c00u ? 1.0 : 0.0;
    }
    float most = top;
#pragma unroll
    for (int i = 32; i > 0; i >>= 1) most = fmaxf(most, __shfl_xor(most, i));
    const double part = wave_sum(top == most ? sum : fabsf(most) <= 65504.f ? sum * (double)exp_of(top, most) : 0.0);
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
        const unsigned least = max(reach >> 11, kMinusInf + 1);
#pragma unroll
        for (int p = 0; p < PIECES; ++p)
            if (keys[p] >= reach) {
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    const unsigned key = key_of(half_at(v[p], e));
                    if (key >= least) list[atomicAdd(&listed, 1u)] = key << 14 | (16383 - ((p * kBeamT + t) * 8 + e));
                }
            }
    }
    __syncthreads();
    const int n = (int)listed;
    v2u *best = a.best + (row * a.slabs + slab) * a.k;
    for (int i = t; i < n; i += kBeamT) {
        const unsigned own = list[i];
        int rank = 0;
        for (int j = 0; j < n; ++j) rank += list[j] > own ? 1 : 0;
        if (rank < a.k) best[rank] = v2u{own >> 14, (unsigned)first + 16383 - (own & 16383)};
    }
    for (int i = n + t; i < a.k; i += kBeamT) best[i] = v2u{0, 0};
    if (t == 0) {
        float whole = wave_top[0];
        for (int w = 1; w < kBeamWaves; ++w) whole = fmaxf(whole, wave_top[w]);
        double all = 0.0;
        for (int w = 0; w < kBeamWaves; ++w)
            if (wave_top[w] == whole) all += wave_sum_[w];
            else if (fabsf(whole) <= 65504.f) all += wave_sum_[w] * (double)exp_of(wave_top[w], whole);
        a.rows[row * a.slabs + slab] = BeamRow{all, whole};
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

// One workgroup per batch element: the rows' sums from their slabs', then the best k of all their candidates, as in beam_rows_kernel: the threads' best,
// a number that k of them reach, the few candidates that reach it ranked.
constexpr int kSurvivors = 2048;
__global__ __launch_bounds__(kBeamT) void beam_select_kernel(const BeamArgs a)
{
    __shared__ Candidate tops[kBeamT], list[kSurvivors];
    __shared__ float top[kBeamMost];
    __shared__ double log_sum[kBeamMost], score[kBeamMost];
    __shared__ int ended[kBeamMost], listed, counts[kBeamWaves];
    const int t = threadIdx.x, l = t & 63, wave = t >> 6, each = a.slabs * a.k, all = a.beams * each;
    const int64_t b = blockIdx.x, row0 = b * a.beams;
    if (t == 0) listed = 0;
    for (int r = wave; r < a.beams; r += kBeamWaves) {
        const bool done = a.done && a.done[row0 + r] != 0;
        float m = -INFINITY;
        double sum = 0.0;
        if (!done) {
            const BeamRow *rows = a.rows + (row0 + r) * a.slabs;
            for (int i = l; i < a.slabs; i += 64) m = fmaxf(m, rows[i].top);
#pragma unroll
            for (int i = 32; i > 0; i >>= 1) m = fmaxf(m, __shfl_xor(m, i));
            for (int i = l; i < a.slabs; i += 64) {
                const BeamRow x = rows[i];
                if (x.top == m) sum += x.sum;
                else if (fabsf(m) <= 65504.f) sum += x.sum * exp((double)x.top - (double)m);
            }
            sum = wave_sum(sum);
        }
        if (l == 0) {
            top[r] = m;
            log_sum[r] = done ? 0.0 : log(sum);
            score[r] = (double)a.scores[row0 + r];
            ended[r] = done;
        }
    }
    __syncthreads();
    auto candidate = [&](int c) {
        const int r = c / each, i = c - r * each;
        Candidate x = {0, 0};
        if (ended[r]) {
            if (i == 0) x.total = total_key(score[r]), x.tie = (u64)(kBeamMost - 1 - r) << kTieBeam | (unsigned)((1 << kTieKey) - 1 - a.eos);
            return x;
        }
        const v2u have = a.best[row0 * each + c];
        if (have[0] == 0) return x;
        const float v = value_of(have[0]), m = top[r];
        if (fabsf(m) > 65504.f && v != m) return x;                   // (beside infinite logits the others have no probability)
        x.total = total_key(score[r] + ((v == m ? 0.0 : (double)v - (double)m) - log_sum[r]));
        x.tie = (u64)(kBeamMost - 1 - r) << kTieBeam | (u64)have[0] << kTieKey | ((1u << kTieKey) - 1 - have[1]);
        return x;
    };
    Candidate mine = {0, 0};
    for (int c = t; c < all; c += kBeamT) {
        const Candidate x = candidate(c);
        if (before(x, mine)) mine = x;
    }
    tops[t] = mine;
    __syncthreads();
    // (all wavefronts the same: four of the threads' best to a lane)
    Candidate four[4], reach = {0, 0};
#pragma unroll
    for (int i = 0; i < 4; ++i) four[i] = tops[4 * l + i];
    auto reached = [&](const Candidate &from) {
        int n = 0;
#pragma unroll
        for (int i = 0; i < 4; ++i) n += __popcll(__ballot(!before(from, four[i])));
        return n;
    };
    // the highest number, bit by bit, that k of them reach, or one that exactly k do
    auto search = [&](auto count) {
        for (int bit = 63 + kTieBeam + 6; bit >= 0; --bit) {
            Candidate next = reach;
            if (bit >= kTieBeam + 6) next.total |= 1ull << (bit - kTieBeam - 6);
            else next.tie |= 1ull << bit;
            const int n = count(next);
            if (n >= a.k) reach = next;
            if (n == a.k) break;
        }
    };
    search(reached);
    auto list_them = [&] {
        if (before(reach, mine)) return;
        for (int c = t; c < all; c += kBeamT) {
            const Candidate x = candidate(c);
            if (x.total == 0 || before(reach, x)) continue;
            const int at = atomicAdd(&listed, 1);
            if (at < kSurvivors) list[at] = x;
        }
    };
    list_them();
    __syncthreads();
    if (listed > kSurvivors) {                                        // many of few threads: count all of them instead
        reach = Candidate{0, 0};
        search([&](const Candidate &from) {
            int n = 0;
            if (!before(from, mine))
                for (int c = t; c < all; c += kBeamT) n += before(from, candidate(c)) ? 0 : 1;
#pragma unroll
            for (int i = 32; i > 0; i >>= 1) n += __shfl_xor(n, i);
            __syncthreads();
            if (l == 0) counts[wave] = n;
            __syncthreads();
            n = 0;
            for (int w = 0; w < kBeamWaves; ++w) n += counts[w];
            return n;
        });
        if (t == 0) listed = 0;
        __syncthreads();
        list_them();
        __syncthreads();
    }
    const int n = min(listed, kSurvivors);
    int32_t *parent = a.parent + b * a.k, *token = a.token + b * a.k, *done_out = a.done_out ? a.done_out + b * a.k : nullptr;
    float *out = a.score + b * a.k;
    for (int i = t; i < n; i += kBeamT) {
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
    for (int i = n + t; i < a.k; i += kBeamT) {
        parent[i] = token[i] = -1;
        out[i] = -INFINITY;
        if (done_out) done_out[i] = 0;
    }
}

// Slabs as large as leave the device its workgroups.
static int beam_pieces(int64_t rows, int vocab)
{
    for (int pieces = 8; pieces > 1; pieces /= 2)
        if (rows * ((vocab + kBeamT * 8 * pieces - 1) / (kBeamT * 8 * pieces)) >= 256) return pieces;
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
    hipLaunchKernelGGL(beam_select_kernel, dim3(batch), block, 0, st, a);
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

// Piece `at` of every sequence that moves: all of them are read before the first is written, so that in place is no matter.
template <int WIDTH, typename V, typename Takes>
__device__ __forceinline__ void move_piece(V *base, int64_t pitch, const Parents &p, Takes takes)
{
    V v[WIDTH];
#pragma unroll
    for (int i = 0; i < WIDTH; ++i)
        if (p.moves >> i & 1) {
            const int n = __builtin_amdgcn_readlane(p.length, i), of = __builtin_amdgcn_readlane(p.parent, i);
            if (takes(n)) v[i] = base[of * pitch];
        }
#pragma unroll
    for (int i = 0; i < WIDTH; ++i)
        if (p.moves >> i & 1) {
            if (takes(__builtin_amdgcn_readlane(p.length, i))) base[i * pitch] = v[i];
        }
}

// One workgroup per group, key head and kibibytes of a block (for all sequences of the group at once), of the unfinished block's rows, or the
// scales; V: what a thread moves of each.
template <int D, int WIDTH, typename V>
__global__ __launch_bounds__(256) void cache8_reorder_kernel(const Cache8View cache, const int32_t *__restrict__ parents, int width,
                                                             const int32_t *__restrict__ lengths, int32_t *__restrict__ lengths_out, int block_groups)
{
    constexpr int BLOCK_V = 2 * kCache8Block * D / (int)sizeof(V), TAIL_V = 2 * BLOCK_V, SPLIT = BLOCK_V / 256, TAIL_SPLIT = TAIL_V / 256;
    const int t = threadIdx.x, h = blockIdx.y;
    const int64_t first = (int64_t)blockIdx.z * width, heads = cache.kv_heads;
    const Parents p = parents_of(parents, lengths, first, width, cache.blocks * kCache8Block);
    if (lengths_out && h == 0 && blockIdx.x == 0 && t < width) lengths_out[first + t] = p.length;
    if (p.moves == 0) return;
    const int64_t head = first * heads + h;                           // of the group's first sequence
    if ((int)blockIdx.x < block_groups) {
        int most = 0;
        for (u64 m = p.moves; m; m &= m - 1) most = max(most, __builtin_amdgcn_readlane(p.length, __builtin_ctzll(m)));
        for (int x = blockIdx.x; x < most / kCache8Block * SPLIT; x += block_groups) {
            const int block = x / SPLIT;
            V *codes = reinterpret_cast<V *>(cache.codes) + (head * cache.blocks + block) * BLOCK_V + (x % SPLIT) * 256 + t;
            move_piece<WIDTH>(codes, heads * cache.blocks * BLOCK_V, p, [&](int n) { return block < n / kCache8Block; });
        }
        return;
    }
    const int x = (int)blockIdx.x - block_groups;
    if (x < TAIL_SPLIT) {
        const int piece = x * 256 + t, row = piece / (D * 2 / (int)sizeof(V)) % kCache8Block;
        V *tail = reinterpret_cast<V *>(cache.tail) + head * TAIL_V + piece;
        move_piece<WIDTH>(tail, heads * TAIL_V, p, [&](int n) { return row < n % kCache8Block; });
        return;
    }
    for (int from = 0; from < cache.blocks; from += 256) {
        const int block = from + t;                                   // (all lanes stay: the lengths are other lanes')
        v2u *scales = reinterpret_cast<v2u *>(cache.scales) + head * cache.blocks + block;
        move_piece<WIDTH>(scales, heads * cache.blocks, p, [&](int n) { return block < n / kCache8Block; });
    }
}

template <int D, int WIDTH, typename V>
static void launch_reorder(const Cache8View &cache, const int32_t *parents, int width, const int32_t *lengths, int longest, int32_t *lengths_out, hipStream_t st)
{
    constexpr int SPLIT = 2 * kCache8Block * D / (int)sizeof(V) / 256;
    const int block_groups = (int)std::min<int64_t>(std::max(1, longest / kCache8Block * SPLIT), 65536);
    for (int group = 0; group < cache.batch / width; group += 65535) {
        Cache8View part = cache;
        const int64_t first = (int64_t)group * width, heads = first * cache.kv_heads;
        part.codes += heads * cache.blocks * 2 * kCache8Block * D;
        part.scales += heads * cache.blocks * 2;
        part.tail += heads * 2 * kCache8Block * D;
        const dim3 grid(block_groups + 2 * SPLIT + 1, cache.kv_heads, std::min(65535, cache.batch / width - group));
        hipLaunchKernelGGL((cache8_reorder_kernel<D, WIDTH, V>), grid, dim3(256), 0, st, part, parents + first, width, lengths + first,
                           lengths_out ? lengths_out + first : nullptr, block_groups);
    }
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
