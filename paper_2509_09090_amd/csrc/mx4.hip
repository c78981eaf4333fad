// Microscaled 4-bit floating point: 32 consecutive channels share a power of two, the elements are 0, 1/2, 1, 3/2, 2, 3, 4, 6 with a
// sign.  Quantizer, packed weight and product; the matrix cores take both operands and their scales as they are.
//
// v_mfma_scale_f32_32x32x64_f8f6f4 with 4-bit operands: lane l holds row l % 32 of an operand and one block of 32 channels (16 bytes), the
// l / 32-th of two, with that block's scale in a byte of a register.  So a fragment of 32 rows x 64 channels is 1 KiB of codes and 64
// scale bytes, and neither is touched by the vector ALU.  Products of two elements are exact, sums are binary32.  (The 16x16x128 form does
// the same work per issued cycle on paper; alone in a loop it reached 5.1 PFLOP/s on random codes, this one 6.2.)
#include <algorithm>

#include "common.h"
#include "mx4_stage.h"

namespace sqap {

typedef int v4i __attribute__((ext_vector_type(4)));
typedef int v8i __attribute__((ext_vector_type(8)));
typedef float v4f __attribute__((ext_vector_type(4)));
typedef float v16f __attribute__((ext_vector_type(16)));
typedef unsigned v2u __attribute__((ext_vector_type(2)));

// ---------------------------------------------------------------- quantizer

// One thread per 8 channels, four threads per block.  The largest magnitude as an integer: the bit patterns of halves order as their
// values do, with infinities and then NaN above all numbers, so that a block which holds one is told by the same maximum.
// e = floor(log2 amax) - 2 puts the largest element into [4, 8): the conversion rounds to nearest, halfway cases to the even code, and
// takes what is above 6 to 6; dividing by 2^e is exact.  One pass: 2368 rows of 4096 in 8.2 us, where their bytes alone take 4.8 at the rate of a
// copy; 148 gathered rows in 4.2 and one row in 1.7, latency.
__global__ __launch_bounds__(256) void mx4_quantize_kernel(const __half *__restrict__ X, int64_t ldx, const int32_t *__restrict__ rows,
                                                           int K, int groups_per_row, uint8_t *__restrict__ Xq, uint8_t *__restrict__ Xs)
{
    const int i = blockIdx.x / groups_per_row, piece = (blockIdx.x - i * groups_per_row) * 256 + threadIdx.x;
    if (piece * 8 >= K) return;                                       // (K is a multiple of 32: the four threads of a block go together)
    const int64_t row = rows ? rows[i] : i;
    const v4i raw = *reinterpret_cast<const v4i *>(X + row * ldx + piece * 8);
    unsigned top = 0;
#pragma unroll
    for (int p = 0; p < 4; ++p) {
        const unsigned w = (unsigned)raw[p] & 0x7fff7fffu;
        top = max(top, max(w & 0xffffu, w >> 16));
    }
    top = max(top, dpp_move<kDppXor1>(top));
    top = max(top, dpp_move<kDppXor2>(top));
    unsigned code = 0, byte;
    if (top >= 0x7c00u) {
        byte = 255;                                                   // the scale that is not a number
    } else if (top == 0) {
        byte = 127;
#pragma unroll
        for (int p = 0; p < 4; ++p) code |= (((unsigned)raw[p] >> 15 & 1u) << 3 | ((unsigned)raw[p] >> 31) << 7) << (8 * p);
    } else {
        byte = (__float_as_uint(__half2float(__ushort_as_half((unsigned short)top))) >> 23) - 2;
        const float scale = __uint_as_float(byte << 23);
#pragma unroll
        for (int p = 0; p < 4; ++p) {
            union { int i; __half2 h; } u = {raw[p]};
            const float2 f = __half22float2(u.h);
            code |= ((unsigned)__builtin_amdgcn_cvt_scalef32_pk_fp4_f32(0u, f.x, f.y, scale, 0) & 255u) << (8 * p);
        }
    }
    reinterpret_cast<unsigned *>(Xq + (int64_t)i * (K >> 1))[piece] = code;
    if ((piece & 3) == 0) Xs[(int64_t)i * (K >> 5) + (piece >> 2)] = (uint8_t)byte;
}

sqap_status launch_mx4_quantize(const __half *X, int64_t ldx, const int32_t *rows, int M, int K, uint8_t *Xq, uint8_t *Xs, hipStream_t st)
{
    const int per_row = (K / 8 + 255) / 256, most = (int)(most_workgroups(256) / per_row);
    for (int64_t first = 0; first < M; first += most) {
        const int n = (int)std::min<int64_t>(most, M - first);
        hipLaunchKernelGGL(mx4_quantize_kernel, dim3((unsigned)n * per_row), dim3(256), 0, st, rows ? X : X + first * ldx, ldx, rows ? rows + first : rows, K,
                           per_row, Xq + first * (K >> 1), Xs + first * (K >> 5));
        SQAP_HIP_CHECK(hipGetLastError());
    }
    return SQAP_OK;
}

// ---------------------------------------------------------------- packed weight

// Fragments of 32 channels x 64 codes in the order in which the lanes hold them: a wavefront reads 1 KiB contiguous.  The channels of a
// span of 64 are dealt to its two fragments so that the 32 results a lane gets from them (fragment c, register i, lane half h:
// channel 32 h + 16 c + i) are neighbours: 64 bytes of an output row.  Scales: a lane's bytes of four fragments along K in one word.
// Past N and K: codes of zero with a scale of one.
__global__ __launch_bounds__(256) void mx4_pack_kernel(const uint8_t *__restrict__ Wq, const uint8_t *__restrict__ Ws, int N, int K, int stages,
                                                       uint8_t *__restrict__ data, unsigned *__restrict__ scales)
{
    const int group = blockIdx.x, l = threadIdx.x & 63, r = l & 31, h = l >> 5;
    const int n = (group >> 1) * 64 + ((r >> 2) & 1) * 32 + (group & 1) * 16 + (r >> 3) * 4 + (r & 3), blocks = K >> 5;
    for (int ks = threadIdx.x >> 6; ks < 4 * stages; ks += 4) {
        const int block = ks * 2 + h;
        v4i v = {0, 0, 0, 0};
        if (n < N && block < blocks) v = *reinterpret_cast<const v4i *>(Wq + (int64_t)n * (K >> 1) + block * 16);
        *reinterpret_cast<v4i *>(data + (((int64_t)group * stages * 4 + ks) * 64 + l) * 16) = v;
    }
    for (int st = threadIdx.x >> 6; st < stages; st += 4) {
        unsigned w = 0;
        for (int s = 0; s < 4; ++s) {
            const int block = st * 8 + s * 2 + h;
            const unsigned b = n < N && block < blocks ? Ws[(int64_t)n * blocks + block] : 127u;
            w |= b << (8 * s);
        }
        scales[((int64_t)group * stages + st) * 64 + l] = w;
    }
}

sqap_status launch_mx4_pack(const uint8_t *Wq, const uint8_t *Ws, const Mx4Weight &w, hipStream_t st)
{
    hipLaunchKernelGGL(mx4_pack_kernel, dim3(w.n_groups), dim3(256), 0, st, Wq, Ws, w.N, w.K, w.stages, w.data, w.scales);
    SQAP_HIP_CHECK(hipGetLastError());
    return SQAP_OK;
}

// ---------------------------------------------------------------- products

// S: which byte of the scales
template <int S>
__device__ __forceinline__ v16f multiply(const v4i &a, const v4i &b, const v16f &c, unsigned scale_a, unsigned scale_b)
{
    const v8i wa = {a[0], a[1], a[2], a[3], 0, 0, 0, 0}, wb = {b[0], b[1], b[2], b[3], 0, 0, 0, 0};
    return __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(wa, wb, c, 4, 4, S, (int)scale_a, S, (int)scale_b);
}

// Eight neighbouring outputs of a row, from channel n on.
__device__ __forceinline__ void store_outputs(__half *__restrict__ row, int n, int N, const float (&v)[8])
{
    union { __half h[8]; halves8_any v; } u;
#pragma unroll
    for (int i = 0; i < 8; ++i) u.h[i] = __float2half_rn(v[i]);
    if (n + 8 <= N) {
        *reinterpret_cast<halves8_any *>(row + n) = u.v;
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i)
            if (n + i < N) row[n + i] = u.h[i];
    }
}
__device__ __forceinline__ void store_fragment(__half *__restrict__ row, int n, int N, const v16f &v)
{
#pragma unroll
    for (int half = 0; half < 2; ++half) {
        float f[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) f[i] = v[8 * half + i];
        store_outputs(row, n + 8 * half, N, f);
    }
}

// A row's eight scale bytes of a stage (256 channels), the even blocks' and the odd ones': the words of the two lane halves.
__device__ __forceinline__ v2u split_scales(const v2u w)
{
    return v2u{__builtin_amdgcn_perm(w[1], w[0], 0x06040200u), __builtin_amdgcn_perm(w[1], w[0], 0x07050301u)};
}
// (The last stage of a K that is no multiple of 256 is read so that it ends with the row; what is missing gets a scale of one.)
__device__ __forceinline__ v2u load_scales(const uint8_t *of_row, int st, int blocks)
{
    v2u w;
    __builtin_memcpy(&w, of_row + min(st * 8, blocks - 8), 8);
    return w;
}
__device__ __forceinline__ v2u place_scales(const v2u loaded, int st, int blocks)
{
    const int over = 8 * max(st * 8 + 8 - blocks, 0);
    unsigned long long w = (unsigned long long)loaded[1] << 32 | loaded[0];
    w = w >> over | (0x7f7f7f7f7f7f7f7full << (63 - over)) << 1;
    return v2u{(unsigned)w, (unsigned)(w >> 32)};
}
// the first stage's, in place; a row may be shorter than a stage
__device__ __forceinline__ v2u first_scales(const uint8_t *of_row, int blocks)
{
    if (blocks >= 8) return load_scales(of_row, 0, blocks);
    unsigned long long w = 0x7f7f7f7f7f7f7f7full;
    for (int b = 0; b < blocks; ++b) w = (w & ~(255ull << (8 * b))) | (unsigned long long)of_row[b] << (8 * b);
    return v2u{(unsigned)w, (unsigned)(w >> 32)};
}

// A window of memory: lane offset + uniform offset, without 64-bit addresses in vector registers; a lane offset behind its end reads zeros, a
// uniform one stays inside.
typedef __amdgpu_buffer_rsrc_t Window;
__device__ __forceinline__ Window window_of(const void *p, unsigned long long bytes)
{
    return __builtin_amdgcn_make_buffer_rsrc(const_cast<void *>(p), 0, (unsigned)(bytes < 0xfffffff0ull ? bytes : 0xfffffff0ull), 0x00027000);
}
__device__ __forceinline__ v4i read16(Window w, unsigned lane, unsigned uniform)
{
    union { __attribute__((ext_vector_type(4))) unsigned u; v4i i; } x;
    x.u = __builtin_amdgcn_raw_buffer_load_b128(w, lane, uniform, 0);
    return x.i;
}

// Up to 32 rows: a workgroup owns 32 channels, its eight wavefronts share K stage by stage (256 channels), and the sums are added in LDS in
// the order of the wavefronts.  Bound by streaming the weight.
constexpr int kFewWaves = 8;
__global__ __launch_bounds__(64 * kFewWaves) void mx4_few_kernel(const uint8_t *__restrict__ Xq, const uint8_t *__restrict__ Xs, int M, int K,
                                                                 const uint8_t *__restrict__ data, const unsigned *__restrict__ scales,
                                                                 int stages, int N, __half *__restrict__ Y, int64_t ldy, int row_tiles, int items,
                                                                 int per_xcd)
{
    __shared__ v4f sums[kFewWaves][4][64];
    const int item = (blockIdx.x & 7) * per_xcd + (blockIdx.x >> 3);  // (row tiles of the same channels behind one L2)
    if (item >= items) return;
    const int group = item / row_tiles, first_row = (item - group * row_tiles) * 32;
    M -= first_row;
    Xq += (int64_t)first_row * (K >> 1);
    Xs += (int64_t)first_row * (K >> 5);
    Y += (int64_t)first_row * ldy;
    const int l = threadIdx.x & 63, wave = threadIdx.x >> 6, h = l >> 5, blocks = K >> 5;
    const int token = min(l & 31, M - 1);
    const uint8_t *x = Xq + (int64_t)token * (K >> 1), *xs = Xs + (int64_t)token * blocks;
    v16f acc;
#pragma unroll
    for (int i = 0; i < 16; ++i) acc[i] = 0.f;
    for (int st = wave; st < stages; st += kFewWaves) {
        v4i w[4], v[4];
        const unsigned sw = scales[((int64_t)group * stages + st) * 64 + l];
#pragma unroll
        for (int s = 0; s < 4; ++s) {
            const int ks = st * 4 + s, block = ks * 2 + h < blocks ? ks * 2 + h : 0;       // (past K: times codes of zero)
            w[s] = *reinterpret_cast<const v4i *>(data + (((int64_t)group * stages * 4 + ks) * 64 + l) * 16);
            v[s] = *reinterpret_cast<const v4i *>(x + block * 16);
        }
        const v2u both = split_scales(st == 0 ? first_scales(xs, blocks) : place_scales(load_scales(xs, st, blocks), st, blocks));
        const unsigned sx = both[h];
        acc = multiply<0>(w[0], v[0], acc, sw, sx);
        acc = multiply<1>(w[1], v[1], acc, sw, sx);
        acc = multiply<2>(w[2], v[2], acc, sw, sx);
        acc = multiply<3>(w[3], v[3], acc, sw, sx);
    }
#pragma unroll
    for (int q = 0; q < 4; ++q) sums[wave][q][l] = v4f{acc[4 * q], acc[4 * q + 1], acc[4 * q + 2], acc[4 * q + 3]};
    __syncthreads();
    if (wave >= 4 || (l & 31) >= M) return;
    v4f sum = sums[0][wave][l];
#pragma unroll
    for (int i = 1; i < kFewWaves; ++i) sum += sums[i][wave][l];
    const int n = (group >> 1) * 64 + h * 32 + (group & 1) * 16 + 4 * wave;
    __half *row = Y + (int64_t)(l & 31) * ldy;
    union { __half h[4]; halves4_any v; } u;
#pragma unroll
    for (int i = 0; i < 4; ++i) u.h[i] = __float2half_rn(sum[i]);
    if (n + 4 <= N) {
        *reinterpret_cast<halves4_any *>(row + n) = u.v;
    } else {
#pragma unroll
        for (int i = 0; i < 4; ++i)
            if (n + i < N) row[n + i] = u.h[i];
    }
}

// More rows: tiles of 32 RM rows x 128 RN channels, a wavefront has RM x RN fragments of results.  K goes by stages of 256 channels.  Rows
// pass through LDS in the order in which the lanes hold them (two buffers, one barrier per stage); they are asked for AHEAD stages
// ahead and wait in registers.  The weight goes from memory to the registers of the wavefront that uses it, DEPTH stages ahead:
// through LDS it would keep that busier than the matrix cores.  Four wavefronts: two workgroups are a compute unit's, so that one
// multiplies while the other waits at its barrier.
constexpr int kTileWaves = 4;
template <int RM, int RN, int DEPTH, int AHEAD>
struct Mx4Tile {
    static constexpr int kRows = 32 * RM, kChannels = 32 * RN * kTileWaves, kThreads = 64 * kTileWaves;
    static constexpr int kPieces = 4 * RM;                            // KiB of a stage
    static constexpr int kScalesAt = 2 * kPieces * 1024, kScaleBytes = kRows * 8, kLds = kScalesAt + 2 * kScaleBytes;
};

template <int RM, int RN, int DEPTH, int AHEAD>
__global__ __launch_bounds__((Mx4Tile<RM, RN, DEPTH, AHEAD>::kThreads), 2)
void mx4_tile_kernel(const uint8_t *__restrict__ Xq, const uint8_t *__restrict__ Xs, int M, int K, const uint8_t *__restrict__ data,
                     const unsigned *__restrict__ scales, int stages, int N, __half *__restrict__ Y, int64_t ldy, int row_tiles, int tiles,
                     int tiles_per_xcd)
{
    using T = Mx4Tile<RM, RN, DEPTH, AHEAD>;
    static_assert(T::kRows <= T::kThreads, "a thread fetches the scales of a row");
    static_assert(DEPTH % AHEAD == 0, "the registers of a stage's rows are told by its number modulo DEPTH");
    constexpr int NW = kTileWaves, LOADS = T::kPieces / NW, STEPS = 4;
    extern __shared__ __attribute__((aligned(16))) uint8_t lds[];
    // tiles that share weights are neighbours and go to one XCD, behind one L2
    const int tile = (blockIdx.x & 7) * tiles_per_xcd + (blockIdx.x >> 3);
    if (tile >= tiles) return;
    const int m0 = tile % row_tiles * T::kRows, first_group = tile / row_tiles * RN * NW;
    const int t = threadIdx.x, l = t & 63, wave = __builtin_amdgcn_readfirstlane(t >> 6), r = l & 31, h = l >> 5;
    const int blocks = K >> 5;

    // rows: a wavefront fetches 8 rows x 128 bytes at a time, whole cache lines (32 rows x 32 bytes, as a fragment has them: 2368 x 22016 x 4096 in 150 us, 140 so).
    // This lane's offsets from the tile's first row; rows past M and blocks past K are behind the window
    const Window rows = window_of(Xq + (int64_t)m0 * (K >> 1), (unsigned long long)min(M - m0, T::kRows) * (K >> 1));
    constexpr unsigned kBehind = 0xfffffff0u;
    unsigned from[LOADS];
#pragma unroll
    for (int i = 0; i < LOADS; ++i) {
        const int p = wave + i * NW, row = p * 8 + (l >> 3);
        from[i] = row < M - m0 ? (unsigned)row * (unsigned)(K >> 1) + (unsigned)(l & 7) * 16u : kBehind;
    }
    v4i fetched[AHEAD][LOADS];
    v2u fetched_scales[AHEAD];
    const uint8_t *scales_of = Xs + (int64_t)min(m0 + t, M - 1) * blocks;
    auto fetch = [&](int st, v4i (&fetched)[LOADS]) {
#pragma unroll
        for (int i = 0; i < LOADS; ++i) {
            fetched[i] = read16(rows, (l & 7) < blocks - st * 8 ? from[i] : kBehind, (unsigned)st * 128u);
        }
    };
    auto fetch_next = [&](int st, auto set_c) {
        constexpr int set = decltype(set_c)::value;
        if (st >= stages) return;
        fetch(st, fetched[set]);
        if (t < T::kRows) fetched_scales[set] = load_scales(scales_of, st, blocks);
    };
    auto keep = [&](int st, const v4i (&fetched)[LOADS], const v2u placed) {
#pragma unroll
        for (int i = 0; i < LOADS; ++i) {
            const int p = wave + i * NW;
            const int row = p * 8 + (l >> 3), q = l & 7;              // block q of its row, for step q / 2, lane half q % 2
            *reinterpret_cast<v4i *>(lds + ((st & 1) * T::kPieces + (row >> 5) * 4) * 1024 + q * 512 + ((row + q) & 31) * 16) = fetched[i];
        }
        if (t < T::kRows) *reinterpret_cast<v2u *>(lds + T::kScalesAt + (st & 1) * T::kScaleBytes + t * 8) = split_scales(placed);
    };

    const int64_t group0 = first_group + wave * RN;
    const Window wdata = window_of(data + group0 * stages * 4096, (unsigned long long)stages * 4096 * RN);
    const Window wscales = window_of(scales + group0 * stages * 64, (unsigned long long)stages * 256 * RN);
    const unsigned lane16 = (unsigned)l * 16u, lane4 = (unsigned)l * 4u;
    v4i wreg[DEPTH][STEPS][RN];
    unsigned ws[DEPTH][RN], ws_next[RN];
    auto fetch_weight = [&](int d, int s, int st) {
#pragma unroll
        for (int c = 0; c < RN; ++c) wreg[d][s][c] = read16(wdata, lane16 + (unsigned)s * 1024u, weight_stage(c, st, stages, 4096u));
    };
    auto fetch_weight_scales = [&](unsigned (&into)[RN], int st) {
#pragma unroll
        for (int c = 0; c < RN; ++c) into[c] = __builtin_amdgcn_raw_buffer_load_b32(wscales, lane4, weight_stage(c, st, stages, 256u), 0);
    };

    v16f acc[RM][RN];
#pragma unroll
    for (int i = 0; i < RM; ++i)
#pragma unroll
        for (int c = 0; c < RN; ++c)
#pragma unroll
            for (int e = 0; e < 16; ++e) acc[i][c][e] = 0.f;
    fetch(0, fetched[0]);
#pragma unroll
    for (int d = 0; d < DEPTH; ++d) {
        fetch_weight_scales(ws[d], d);
#pragma unroll
        for (int s = 0; s < STEPS; ++s) fetch_weight(d, s, d);
    }
    v2u first = {0u, 0u};
    if (t < T::kRows) first = first_scales(scales_of, blocks);
    keep(0, fetched[0], first);
    if constexpr (AHEAD > 1) fetch_next(1, std::integral_constant<int, 1>{});
    auto stage = [&](int st, auto depth_c) {
        constexpr int d = decltype(depth_c)::value;
        lds_barrier();                                                // this stage is in LDS; nobody reads the other buffer any more
        fetch_weight_scales(ws_next, st + DEPTH);
        fetch_next(st + AHEAD, std::integral_constant<int, (d + AHEAD) % AHEAD>{});
        const uint8_t *at = lds + (st & 1) * T::kPieces * 1024;
        unsigned xs[RM];
#pragma unroll
        for (int i = 0; i < RM; ++i)
            xs[i] = *reinterpret_cast<const unsigned *>(lds + T::kScalesAt + (st & 1) * T::kScaleBytes + (i * 32 + r) * 8 + h * 4);
        // a step's fragments are read while the one before is multiplied; no further ahead, there are no registers for them
        v4i x[2][RM];
        auto read = [&](int s) {
#pragma unroll
            for (int i = 0; i < RM; ++i) x[s & 1][i] = *reinterpret_cast<const v4i *>(at + (i * 4 + s) * 1024 + h * 512 + ((r + 2 * s + h) & 31) * 16);
        };
        read(0);
#pragma unroll
        for (int s = 0; s < STEPS; ++s) {
            __builtin_amdgcn_sched_barrier(0);
            if (s + 1 < STEPS) read(s + 1);
#pragma unroll
            for (int i = 0; i < RM; ++i)
#pragma unroll
                for (int c = 0; c < RN; ++c)
                    acc[i][c] = s == 0   ? multiply<0>(wreg[d][s][c], x[s & 1][i], acc[i][c], ws[d][c], xs[i])
                                : s == 1 ? multiply<1>(wreg[d][s][c], x[s & 1][i], acc[i][c], ws[d][c], xs[i])
                                : s == 2 ? multiply<2>(wreg[d][s][c], x[s & 1][i], acc[i][c], ws[d][c], xs[i])
                                         : multiply<3>(wreg[d][s][c], x[s & 1][i], acc[i][c], ws[d][c], xs[i]);
            // the weight's next fragments take these registers: not asked for before they are free
#pragma unroll
            for (int i = 0; i < RM; ++i)
#pragma unroll
                for (int c = 0; c < RN; ++c) asm volatile("" : "+v"(acc[i][c]));
            __builtin_amdgcn_sched_barrier(0);
            fetch_weight(d, s, st + DEPTH);
        }
#pragma unroll
        for (int c = 0; c < RN; ++c) ws[d][c] = ws_next[c];
        keep(st + 1, fetched[(d + 1) % AHEAD], place_scales(fetched_scales[(d + 1) % AHEAD], st + 1, blocks));
    };
    int st = 0;
    auto several = [&](auto count_c, auto self) {                     // stages st .. st + count - 1, of which the last may be missing
        constexpr int d = decltype(count_c)::value;
        if constexpr (d < DEPTH) {
            if (st + d >= stages) return;
            stage(st + d, count_c);
            self(std::integral_constant<int, d + 1>{}, self);
        }
    };
    for (; st + DEPTH <= stages; st += DEPTH) {
        stage(st, std::integral_constant<int, 0>{});
        if constexpr (DEPTH > 1) stage(st + 1, std::integral_constant<int, 1>{});
        if constexpr (DEPTH > 2) {
            stage(st + 2, std::integral_constant<int, 2>{});
            stage(st + 3, std::integral_constant<int, 3>{});
        }
    }
    if constexpr (DEPTH > 1) several(std::integral_constant<int, 0>{}, several);
    auto row_of = [&](int i) { return m0 + i * 32 + r; };
    auto channel = [&](int c) {
        const int group = first_group + wave * RN + c;
        return (group >> 1) * 64 + 32 * h + (group & 1) * 16;
    };
#pragma unroll
    for (int i = 0; i < RM; ++i)
        if (row_of(i) < M)
#pragma unroll
            for (int c = 0; c < RN; ++c) store_fragment(Y + (int64_t)row_of(i) * ldy, channel(c), N, acc[i][c]);
}

template <int RM, int RN, int DEPTH, int AHEAD>
static sqap_status launch_tile(const uint8_t *Xq, const uint8_t *Xs, int M, const Mx4Weight &w, __half *Y, int64_t ldy, hipStream_t st)
{
    using T = Mx4Tile<RM, RN, DEPTH, AHEAD>;
    static std::atomic<bool> ready[kMaxDeviceSlots];
    if (T::kLds > 65536 && !ready[device_slot()].load(std::memory_order_relaxed)) {
        SQAP_HIP_CHECK(hipFuncSetAttribute(reinterpret_cast<const void *>(mx4_tile_kernel<RM, RN, DEPTH, AHEAD>),
                                           hipFuncAttributeMaxDynamicSharedMemorySize, T::kLds));
        ready[device_slot()].store(true, std::memory_order_relaxed);
    }
    const int row_tiles = (M + T::kRows - 1) / T::kRows, tiles = row_tiles * ((w.N + T::kChannels - 1) / T::kChannels), per_xcd = (tiles + 7) / 8;
    hipLaunchKernelGGL((mx4_tile_kernel<RM, RN, DEPTH, AHEAD>), dim3(per_xcd * 8), dim3(T::kThreads), T::kLds, st, Xq, Xs, M, w.K, w.data,
                       w.scales, w.stages, w.N, Y, ldy, row_tiles, tiles, per_xcd);
    SQAP_HIP_CHECK(hipGetLastError());
    return SQAP_OK;
}

// 32 x 32 outputs per workgroup, K shared by its wavefronts, up to two workgroups per compute unit: 148 x 4096 x 4096 (640 of them) takes
// 11.4 us so and 8.9 in tiles, 100 x 4096 x 4096 (512) 8.6 and 8.8, 100 x 4096 x 11008 17.6 and 24.2.
// Otherwise the tile whose rounds over the 256 compute units cost least.  A round's cost is what was measured, in 0.1 us at K = 4096 (the first
// costs some 3 us more for all of them; other K scale all alike): 320 x 4096 takes 9.5 / 12.7 / 14.6 / 17.8 us in the four kinds, 148 x 12288
// 16.9 / 14.4 / 17.2 / 20.7, 148 x 22016 21.9 / 23.2 / 19.3 / 22.3, 800 x 12288 38.1 / 35.6 / 31.7 / 34.1, 2368 x 22016 190 / 159 / 155 / 132.
// Over 44 shapes of 40 to 2368 rows the choice is 1.4 in 100 from the best of them on average.
sqap_status launch_mx4_linear(const uint8_t *Xq, const uint8_t *Xs, int M, const Mx4Weight &w, __half *Y, int64_t ldy, hipStream_t st)
{
    const auto tiles = [&](int rows, int channels) { return ((int64_t)M + rows - 1) / rows * ((w.N + channels - 1) / channels); };
    if (M <= 32 || tiles(32, 32) <= 512) {
        const int row_tiles = (M + 31) / 32, items = (w.N + 63) / 64 * 2 * row_tiles, per_xcd = (items + 7) / 8;
        hipLaunchKernelGGL(mx4_few_kernel, dim3(per_xcd * 8), dim3(64 * kFewWaves), 0, st, Xq, Xs, M, w.K, w.data, w.scales, w.stages, w.N, Y, ldy,
                           row_tiles, items, per_xcd);
        SQAP_HIP_CHECK(hipGetLastError());
        return SQAP_OK;
    }
    const auto cost = [&](int rows, int channels, int64_t round) { return (tiles(rows, channels) + 255) / 256 * round; };
    const int64_t c64 = cost(64, 128, 65), c128 = cost(128, 128, 95), c160 = cost(160, 128, 115), wide = cost(128, 256, 140);
    const int64_t least = std::min({c64, c128, c160, wide});
    if (c64 == least) return launch_tile<2, 1, 4, 2>(Xq, Xs, M, w, Y, ldy, st);
    if (c128 == least) return launch_tile<4, 1, 2, 2>(Xq, Xs, M, w, Y, ldy, st);
    if (c160 == least) return launch_tile<5, 1, 2, 2>(Xq, Xs, M, w, Y, ldy, st);
    return launch_tile<4, 2, 1, 1>(Xq, Xs, M, w, Y, ldy, st);
}

}  // namespace sqap
