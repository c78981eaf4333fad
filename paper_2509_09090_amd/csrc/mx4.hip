// Microscaled 4-bit floating point: 32 consecutive channels share a power of two, the elements are 0, 1/2, 1, 3/2, 2, 3, 4, 6 with a
// sign.  Quantizer, packed weight and product; the matrix cores take both operands and their scales as they are.
//
// v_mfma_scale_f32_16x16x128_f8f6f4 with 4-bit operands: lane l holds row l % 16 of an operand and the 32 channels (one block, 16 bytes)
// 32 (l / 16) of the 128, with that block's scale in a byte of a register.  So a fragment of 16 rows x 128 channels is 1 KiB of codes
// and 64 scale bytes, and neither is touched by the vector ALU.  Products of two elements are exact, sums are binary32.
#include "common.h"

namespace sqap {

typedef int v4i __attribute__((ext_vector_type(4)));
typedef int v8i __attribute__((ext_vector_type(8)));
typedef float v4f __attribute__((ext_vector_type(4)));
typedef unsigned v2u __attribute__((ext_vector_type(2)));

// ---------------------------------------------------------------- quantizer

// One thread per 8 channels, four threads per block.  The largest magnitude as an integer: the bit patterns of halves order as their
// values do, with infinities and then NaN above all numbers, so that a block which holds one is told by the same maximum.
// e = floor(log2 amax) - 2 puts the largest element into [4, 8): the conversion rounds to nearest, halfway cases to the even code, and
// takes what is above 6 to 6; dividing by 2^e is exact.
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
    const int per_row = (K / 8 + 255) / 256;
    hipLaunchKernelGGL(mx4_quantize_kernel, dim3((unsigned)M * per_row), dim3(256), 0, st, X, ldx, rows, K, per_row, Xq, Xs);
    SQAP_HIP_CHECK(hipGetLastError());
    return SQAP_OK;
}

// ---------------------------------------------------------------- packed weight

// Fragments of 16 channels x 128 codes in the order in which the lanes hold them: a wavefront reads 1 KiB contiguous.  The channels of a
// span of 64 are dealt to its four fragments so that the sixteen results a lane gets from them (fragment c, register i, lane group g:
// channel 16 g + 4 c + i) are neighbours: 32 bytes of an output row.  Scales: a lane's bytes of four fragments along K in one word.
// Past N and K: codes of zero with a scale of one.
__global__ __launch_bounds__(256) void mx4_pack_kernel(const uint8_t *__restrict__ Wq, const uint8_t *__restrict__ Ws, int N, int K, int ksteps,
                                                       int kquads, uint8_t *__restrict__ data, unsigned *__restrict__ scales)
{
    const int group = blockIdx.x, l = threadIdx.x & 63, r = l & 15, g = l >> 4;
    const int n = (group >> 2) * 64 + (r >> 2) * 16 + (group & 3) * 4 + (r & 3), blocks = K >> 5;
    for (int ks = threadIdx.x >> 6; ks < ksteps; ks += 4) {
        const int block = ks * 4 + g;
        v4i v = {0, 0, 0, 0};
        if (n < N && block < blocks) v = *reinterpret_cast<const v4i *>(Wq + (int64_t)n * (K >> 1) + block * 16);
        *reinterpret_cast<v4i *>(data + (((int64_t)group * ksteps + ks) * 64 + l) * 16) = v;
    }
    for (int kq = threadIdx.x >> 6; kq < kquads; kq += 4) {
        unsigned w = 0;
        for (int s = 0; s < 4; ++s) {
            const int block = kq * 16 + s * 4 + g;
            const unsigned b = n < N && block < blocks ? Ws[(int64_t)n * blocks + block] : 127u;
            w |= b << (8 * s);
        }
        scales[((int64_t)group * kquads + kq) * 64 + l] = w;
    }
}

sqap_status launch_mx4_pack(const uint8_t *Wq, const uint8_t *Ws, const Mx4Weight &w, hipStream_t st)
{
    hipLaunchKernelGGL(mx4_pack_kernel, dim3(w.n_groups), dim3(256), 0, st, Wq, Ws, w.N, w.K, w.ksteps, w.kquads, w.data, w.scales);
    SQAP_HIP_CHECK(hipGetLastError());
    return SQAP_OK;
}

// ---------------------------------------------------------------- products

template <int SA, int SB>
__device__ __forceinline__ v4f multiply(const v4i &a, const v4i &b, const v4f &c, unsigned scale_a, unsigned scale_b)
{
    const v8i wa = {a[0], a[1], a[2], a[3], 0, 0, 0, 0}, wb = {b[0], b[1], b[2], b[3], 0, 0, 0, 0};
    return __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(wa, wb, c, 4, 4, SA, (int)scale_a, SB, (int)scale_b);
}

// Four neighbouring outputs of a row, from channel n on.
__device__ __forceinline__ void store_outputs(__half *__restrict__ Y, int64_t at, int n, int N, const v4f &v)
{
    union { __half h[4]; halves4_any v; } u;
#pragma unroll
    for (int i = 0; i < 4; ++i) u.h[i] = __float2half_rn(v[i]);
    if (n + 4 <= N) {
        *reinterpret_cast<halves4_any *>(Y + at + n) = u.v;
    } else {
#pragma unroll
        for (int i = 0; i < 4; ++i)
            if (n + i < N) Y[at + n + i] = u.h[i];
    }
}

// Up to 16 rows: a workgroup owns 16 channels, its eight wavefronts share K in quads of four fragments, and the sums are added in LDS in
// the order of the wavefronts.  Bound by streaming the weight.
constexpr int kFewWaves = 8;
__global__ __launch_bounds__(64 * kFewWaves) void mx4_few_kernel(const uint8_t *__restrict__ Xq, const uint8_t *__restrict__ Xs, int M, int K,
                                                                 const uint8_t *__restrict__ data, const unsigned *__restrict__ scales,
                                                                 int ksteps, int kquads, int N, __half *__restrict__ Y, int64_t ldy)
{
    __shared__ v4f sums[kFewWaves - 1][64];
    const int group = blockIdx.x, l = threadIdx.x & 63, wave = threadIdx.x >> 6, g = l >> 4, blocks = K >> 5;
    const int token = min(l & 15, M - 1);
    const uint8_t *x = Xq + (int64_t)token * (K >> 1), *xs = Xs + (int64_t)token * blocks;
    v4f acc = {0.f, 0.f, 0.f, 0.f};
    for (int kq = wave; kq < kquads; kq += kFewWaves) {
        v4i w[4], v[4];
        unsigned sx[4];
        const unsigned sw = scales[((int64_t)group * kquads + kq) * 64 + l];
#pragma unroll
        for (int s = 0; s < 4; ++s) {
            const int ks = kq * 4 + s, block = ks * 4 + g < blocks ? ks * 4 + g : 0;       // (past K: times codes of zero, and the row's own scale)
            w[s] = v4i{0, 0, 0, 0};
            if (ks < ksteps) w[s] = *reinterpret_cast<const v4i *>(data + (((int64_t)group * ksteps + ks) * 64 + l) * 16);
            v[s] = *reinterpret_cast<const v4i *>(x + block * 16);
            sx[s] = xs[block];
        }
        acc = multiply<0, 0>(w[0], v[0], acc, sw, sx[0]);
        acc = multiply<1, 0>(w[1], v[1], acc, sw, sx[1]);
        acc = multiply<2, 0>(w[2], v[2], acc, sw, sx[2]);
        acc = multiply<3, 0>(w[3], v[3], acc, sw, sx[3]);
    }
    if (wave > 0) sums[wave - 1][l] = acc;
    __syncthreads();
    if (wave > 0 || (l & 15) >= M) return;
    for (int i = 0; i < kFewWaves - 1; ++i) acc += sums[i][l];
    store_outputs(Y, (int64_t)(l & 15) * ldy, (group >> 2) * 64 + g * 16 + (group & 3) * 4, N, acc);
}

// More rows: tiles of 16 RM WM rows x 64 WN channels; a wavefront has RM x 4 fragments of results (64 channels: one span).  Rows pass
// through LDS in the order in which the lanes hold them, two fragments along K per stage and two stages; they are loaded straight to LDS.
// The weight goes from memory to the registers of the wavefronts that use it.  WK wavefronts share K: each takes one of a stage's two
// fragments, and the sums are added in LDS at the end.
template <int RM, int WM, int WN, int WK>
struct Mx4Tile {
    static constexpr int kRows = 16 * RM * WM, kChannels = 64 * WN, kWaves = WM * WN * WK, kThreads = 64 * kWaves;
    static constexpr int kGroups = RM * WM, kPieces = 2 * kGroups;                         // KiB of a stage
    static constexpr int kScalesAt = 2 * kPieces * 1024, kScaleBytes = kRows * 8;
    static constexpr int kMerge = WK > 1 ? (WK - 1) * WM * WN * RM * 4 * 64 * 16 : 0;
    static constexpr int kLds = kScalesAt + 2 * kScaleBytes > kMerge ? kScalesAt + 2 * kScaleBytes : kMerge;
};

template <int RM, int WM, int WN, int WK>
__global__ __launch_bounds__((Mx4Tile<RM, WM, WN, WK>::kThreads))
void mx4_tile_kernel(const uint8_t *__restrict__ Xq, const uint8_t *__restrict__ Xs, int M, int K, const uint8_t *__restrict__ data,
                     const unsigned *__restrict__ scales, int ksteps, int kquads, int N, __half *__restrict__ Y, int64_t ldy, int row_tiles,
                     int tiles, int tiles_per_xcd)
{
    using T = Mx4Tile<RM, WM, WN, WK>;
    constexpr int NW = T::kWaves, LOADS = (T::kPieces + NW - 1) / NW;
    static_assert(WK == 1 || WK == 2, "a stage has two fragments along K");
    static_assert(T::kRows <= T::kThreads, "a thread fetches the scales of a row");
    extern __shared__ __attribute__((aligned(16))) uint8_t lds[];
    // tiles that share weights are neighbours and go to one XCD, behind one L2
    const int tile = (blockIdx.x & 7) * tiles_per_xcd + (blockIdx.x >> 3);
    if ((int)(blockIdx.x >> 3) >= tiles_per_xcd || tile >= tiles) return;
    const int m0 = tile % row_tiles * T::kRows, span0 = tile / row_tiles * WN;
    const int t = threadIdx.x, l = t & 63, wave = __builtin_amdgcn_readfirstlane(t >> 6), r = l & 15, g = l >> 4;
    const int wk = wave / (WM * WN), wm = wave % (WM * WN) / WN, wn = wave % WN;
    const int blocks = K >> 5, stages = ksteps >> 1;

    // this lane's rows of the pieces that the wavefront fetches, and the row whose scales the thread fetches
    const uint8_t *from[LOADS];
#pragma unroll
    for (int i = 0; i < LOADS; ++i) from[i] = Xq + (int64_t)min(m0 + ((wave + i * NW) >> 1) * 16 + r, M - 1) * (K >> 1);
    const uint8_t *scales_of = Xs + (int64_t)min(m0 + t, M - 1) * blocks;
    auto fetch = [&](int st) {
#pragma unroll
        for (int i = 0; i < LOADS; ++i) {
            const int p = wave + i * NW;
            if (T::kPieces % NW != 0 && p >= T::kPieces) break;
            const int block = (st * 2 + (p & 1)) * 4 + g;
            const uint8_t *at = from[i] + (block < blocks ? block : 0) * 16;                // (past K: times codes of zero)
            __builtin_amdgcn_global_load_lds((const __attribute__((address_space(1))) v4i *)at,
                                             (__attribute__((address_space(3))) void *)(lds + ((st & 1) * T::kPieces + p) * 1024), 16, 0, 0);
        }
    };
    auto fetch_scales = [&](int st) {
        v2u w = {0x7f7f7f7fu, 0x7f7f7f7fu};
        if (t < T::kRows) {
            if (st * 8 + 8 <= blocks) {
                __builtin_memcpy(&w, scales_of + st * 8, 8);
            } else {
                for (int b = st * 8; b < blocks; ++b) {
                    const unsigned shift = 8 * (b & 3), s = scales_of[b];
                    if (b & 4) w[1] = (w[1] & ~(255u << shift)) | s << shift;
                    else w[0] = (w[0] & ~(255u << shift)) | s << shift;
                }
            }
        }
        return w;
    };
    // two bytes per lane group: the group's blocks of the stage's two fragments
    auto keep_scales = [&](int st, const v2u w) {
        if (t < T::kRows)
            *reinterpret_cast<v2u *>(lds + T::kScalesAt + (st & 1) * T::kScaleBytes + t * 8) =
                v2u{__builtin_amdgcn_perm(w[1], w[0], 0x05010400u), __builtin_amdgcn_perm(w[1], w[0], 0x07030602u)};
    };

    const int64_t group0 = (int64_t)(span0 + wn) * 4;
    const uint8_t *wdata = data + (group0 * ksteps * 64 + l) * 16;
    const unsigned *wscales = scales + group0 * kquads * 64 + l;
    constexpr int STEPS = 2 / WK;                                     // fragments along K that this wavefront takes of a stage
    v4i wreg[STEPS][4];
    unsigned ws[4];
    auto fetch_weight = [&](int st) {
#pragma unroll
        for (int s = 0; s < STEPS; ++s)
#pragma unroll
            for (int c = 0; c < 4; ++c) wreg[s][c] = *reinterpret_cast<const v4i *>(wdata + ((int64_t)c * ksteps + 2 * st + s * WK + wk) * 1024);
    };

    v4f acc[RM][4];
#pragma unroll
    for (int i = 0; i < RM; ++i)
#pragma unroll
        for (int c = 0; c < 4; ++c) acc[i][c] = v4f{0.f, 0.f, 0.f, 0.f};
    fetch(0);
    keep_scales(0, fetch_scales(0));
    for (int st = 0; st < stages; ++st) {
        if ((st & 1) == 0) {
#pragma unroll
            for (int c = 0; c < 4; ++c) ws[c] = wscales[((int64_t)c * kquads + (st >> 1)) * 64];
        } else {
#pragma unroll
            for (int c = 0; c < 4; ++c) ws[c] >>= 16;
        }
        fetch_weight(st);
        __syncthreads();                                              // this stage has arrived; nobody reads the other buffer any more
        v2u next = {0u, 0u};
        if (st + 1 < stages) {
            fetch(st + 1);
            next = fetch_scales(st + 1);
        }
#pragma unroll
        for (int s = 0; s < STEPS; ++s) {
            const int f = s * WK + wk;
            v4i x[RM];
            unsigned xs[RM];
#pragma unroll
            for (int i = 0; i < RM; ++i) {
                const int group = wm * RM + i;
                x[i] = *reinterpret_cast<const v4i *>(lds + (((st & 1) * T::kPieces) + group * 2 + f) * 1024 + l * 16);
                xs[i] = *reinterpret_cast<const unsigned short *>(lds + T::kScalesAt + (st & 1) * T::kScaleBytes + (group * 16 + r) * 8 + g * 2);
            }
            if (WK == 1) {
#pragma unroll
                for (int i = 0; i < RM; ++i)
#pragma unroll
                    for (int c = 0; c < 4; ++c)
                        acc[i][c] = s == 0 ? multiply<0, 0>(wreg[s][c], x[i], acc[i][c], ws[c], xs[i]) : multiply<1, 1>(wreg[s][c], x[i], acc[i][c], ws[c], xs[i]);
            } else {
                const int shift = 8 * wk;
#pragma unroll
                for (int i = 0; i < RM; ++i)
#pragma unroll
                    for (int c = 0; c < 4; ++c) acc[i][c] = multiply<0, 0>(wreg[s][c], x[i], acc[i][c], ws[c] >> shift, xs[i] >> shift);
            }
        }
        if (st + 1 < stages) keep_scales(st + 1, next);
    }
    if (WK > 1) {
        __syncthreads();
        v4f *merge = reinterpret_cast<v4f *>(lds) + (wm * WN + wn) * RM * 4 * 64 + l;
        if (wk > 0) {
#pragma unroll
            for (int i = 0; i < RM; ++i)
#pragma unroll
                for (int c = 0; c < 4; ++c) merge[(i * 4 + c) * 64] = acc[i][c];
        }
        __syncthreads();
        if (wk > 0) return;
#pragma unroll
        for (int i = 0; i < RM; ++i)
#pragma unroll
            for (int c = 0; c < 4; ++c) acc[i][c] += merge[(i * 4 + c) * 64];
    }
#pragma unroll
    for (int i = 0; i < RM; ++i) {
        const int m = m0 + (wm * RM + i) * 16 + r;
        if (m >= M) continue;
        const int n = (span0 + wn) * 64 + g * 16;
        const int64_t at = (int64_t)m * ldy;
#pragma unroll
        for (int c = 0; c < 4; c += 2) {
            if (n + 4 * c + 8 <= N) {
                union { __half h[8]; halves8_any v; } u;
#pragma unroll
                for (int e = 0; e < 8; ++e) u.h[e] = __float2half_rn(acc[i][c + (e >> 2)][e & 3]);
                *reinterpret_cast<halves8_any *>(Y + at + n + 4 * c) = u.v;
            } else {
                store_outputs(Y, at, n + 4 * c, N, acc[i][c]);
                store_outputs(Y, at, n + 4 * c + 4, N, acc[i][c + 1]);
            }
        }
    }
}

template <int RM, int WM, int WN, int WK>
static sqap_status launch_tile(const uint8_t *Xq, const uint8_t *Xs, int M, const Mx4Weight &w, __half *Y, int64_t ldy, hipStream_t st)
{
    using T = Mx4Tile<RM, WM, WN, WK>;
    static std::atomic<bool> ready[kMaxDeviceSlots];
    if (T::kLds > 65536 && !ready[device_slot()].load(std::memory_order_relaxed)) {
        SQAP_HIP_CHECK(hipFuncSetAttribute(reinterpret_cast<const void *>(mx4_tile_kernel<RM, WM, WN, WK>),
                                           hipFuncAttributeMaxDynamicSharedMemorySize, T::kLds));
        ready[device_slot()].store(true, std::memory_order_relaxed);
    }
    const int row_tiles = (M + T::kRows - 1) / T::kRows, tiles = row_tiles * ((w.N + T::kChannels - 1) / T::kChannels), per_xcd = (tiles + 7) / 8;
    hipLaunchKernelGGL((mx4_tile_kernel<RM, WM, WN, WK>), dim3(per_xcd * 8), dim3(T::kThreads), T::kLds, st, Xq, Xs, M, w.K, w.data, w.scales,
                       w.ksteps, w.kquads, w.N, Y, ldy, row_tiles, tiles, per_xcd);
    SQAP_HIP_CHECK(hipGetLastError());
    return SQAP_OK;
}

sqap_status launch_mx4_linear(const uint8_t *Xq, const uint8_t *Xs, int M, const Mx4Weight &w, __half *Y, int64_t ldy, hipStream_t st)
{
    if (M <= 16) {
        hipLaunchKernelGGL(mx4_few_kernel, dim3((w.N + 63) / 64 * 4), dim3(64 * kFewWaves), 0, st, Xq, Xs, M, w.K, w.data, w.scales, w.ksteps,
                           w.kquads, w.N, Y, ldy);
        SQAP_HIP_CHECK(hipGetLastError());
        return SQAP_OK;
    }
    if (M <= 64) return launch_tile<2, 2, 1, 2>(Xq, Xs, M, w, Y, ldy, st);
    if (M <= 512) return launch_tile<5, 2, 1, 2>(Xq, Xs, M, w, Y, ldy, st);
    return launch_tile<8, 2, 4, 1>(Xq, Xs, M, w, Y, ldy, st);
}

}  // namespace sqap
