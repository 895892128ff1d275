// Matrix products with bias, activation and residual in their epilogue, and their gradients (flashbev_linear of flashbev.h).
//
// One kernel, gemm_kernel, forms D[M x N] = A[M x K] B[N x K]^T on the fifth-generation tensor cores for the three products
//
//     out         = x       weight^T     A = x  (K-major),      B = weight   (K-major)
//     grad_x      = dz      weight       A = dz (K-major),      B = weight^T (contiguous along N: MN-major)
//     grad_weight = dz^T    x            A = dz^T (MN-major),   B = x^T      (MN-major)
//
// persistent CTAs, one per SM: one thread fills a ring of shared-memory stages by TMA, one issues the products into
// tensor memory, and 8 or 16 warps take finished sums from there through bias, activation and residual to global memory.  In every tile,
// operands are rows of bf16 numbers with the swizzle of TMA, whether a row runs along K or along M or N.
//
// Operands that TMA cannot read so -- float32 ones, which become three bf16 pieces, and bf16 ones whose rows are no whole 16-byte
// vectors -- are laid out in the caller's scratch by a kernel ahead of the product.  (Sixteen warps that load, split and store the
// stages in the product itself were bound by the latency of what they can have in flight: 40000 x 1024 x 256, float32: 172 us,
// tensor cores busy for 39 %.)
#include "flashbev.h"
#include "launch.cuh"
#include "tcgen05.cuh"

#include <cuda_bf16.h>
#include <math.h>
#include <stdio.h>
#include <stdlib.h>
#include <string.h>

#include <algorithm>
#include <type_traits>

using namespace flashbev_host;
using namespace flashbev_sm100;

namespace {

using bf16 = __nv_bfloat16;

constexpr int kBM = 128;            // rows of a tile: the 128 lanes of tensor memory
constexpr int kSmemLimit = 227 * 1024;
constexpr int kControlBytes = 512;  // barriers and the like

// Elements of float32 operands: x = p0 + p1 + p2, each piece the bf16 number nearest to what is left.  Every difference is exact and
// 8 + 8 + 8 bits hold the 24 of x.  Of the nine products the three left out, p1 p2, p2 p1 and p2 p2, are at most 2^-24 |a| |b|.  Two tf32
// pieces cost the same tensor time (three products at half the rate) and lose two bits.
__device__ __forceinline__ uint32_t pack(float lo, float hi)
{
    __nv_bfloat162 v = __floats2bfloat162_rn(lo, hi);
    uint32_t r;
    memcpy(&r, &v, 4);
    return r;
}

__device__ __forceinline__ float low(uint32_t v) { return __uint_as_float(v << 16); }
__device__ __forceinline__ float high(uint32_t v) { return __uint_as_float(v & 0xffff0000u); }

__device__ __forceinline__ float to_float(float v) { return v; }
__device__ __forceinline__ float to_float(bf16 v) { return __bfloat162float(v); }
template <typename T>
__device__ __forceinline__ T from_float(float v)
{
    if constexpr (std::is_same<T, float>::value) return v;
    else return __float2bfloat16_rn(v);
}

// ---- activations ------------------------------------------------------------------------------------------------------------

__device__ __forceinline__ float exp2_approx(float v)
{
    float r;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(v));
    return r;
}

__device__ __forceinline__ float rcp_approx(float v)
{
    float r;
    asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(v));
    return r;
}

__device__ __forceinline__ float max_nan(float a, float b)
{
    float r;
    asm("max.NaN.f32 %0, %1, %2;" : "=f"(r) : "f"(a), "f"(b));
    return r;
}

__device__ __forceinline__ float2 both(float v) { return make_float2(v, v); }

// Phi(-a) of the standard normal distribution for 0 <= a <= 14, to 3e-5 of itself up to a = 6 (bf16 rounds to 2e-3): log2 Phi(-a)
// is smooth, and the polynomial below is its least-maximum fit of degree 8 over that range, the error weighted by 1 / (1 + 20 (a -
// 6)) behind 6 (reweighted least squares).  Eight two-wide multiply-adds and one special function; erfc by rational forms takes two
// of those, and with them the epilogue of 184950 x 256 numbers waits for the special function unit: 54 us against 36 without an
// activation, 45 so.
__device__ __forceinline__ float2 normal_tail(float2 a)
{
    float2 q = __ffma2_rn(a, both(3.97813622e-8f), both(-2.38079224e-6f));
    q = __ffma2_rn(q, a, both(6.07985676e-5f));
    q = __ffma2_rn(q, a, both(-8.80368869e-4f));
    q = __ffma2_rn(q, a, both(8.17755144e-3f));
    q = __ffma2_rn(q, a, both(-5.30334003e-2f));
    q = __ffma2_rn(q, a, both(-4.59630847e-1f));
    q = __ffma2_rn(q, a, both(-1.15070558f));
    q = __ffma2_rn(q, a, both(-1.00003982f));
    return make_float2(exp2_approx(q.x), exp2_approx(q.y));
}

// |z|, at most 14, where Phi(-a) is less than float32 holds (and NaN is 14)
__device__ __forceinline__ float2 magnitude(float2 z) { return make_float2(fminf(fabsf(z.x), 14.0f), fminf(fabsf(z.y), 14.0f)); }

template <bool FAST>
__device__ __forceinline__ float normal_cdf(float z)
{
    if constexpr (!FAST) return 0.5f * erfcf(-0.70710678f * z);
    const float s = normal_tail(magnitude(both(z))).x;
    return z < 0.0f ? s : 1.0f - s;
}

template <bool FAST>
__device__ __forceinline__ float sigmoid(float z)
{
    return FAST ? rcp_approx(1.0f + exp2_approx(-1.44269504f * z)) : 1.0f / (1.0f + expf(-z));
}

// Two numbers at a time.  GELU, where it is FAST, as max(z, 0) - |z| Phi(-|z|): no difference of near numbers on either side.  (Phi(-20)
// is 0 in float32, and no infinity is multiplied by it.)  FAST is for bf16 results whose kernel the special functions bound; GELU is
// then 3e-5 of its negative part off, a hundredth of its rounding.
template <bool FAST, int ACT>
__device__ __forceinline__ float2 activate(float2 z)
{
    if (ACT == FLASHBEV_ACT_RELU) return make_float2(max_nan(z.x, 0.0f), max_nan(z.y, 0.0f));
    if (ACT == FLASHBEV_ACT_GELU) {
        if constexpr (!FAST) return make_float2(fmaxf(z.x, -20.0f) * normal_cdf<false>(z.x), fmaxf(z.y, -20.0f) * normal_cdf<false>(z.y));
        const float2 a = magnitude(z), s = normal_tail(a), m = make_float2(max_nan(z.x, 0.0f), max_nan(z.y, 0.0f));
        return __ffma2_rn(make_float2(-a.x, -a.y), s, m);
    }
    if (ACT == FLASHBEV_ACT_SILU) return __fmul2_rn(z, make_float2(sigmoid<FAST>(z.x), sigmoid<FAST>(z.y)));
    return z;
}

template <bool FAST, int ACT, int N>
__device__ __forceinline__ void activate(float (&v)[N])
{
#pragma unroll
    for (int i = 0; i < N; i += 2) {
        const float2 q = activate<FAST, ACT>(make_float2(v[i], v[i + 1]));
        v[i] = q.x, v[i + 1] = q.y;
    }
}

template <bool FAST, bool FAST_GELU = FAST, int N>
__device__ __forceinline__ void activate_all(float (&v)[N], int act)
{
    if (act == FLASHBEV_ACT_RELU) activate<FAST, FLASHBEV_ACT_RELU>(v);
    else if (act == FLASHBEV_ACT_GELU) activate<FAST_GELU, FLASHBEV_ACT_GELU>(v);
    else if (act == FLASHBEV_ACT_SILU) activate<FAST, FLASHBEV_ACT_SILU>(v);
}

// g act'(z).  Where the slope is 0 the product is, whatever g.
template <bool FAST>
__device__ __forceinline__ float2 slope_times(float2 g, float2 z, int act)
{
    if (act == FLASHBEV_ACT_RELU) return make_float2(z.x > 0.0f ? g.x : 0.0f, z.y > 0.0f ? g.y : 0.0f);
    if (act == FLASHBEV_ACT_GELU) {  // Phi(z) + z phi(z)
        float2 cdf, e = __fmul2_rn(__fmul2_rn(z, z), both(FAST ? -0.5f * 1.44269504f : -0.5f));
        if constexpr (FAST) {
            const float2 s = normal_tail(magnitude(z));
            cdf = make_float2(z.x < 0.0f ? s.x : 1.0f - s.x, z.y < 0.0f ? s.y : 1.0f - s.y);
            e.x = exp2_approx(e.x), e.y = exp2_approx(e.y);
        } else {
            cdf = make_float2(normal_cdf<false>(z.x), normal_cdf<false>(z.y));
            e.x = expf(e.x), e.y = expf(e.y);
        }
        return __fmul2_rn(g, __ffma2_rn(__fmul2_rn(z, both(0.39894228f)), e, cdf));
    }
    if (act == FLASHBEV_ACT_SILU) {
        const float2 s = make_float2(sigmoid<FAST>(z.x), sigmoid<FAST>(z.y));
        return __fmul2_rn(__fmul2_rn(g, s), __ffma2_rn(z, __fadd2_rn(both(1.0f), make_float2(-s.x, -s.y)), both(1.0f)));
    }
    return g;
}

// ---- the product ------------------------------------------------------------------------------------------------------------

constexpr int kBK = 64;             // K of a stage: a swizzled row of 128 bytes (with rows of 64, TMA takes twice as long for the same bytes)
constexpr int kMostStages = 12;
constexpr int kSlot = 16 * 1024;    // float32 operands: a tile of one piece

// Warps of the epilogue (EW): 16 for short sums, as it is their latency that those wait for (64-column sums of 184950 rows, 64
// columns: 25 us with eight, 20 us with 16); eight for long ones, which leaves shared memory for a fourth stage of 48 KB, and for
// pieces (12 slots).  (Registers are those of a quarter of an SM: the last warps of four, which do nothing, cost none.)
__host__ __device__ constexpr int gemm_threads(int ew) { return 32 * (ew + 4); }
// Bytes behind the ring: a buffer of 32 rows x 128 bytes and a bias of 64 columns per epilogue warp.
__host__ __device__ constexpr int epilogue_bytes(int ew) { return ew * (4096 + 256); }
__host__ __device__ constexpr int ring_bytes(int ew) { return (kSmemLimit - kControlBytes - epilogue_bytes(ew)) / 1024 * 1024; }
constexpr int kAccs = 4;            // most accumulators in tensor memory

struct alignas(64) GemmParams {
    CUtensorMap ta, tb;         // operands
    CUtensorMap tout, tpre;     // results, with store_tma
    int a_mn, b_mn;             // the operand's rows run along M / N, one per k
    int M, N;
    int bn, stages;             // columns of a tile; stages in the ring
    int tiles_n, tiles, kblocks, kshare, splits;  // a tile's sum is cut into `splits` of `kshare` blocks of K (the last may have fewer)
    int run;                    // blocks after which the sum is added to the running one; kshare or more: never
    int columns;                // of tensor memory
    int accs;                   // accumulators in it
    int groups;                 // of epilogue warps, which take accumulators in turn
    int store_tma;              // the results leave through TMA stores
    int wide;                   // ... of 64 columns
    int kept;                   // bytes of B that stay in shared memory: all of the CTA's columns, one tile per block of K; or 0
    void *out, *pre;            // pre: z, or NULL
    const void *residual, *bias;
    long long ld_out, ld_pre, ld_res;
    int out_vec, pre_vec, res_vec;  // bytes that every row's start is a multiple of: 16, 4 or 2
    int act;
    float *partial;             // instead of the epilogue: [splits][M][ld_partial] sums
    long long ld_partial;
    uint32_t *error_word;
#ifdef FLASHBEV_DEBUG_BOUNDS
    long long limits[3];        // of the waits of loads, products and epilogue
#endif
};

// The cycles after which a wait gives up.  The checked build takes them from its environment, so that waits can be made to run out.
enum Role { kLoads, kProducts, kResults };

__device__ __forceinline__ long long wait_limit(const GemmParams &p, Role role)
{
#ifdef FLASHBEV_DEBUG_BOUNDS
    return p.limits[role];
#else
    return kWaitCycles;
#endif
}

// A tile of the epilogue is 32 rows x 32 columns of a result: rows of eight (float32) or four pieces of 16 bytes, swizzled as TMA has
// them.  In tensor memory's layout a lane has a row; in global memory's neighbouring lanes have a row's pieces.  Neither side has bank
// conflicts.
template <typename T>
constexpr int kPiece = 16 / (int)sizeof(T);  // elements of a piece
template <typename T>
constexpr int kPieces32 = 32 / kPiece<T>;    // pieces of a row; also the warp's accesses to the tile
template <typename T>
constexpr int kRows32 = 32 / kPieces32<T>;   // rows of an access

// Where a row's piece lies.  Rows of 128 bytes: float32 tiles, and bf16 ones that are half of a tile of 64 columns (`half` 0 or 1);
// rows of 64 bytes: bf16 tiles by themselves (`half` -1).
template <typename T>
__device__ __forceinline__ int piece_at(int row, int piece, int half)
{
    if (kPieces32<T> == 8) return row * 128 + ((piece ^ (row & 7)) << 4);
    return half < 0 ? row * 64 + ((piece ^ (row >> 1 & 3)) << 4) : row * 128 + (((piece + 4 * half) ^ (row & 7)) << 4);
}

template <typename T>
__device__ __forceinline__ uint4 load_piece(const T *p, int have)
{
    constexpr int E = kPiece<T>;
    if (have >= E) return *reinterpret_cast<const uint4 *>(p);
    T v[E];
#pragma unroll
    for (int i = 0; i < E; ++i) v[i] = i < have ? p[i] : from_float<T>(0.0f);
    uint4 r;
    memcpy(&r, v, 16);
    return r;
}

template <typename T>
__device__ __forceinline__ void store_piece(T *p, uint4 r, int have)
{
    constexpr int E = kPiece<T>;
    if (have >= E) {
        *reinterpret_cast<uint4 *>(p) = r;
        return;
    }
    T v[E];
    memcpy(v, &r, 16);
#pragma unroll
    for (int i = 0; i < E; ++i)
        if (i < have) p[i] = v[i];
}

template <typename T>
__device__ __forceinline__ uint4 piece_of(const float *v)
{
    if constexpr (sizeof(T) == 4)
        return make_uint4(__float_as_uint(v[0]), __float_as_uint(v[1]), __float_as_uint(v[2]), __float_as_uint(v[3]));
    else
        return make_uint4(pack(v[0], v[1]), pack(v[2], v[3]), pack(v[4], v[5]), pack(v[6], v[7]));
}

// The lane's row into a tile
template <typename T>
__device__ __forceinline__ void row_store(const float (&v)[32], unsigned char *tile, int half, int lane)
{
#pragma unroll
    for (int c = 0; c < kPieces32<T>; ++c) *reinterpret_cast<uint4 *>(tile + piece_at<T>(lane, c, half)) = piece_of<T>(v + kPiece<T> * c);
}

// ... and added to from one
template <typename T>
__device__ __forceinline__ void row_add(float (&v)[32], const unsigned char *tile, int half, int lane)
{
#pragma unroll
    for (int c = 0; c < kPieces32<T>; ++c) {
        const uint4 q = *reinterpret_cast<const uint4 *>(tile + piece_at<T>(lane, c, half));
        const uint32_t w[4] = {q.x, q.y, q.z, q.w};
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            if constexpr (kPiece<T> == 4) v[4 * c + j] += __uint_as_float(w[j]);
            else v[8 * c + 2 * j] += low(w[j]), v[8 * c + 2 * j + 1] += high(w[j]);
        }
    }
}

// The lane's row through the activation.  Without the short formulas a number takes about 40 instructions; 32 of them in a row are
// more code than the instruction cache brings in the time of a call (1846 x 72 x 846, GELU: 20 us against 17), so the row goes
// through the warp's buffer, four numbers at a time.
template <bool FAST>
__device__ __forceinline__ void activate_row(float (&v)[32], int act, unsigned char *buffer, int lane)
{
    if (FAST || act < FLASHBEV_ACT_GELU) {
        activate_all<FAST>(v, act);
        return;
    }
    row_store<float>(v, buffer, -1, lane);
#pragma unroll 1
    for (int c = 0; c < 8; ++c) {
        float4 *const at = reinterpret_cast<float4 *>(buffer + piece_at<float>(lane, c, -1));
        float q[4] = {at->x, at->y, at->z, at->w};
        activate_all<FAST>(q, act);
        *at = make_float4(q[0], q[1], q[2], q[3]);
    }
#pragma unroll
    for (int c = 0; c < 8; ++c) {
        const float4 q = *reinterpret_cast<const float4 *>(buffer + piece_at<float>(lane, c, -1));
        v[4 * c] = q.x, v[4 * c + 1] = q.y, v[4 * c + 2] = q.z, v[4 * c + 3] = q.w;
    }
    __syncwarp();
}

// A tile from a matrix to registers, and from there to shared memory.  vec: bytes that every row's start is a multiple of.  16:
// pieces.  Less: a lane has a column, or of bf16 rows on 4-byte boundaries two, so that the warp touches every sector of a row
// once.
template <typename T>
__device__ __forceinline__ void tile_load(uint4 (&r)[kPieces32<T>], const T *base, long long ld, int vec, int row0, int col0, int M, int N, int lane)
{
    if (sizeof(T) == 2 && vec == 4) {
        const T *p = base + (row0 + lane / 16) * ld + col0 + lane % 16 * 2;
        uint32_t w[16];
#pragma unroll
        for (int i = 0; i < 16; ++i, p += 2 * ld) {
            const int have = row0 + 2 * i + lane / 16 < M ? N - (col0 + lane % 16 * 2) : 0;
            w[i] = have >= 2 ? *reinterpret_cast<const uint32_t *>(p) : (have == 1 ? *reinterpret_cast<const unsigned short *>(p) : 0);
        }
        memcpy(r, w, sizeof(w));
        return;
    }
    if (vec == 16) {
        const int row = row0 + lane / kPieces32<T>, col = col0 + lane % kPieces32<T> * kPiece<T>;
        const T *p = base + row * ld + col;
#pragma unroll
        for (int i = 0; i < kPieces32<T>; ++i, p += kRows32<T> * ld)
            if (row + kRows32<T> * i < M && col < N) r[i] = load_piece(p, N - col);
    } else {
        const T *p = base + row0 * ld + col0 + lane;
        T v[32];
#pragma unroll
        for (int i = 0; i < 32; ++i, p += ld) v[i] = row0 + i < M && col0 + lane < N ? *p : from_float<T>(0.0f);
        memcpy(r, v, sizeof(v));
    }
}

template <typename T>
__device__ __forceinline__ void tile_stage(const uint4 (&r)[kPieces32<T>], int vec, unsigned char *tile, int half, int lane)
{
    if (sizeof(T) == 2 && vec == 4) {
        uint32_t w[16];
        memcpy(w, r, sizeof(w));
#pragma unroll
        for (int i = 0; i < 16; ++i)
            reinterpret_cast<uint32_t *>(tile + piece_at<T>(2 * i + lane / 16, lane % 16 / 4, half))[lane % 4] = w[i];
    } else if (vec == 16) {
#pragma unroll
        for (int i = 0; i < kPieces32<T>; ++i)
            *reinterpret_cast<uint4 *>(tile + piece_at<T>(kRows32<T> * i + lane / kPieces32<T>, lane % kPieces32<T>, half)) = r[i];
    } else {
        T v[32];
        memcpy(v, r, sizeof(v));
#pragma unroll
        for (int i = 0; i < 32; ++i) reinterpret_cast<T *>(tile + piece_at<T>(i, lane / kPiece<T>, half))[lane % kPiece<T>] = v[i];
    }
    __syncwarp();
}

// A tile leaves: by one TMA store, which goes on while the warp does, or by ordinary ones.
template <typename T>
__device__ __forceinline__ void tile_leave(const unsigned char *tile, const CUtensorMap *map, T *base, long long ld, int vec, int row0, int col0, int M,
                                           int N, int layer, int lane)
{
    if (map) {
        asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
        __syncwarp();
        if (lane == 0) tma_store_3d(map, col0, row0, layer, smem_u32(tile));
        return;
    }
    __syncwarp();
    if (sizeof(T) == 2 && vec == 4) {
        T *p = base + (row0 + lane / 16) * ld + col0 + lane % 16 * 2;
        const int have = N - (col0 + lane % 16 * 2), rows = M - row0 - lane / 16;
#pragma unroll 8
        for (int i = 0; i < 16; ++i, p += 2 * ld) {
            const uint32_t w = reinterpret_cast<const uint32_t *>(tile + piece_at<T>(2 * i + lane / 16, lane % 16 / 4, -1))[lane % 4];
            if (2 * i < rows && have >= 2) *reinterpret_cast<uint32_t *>(p) = w;
            else if (2 * i < rows && have == 1) *reinterpret_cast<unsigned short *>(p) = (unsigned short)w;
        }
    } else if (vec == 16) {
        const int row = row0 + lane / kPieces32<T>, col = col0 + lane % kPieces32<T> * kPiece<T>;
        T *p = base + row * ld + col;
#pragma unroll
        for (int i = 0; i < kPieces32<T>; ++i, p += kRows32<T> * ld) {
            const uint4 q = *reinterpret_cast<const uint4 *>(tile + piece_at<T>(kRows32<T> * i + lane / kPieces32<T>, lane % kPieces32<T>, -1));
            if (row + kRows32<T> * i < M && col < N) store_piece(p, q, N - col);
        }
    } else if (col0 + lane < N) {
        T *p = base + row0 * ld + col0 + lane;
#pragma unroll 8
        for (int i = 0; i < min(32, M - row0); ++i, p += ld) *p = reinterpret_cast<const T *>(tile + piece_at<T>(i, lane / kPiece<T>, -1))[lane % kPiece<T>];
    }
    __syncwarp();
}

// The shares of tiles' sums that a CTA takes, every gridDim.x-th: tile (m0, n0) and the blocks [k, end) of K.
struct Shares {
    int w, m, n, dm, dn, m0, n0, k, end, split;

    __device__ __forceinline__ explicit Shares(const GemmParams &p)
    {
        w = blockIdx.x, split = w / p.tiles;
        const int t = w - split * p.tiles;
        m = t / p.tiles_n, n = t - m * p.tiles_n;
        dm = gridDim.x / p.tiles_n, dn = gridDim.x - dm * p.tiles_n;
        k = split * p.kshare, end = min(k + p.kshare, p.kblocks);
        m0 = m * kBM, n0 = n * p.bn;
    }
    __device__ __forceinline__ bool more(const GemmParams &p) const { return w < p.tiles * p.splits; }
    // (with several shares to a tile the grid has a CTA for each of them)
    __device__ __forceinline__ void next(const GemmParams &p)
    {
        w += gridDim.x, m += dm, n += dn;
        if (n >= p.tiles_n) n -= p.tiles_n, ++m;
        m0 = m * kBM, n0 = n * p.bn;
    }
};

// float32 operands: every tile of a piece has a slot of shared memory and barriers of its own, twelve in all, six of one block and
// six of the next.  A block's tiles come in the order below, and are released, from the first product that is their last on, in the
// order of `released`; the tiles of the block after the next take the slots in that order, so that they are on their way while the
// last two sixths of this block's products and all of the next one's run.  (40000 x 256 x 256: 36 us, of which the loads by
// themselves take 17 and loads and products 25.)
enum PieceTile { kA0 = 0, kB0 = 1, kB1 = 2, kA1 = 3, kB2 = 4, kA2 = 5 };

struct Slots {
    unsigned now = 0x543210u, after = 0xba9876u;  // slot of tile i of this block and of the next: four bits each
    unsigned turn = 0;                            // parity of every slot's next use

    __device__ __forceinline__ int of(int tile) const { return (int)(now >> 4 * tile & 15u); }
    __device__ __forceinline__ void released()
    {
        const unsigned a0 = now & 15u, b0 = now >> 4 & 15u, b1 = now >> 8 & 15u, a1 = now >> 12 & 15u, b2 = now >> 16 & 15u, a2 = now >> 20 & 15u;
        now = after;
        after = b1 | a1 << 4 | a0 << 8 | b2 << 12 | b0 << 16 | a2 << 20;
    }
};

// MODE: an activation, for results of unshared sums that leave by TMA, or kAny: everything as the parameters say.  What an instance
// does not need would be in its way: the code of the other activations and of rows of any alignment, skipped, cost 8 of 37 us
// (184950 x 64 x 256) in instruction fetches.
//
// Measured: 8192 x 4096 x 4096, bf16, SiLU: 180 to 190 us by itself, the tensor cores busy for 85 % (232 us and 1.18 PFLOP/s in a long
// run, where the power limit holds the clock down); 184950 x 256 x 256: 34 to 39 us, 4.9 TB/s, bound by what is read and written;
// with 1024 columns, GELU and its argument kept, 40000 rows: 42 to 50 us, bound by the 164 MB that it writes (a memset of as much takes
// 45 us; without the activation 37) and, where z is not kept, by the epilogue's instructions (38 us, 28 without the activation); float32
// 40000 x 256 x 256: 36 to 38 us, bound by the tensor cores (54 %) and the loads in turn.  20 warps on an SM leave a
// thread 96 registers: the instances of 16 epilogue warps with float32 results spill 48 to 68 bytes, those for anything 108 and 304.
constexpr int kAny = 4;

// Blocks that have given up on this device (flashbev_linear_given_up)
__device__ unsigned given_up;

template <int kPieces, typename TOUT, int kEpilogue, int MODE>
__global__ void __launch_bounds__(gemm_threads(kEpilogue), 1) gemm_kernel(const __grid_constant__ GemmParams p)
{
    using TIN = typename std::conditional<kPieces == 3, float, bf16>::type;
    constexpr int BK = kBK, kRing = ring_bytes(kEpilogue);
    extern __shared__ __align__(1024) unsigned char ring[];  // (the kernel declares no other: it starts on a swizzle's boundary)
    unsigned char *const staging = ring + kRing;
    float *const bias_rows = reinterpret_cast<float *>(staging + kEpilogue * 4096);  // 64 per warp
    uint64_t *const bars = reinterpret_cast<uint64_t *>(staging + epilogue_bytes(kEpilogue));  // 2 * kMostStages + 2 * kAccs + 2
    uint32_t &tmem_slot = *reinterpret_cast<uint32_t *>(bars + 2 * kMostStages + 2 * kAccs + 2);
    volatile int &failed = *reinterpret_cast<volatile int *>(&tmem_slot + 1);
    const int warp = threadIdx.x / 32, lane = threadIdx.x % 32;
    const uint32_t full = smem_u32(bars), empty = full + 8 * kMostStages, acc_full = empty + 8 * kMostStages, acc_empty = acc_full + 8 * kAccs,
                   last = acc_empty + 8 * kAccs, kept_full = last + 8;
    // Tensor memory.  Two or four accumulators, so that some are taken out while another is filled (long runs may have one).  The tensor cores cut a sum
    // off, not round it, at every instruction, by 3e-8 of the sum on the average (2e-7 where all terms have one sign).  So (1) pieces have a second accumulator for all
    // products but p0 p0, which keeps the five small products of each step from cutting at the large sum; (2) after `run` blocks
    // the sum is added to a running one that stays in tensor memory too, behind the accumulators, and so does the small products'
    // then.
    constexpr int kParts = kPieces == 3 ? 2 : 1;
    const bool runs = MODE == kAny && p.run < p.kshare;
    const int acc_step = runs ? p.bn : kParts * p.bn, sum_at = p.accs * p.bn;
    const unsigned acc_mask = p.accs - 1, acc_shift = p.accs / 2;

    if (threadIdx.x == 0) {
        failed = 0;
        for (int s = 0; s < (kPieces == 3 ? kMostStages : p.stages); ++s) {
            mbar_init(full + 8 * s, 1);
            mbar_init(empty + 8 * s, 1);
        }
        for (int b = 0; b < p.accs; ++b) mbar_init(acc_full + 8 * b, 1), mbar_init(acc_empty + 8 * b, kEpilogue / p.groups);
        mbar_init(last, 1);
        mbar_init(kept_full, 1);
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
        asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
    }
    if (warp == kEpilogue) tmem_alloc(smem_u32(&tmem_slot), p.columns);
    tcgen05_fence_before();
    __syncthreads();
    tcgen05_fence_after();
    const uint32_t tmem = tmem_slot;
    asm volatile("griddepcontrol.wait;" ::: "memory");
    asm volatile("griddepcontrol.launch_dependents;");

    const int a_bytes = kBM * 2 * BK, b_bytes = p.bn * 2 * BK, stage_bytes = a_bytes + (p.kept ? 0 : b_bytes);
    const uint32_t stages_at = smem_u32(ring) + p.kept;

    if (warp < kEpilogue) {
        // ---- epilogue: the 32 lanes 32 (warp % 4) and up, parts of 64 columns in two tiles of 32.  16 warps are as many as the widest product
        // has such parts; for narrower ones they form groups that take the accumulators in turn.
        const int in_group = kEpilogue / 4 / p.groups, group = warp / 4 / in_group, part = warp / 4 % in_group;
        unsigned char *const buffer = staging + warp * 4096;  // a float32 tile, or two bf16 ones: for the part's two, or for the result and z
        float *const bias = bias_rows + warp * 64;
        const uint32_t lanes = tmem + ((uint32_t)(warp % 4 * 32) << 16);
        const bool tma = MODE != kAny || p.store_tma, partial = MODE == kAny && p.partial;
        const int res_vec = MODE != kAny ? 16 : p.res_vec;
        const CUtensorMap *const tout = tma ? &p.tout : nullptr, *const tpre = tma ? &p.tpre : nullptr;
        unsigned u = 0;          // accumulators of the CTA so far
        int bias_at = -1;        // the column that the bias in shared memory starts at
        const auto stores_done = [&] {  // (with the buffer)
            if (lane == 0) tma_store_wait<0>();
            __syncwarp();
        };
        bool ok = true;
        for (Shares s(p); s.more(p) && ok; s.next(p)) {
            const int row0 = s.m0 + warp % 4 * 32, tiles = row0 < p.M ? (min(p.bn, p.N - s.n0) + 31) / 32 : 0;
            for (int k0 = s.k; k0 < s.end; k0 += p.run, ++u) {
                if (u % p.groups != group) continue;
                const bool first = k0 == s.k, ends = k0 + p.run >= s.end;
                const unsigned a = u & acc_mask;
                bool waited = false;
                for (int h0 = 2 * part; h0 < tiles; h0 += 2 * in_group) {
                    const int c0 = s.n0 + 32 * h0;
                    uint4 res[kPieces32<TOUT>];
                    const auto bring = [&](int col0) {
                        tile_load<TOUT>(res, static_cast<const TOUT *>(p.residual), p.ld_res, res_vec, row0, col0, p.M, p.N, lane);
                    };
                    if (ends && !partial) {  // what does not need the sums
                        if (p.residual) bring(c0);
                        if (bias_at != c0) {
                            bias_at = c0;
#pragma unroll
                            for (int j = 0; j < 64; j += 32)
                                bias[j + lane] = p.bias && c0 + j + lane < p.N ? to_float(static_cast<const TIN *>(p.bias)[c0 + j + lane]) : 0.0f;
                        }
                        stores_done();
                    }
                    if (!waited) {
                        if (!(ok = __all_sync(0xffffffffu, mbar_wait(acc_full + 8 * a, u >> acc_shift & 1, &failed, wait_limit(p, kResults))))) break;
                        tcgen05_fence_after();
                        waited = true;
                    }
#pragma unroll 1
                    for (int odd = 0; odd < 2; ++odd) {
                        const int h = h0 + odd, col0 = c0 + 32 * odd;
                        if (h >= tiles) break;
                        const uint32_t acc = lanes + a * acc_step + 32 * h, sum = lanes + sum_at + 32 * h;
                        uint32_t r[32];
                        float v[32];
                        tmem_load32(r, acc);
                        tmem_wait(r);
#pragma unroll
                        for (int i = 0; i < 32; ++i) v[i] = __uint_as_float(r[i]);
                        const auto add = [&](uint32_t at) {
                            tmem_load32(r, at);
                            tmem_wait(r);
#pragma unroll
                            for (int i = 0; i < 32; ++i) v[i] += __uint_as_float(r[i]);
                        };
                        if (runs && !first) add(sum);
                        if (!ends) {
#pragma unroll
                            for (int i = 0; i < 32; ++i) r[i] = __float_as_uint(v[i]);
                            tmem_store32(sum, r);
                            continue;
                        }
                        if (kParts == 2) add(runs ? sum + p.bn : acc + p.bn);
                        if (partial) {
                            stores_done();
                            row_store<float>(v, buffer, -1, lane);
                            tile_leave<float>(buffer, &p.tout, nullptr, 0, 16, row0, col0, p.M, p.N, s.split, lane);
                            continue;
                        }
#pragma unroll
                        for (int c = 0; c < 8; ++c) {
                            const float4 q = reinterpret_cast<const float4 *>(bias + 32 * odd)[c];
                            const float2 x = __fadd2_rn(make_float2(v[4 * c], v[4 * c + 1]), make_float2(q.x, q.y));
                            const float2 y = __fadd2_rn(make_float2(v[4 * c + 2], v[4 * c + 3]), make_float2(q.z, q.w));
                            v[4 * c] = x.x, v[4 * c + 1] = x.y, v[4 * c + 2] = y.x, v[4 * c + 3] = y.y;
                        }
                        // z leaves from the buffer's second half, or from the whole of it before the result comes
                        if (p.pre) {
                            unsigned char *const tile = buffer + (sizeof(TIN) == 2 && sizeof(TOUT) == 2 ? 2048 : 0);
                            if (odd) stores_done();
                            row_store<TIN>(v, tile, -1, lane);
                            tile_leave<TIN>(tile, tpre, static_cast<TIN *>(p.pre), p.ld_pre, p.pre_vec, row0, col0, p.M, p.N, 0, lane);
                        }
                        if (p.pre ? sizeof(TIN) == 4 || sizeof(TOUT) == 4 : odd && sizeof(TOUT) == 4) stores_done();
                        activate_row<std::is_same<TOUT, bf16>::value>(v, MODE == kAny ? p.act : MODE, buffer, lane);
                        // (a bf16 result without z: both halves leave at once, in rows of 128 bytes, where no other CTA has the
                        // second half's columns)
                        const int half = p.wide ? odd : -1;
                        unsigned char *const tile = buffer + (sizeof(TOUT) == 2 && odd && !p.pre && !p.wide ? 2048 : 0);
                        if (p.residual) {
                            tile_stage<TOUT>(res, res_vec, tile, half, lane);
                            if (!odd && h + 1 < tiles) bring(col0 + 32);
                            row_add<TOUT>(v, tile, half, lane);
                        }
                        row_store<TOUT>(v, tile, half, lane);
                        if (!p.wide) tile_leave<TOUT>(tile, tout, static_cast<TOUT *>(p.out), p.ld_out, p.out_vec, row0, col0, p.M, p.N, 0, lane);
                        else if (odd || h + 1 == tiles) tile_leave<TOUT>(tile, tout, nullptr, 0, 16, row0, c0, p.M, p.N, 0, lane);
                    }
                }
                if (ok && !waited) ok = __all_sync(0xffffffffu, mbar_wait(acc_full + 8 * a, u >> acc_shift & 1, &failed, wait_limit(p, kResults)));
                if (!ok) break;
                tcgen05_fence_before();
                __syncwarp();
                if (lane == 0) mbar_arrive(acc_empty + 8 * a);
            }
        }
        if (lane == 0) tma_store_wait<0>();
        __syncwarp();
    } else if (warp == kEpilogue) {
        // ---- products, by one thread
        if (elect_one()) {
            const uint32_t idesc = mma_idesc(p.bn, p.a_mn, p.b_mn);
            const int a_step = p.a_mn ? 2048 >> 4 : 32 >> 4, b_step = p.b_mn ? 2048 >> 4 : 32 >> 4;  // 16 of K further
            int stage = 0, phase = 0;
            const long long limit = wait_limit(p, kProducts);
            Slots slots;
            unsigned u = 0;  // accumulators filled so far
            bool ok = !p.kept || mbar_wait(kept_full, 0, &failed, limit);
            for (Shares s(p); s.more(p) && ok; s.next(p)) {
                for (int k0 = s.k; k0 < s.end && ok; k0 += p.run, ++u) {
                    const unsigned acc = u & acc_mask;
                    ok = mbar_wait(acc_empty + 8 * acc, (u >> acc_shift & 1) ^ 1, &failed, limit);
                    // (the one accumulator of the small products: the tile before has been taken out)
                    if (ok && kParts == 2 && runs && k0 == s.k) ok = mbar_wait(acc_empty + 8 * ((u + 1) & 1), ((u + 1) >> 1 & 1) ^ 1, &failed, limit);
                    if (!ok) break;
                    tcgen05_fence_after();
                    const uint32_t d = tmem + acc * acc_step, small = runs ? tmem + 3 * p.bn : d + p.bn;
                    const int k1 = min(k0 + p.run, s.end);
                    for (int k = k0; k < k1; ++k) {
                        if constexpr (kPieces == 1) {
                            if (!(ok = mbar_wait(full + 8 * stage, phase, &failed, limit))) break;
                            tcgen05_fence_after();
                            const uint32_t at = stages_at + stage * stage_bytes, b_at = p.kept ? smem_u32(ring) + k * b_bytes : at + a_bytes;
                            const uint64_t a = smem_desc(at, p.a_mn, 128 * BK), b = smem_desc(b_at, p.b_mn, 128 * BK);
#pragma unroll
                            for (int i = 0; i < BK / 16; ++i) mma_bf16(d, a + i * a_step, b + i * b_step, idesc, k > k0 || i > 0);
                            mma_commit(empty + 8 * stage);
                            if (++stage == p.stages) stage = 0, phase ^= 1;
                        } else {
                            const auto arrived = [&](int tile) {
                                const int slot = slots.of(tile);
                                ok = ok && mbar_wait(full + 8 * slot, slots.turn >> slot & 1, &failed, limit);
                                slots.turn ^= 1u << slot;
                            };
                            const auto multiply = [&](uint32_t to, int ta, int tb, bool add) {
                                const uint64_t a = smem_desc(smem_u32(ring) + slots.of(ta) * kSlot, p.a_mn, 128 * BK),
                                               b = smem_desc(smem_u32(ring) + slots.of(tb) * kSlot, p.b_mn, 128 * BK);
#pragma unroll
                                for (int i = 0; i < BK / 16; ++i) mma_bf16(to, a + i * a_step, b + i * b_step, idesc, add || i > 0);
                            };
                            const auto release = [&](int tile) { mma_commit(empty + 8 * slots.of(tile)); };
                            arrived(kA0), arrived(kB0);
                            if (!ok) break;
                            tcgen05_fence_after();
                            multiply(d, kA0, kB0, k > k0);
                            arrived(kB1);
                            if (!ok) break;
                            tcgen05_fence_after();
                            multiply(small, kA0, kB1, k > s.k);
                            arrived(kA1);
                            if (!ok) break;
                            tcgen05_fence_after();
                            multiply(small, kA1, kB0, true), multiply(small, kA1, kB1, true);
                            release(kB1), release(kA1);
                            arrived(kB2);
                            if (!ok) break;
                            tcgen05_fence_after();
                            multiply(small, kA0, kB2, true);
                            release(kA0), release(kB2);
                            arrived(kA2);
                            if (!ok) break;
                            tcgen05_fence_after();
                            multiply(small, kA2, kB0, true);
                            release(kB0), release(kA2);
                            slots.released();
                        }
                    }
                    if (ok) mma_commit(acc_full + 8 * acc);
                }
            }
            // No product may be under way when the CTA gives its memory back.  The epilogue has waited for every one of them, unless
            // some wait ran out, whoever's it was.
            mma_commit(last);
            mbar_drain(last, 0, &failed);
        }
        __syncwarp();
    } else if (warp == kEpilogue + 1) {
        // ---- loads, by one thread
        if (elect_one()) {
            int stage = 0, phase = 0;
            const long long limit = wait_limit(p, kLoads);
            bool ok = true;
            const auto load_b = [&](uint32_t at, int n0, int k, int piece, uint32_t bar) {  // (an operand whose rows run along M or N: 64 of it at a time)
                if (!p.b_mn) tma_load_3d(at, &p.tb, k * BK, n0, piece, bar);
                else
                    for (int i = 0; i < p.bn / 64; ++i) tma_load_3d(at + 128 * BK * i, &p.tb, n0 + 64 * i, k * BK, piece, bar);
            };
            const auto load_a = [&](uint32_t at, int m0, int k, int piece, uint32_t bar) {
                if (!p.a_mn) tma_load_3d(at, &p.ta, k * BK, m0, piece, bar);
                else
                    for (int i = 0; i < kBM / 64; ++i) tma_load_3d(at + 128 * BK * i, &p.ta, m0 + 64 * i, k * BK, piece, bar);
            };
            if (p.kept) {  // (the CTAs' number is a multiple of the tiles along N: a CTA's tiles all have the same columns)
                mbar_expect(kept_full, p.kept);
                for (int k = 0; k < p.kblocks; ++k) load_b(smem_u32(ring) + k * b_bytes, Shares(p).n0, k, 0, kept_full);
            }
            Slots slots;
            for (Shares s(p); s.more(p) && ok; s.next(p)) {
                for (int k = s.k; k < s.end; ++k) {
                    if constexpr (kPieces == 1) {
                        if (!(ok = mbar_wait(empty + 8 * stage, phase ^ 1, &failed, limit))) break;
                        const uint32_t bar = full + 8 * stage, at = stages_at + stage * stage_bytes;
                        mbar_expect(bar, stage_bytes);
                        load_a(at, s.m0, k, 0, bar);
                        if (!p.kept) load_b(at + a_bytes, s.n0, k, 0, bar);
                        if (++stage == p.stages) stage = 0, phase ^= 1;
                    } else {
#pragma unroll
                        for (int tile = 0; tile < 6; ++tile) {
                            const int slot = slots.of(tile), piece = tile == kA0 || tile == kB0 ? 0 : (tile == kA1 || tile == kB1 ? 1 : 2);
                            if (!(ok = ok && mbar_wait(empty + 8 * slot, (slots.turn >> slot & 1) ^ 1, &failed, limit))) break;
                            slots.turn ^= 1u << slot;
                            const bool is_a = tile == kA0 || tile == kA1 || tile == kA2;
                            const uint32_t bar = full + 8 * slot, at = smem_u32(ring) + slot * kSlot;
                            mbar_expect(bar, is_a ? a_bytes : b_bytes);
                            if (is_a) load_a(at, s.m0, k, piece, bar);
                            else load_b(at, s.n0, k, piece, bar);
                        }
                        slots.released();
                        if (!ok) break;
                    }
                }
            }
            // Nor any load: the products have waited for them, unless some wait ran out.  The last one into every stage: the ones
            // before `stage` in this round of the ring, the others in the round before.
            if (p.kept) mbar_drain(kept_full, 0, &failed);
            if (kPieces == 1)
                for (int i = 0; i < p.stages; ++i) mbar_drain(full + 8 * i, i < stage ? phase : phase ^ 1, &failed);
            else
                for (int i = 0; i < kMostStages; ++i) mbar_drain(full + 8 * i, (slots.turn >> i & 1) ^ 1, &failed);
        }
        __syncwarp();
    }
    tcgen05_fence_before();
    __syncthreads();
    if (warp == kEpilogue) {
        tcgen05_fence_after();
        tmem_free(tmem, p.columns);
    }
    if (threadIdx.x == 0 && failed) {
        atomicAdd(&given_up, 1u);
        if (p.error_word) atomicAdd(p.error_word, 1u);
    }
}

// ---- sums that several CTAs shared ----------------------------------------------------------------------------------------

// Column sums of partial sums, `rows` rows of N: 8 columns per block, whose threads have 32 rows of them at a time.
constexpr int kSumColumns = 8;
template <typename T>
struct ColumnSums {
    const float *sums;
    int rows, N;
    T *out;   // NULL: none
};

template <typename T>
__device__ __forceinline__ void column_sums(const ColumnSums<T> &q, int block, float (&part)[8][kSumColumns])
{
    const int warp = threadIdx.x / 32, lane = threadIdx.x % 32, col = block * kSumColumns + lane % 8;
    float v = 0.0f;
    if (col < q.N)
#pragma unroll 20
        for (int r = threadIdx.x / 8; r < q.rows; r += 32) v += q.sums[(long long)r * q.N + col];
    v += __shfl_xor_sync(0xffffffffu, v, 8);
    v += __shfl_xor_sync(0xffffffffu, v, 16);
    if (lane < 8) part[warp][lane] = v;
    __syncthreads();
    if (threadIdx.x < 8 && col < q.N) {
        v = 0.0f;
#pragma unroll
        for (int w = 0; w < 8; ++w) v += part[w][lane];
        q.out[col] = from_float<T>(v);
    }
}

template <typename T>
__global__ void __launch_bounds__(256) column_sum_kernel(const ColumnSums<T> q)
{
    __shared__ float part[8][kSumColumns];
    asm volatile("griddepcontrol.wait;" ::: "memory");
    asm volatile("griddepcontrol.launch_dependents;");
    column_sums(q, blockIdx.x, part);
}

// Adds the shares up in a fixed order and does what the epilogue would have done.  Four columns of a row per thread; with few of
// them (`groups` > 1) as many threads take every so manieth share, and the first of them joins their sums.  The first blocks
// (`sum_blocks`, which take longest) add up column sums.  Bound by latency: 8 to 9 us for nine shares of a 1024 x 256 gradient (9.4 MB).
template <typename TIN, typename TOUT>
__global__ void __launch_bounds__(256) join_kernel(const float *__restrict__ partial, long long ld_partial, int splits, int groups, int M, int N,
                                                   const TIN *__restrict__ bias, const TOUT *residual, long long ld_res, TOUT *out, long long ld_out,
                                                   TIN *pre, long long ld_pre, int act, const ColumnSums<TIN> columns, int sum_blocks)
{
    __shared__ float4 joined[8 * 33];
    asm volatile("griddepcontrol.wait;" ::: "memory");
    asm volatile("griddepcontrol.launch_dependents;");
    const int block = (int)blockIdx.x - sum_blocks, blocks = (int)gridDim.x - sum_blocks;
    if (block < 0) {
        column_sums(columns, blockIdx.x, reinterpret_cast<float (&)[8][kSumColumns]>(joined));
        return;
    }
    const int quads = (int)(ld_partial / 4), width = 256 / groups, group = threadIdx.x / width, t = threadIdx.x % width;
    const long long all = (long long)M * quads, step = (long long)M * ld_partial / 4;
    for (long long i0 = (long long)block * width; i0 < all; i0 += (long long)blocks * width) {
        const long long i = i0 + t, row = i / quads;
        const int col = (int)(i - row * quads) * 4;
        const float4 *src = reinterpret_cast<const float4 *>(partial) + row * (ld_partial / 4) + col / 4;
        float v[4] = {0.0f, 0.0f, 0.0f, 0.0f};
        if (i < all)
#pragma unroll 8
            for (int s = group; s < splits; s += groups) {
                const float4 q = __ldcs(src + s * step);
                v[0] += q.x, v[1] += q.y, v[2] += q.z, v[3] += q.w;
            }
        if (groups > 1) {
            joined[threadIdx.x] = make_float4(v[0], v[1], v[2], v[3]);
            __syncthreads();
            if (group == 0)
                for (int g = 1; g < groups; ++g) {
                    const float4 q = joined[g * width + t];
                    v[0] += q.x, v[1] += q.y, v[2] += q.z, v[3] += q.w;
                }
            __syncthreads();
        }
        if (group || i >= all) continue;
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            if (col + j >= N) break;
            if (bias) v[j] += to_float(bias[col + j]);
            if (pre) pre[row * ld_pre + col + j] = from_float<TIN>(v[j]);
        }
        activate_all<std::is_same<TOUT, bf16>::value, false>(v, act);
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            if (col + j >= N) break;
            if (residual) v[j] += to_float(residual[row * ld_res + col + j]);
            out[row * ld_out + col + j] = from_float<TOUT>(v[j]);
        }
    }
}

// ---- operands laid out for TMA --------------------------------------------------------------------------------------------

__device__ __forceinline__ void split(float2 v, uint32_t (&p)[3])
{
    p[0] = pack(v.x, v.y);
    v = __fadd2_rn(v, make_float2(-low(p[0]), -high(p[0])));
    p[1] = pack(v.x, v.y);
    v = __fadd2_rn(v, make_float2(-low(p[1]), -high(p[1])));
    p[2] = pack(v.x, v.y);
}

// Eight neighbours as bf16 pieces, 16 bytes of each of the operand's matrices (`layer` apart)
__device__ __forceinline__ void store_pieces(const float (&v)[8], bf16 *to, long long layer)
{
    uint32_t p[3][4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        uint32_t q[3];
        split(make_float2(v[2 * i], v[2 * i + 1]), q);
        p[0][i] = q[0], p[1][i] = q[1], p[2][i] = q[2];
    }
#pragma unroll
    for (int j = 0; j < 3; ++j) *reinterpret_cast<uint4 *>(to + j * layer) = make_uint4(p[j][0], p[j][1], p[j][2], p[j][3]);
}

struct LayoutJob {
    const void *from;
    bf16 *to;               // [pieces][rows][ld_to]
    long long ld, ld_to, layer;
    int rows, width;        // width 0: no job
    int vec;                // neighbours that a load may take at once: 8 (all of the row is in such eights), 2 or 1
    unsigned lanes;         // threads of a row: one for eight elements
};

// A thread has eight elements of a row at a time and stores them as whole vectors, with zeros behind the row's end.  (184950 x 82 bf16
// numbers, rows on 4-byte boundaries, and their product with 82 x 128: 34 us; with two elements for a thread 41.)
template <typename T>
__device__ __forceinline__ void lay_out(const LayoutJob &q, unsigned block, unsigned blocks)
{
    constexpr int kP = sizeof(T) == 4 ? 3 : 1;
    // (place in the row and row, a grid's step on: no division for every piece)
    const unsigned start = block * 256 + threadIdx.x, step = blocks * 256;
    unsigned row = start / q.lanes, lane = start - row * q.lanes;
    const unsigned step_rows = step / q.lanes, step_lanes = step - step_rows * q.lanes;
#pragma unroll 4
    for (; row < (unsigned)q.rows; row += step_rows, lane += step_lanes, row += lane >= q.lanes, lane -= lane >= q.lanes ? q.lanes : 0) {
        const T *src = static_cast<const T *>(q.from) + row * q.ld;
        bf16 *dst = q.to + row * q.ld_to;
        src += 8 * lane, dst += 8 * lane;
        if (q.vec == 8) {
            if constexpr (kP == 3) {
                const uint4 a = __ldcs(reinterpret_cast<const uint4 *>(src)), b = __ldcs(reinterpret_cast<const uint4 *>(src) + 1);
                const float v[8] = {__uint_as_float(a.x), __uint_as_float(a.y), __uint_as_float(a.z), __uint_as_float(a.w),
                                    __uint_as_float(b.x), __uint_as_float(b.y), __uint_as_float(b.z), __uint_as_float(b.w)};
                store_pieces(v, dst, q.layer);
            } else {
                *reinterpret_cast<uint4 *>(dst) = __ldcs(reinterpret_cast<const uint4 *>(src));
            }
        } else {
            using W = typename std::conditional<kP == 3, uint2, uint32_t>::type;  // two neighbours
            const int have = q.width - 8 * (int)lane;
            T v[8];
            if (q.vec == 2) {
                W w[4];
#pragma unroll
                for (int i = 0; i < 4; ++i) w[i] = 2 * i < have ? __ldg(reinterpret_cast<const W *>(src) + i) : W{};
                memcpy(v, w, sizeof(v));
            } else {
#pragma unroll
                for (int i = 0; i < 8; ++i) v[i] = i < have ? __ldg(src + i) : from_float<T>(0.0f);
            }
            if constexpr (kP == 3) {
                store_pieces(v, dst, q.layer);
            } else {
                uint4 w;
                memcpy(&w, v, sizeof(w));
                *reinterpret_cast<uint4 *>(dst) = w;
            }
        }
    }
}

// Two jobs, x and the weights: whole blocks of either.  Bound by traffic: 15 us for 40000 x 256 float32 numbers and their pieces (102 MB).
struct LayoutJobs {
    LayoutJob first, second;
    unsigned first_blocks, blocks;  // 0: none

    template <typename T>
    __device__ __forceinline__ void run(unsigned block) const
    {
        if (block < first_blocks) lay_out<T>(first, block, first_blocks);
        else lay_out<T>(second, block - first_blocks, blocks - first_blocks);
    }
};

template <typename T>
__global__ void __launch_bounds__(256) layout_kernel(const __grid_constant__ LayoutJobs jobs)
{
    asm volatile("griddepcontrol.wait;" ::: "memory");
    asm volatile("griddepcontrol.launch_dependents;");
    jobs.run<T>(blockIdx.x);
}

// ---- dz = grad_out act'(z), and its column sums ---------------------------------------------------------------------------

constexpr int kSlopeRows = 8;    // warps of a block: each takes every eighth row of the block's
constexpr int kSlopeBlocks = 3;  // blocks of an SM

// VEC neighbours, aligned as a whole; `once`: nobody else reads them.
template <typename T, int VEC>
struct Loaded {
    using W = typename std::conditional<VEC * sizeof(T) >= 16, uint4,
                                        typename std::conditional<VEC * sizeof(T) == 8, uint2,
                                                                  typename std::conditional<VEC * sizeof(T) == 4, uint32_t, uint16_t>::type>::type>::type;
    W w[VEC * sizeof(T) / sizeof(W)];
};

template <typename T, int VEC>
__device__ __forceinline__ void load(Loaded<T, VEC> &to, const T *from, bool once)
{
    using W = typename Loaded<T, VEC>::W;
    const W *const p = reinterpret_cast<const W *>(from);
#pragma unroll
    for (int i = 0; i < (int)(sizeof(to) / sizeof(W)); ++i) to.w[i] = once ? __ldcs(p + i) : __ldg(p + i);
}

// A lane has VEC neighbouring columns, a warp a stretch of a row, the block `per` rows.  dz, in bf16 numbers or three pieces
// `layer` apart, may be NULL (column sums only), sums too; ACT: there is a z.  Of bf16 operands dz is rounded once, to bf16, also where
// grad_out is float32: half a step for each of its numbers, as large as the roundings of the operands and gradients (which are 2.4e-3 off by
// both, 1.7e-3 by their own alone).  Two pieces of it would double both products and what is written here.  One pass over g and z, bound by traffic (column sums of
// 40000 x 1024 bf16 numbers and the kernel that joins them: 19 us, 4.4 TB/s).  The loads of a batch of rows are under way together, and
// all blocks are on the SMs at once: all gradients of 40000 x 256 -> 1024 with GELU take 106 us so, 112 with two blocks of longer
// batches, 111 by a loop over single rows.
template <typename TG, typename TZ, int VEC, bool ACT>
__global__ void __launch_bounds__(32 * kSlopeRows, kSlopeBlocks) slope_kernel(const TG *__restrict__ g, long long ld_g, const TZ *__restrict__ z, long long ld_z,
                                                                bf16 *__restrict__ dz, long long ld_dz, long long layer, float *__restrict__ sums, int M,
                                                                int N, int per, int act, const __grid_constant__ LayoutJobs jobs)
{
    constexpr bool kFast = std::is_same<TZ, bf16>::value;
    asm volatile("griddepcontrol.wait;" ::: "memory");
    asm volatile("griddepcontrol.launch_dependents;");
    if constexpr (sizeof(TZ) == 4) {
        const unsigned y = blockIdx.y - ((unsigned)M + per - 1) / per;
        if ((int)y >= 0) {
            if (y * gridDim.x + blockIdx.x < jobs.blocks) jobs.run<TZ>(y * gridDim.x + blockIdx.x);
            return;
        }
    }
    const int warp = threadIdx.x / 32, lane = threadIdx.x % 32;
    const int col = (blockIdx.x * 32 + lane) * VEC;
    const long long row1 = min((long long)M, (long long)(blockIdx.y + 1) * per);
    float acc[VEC];
#pragma unroll
    for (int j = 0; j < VEC; ++j) acc[j] = 0.0f;
    // (all loads of a batch of rows ahead of their arithmetic, the last batch's too)
    constexpr int kBatch = VEC == 8 && (sizeof(TZ) == 4 || ACT) ? 2 : 4;
    if (col < N)
        for (long long first = (long long)blockIdx.y * per + warp; first < row1; first += kBatch * kSlopeRows) {
            Loaded<TG, VEC> gq[kBatch];
            Loaded<TZ, VEC> zq[kBatch];
#pragma unroll
            for (int k = 0; k < kBatch; ++k) {
                const long long row = first + k * kSlopeRows;
                if (row >= row1) break;
                load(gq[k], g + row * ld_g + col, dz != nullptr);  // (without dz the products read it too)
                if constexpr (ACT) load(zq[k], z + row * ld_z + col, true);
            }
#pragma unroll
            for (int k = 0; k < kBatch; ++k) {
                const long long row = first + k * kSlopeRows;
                if (row >= row1) break;
                TG gv[VEC];
                TZ zv[VEC] = {};
                memcpy(gv, &gq[k], sizeof(gv));
                if constexpr (ACT) memcpy(zv, &zq[k], sizeof(zv));
                float d[VEC];
                if constexpr (VEC == 1) {
                    d[0] = ACT ? slope_times<kFast>(both(to_float(gv[0])), both(to_float(zv[0])), act).x : to_float(gv[0]);
                    acc[0] += d[0];
                } else {
#pragma unroll
                    for (int j = 0; j < VEC; j += 2) {
                        float2 v = make_float2(to_float(gv[j]), to_float(gv[j + 1]));
                        if constexpr (ACT) v = slope_times<kFast>(v, make_float2(to_float(zv[j]), to_float(zv[j + 1])), act);
                        d[j] = v.x, d[j + 1] = v.y;
                        v = __fadd2_rn(v, make_float2(acc[j], acc[j + 1]));
                        acc[j] = v.x, acc[j + 1] = v.y;
                    }
                }
                if (dz) {
                    bf16 *const to = dz + row * ld_dz + col;
                    if constexpr (VEC == 8 && sizeof(TZ) == 4) {
                        store_pieces(d, to, layer);
                    } else if constexpr (VEC == 8) {
                        *reinterpret_cast<uint4 *>(to) = make_uint4(pack(d[0], d[1]), pack(d[2], d[3]), pack(d[4], d[5]), pack(d[6], d[7]));
                    } else if constexpr (sizeof(TZ) == 4) {
                        uint32_t p[3];
                        split(make_float2(d[0], VEC > 1 ? d[VEC - 1] : 0.0f), p);
#pragma unroll
                        for (int j = 0; j < 3; ++j)
                            if constexpr (VEC == 2) *reinterpret_cast<uint32_t *>(to + j * layer) = p[j];
                            else to[j * layer] = __ushort_as_bfloat16((unsigned short)p[j]);
                    } else if constexpr (VEC == 2) {
                        *reinterpret_cast<uint32_t *>(to) = pack(d[0], d[1]);
                    } else {
                        *to = from_float<bf16>(d[0]);
                    }
                }
            }
        }
    if (!sums) return;
    __shared__ float part[kSlopeRows][32 * VEC + 1];
#pragma unroll
    for (int j = 0; j < VEC; ++j) part[warp][lane * VEC + j] = acc[j];
    __syncthreads();
    for (int c = threadIdx.x; c < 32 * VEC; c += 32 * kSlopeRows) {
        const int at = blockIdx.x * 32 * VEC + c;
        if (at >= N) break;
        float v = 0.0f;
#pragma unroll
        for (int w = 0; w < kSlopeRows; ++w) v += part[w][c];
        sums[(long long)blockIdx.y * N + at] = v;
    }
}

// ---- few rows ---------------------------------------------------------------------------------------------------------------

// Up to R rows of x: bound by reading the weights once, so no tensor cores (their tiles would be empty rows).  A warp forms NC
// neighbouring columns of all rows, its lanes 8 elements of the sum each at a time.  Where that leaves most SMs without a warp, the block's
// eight warps share the sum of the same columns (`shared`).  VEC: bytes that every row's start is a multiple of, 16 or an element.
// Measured: 1 x 1024 -> 4096, bf16: 5 us a call, of which launch and latency are most (the weights' 8 MB take 1.3 us at the card's rate).
template <typename TIN, typename TOUT, int R, int NC, bool VEC>
__global__ void __launch_bounds__(256) rows_kernel(const TIN *__restrict__ x, long long ld_x, const TIN *__restrict__ weight, long long ld_w, int M,
                                                   int N, int K, int shared, const TIN *__restrict__ bias, const TOUT *residual, long long ld_res,
                                                   TOUT *out, long long ld_out, TIN *pre, long long ld_pre, int act)
{
    constexpr int Q = 8 * (int)sizeof(TIN) / 16;
    __shared__ float joined[8][R * NC];
    asm volatile("griddepcontrol.wait;" ::: "memory");
    asm volatile("griddepcontrol.launch_dependents;");
    const int lane = threadIdx.x % 32, warp = threadIdx.x / 32, n0 = (shared ? blockIdx.x : blockIdx.x * 8 + warp) * NC;
    if (n0 >= N) return;  // (all of the block where it shares)
    float acc[R][NC];
#pragma unroll
    for (int r = 0; r < R; ++r)
#pragma unroll
        for (int c = 0; c < NC; ++c) acc[r][c] = 0.0f;
    // VEC: the lane's eight elements are neighbours, else every 32nd of the warp's 256, so that its loads are too
    const auto bring = [&](float (&v)[8], const TIN *row, int k) {
        if constexpr (VEC) {
            uint4 q[Q];
            TIN t[8];
#pragma unroll
            for (int i = 0; i < Q; ++i) q[i] = k + lane * 8 < K ? __ldg(reinterpret_cast<const uint4 *>(row + k + lane * 8) + i) : make_uint4(0, 0, 0, 0);
            memcpy(t, q, sizeof(t));
#pragma unroll
            for (int i = 0; i < 8; ++i) v[i] = to_float(t[i]);
        } else {
#pragma unroll
            for (int i = 0; i < 8; ++i) v[i] = k + lane + 32 * i < K ? to_float(__ldg(row + k + lane + 32 * i)) : 0.0f;
        }
    };
#pragma unroll(R <= 2 ? 4 : 2)
    for (int k = shared ? warp * 256 : 0; k < K; k += shared ? 2048 : 256) {
        float wv[NC][8];
#pragma unroll
        for (int c = 0; c < NC; ++c) bring(wv[c], weight + min(n0 + c, N - 1) * ld_w, k);
#pragma unroll
        for (int r = 0; r < R; ++r) {
            float xv[8];
            bring(xv, x + min(r, M - 1) * ld_x, k);
#pragma unroll
            for (int c = 0; c < NC; ++c)
#pragma unroll
                for (int i = 0; i < 8; ++i) acc[r][c] = fmaf(xv[i], wv[c][i], acc[r][c]);
        }
    }
#pragma unroll
    for (int r = 0; r < R; ++r)
#pragma unroll
        for (int c = 0; c < NC; ++c)
#pragma unroll
            for (int d = 16; d; d /= 2) acc[r][c] += __shfl_xor_sync(0xffffffffu, acc[r][c], d);
    // lane r NC + c has row r's column c
    const int r = lane / NC, n = n0 + lane % NC;
    float z[2] = {0.0f, 0.0f};
#pragma unroll
    for (int i = 0; i < R * NC; ++i)
        if (lane == i) z[0] = acc[i / NC][i % NC];
    if (shared) {
        if (lane < R * NC) joined[warp][lane] = z[0];
        __syncthreads();
        if (warp) return;
        if (lane < R * NC)
            for (int w = 1; w < 8; ++w) z[0] += joined[w][lane];
    }
    if (r >= min(R, M) || n >= N) return;
    if (bias) z[0] += to_float(bias[n]);
    if (pre) pre[r * ld_pre + n] = from_float<TIN>(z[0]);
    activate_all<std::is_same<TOUT, bf16>::value, false>(z, act);
    if (residual) z[0] += to_float(residual[r * ld_res + n]);
    out[r * ld_out + n] = from_float<TOUT>(z[0]);
}

// ---- host -------------------------------------------------------------------------------------------------------------------

constexpr int kMaxFeatures = 1 << 24;
constexpr int kFewRows = 8;

// One of the kernel's operands: rows of contiguous bf16 numbers, ld apart; of pieces three such matrices, `layer` apart.
struct Operand {
    const void *p;
    long long ld;
    bool mn;  // a row per k
    long long layer = 0;
};

// (a tensor map's strides end at 2^40 bytes)
bool tma_ok(const void *p, long long ld) { return (uintptr_t)p % 16 == 0 && ld % 8 == 0 && ld < (1LL << 38); }

size_t round_up(size_t v) { return (v + 255) / 256 * 256; }

// Distance of the rows, and bytes, of an operand that has to be laid out in the scratch
long long laid_out_ld(int width) { return (width + 7LL) / 8 * 8; }
size_t laid_out_bytes(long long rows, int width, bool f32) { return round_up((size_t)rows * laid_out_ld(width) * (f32 ? 6 : 2)); }

using EncodeTiled = CUresult (*)(CUtensorMap *, CUtensorMapDataType, cuuint32_t, void *, const cuuint64_t *, const cuuint64_t *, const cuuint32_t *,
                                 const cuuint32_t *, CUtensorMapInterleave, CUtensorMapSwizzle, CUtensorMapL2promotion, CUtensorMapFloatOOBfill);

EncodeTiled encode_tiled()
{
    static std::atomic<void *> found{nullptr};  // (concurrent callers may both look: same answer)
    void *f = found.load(std::memory_order_acquire);
    if (!f) {
        cudaDriverEntryPointQueryResult how;
        if (cudaGetDriverEntryPointByVersion("cuTensorMapEncodeTiled", &f, 12000, cudaEnableDefault, &how) != cudaSuccess ||
            how != cudaDriverEntryPointSuccess) {
            cudaGetLastError();
            return nullptr;
        }
        found.store(f, std::memory_order_release);
    }
    return reinterpret_cast<EncodeTiled>(f);
}

// `across`: extent along M or N; box: rows of the tile
bool make_map(CUtensorMap &map, const Operand &o, int pieces, int across, int K, int rows)
{
    const EncodeTiled encode = encode_tiled();
    if (!encode) return false;
    constexpr int bk = kBK;
    const cuuint64_t size[3] = {(cuuint64_t)(o.mn ? across : K), (cuuint64_t)(o.mn ? K : across), (cuuint64_t)pieces};
    const cuuint64_t pitch[2] = {(cuuint64_t)o.ld * 2, (cuuint64_t)(pieces == 1 ? o.ld : o.layer) * 2};
    const cuuint32_t box[3] = {(cuuint32_t)(o.mn ? 64 : bk), (cuuint32_t)(o.mn ? bk : rows), 1}, step[3] = {1, 1, 1};
    return encode(&map, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 3, const_cast<void *>(o.p), size, pitch, box, step, CU_TENSOR_MAP_INTERLEAVE_NONE,
                  CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
                  CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

// A TMA store clips a row's end to 16 bytes, not to its last element, and writes zeros behind that: rows that have something else there
// are not for it.
bool whole(int width, bool f32) { return width % (f32 ? 4 : 8) == 0; }

// Results: `layers` matrices of M rows, stored in tiles of 32 x 32 (wide: 64 columns of bf16)
bool make_store_map(CUtensorMap &map, void *p, bool f32, bool wide, int M, int N, long long ld, int layers)
{
    const EncodeTiled encode = encode_tiled();
    if (!encode) return false;
    const int elem = f32 ? 4 : 2;
    const cuuint64_t size[3] = {(cuuint64_t)N, (cuuint64_t)M, (cuuint64_t)layers};
    const cuuint64_t pitch[2] = {(cuuint64_t)ld * elem, (cuuint64_t)ld * elem * (cuuint64_t)(layers > 1 ? M : 1)};
    const cuuint32_t box[3] = {wide ? 64u : 32u, 32, 1}, step[3] = {1, 1, 1};
    return encode(&map, f32 ? CU_TENSOR_MAP_DATA_TYPE_FLOAT32 : CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 3, p, size, pitch, box, step,
                  CU_TENSOR_MAP_INTERLEAVE_NONE, f32 || wide ? CU_TENSOR_MAP_SWIZZLE_128B : CU_TENSOR_MAP_SWIZZLE_64B, CU_TENSOR_MAP_L2_PROMOTION_NONE,
                  CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

// K after which a float32 result's sum is taken out of the tensor cores: 24 instructions that cut it off, 8e-7 of it.
constexpr int kRun = 384;

// ... and a bf16 result's: 2048 instructions.  Of terms of one sign each cuts off 2e-7 of the sum so far (of random signs 3e-8), all of them 2e-4
// of the whole, a tenth of the half step that the result is rounded by, or less.  (Sums of a million terms of one sign lost 6e-3 without.)
constexpr int kLongRun = 32768;

// Sums up to this long wait for the epilogue.
constexpr int kShort = 256;

// Tiles and shares of a product.
struct Plan {
    int ew, bn, stages, grid, kept, tiles_m, tiles_n, kblocks, kshare, splits, run, columns, accs, groups;
    long long ld_partial;
    size_t partial_bytes;  // 0: every tile's sum belongs to one CTA
};

Plan plan_product(bool b_mn, bool f32, bool out_f32, bool heavy, int M, int N, int K, bool may_split)
{
    Plan q = {};
    const int sms = sm_count();
    q.tiles_m = (M + kBM - 1) / kBM;
    constexpr int bk = kBK;
    q.kblocks = (K + bk - 1) / bk;
    const bool runs = out_f32 && K > kRun;
    // Widths: the columns in equal parts, at most 256 (128 where accumulators for pieces or a running sum take tensor memory); and
    // shares of long sums where there are few tiles.  By estimated cycles of the CTA with the most to do: a block of K, a tile's
    // epilogue 12 cycles a column and 800 more, beside the products of the next tile if there is one; partial sums are written and
    // read again by another kernel, which takes 7000 cycles and all CTAs together 2000 bytes a cycle.  With these constants the
    // choices are 2 % slower than the best of nine sets in the mean over 45 sizes of 9 to 184950 rows, 14 % at most; 200 x 256
    // numbers that are sums of 256 take 4.7 us by themselves, 7.7 shared.
    const int widest = f32 || runs ? 128 : 256, grain = b_mn ? 64 : 32;
    double best = 0.0;
    for (int most_bn = widest; q.bn == 0 || most_bn >= 64; most_bn -= grain) {
        const int t = (N + most_bn - 1) / most_bn, bn = ((N + t - 1) / t + grain - 1) / grain * grain;
        if (bn == q.bn) continue;
        const long long tiles = (long long)q.tiles_m * ((N + bn - 1) / bn);
        int parts = may_split && tiles * 2 <= sms ? (int)std::min<long long>(sms / tiles, (long long)q.kblocks * bk / 128) : 1;
        for (parts = std::max(1, parts); parts >= 1; parts /= 2) {
            const int share = (q.kblocks + parts - 1) / parts, splits = (q.kblocks + share - 1) / share;
            const double items = (double)((tiles * splits + sms - 1) / sms), main = share * (f32 ? 10.0 : 2.15) * std::max(kBM + bn, f32 ? 0 : 240);
            const double rest = 12.0 * bn + 800.0, join = splits > 1 ? 7000.0 + splits * 8.0 * M * N / 2000.0 : 0.0;
            const double cost = items * std::max(main, rest) + std::min(main, rest) + join;
            if (q.bn == 0 || cost < best) best = cost, q.bn = bn, q.kshare = share, q.splits = splits;
        }
    }
    q.tiles_n = (N + q.bn - 1) / q.bn;
    // B stays in shared memory where all of K fits beside three stages of A and a CTA has several tiles: its loads are two thirds
    // of a 128 x 256 tile's.
    const long long tiles = (long long)q.tiles_m * q.tiles_n;
    const long long kept = (long long)q.kblocks * q.bn * 2 * bk;
    const int a_bytes = kBM * 2 * bk, spread = sms / q.tiles_n * q.tiles_n;
    q.grid = (int)std::min<long long>(tiles * q.splits, sms);
    if (!f32 && !heavy && q.splits == 1 && kept + 3 * a_bytes <= ring_bytes(8) && tiles > spread && spread > 0 && spread * 20 >= sms * 19)
        q.kept = (int)kept, q.grid = spread;
    q.ew = f32 || q.kept || q.kshare * bk > kShort ? 8 : 16;
    q.stages = std::min(8, (ring_bytes(q.ew) - q.kept) / (a_bytes + (q.kept ? 0 : q.bn * 2 * bk)));  // (of bf16 operands)
    q.run = std::min(q.kshare, (out_f32 ? kRun : kLongRun) / bk);
    // Accumulators: with runs two (one beside the running sum of more than 128 columns: its runs are long ones, and taking a sum out every 260000
    // cycles takes a few thousand), the running sum and, of float32 operands, that of the small products; else four where they fit
    // (float32 operands: pairs).  Groups of epilogue warps: as many 64-column parts as the tile has in each, and no more of them than accumulators.
    const int parts = f32 ? 2 : 1, warps = q.ew / 4, wide = (q.bn + 63) / 64;
    const bool in_runs = q.run < q.kshare;
    q.accs = in_runs ? (q.bn > 128 ? 1 : 2) : (4 * parts * q.bn <= 512 ? 4 : 2);
    const int used = in_runs ? (q.accs + parts) * q.bn : q.accs * parts * q.bn;
    for (q.columns = 32; q.columns < used;) q.columns *= 2;
    q.groups = 1;
    while (!in_runs && q.groups < q.accs && q.groups * 2 * wide <= warps) q.groups *= 2;
    if (q.splits > 1) {
        q.ld_partial = (N + 3) / 4 * 4;
        q.partial_bytes = (size_t)q.splits * M * q.ld_partial * sizeof(float);
    }
    return q;
}

// What the epilogue does.
struct Epilogue {
    const void *bias = nullptr, *residual = nullptr;
    void *out = nullptr, *pre = nullptr;
    long long ld_res = 0, ld_out = 0, ld_pre = 0;
    int act = FLASHBEV_ACT_NONE;
    bool out_f32 = false;
    // column sums that a kernel which joins shares adds up beside them
    const float *sums = nullptr;
    int sum_rows = 0, sum_columns = 0;
    void *sum_out = nullptr;
};

bool vec_ok(const void *p, long long ld, bool f32)
{
    return ((uintptr_t)p | (uintptr_t)(ld * (f32 ? 4 : 2))) % 16 == 0 && ld < (1LL << 37);
}

int row_bytes(const void *p, long long ld, bool f32)
{
    if (vec_ok(p, ld, f32)) return 16;
    return ((uintptr_t)p | (uintptr_t)(ld * (f32 ? 4 : 2))) % 4 == 0 ? 4 : 2;
}

template <int PIECES, typename TOUT, int EW, int MODE>
cudaError_t launch_gemm(const GemmParams &g, int grid, cudaStream_t stream)
{
    const auto kernel = gemm_kernel<PIECES, TOUT, EW, MODE>;
    constexpr int smem = ring_bytes(EW) + epilogue_bytes(EW) + kControlBytes;
    static_assert(smem <= kSmemLimit && ring_bytes(8) >= kMostStages * kSlot && ring_bytes(16) >= 3 * 48 * 1024, "");
    const cudaError_t e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, smem);
    if (e != cudaSuccess) return e;
    return launch_dependent(kernel, dim3((unsigned)grid), dim3((unsigned)gemm_threads(EW)), smem, stream, g);
}

template <int PIECES, typename TOUT, int EW>
cudaError_t launch_mode(const GemmParams &g, int grid, cudaStream_t stream)
{
    if (g.partial || g.run < g.kshare || !g.store_tma || (g.residual && g.res_vec != 16)) return launch_gemm<PIECES, TOUT, EW, kAny>(g, grid, stream);
    switch (g.act) {
    case FLASHBEV_ACT_RELU: return launch_gemm<PIECES, TOUT, EW, FLASHBEV_ACT_RELU>(g, grid, stream);
    case FLASHBEV_ACT_GELU: return launch_gemm<PIECES, TOUT, EW, FLASHBEV_ACT_GELU>(g, grid, stream);
    case FLASHBEV_ACT_SILU: return launch_gemm<PIECES, TOUT, EW, FLASHBEV_ACT_SILU>(g, grid, stream);
    default: return launch_gemm<PIECES, TOUT, EW, FLASHBEV_ACT_NONE>(g, grid, stream);
    }
}

// Operands to be laid out in the scratch
struct Layouts {
    LayoutJobs jobs = {};
    int count = 0;

    // `o` becomes the operand's place in the scratch
    void add(Operand &o, char *to, int rows, int width, bool f32)
    {
        LayoutJob &q = count++ ? jobs.second : jobs.first;
        q.from = o.p, q.to = reinterpret_cast<bf16 *>(to), q.ld = o.ld, q.rows = rows, q.width = width;
        q.ld_to = laid_out_ld(width), q.layer = rows * q.ld_to;
        const uintptr_t starts = (uintptr_t)q.from | (uintptr_t)(q.ld * (f32 ? 4 : 2));
        q.vec = width % 8 == 0 && starts % 16 == 0 ? 8 : (width % 2 == 0 && starts % (f32 ? 8 : 4) == 0 ? 2 : 1);
        q.lanes = (unsigned)(width + 7) / 8;
        jobs.blocks += (unsigned)std::min<long long>(((long long)rows * q.lanes + 255) / 256, 8LL * sm_count());
        if (count == 1) jobs.first_blocks = jobs.blocks;
        o = {q.to, q.ld_to, o.mn, q.layer};
    }
    cudaError_t launch(bool f32, cudaStream_t stream) const
    {
        return launch_dependent(f32 ? layout_kernel<float> : layout_kernel<bf16>, dim3(jobs.blocks), dim3(256), 0, stream, jobs);
    }
};

template <typename TIN, typename TOUT>
cudaError_t launch_join(const Plan &q, const float *partial, int M, int N, const Epilogue &e, cudaStream_t stream)
{
    const long long quads = (long long)M * (q.ld_partial / 4);
    int groups = 1;
    while (groups < 16 && groups * 2 <= q.splits && quads * groups < 1024LL * sm_count()) groups *= 2;
    const unsigned blocks = (unsigned)std::min<long long>((quads * groups + 255) / 256, 8LL * sm_count());
    const ColumnSums<TIN> columns = {e.sums, e.sum_rows, e.sum_columns, static_cast<TIN *>(e.sum_out)};
    const unsigned sum_blocks = e.sum_out ? (unsigned)(e.sum_columns + kSumColumns - 1) / kSumColumns : 0;
    return launch_dependent(join_kernel<TIN, TOUT>, dim3(sum_blocks + blocks), dim3(256), 0, stream, partial, q.ld_partial, q.splits, groups, M, N,
                            static_cast<const TIN *>(e.bias), static_cast<const TOUT *>(e.residual), e.ld_res, static_cast<TOUT *>(e.out), e.ld_out,
                            static_cast<TIN *>(e.pre), e.ld_pre, e.act, columns, (int)sum_blocks);
}

// Enqueues one product; adds the kernels to `launches`.
flashbev_status run_product(const Plan &q, const Operand &a, const Operand &b, bool f32, int M, int N, int K, const Epilogue &e, float *partial,
                            uint32_t *error_word, cudaStream_t stream, int &launches)
{
    GemmParams g = {};
    const int pieces = f32 ? 3 : 1;
    if (!make_map(g.ta, a, pieces, M, K, kBM) || !make_map(g.tb, b, pieces, N, K, q.bn)) return FLASHBEV_CUDA_ERROR;
    g.a_mn = a.mn, g.b_mn = b.mn;
    g.M = M, g.N = N, g.bn = q.bn, g.stages = q.stages;
    g.run = q.run, g.columns = q.columns, g.accs = q.accs, g.groups = q.groups, g.kept = q.kept;
    g.tiles_n = q.tiles_n, g.tiles = q.tiles_m * q.tiles_n, g.kblocks = q.kblocks, g.kshare = q.kshare, g.splits = q.splits;
    g.out = e.out, g.pre = e.pre, g.residual = e.residual, g.bias = e.bias, g.act = e.act;
    g.ld_out = e.ld_out, g.ld_pre = e.ld_pre, g.ld_res = e.ld_res;
    g.out_vec = row_bytes(e.out, e.ld_out, e.out_f32), g.pre_vec = row_bytes(e.pre, e.ld_pre, f32), g.res_vec = row_bytes(e.residual, e.ld_res, e.out_f32);
    g.error_word = error_word;
#ifdef FLASHBEV_DEBUG_BOUNDS
    {
        long long *const t = g.limits;
        t[0] = t[1] = t[2] = kWaitCycles;
        if (const char *given = getenv("FLASHBEV_WAIT_CYCLES")) sscanf(given, "%lld,%lld,%lld", t, t + 1, t + 2);
    }
#endif
    if (q.splits > 1) {
        g.partial = partial, g.ld_partial = q.ld_partial;
        // (partial sums have no other results; what lies behind their rows' ends is nobody's)
        if (!make_store_map(g.tout, partial, true, false, M, N, q.ld_partial, q.splits)) return FLASHBEV_CUDA_ERROR;
    } else if (g.out_vec == 16 && whole(N, e.out_f32) && (!e.pre || (g.pre_vec == 16 && whole(N, f32)))) {
        g.store_tma = 1;
        g.wide = !e.out_f32 && !e.pre && (q.bn % 64 == 0 || q.tiles_n == 1);
        if (!make_store_map(g.tout, e.out, e.out_f32, g.wide, M, N, e.ld_out, 1)) return FLASHBEV_CUDA_ERROR;
        if (e.pre && !make_store_map(g.tpre, e.pre, f32, false, M, N, e.ld_pre, 1)) return FLASHBEV_CUDA_ERROR;
    }
    cudaError_t err;
    // (partial sums are float32)
    const bool out_f32 = e.out_f32 || g.partial;
    if (f32) err = out_f32 ? launch_mode<3, float, 8>(g, q.grid, stream) : launch_mode<3, bf16, 8>(g, q.grid, stream);
    else if (out_f32) err = q.ew == 8 ? launch_mode<1, float, 8>(g, q.grid, stream) : launch_mode<1, float, 16>(g, q.grid, stream);
    else err = q.ew == 8 ? launch_mode<1, bf16, 8>(g, q.grid, stream) : launch_mode<1, bf16, 16>(g, q.grid, stream);
    ++launches;
    if (err == cudaSuccess && q.splits > 1) {
        if (f32) err = e.out_f32 ? launch_join<float, float>(q, partial, M, N, e, stream) : launch_join<float, bf16>(q, partial, M, N, e, stream);
        else err = e.out_f32 ? launch_join<bf16, float>(q, partial, M, N, e, stream) : launch_join<bf16, bf16>(q, partial, M, N, e, stream);
        ++launches;
    }
    if (err != cudaSuccess || cudaGetLastError() != cudaSuccess) {
        cudaGetLastError();
        return FLASHBEV_CUDA_ERROR;
    }
    return FLASHBEV_OK;
}

template <typename TIN, typename TOUT>
cudaError_t launch_rows(const void *x, long long ld_x, const void *weight, long long ld_w, int M, int N, int K, const Epilogue &e, cudaStream_t stream)
{
    const bool vec = K % 8 == 0 && (((uintptr_t)x | (uintptr_t)weight) | (uintptr_t)((ld_x | ld_w) * (long long)sizeof(TIN))) % 16 == 0;
    const auto go = [&](auto kernel, int nc) {
        const int warps = (N + nc - 1) / nc, shared = K > 512 && warps < 4 * sm_count();
        return launch_dependent(kernel, dim3((unsigned)(shared ? warps : (warps + 7) / 8)), dim3(256), 0, stream, static_cast<const TIN *>(x), ld_x,
                                static_cast<const TIN *>(weight), ld_w, M, N, K, shared, static_cast<const TIN *>(e.bias), static_cast<const TOUT *>(e.residual),
                                e.ld_res, static_cast<TOUT *>(e.out), e.ld_out, static_cast<TIN *>(e.pre), e.ld_pre, e.act);
    };
    if (M == 1) return vec ? go(rows_kernel<TIN, TOUT, 1, 2, true>, 2) : go(rows_kernel<TIN, TOUT, 1, 2, false>, 2);
    if (M == 2) return vec ? go(rows_kernel<TIN, TOUT, 2, 2, true>, 2) : go(rows_kernel<TIN, TOUT, 2, 2, false>, 2);
    if (M <= 4) return vec ? go(rows_kernel<TIN, TOUT, 4, 2, true>, 2) : go(rows_kernel<TIN, TOUT, 4, 2, false>, 2);
    return vec ? go(rows_kernel<TIN, TOUT, 8, 2, true>, 2) : go(rows_kernel<TIN, TOUT, 8, 2, false>, 2);
}

bool dtype_ok(int d) { return d == FLASHBEV_F32 || d == FLASHBEV_BF16; }
size_t elem_size(int d) { return d == FLASHBEV_F32 ? 4 : 2; }
bool aligned(const void *p, int dtype) { return (uintptr_t)p % elem_size(dtype) == 0; }
bool stride_ok(long long ld, int width) { return ld == 0 || ld >= width; }
long long dense(long long ld, int width) { return ld ? ld : width; }

// rows x ld has to stay within what 64-bit byte offsets hold with room to spare
bool extent_ok(long long rows, long long ld) { return (double)rows * (double)ld < 2305843009213693952.0; }

flashbev_status check_linear(const flashbev_linear_params *p)
{
    if (!p || p->struct_size < sizeof(flashbev_linear_params)) return FLASHBEV_INVALID_ARG;
    if (p->rows < 0 || p->in_features <= 0 || p->out_features <= 0) return FLASHBEV_INVALID_ARG;
    if (!dtype_ok(p->dtype) || !dtype_ok(p->out_dtype) || p->act < 0 || p->act > FLASHBEV_ACT_SILU || p->reserved) return FLASHBEV_INVALID_ARG;
    if (!stride_ok(p->ld_x, p->in_features) || !stride_ok(p->ld_weight, p->in_features) || !stride_ok(p->ld_residual, p->out_features) ||
        !stride_ok(p->ld_out, p->out_features) || !stride_ok(p->ld_preact, p->out_features))
        return FLASHBEV_INVALID_ARG;
    if (!p->weight || (p->rows && (!p->x || !p->out))) return FLASHBEV_INVALID_ARG;
    if (p->rows > 2147483647LL - kBM || p->in_features > kMaxFeatures || p->out_features > kMaxFeatures) return FLASHBEV_UNSUPPORTED;
    for (long long ld : {p->ld_x, p->ld_weight, p->ld_residual, p->ld_out, p->ld_preact})
        if (!extent_ok(std::max<long long>(p->rows, p->out_features), dense(ld, std::max(p->in_features, p->out_features)))) return FLASHBEV_UNSUPPORTED;
    if (((double)p->rows / kBM + 1.0) * (p->out_features / 64.0 + 1.0) > 2.0e9) return FLASHBEV_UNSUPPORTED;
    if (!aligned(p->x, p->dtype) || !aligned(p->weight, p->dtype) || !aligned(p->bias, p->dtype) || !aligned(p->preact_out, p->dtype) ||
        !aligned(p->out, p->out_dtype) || !aligned(p->residual, p->out_dtype) || (uintptr_t)p->workspace % 16 || (uintptr_t)p->error_word % 4)
        return FLASHBEV_MISALIGNED;
    return FLASHBEV_OK;
}

// Scratch of a forward call: operands that have to be laid out, then partial sums.
struct ForwardPlan {
    Plan product;
    bool lay_x, lay_w;
    size_t x_at, w_at, partial_at, needed, total;  // needed: without partial sums
};

// An epilogue that 16 warps are worth more for than weights that stay in shared memory: special functions, a residual to wait for
// (184950 x 256 x 256, GELU 52 us with eight, 40 with 16; with a residual 59 and 49)
bool heavy_epilogue(const flashbev_linear_params *p)
{
    const bool out_f32 = p->out_dtype == FLASHBEV_F32;
    return p->act >= FLASHBEV_ACT_GELU || (p->residual && vec_ok(p->residual, dense(p->ld_residual, p->out_features), out_f32) &&
                                           vec_ok(p->out, dense(p->ld_out, p->out_features), out_f32));
}

ForwardPlan plan_forward(const flashbev_linear_params *p)
{
    ForwardPlan q = {};
    const bool f32 = p->dtype == FLASHBEV_F32;
    const int M = (int)p->rows, N = p->out_features, K = p->in_features;
    q.lay_x = f32 || !tma_ok(p->x, dense(p->ld_x, K)), q.lay_w = f32 || !tma_ok(p->weight, dense(p->ld_weight, K));
    size_t at = 0;
    if (q.lay_x) q.x_at = at, at += laid_out_bytes(M, K, f32);
    if (q.lay_w) q.w_at = at, at += laid_out_bytes(N, K, f32);
    q.needed = q.partial_at = at;
    q.product = plan_product(false, f32, p->out_dtype == FLASHBEV_F32, heavy_epilogue(p), M, N, K, true);
    q.total = at + round_up(q.product.partial_bytes);
    return q;
}

// ---- backward

struct BackwardPlan {
    bool need_dz, need_x, need_w, need_b, lay_x, lay_w;
    Plan gx, gw;
    int per, chunks;                                // rows of a block of slope_kernel; blocks along the rows
    size_t dz_at, x_at, w_at, sums_at, partial_at, total;
};

flashbev_status check_backward(const flashbev_linear_backward_params *p)
{
    if (!p || p->struct_size < sizeof(flashbev_linear_backward_params)) return FLASHBEV_INVALID_ARG;
    if (p->rows < 0 || p->in_features <= 0 || p->out_features <= 0) return FLASHBEV_INVALID_ARG;
    if (!dtype_ok(p->dtype) || !dtype_ok(p->grad_dtype) || p->act < 0 || p->act > FLASHBEV_ACT_SILU || p->reserved) return FLASHBEV_INVALID_ARG;
    if (!stride_ok(p->ld_grad_out, p->out_features) || !stride_ok(p->ld_x, p->in_features) || !stride_ok(p->ld_weight, p->in_features) ||
        !stride_ok(p->ld_preact, p->out_features) || !stride_ok(p->ld_grad_x, p->in_features) || !stride_ok(p->ld_grad_weight, p->in_features))
        return FLASHBEV_INVALID_ARG;
    if (p->rows && (!p->grad_out || (p->act != FLASHBEV_ACT_NONE && !p->preact) || (p->grad_x && !p->weight) || (p->grad_weight && !p->x)))
        return FLASHBEV_INVALID_ARG;
    if (p->dtype == FLASHBEV_F32 && p->grad_dtype != FLASHBEV_F32) return FLASHBEV_UNSUPPORTED;
    if (p->rows > 2147483647LL - kBM || p->in_features > kMaxFeatures || p->out_features > kMaxFeatures) return FLASHBEV_UNSUPPORTED;
    for (long long ld : {p->ld_grad_out, p->ld_x, p->ld_weight, p->ld_preact, p->ld_grad_x, p->ld_grad_weight})
        if (!extent_ok(std::max<long long>(p->rows, p->out_features), dense(ld, std::max(p->in_features, p->out_features)))) return FLASHBEV_UNSUPPORTED;
    if (((double)std::max<long long>(p->rows, p->out_features) / kBM + 1.0) * (p->in_features / 64.0 + 1.0) > 2.0e9) return FLASHBEV_UNSUPPORTED;
    if (!aligned(p->grad_out, p->grad_dtype) || !aligned(p->x, p->dtype) || !aligned(p->weight, p->dtype) || !aligned(p->preact, p->dtype) ||
        !aligned(p->grad_x, p->dtype) || !aligned(p->grad_weight, p->dtype) || !aligned(p->grad_bias, p->dtype) || (uintptr_t)p->workspace % 16 ||
        (uintptr_t)p->error_word % 4)
        return FLASHBEV_MISALIGNED;
    return FLASHBEV_OK;
}

BackwardPlan plan_backward(const flashbev_linear_backward_params *p)
{
    BackwardPlan q = {};
    const bool f32 = p->dtype == FLASHBEV_F32;
    const int M = (int)p->rows, N = p->out_features, K = p->in_features;
    q.need_x = p->grad_x, q.need_w = p->grad_weight, q.need_b = p->grad_bias;
    if (!M) return q;
    q.need_dz = (q.need_x || q.need_w) && (f32 || p->act != FLASHBEV_ACT_NONE || p->dtype != p->grad_dtype ||
                                           !tma_ok(p->grad_out, dense(p->ld_grad_out, N)));
    q.lay_x = q.need_w && (f32 || !tma_ok(p->x, dense(p->ld_x, K)));
    q.lay_w = q.need_x && (f32 || !tma_ok(p->weight, dense(p->ld_weight, K)));
    size_t at = 0;
    if (q.need_dz) q.dz_at = at, at += laid_out_bytes(M, N, f32);
    if (q.lay_x) q.x_at = at, at += laid_out_bytes(M, K, f32);
    if (q.lay_w) q.w_at = at, at += laid_out_bytes(N, K, f32);
    if (q.need_dz || q.need_b) {
        // as many blocks as the SMs hold, but no fewer than 32 rows for each
        const int across = std::max(1, (N + 255) / 256);
        const long long blocks = std::max(1, kSlopeBlocks * sm_count() / across);
        q.per = (int)std::max<long long>(32, (M + blocks - 1) / blocks);
        q.chunks = (int)(((long long)M + q.per - 1) / q.per);
        if (q.need_b) q.sums_at = at, at += round_up((size_t)q.chunks * N * sizeof(float));
    }
    if (q.need_x) q.gx = plan_product(true, f32, f32, false, M, K, N, true);
    if (q.need_w) q.gw = plan_product(true, f32, f32, false, N, K, M, true);
    q.partial_at = at;  // (the products run one after the other)
    q.total = at + round_up(std::max(q.gx.partial_bytes, q.gw.partial_bytes));
    return q;
}

template <typename TG, typename TZ>
cudaError_t launch_slope(const flashbev_linear_backward_params *p, const BackwardPlan &q, const LayoutJobs &jobs, cudaStream_t stream)
{
    const int M = (int)p->rows, N = p->out_features;
    char *const ws = static_cast<char *>(p->workspace);
    bf16 *const dz = q.need_dz ? reinterpret_cast<bf16 *>(ws + q.dz_at) : nullptr;
    const long long ld_dz = laid_out_ld(N);
    float *const sums = q.need_b ? reinterpret_cast<float *>(ws + q.sums_at) : nullptr;
    const TZ *const z = p->act == FLASHBEV_ACT_NONE ? nullptr : static_cast<const TZ *>(p->preact);
    const long long ld_g = dense(p->ld_grad_out, N), ld_z = dense(p->ld_preact, N);
    // (dz's rows start on 16-byte boundaries)
    const auto starts_on = [&](int numbers) {
        return N % numbers == 0 && ((uintptr_t)p->grad_out | (uintptr_t)(ld_g * (long long)sizeof(TG))) % (numbers == 8 ? 16 : numbers * sizeof(TG)) == 0 &&
               (!z || ((uintptr_t)z | (uintptr_t)(ld_z * (long long)sizeof(TZ))) % (numbers == 8 ? 16 : numbers * sizeof(TZ)) == 0);
    };
    const int vec = starts_on(8) ? 8 : (starts_on(2) ? 2 : 1), width = 32 * vec;
    const auto pick = [&](auto eight, auto two, auto one) { return vec == 8 ? eight : (vec == 2 ? two : one); };
    const auto kernel = z ? pick(slope_kernel<TG, TZ, 8, true>, slope_kernel<TG, TZ, 2, true>, slope_kernel<TG, TZ, 1, true>)
                          : pick(slope_kernel<TG, TZ, 8, false>, slope_kernel<TG, TZ, 2, false>, slope_kernel<TG, TZ, 1, false>);
    const unsigned across = (unsigned)((N + width - 1) / width);
    const dim3 grid(across, (unsigned)q.chunks + (jobs.blocks + across - 1) / across);
    return launch_dependent(kernel, grid, dim3(32 * kSlopeRows), 0, stream,
                            static_cast<const TG *>(p->grad_out), ld_g, z, ld_z, dz, ld_dz, M * ld_dz, sums, M, N, q.per, p->act, jobs);
}

}  // namespace

extern "C" {

flashbev_status flashbev_linear(const flashbev_linear_params *p, void *stream_)
{
    const flashbev_status st = check_linear(p);
    if (st != FLASHBEV_OK) return st;
    cudaStream_t stream = static_cast<cudaStream_t>(stream_);
    int launches = 0;
    if (p->rows) {
        const bool f32 = p->dtype == FLASHBEV_F32;
        const int M = (int)p->rows, N = p->out_features, K = p->in_features;
        const long long ld_x = dense(p->ld_x, K), ld_w = dense(p->ld_weight, K);
        Epilogue e;
        e.bias = p->bias, e.residual = p->residual, e.out = p->out, e.pre = p->preact_out, e.act = p->act;
        e.ld_res = dense(p->ld_residual, N), e.ld_out = dense(p->ld_out, N), e.ld_pre = dense(p->ld_preact, N);
        e.out_f32 = p->out_dtype == FLASHBEV_F32;
        if (M <= kFewRows) {
            cudaError_t err;
            const auto go = [&](auto run) { return run(p->x, ld_x, p->weight, ld_w, M, N, K, e, stream); };
            if (f32) err = e.out_f32 ? go(launch_rows<float, float>) : go(launch_rows<float, bf16>);
            else err = e.out_f32 ? go(launch_rows<bf16, float>) : go(launch_rows<bf16, bf16>);
            if (err != cudaSuccess || cudaGetLastError() != cudaSuccess) {
                cudaGetLastError();
                return FLASHBEV_CUDA_ERROR;
            }
            launches = 1;
            t_last_kernel = "linear_rows";
        } else {
            ForwardPlan q = plan_forward(p);
            const size_t have = p->workspace ? p->workspace_bytes : 0;
            if (have < q.needed) return FLASHBEV_TOO_SMALL;
            if (have < q.total) q.product = plan_product(false, f32, e.out_f32, heavy_epilogue(p), M, N, K, false);
            char *const ws = static_cast<char *>(p->workspace);
            Operand x = {p->x, ld_x, false}, w = {p->weight, ld_w, false};
            Layouts layouts;
            if (q.lay_x) layouts.add(x, ws + q.x_at, M, K, f32);
            if (q.lay_w) layouts.add(w, ws + q.w_at, N, K, f32);
            if (layouts.count) {
                if (layouts.launch(f32, stream) != cudaSuccess) {
                    cudaGetLastError();
                    return FLASHBEV_CUDA_ERROR;
                }
                ++launches;
            }
            const flashbev_status run =
                run_product(q.product, x, w, f32, M, N, K, e, reinterpret_cast<float *>(ws + q.partial_at), p->error_word, stream, launches);
            if (run != FLASHBEV_OK) return run;
            t_last_kernel = f32 ? "linear_f32" : (layouts.count ? "linear_bf16_laid_out" : "linear_bf16");
        }
    }
    t_last_launches = launches;
    return FLASHBEV_OK;
}

size_t flashbev_linear_workspace_bytes(const flashbev_linear_params *p)
{
    if (check_linear(p) != FLASHBEV_OK || p->rows <= kFewRows) return 0;
    return plan_forward(p).total;
}

flashbev_status flashbev_linear_backward(const flashbev_linear_backward_params *p, void *stream_)
{
    const flashbev_status st = check_backward(p);
    if (st != FLASHBEV_OK) return st;
    cudaStream_t stream = static_cast<cudaStream_t>(stream_);
    const bool f32 = p->dtype == FLASHBEV_F32;
    const int M = (int)p->rows, N = p->out_features, K = p->in_features;
    const BackwardPlan q = plan_backward(p);
    if (q.total && (!p->workspace || p->workspace_bytes < q.total)) return FLASHBEV_TOO_SMALL;
    int launches = 0;
    if (!M) {
        const size_t e = elem_size(p->dtype), ld = (size_t)dense(p->ld_grad_weight, K) * e;
        if ((p->grad_weight && cudaMemset2DAsync(p->grad_weight, ld, 0, K * e, N, stream) != cudaSuccess) ||
            (p->grad_bias && cudaMemsetAsync(p->grad_bias, 0, N * e, stream) != cudaSuccess)) {
            cudaGetLastError();
            return FLASHBEV_CUDA_ERROR;
        }
        t_last_launches = 0;
        return FLASHBEV_OK;
    }
    char *const ws = static_cast<char *>(p->workspace);
    cudaError_t err = cudaSuccess;
    Operand dz = {p->grad_out, dense(p->ld_grad_out, N), false};
    if (q.need_dz) dz = {ws + q.dz_at, laid_out_ld(N), false, M * laid_out_ld(N)};
    Operand x = {p->x, dense(p->ld_x, K), true}, w = {p->weight, dense(p->ld_weight, K), true};
    Layouts layouts;
    if (q.lay_x) layouts.add(x, ws + q.x_at, M, K, f32);
    if (q.lay_w) layouts.add(w, ws + q.w_at, N, K, f32);
    if (q.need_dz || q.need_b) {
        if (f32) err = launch_slope<float, float>(p, q, layouts.jobs, stream);
        else err = p->grad_dtype == FLASHBEV_F32 ? launch_slope<float, bf16>(p, q, {}, stream) : launch_slope<bf16, bf16>(p, q, {}, stream);
        ++launches;
    }
    if (err == cudaSuccess && layouts.count && !(f32 && launches)) {
        err = layouts.launch(f32, stream);
        ++launches;
    }
    if (err != cudaSuccess) {
        cudaGetLastError();
        return FLASHBEV_CUDA_ERROR;
    }
    float *const partial = reinterpret_cast<float *>(ws + q.partial_at);
    Epilogue e;
    e.out_f32 = f32;
    const float *const sums = reinterpret_cast<const float *>(ws + q.sums_at);
    const bool joins = q.need_w && q.gw.splits > 1;  // the bias' gradient from the kernel that joins the weights'
    if (q.need_b && !joins) {
        const dim3 grid((unsigned)((N + kSumColumns - 1) / kSumColumns));
        if (f32) err = launch_dependent(column_sum_kernel<float>, grid, dim3(256), 0, stream, ColumnSums<float>{sums, q.chunks, N, static_cast<float *>(p->grad_bias)});
        else err = launch_dependent(column_sum_kernel<bf16>, grid, dim3(256), 0, stream, ColumnSums<bf16>{sums, q.chunks, N, static_cast<bf16 *>(p->grad_bias)});
        ++launches;
        if (err != cudaSuccess) {
            cudaGetLastError();
            return FLASHBEV_CUDA_ERROR;
        }
    }
    if (q.need_x) {
        e.out = p->grad_x, e.ld_out = dense(p->ld_grad_x, K);
        const flashbev_status run = run_product(q.gx, dz, w, f32, M, K, N, e, partial, p->error_word, stream, launches);
        if (run != FLASHBEV_OK) return run;
    }
    if (q.need_w) {
        Operand dzt = dz;
        dzt.mn = true;
        e.out = p->grad_weight, e.ld_out = dense(p->ld_grad_weight, K);
        if (q.need_b && joins) e.sums = sums, e.sum_rows = q.chunks, e.sum_columns = N, e.sum_out = p->grad_bias;
        const flashbev_status run = run_product(q.gw, dzt, x, f32, N, K, M, e, partial, p->error_word, stream, launches);
        if (run != FLASHBEV_OK) return run;
    }
    t_last_launches = launches;
    t_last_kernel = f32 ? "linear_backward_f32" : "linear_backward_bf16";
    return FLASHBEV_OK;
}

flashbev_status flashbev_linear_given_up(uint32_t *blocks)
{
    if (!blocks) return FLASHBEV_INVALID_ARG;
    if (cudaDeviceSynchronize() != cudaSuccess || cudaMemcpyFromSymbol(blocks, given_up, sizeof(*blocks)) != cudaSuccess) {
        cudaGetLastError();
        return FLASHBEV_CUDA_ERROR;
    }
    return FLASHBEV_OK;
}

size_t flashbev_linear_backward_workspace_bytes(const flashbev_linear_backward_params *p)
{
    // (the scratch's own address and size do not matter here)
    return check_backward(p) == FLASHBEV_OK ? plan_backward(p).total : 0;
}

}  // extern "C"
