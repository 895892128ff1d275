// Matrix products with bias, activation and residual in their epilogue, and their gradients (flashbev_linear of flashbev.h).
//
// One kernel, gemm_kernel, forms D[M x N] = A[M x K] B[N x K]^T on the fifth-generation tensor cores for the three products
//
//     out         = x       weight^T     A = x  (K-major),      B = weight   (K-major)
//     grad_x      = dz      weight       A = dz (K-major),      B = weight^T (contiguous along N: MN-major)
//     grad_weight = dz^T    x            A = dz^T (MN-major),   B = x^T      (MN-major)
//
// persistent CTAs, one per SM: a producer fills a ring of shared-memory stages (64 of K each), one thread issues the products into
// one half of tensor memory, eight warps take the other half through bias, activation and residual to global memory.  In every
// tile, operands are 128-byte rows of 64 bf16 numbers with 128-byte swizzle, whether a row runs along K or along M or N.
#include "flashbev.h"
#include "launch.cuh"
#include "tcgen05.cuh"

#include <cuda_bf16.h>
#include <math.h>
#include <string.h>

#include <algorithm>
#include <type_traits>

using namespace flashbev_host;
using namespace flashbev_sm100;

namespace {

using bf16 = __nv_bfloat16;

constexpr int kBM = 128;            // rows of a tile: the 128 lanes of tensor memory
constexpr int kBK = 64;             // K of a stage: one swizzled 128-byte row of bf16
constexpr int kEpilogueWarps = 8;   // two per 32 lanes of tensor memory
constexpr int kProducerWarps = 8;   // of the loaders without TMA
constexpr int kRing = 192 * 1024;   // bytes of the operand stages
constexpr int kSmem = 1024 + kRing + kEpilogueWarps * 4096 + 1024;  // alignment, stages, staging of the epilogue, barriers and bias

// How a stage is filled.
enum Loader {
    kTma = 0,     // bf16, 16-byte aligned rows: TMA
    kCopy = 1,    // bf16 rows of any alignment: loads and shared-memory stores by eight warps
    kSplit = 2    // float32: the same warps take every number apart into three bf16 pieces
};

// Elements of float32 operands: x = p0 + p1 + p2, each piece the bf16 number nearest to what is left.  Every difference is exact and
// 8 + 8 + 8 bits hold the 24 of x.  Of the nine products the three left out, p1 p2, p2 p1 and p2 p2, are below 2^-25 |a| |b|.  Two tf32
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

// Phi(z) = erfc(-z / sqrt 2) / 2.  Results that are rounded to bf16 take erfc from Abramowitz and Stegun, Handbook of Mathematical
// Functions, 7.1.26 (within 1.5e-7; for z < 0 without a difference): 14 instructions instead of about 30, and the epilogue of a short sum is as long
// as its memory traffic.
template <bool FAST>
__device__ __forceinline__ float normal_cdf(float z)
{
    if constexpr (!FAST) return 0.5f * erfcf(-0.70710678f * z);
    const float a = fabsf(z) * 0.70710678f;
    const float t = __fdividef(1.0f, fmaf(0.3275911f, a, 1.0f));
    float s = fmaf(1.061405429f, t, -1.453152027f);
    s = fmaf(s, t, 1.421413741f);
    s = fmaf(s, t, -0.284496736f);
    s = fmaf(s, t, 0.254829592f);
    s = 0.5f * s * t * __expf(-a * a);
    return z < 0.0f ? s : 1.0f - s;
}

template <bool FAST>
__device__ __forceinline__ float sigmoid(float z)
{
    return FAST ? __fdividef(1.0f, 1.0f + __expf(-z)) : 1.0f / (1.0f + expf(-z));
}

template <bool FAST, int ACT>
__device__ __forceinline__ float activate(float z)
{
    if (ACT == FLASHBEV_ACT_RELU) return z < 0.0f ? 0.0f : z;  // (NaN stays)
    if (ACT == FLASHBEV_ACT_GELU) return z * normal_cdf<FAST>(z);
    if (ACT == FLASHBEV_ACT_SILU) return z * sigmoid<FAST>(z);
    return z;
}

// g act'(z)
template <bool FAST>
__device__ __forceinline__ float slope_times(float g, float z, int act)
{
    if (act == FLASHBEV_ACT_RELU) return z > 0.0f ? g : 0.0f;
    if (act == FLASHBEV_ACT_GELU) {
        const float e = FAST ? __expf(-0.5f * z * z) : expf(-0.5f * z * z);
        return g * fmaf(z * 0.39894228f, e, normal_cdf<FAST>(z));
    }
    if (act == FLASHBEV_ACT_SILU) {
        const float s = sigmoid<FAST>(z);
        return g * s * fmaf(z, 1.0f - s, 1.0f);
    }
    return g;
}

// ---- the product ------------------------------------------------------------------------------------------------------------

struct alignas(64) GemmParams {
    CUtensorMap ta, tb;         // kTma
    const void *a, *b;          // the other loaders
    long long lda, ldb;
    int a_mn, b_mn;             // the operand's rows run along M / N, one per k
    int a_vec, b_vec;           // bytes that every row's start is a multiple of: 16, 4 or less
    int M, N, K;
    int bn, stages;             // columns of a tile; stages in the ring
    int tiles_n, tiles, kblocks, kshare, splits;  // a tile's sum is cut into `splits` of `kshare` blocks of 64 (the last may have fewer)
    void *out, *pre;            // pre: z, or NULL
    const void *residual, *bias;
    long long ld_out, ld_pre, ld_res;
    int out_vec, pre_vec, res_vec;  // 16-byte accesses are allowed
    int act;
    float *partial;             // instead of the epilogue: [splits][M][ld_partial] sums
    long long ld_partial;
    uint32_t *error_word;
};

// A chunk of 32 rows x 32 columns between tensor memory's layout (a lane has a row) and global memory's (16 bytes of a row per lane,
// whole rows side by side), through 4 KB of the warp's own shared memory.  16-byte pieces are swizzled so that neither side has bank
// conflicts.
template <typename T>
struct Chunk {
    static constexpr int E = 16 / (int)sizeof(T);  // elements of 16 bytes
    static constexpr int P = 32 / E;               // pieces of a row: 8 (float32) or 4
    static constexpr int R = 32 / P;               // rows of one warp access
    static __device__ __forceinline__ uint32_t at(int row, int piece)
    {
        return P == 8 ? row * 128 + ((piece ^ (row & 7)) << 4) : row * 64 + ((piece ^ ((row >> 1) & 3)) << 4);
    }
};

template <typename T>
__device__ __forceinline__ uint4 load_piece(const T *p, int have, bool vec)
{
    constexpr int E = Chunk<T>::E;
    if (vec && have >= E) return *reinterpret_cast<const uint4 *>(p);
    T v[E];
#pragma unroll
    for (int i = 0; i < E; ++i) v[i] = i < have ? p[i] : from_float<T>(0.0f);
    uint4 r;
    memcpy(&r, v, 16);
    return r;
}

template <typename T>
__device__ __forceinline__ void store_piece(T *p, uint4 r, int have, bool vec)
{
    constexpr int E = Chunk<T>::E;
    if (vec && have >= E) {
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
__device__ __forceinline__ void chunk_load(uint4 (&r)[Chunk<T>::P], const T *base, long long ld, int row0, int col0, int M, int N, bool vec,
                                           int lane)
{
    using C = Chunk<T>;
    const int col = col0 + lane % C::P * C::E;
#pragma unroll
    for (int i = 0; i < C::P; ++i) {
        const int row = row0 + i * C::R + lane / C::P;
        if (row < M && col < N) r[i] = load_piece(base + row * ld + col, N - col, vec);
    }
}

// Adds the chunk that `chunk_load` brought to the lane's row.
template <typename T>
__device__ __forceinline__ void chunk_add(float (&v)[32], const uint4 (&r)[Chunk<T>::P], unsigned char *stage, int lane)
{
    using C = Chunk<T>;
#pragma unroll
    for (int i = 0; i < C::P; ++i) *reinterpret_cast<uint4 *>(stage + C::at(i * C::R + lane / C::P, lane % C::P)) = r[i];
    __syncwarp();
#pragma unroll
    for (int c = 0; c < C::P; ++c) {
        const uint4 q = *reinterpret_cast<const uint4 *>(stage + C::at(lane, c));
        const uint32_t w[4] = {q.x, q.y, q.z, q.w};
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            if constexpr (C::E == 4) v[4 * c + j] += __uint_as_float(w[j]);
            else v[8 * c + 2 * j] += low(w[j]), v[8 * c + 2 * j + 1] += high(w[j]);
        }
    }
    __syncwarp();
}

template <typename T>
__device__ __forceinline__ void chunk_store(const float (&v)[32], T *base, long long ld, int row0, int col0, int M, int N, bool vec,
                                            unsigned char *stage, int lane)
{
    using C = Chunk<T>;
#pragma unroll
    for (int c = 0; c < C::P; ++c) {
        uint4 q;
        if constexpr (C::E == 4)
            q = make_uint4(__float_as_uint(v[4 * c]), __float_as_uint(v[4 * c + 1]), __float_as_uint(v[4 * c + 2]), __float_as_uint(v[4 * c + 3]));
        else
            q = make_uint4(pack(v[8 * c], v[8 * c + 1]), pack(v[8 * c + 2], v[8 * c + 3]), pack(v[8 * c + 4], v[8 * c + 5]),
                           pack(v[8 * c + 6], v[8 * c + 7]));
        *reinterpret_cast<uint4 *>(stage + C::at(lane, c)) = q;
    }
    __syncwarp();
    const int col = col0 + lane % C::P * C::E;
#pragma unroll
    for (int i = 0; i < C::P; ++i) {
        const int row = row0 + i * C::R + lane / C::P;
        const uint4 q = *reinterpret_cast<const uint4 *>(stage + C::at(i * C::R + lane / C::P, lane % C::P));
        if (row < M && col < N) store_piece(base + row * ld + col, q, N - col, vec);
    }
    __syncwarp();
}

// One row of 64 elements of an operand's tile, the eight that this lane brings.  `unit`: row of 128 bytes in the tile.  K-major: one
// per m (or n); MN-major: 64 of them, one per k, for every 64 of M (or N).
template <int LOADER>
struct Eight {
    uint32_t w[LOADER == kSplit ? 8 : 4];
};

template <int LOADER>
__device__ __forceinline__ Eight<LOADER> operand_load(const void *base, long long ld, bool mn, int vec, int mn0, int k0, int MN, int K, int unit,
                                                      int piece)
{
    const int slow = mn ? k0 + unit % 64 : mn0 + unit, slows = mn ? K : MN;
    const int fast = (mn ? mn0 + unit / 64 * 64 : k0) + piece * 8, fasts = mn ? MN : K;
    Eight<LOADER> e;
#pragma unroll
    for (int i = 0; i < (LOADER == kSplit ? 8 : 4); ++i) e.w[i] = 0;
    const int have = slow < slows ? fasts - fast : 0;
    if (have <= 0) return e;
    if constexpr (LOADER == kSplit) {
        const float *p = static_cast<const float *>(base) + slow * ld + fast;
        if (vec >= 16 && have >= 8) {
            const uint4 u = __ldg(reinterpret_cast<const uint4 *>(p)), v = __ldg(reinterpret_cast<const uint4 *>(p) + 1);
            e.w[0] = u.x, e.w[1] = u.y, e.w[2] = u.z, e.w[3] = u.w, e.w[4] = v.x, e.w[5] = v.y, e.w[6] = v.z, e.w[7] = v.w;
        } else {
#pragma unroll
            for (int i = 0; i < 8; ++i)
                if (i < have) e.w[i] = __float_as_uint(__ldg(p + i));
        }
    } else {
        const unsigned short *p = static_cast<const unsigned short *>(base) + slow * ld + fast;
        if (vec >= 16 && have >= 8) {
            const uint4 u = __ldg(reinterpret_cast<const uint4 *>(p));
            e.w[0] = u.x, e.w[1] = u.y, e.w[2] = u.z, e.w[3] = u.w;
        } else if (vec >= 4) {
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                if (2 * i + 2 <= have) e.w[i] = __ldg(reinterpret_cast<const uint32_t *>(p) + i);
                else if (2 * i < have) e.w[i] = __ldg(p + 2 * i);
            }
        } else {
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                if (2 * i < have) e.w[i] = __ldg(p + 2 * i);
                if (2 * i + 1 < have) e.w[i] |= (uint32_t)__ldg(p + 2 * i + 1) << 16;
            }
        }
    }
    return e;
}

template <int LOADER>
__device__ __forceinline__ void operand_store(const Eight<LOADER> &e, unsigned char *tile, int tile_bytes, int unit, int piece)
{
    const int at = unit * 128 + ((piece ^ (unit & 7)) << 4);
    if constexpr (LOADER != kSplit) {
        *reinterpret_cast<uint4 *>(tile + at) = make_uint4(e.w[0], e.w[1], e.w[2], e.w[3]);
    } else {
        uint32_t p0[4], p1[4], p2[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            float u = __uint_as_float(e.w[2 * i]), v = __uint_as_float(e.w[2 * i + 1]);
            p0[i] = pack(u, v);
            u -= low(p0[i]), v -= high(p0[i]);
            p1[i] = pack(u, v);
            p2[i] = pack(u - low(p1[i]), v - high(p1[i]));
        }
        *reinterpret_cast<uint4 *>(tile + at) = make_uint4(p0[0], p0[1], p0[2], p0[3]);
        *reinterpret_cast<uint4 *>(tile + tile_bytes + at) = make_uint4(p1[0], p1[1], p1[2], p1[3]);
        *reinterpret_cast<uint4 *>(tile + 2 * tile_bytes + at) = make_uint4(p2[0], p2[1], p2[2], p2[3]);
    }
}

// A share of a tile's sum: tile (m0, n0) and the blocks [k, end) of 64.
struct Share {
    int m0, n0, k, end, split;
};

__device__ __forceinline__ Share share_of(const GemmParams &p, int w)
{
    Share s;
    s.split = w / p.tiles;
    const int t = w - s.split * p.tiles;
    const int m = t / p.tiles_n;
    s.m0 = m * kBM, s.n0 = (t - m * p.tiles_n) * p.bn;
    s.k = s.split * p.kshare;
    s.end = min(s.k + p.kshare, p.kblocks);
    return s;
}

template <typename TIN, typename TOUT, int ACT>
__device__ __forceinline__ void finish_chunk(const GemmParams &p, float (&v)[32], int row0, int col0, unsigned char *stage, const float *bias,
                                             const uint4 (&res)[Chunk<TOUT>::P], int lane)
{
    constexpr bool kFast = std::is_same<TOUT, bf16>::value;
#pragma unroll
    for (int c = 0; c < 8; ++c) {
        const float4 b = reinterpret_cast<const float4 *>(bias)[c];
        v[4 * c] += b.x, v[4 * c + 1] += b.y, v[4 * c + 2] += b.z, v[4 * c + 3] += b.w;
    }
    if (p.pre) chunk_store<TIN>(v, static_cast<TIN *>(p.pre), p.ld_pre, row0, col0, p.M, p.N, p.pre_vec, stage, lane);
#pragma unroll
    for (int i = 0; i < 32; ++i) v[i] = activate<kFast, ACT>(v[i]);
    if (p.residual) chunk_add<TOUT>(v, res, stage, lane);
    chunk_store<TOUT>(v, static_cast<TOUT *>(p.out), p.ld_out, row0, col0, p.M, p.N, p.out_vec, stage, lane);
}

template <int LOADER, typename TOUT>
__global__ void __launch_bounds__(LOADER == kTma ? 32 * (kEpilogueWarps + 2) : 32 * (kEpilogueWarps + 1 + kProducerWarps), 1)
    gemm_kernel(const __grid_constant__ GemmParams p)
{
    using TIN = typename std::conditional<LOADER == kSplit, float, bf16>::type;
    constexpr int kPieces = LOADER == kSplit ? 3 : 1;
    extern __shared__ unsigned char raw[];
    unsigned char *const ring = raw + ((1024 - (smem_u32(raw) & 1023)) & 1023);
    unsigned char *const staging = ring + kRing;
    float *const bias_rows = reinterpret_cast<float *>(staging + kEpilogueWarps * 4096);  // 32 per warp
    __shared__ __align__(8) uint64_t bars[2 * 8 + 4 + 1];
    __shared__ uint32_t tmem_slot;
    __shared__ volatile int failed;
    const int warp = threadIdx.x / 32, lane = threadIdx.x % 32;
    const uint32_t full = smem_u32(bars), empty = full + 64, acc_full = full + 128, acc_empty = full + 144, last = full + 160;
    // Tensor memory: two accumulators, so that one is taken out while the other is filled.  With pieces each has a second one behind it
    // for all products but p0 p0: the tensor cores cut the sum off, not round it, at every instruction, and the five small products
    // would do so to the whole sum five times as often as the large one does (float32, K = 4096, 16 rows: relative error 3.2e-6
    // with one accumulator).
    constexpr int kParts = kPieces == 3 ? 2 : 1;
    const uint32_t columns = 2 * kParts * p.bn;

    if (threadIdx.x == 0) {
        failed = 0;
        for (int s = 0; s < p.stages; ++s) {
            mbar_init(full + 8 * s, LOADER == kTma ? 1 : kProducerWarps);
            mbar_init(empty + 8 * s, 1);
        }
        for (int b = 0; b < 2; ++b) mbar_init(acc_full + 8 * b, 1), mbar_init(acc_empty + 8 * b, kEpilogueWarps);
        mbar_init(last, 1);
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
        asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
    }
    if (warp == kEpilogueWarps) tmem_alloc(smem_u32(&tmem_slot), columns);
    tcgen05_fence_before();
    __syncthreads();
    tcgen05_fence_after();
    const uint32_t tmem = tmem_slot;
    asm volatile("griddepcontrol.wait;" ::: "memory");
    asm volatile("griddepcontrol.launch_dependents;");

    const int total = p.tiles * p.splits;
    const int a_bytes = kBM * 128, b_bytes = p.bn * 128, stage_bytes = kPieces * (a_bytes + b_bytes);

    if (warp < kEpilogueWarps) {
        // ---- epilogue: warps w and w + 4 share the 32 lanes 32 (w % 4) and up, every other chunk of 32 columns each
        unsigned char *const stage = staging + warp * 4096;
        float *const bias = bias_rows + warp * 32;
        const uint32_t lanes = tmem + ((uint32_t)(warp % 4 * 32) << 16);
        int buf = 0, phase = 0;
        for (int w = blockIdx.x; w < total; w += gridDim.x) {
            const Share s = share_of(p, w);
            const int row0 = s.m0 + warp % 4 * 32;
            bool waited = false, ok = true;
            for (int c = warp / 4; c < p.bn / 32; c += 2) {
                const int col0 = s.n0 + 32 * c;
                if (col0 >= p.N || row0 >= p.M) break;
                uint4 res[Chunk<TOUT>::P];
                if (!p.partial) {
                    if (p.residual) chunk_load<TOUT>(res, static_cast<const TOUT *>(p.residual), p.ld_res, row0, col0, p.M, p.N, p.res_vec, lane);
                    const int col = col0 + lane;
                    bias[lane] = p.bias && col < p.N ? to_float(static_cast<const TIN *>(p.bias)[col]) : 0.0f;
                    __syncwarp();
                }
                if (!waited) {
                    if (!(ok = __all_sync(0xffffffffu, mbar_wait(acc_full + 8 * buf, phase, &failed)))) break;
                    tcgen05_fence_after();
                    waited = true;
                }
                float v[32];
                tmem_load32(v, lanes + buf * kParts * p.bn + 32 * c);
                if constexpr (kParts == 2) {
                    float small[32];
                    tmem_load32(small, lanes + (2 * buf + 1) * p.bn + 32 * c);
#pragma unroll
                    for (int i = 0; i < 32; ++i) v[i] += small[i];
                }
                if (p.partial) {
                    float *const out = p.partial + (long long)s.split * p.M * p.ld_partial;
                    chunk_store<float>(v, out, p.ld_partial, row0, col0, p.M, p.N, true, stage, lane);
                } else if (p.act == FLASHBEV_ACT_NONE) {
                    finish_chunk<TIN, TOUT, FLASHBEV_ACT_NONE>(p, v, row0, col0, stage, bias, res, lane);
                } else if (p.act == FLASHBEV_ACT_RELU) {
                    finish_chunk<TIN, TOUT, FLASHBEV_ACT_RELU>(p, v, row0, col0, stage, bias, res, lane);
                } else if (p.act == FLASHBEV_ACT_GELU) {
                    finish_chunk<TIN, TOUT, FLASHBEV_ACT_GELU>(p, v, row0, col0, stage, bias, res, lane);
                } else {
                    finish_chunk<TIN, TOUT, FLASHBEV_ACT_SILU>(p, v, row0, col0, stage, bias, res, lane);
                }
            }
            if (ok && !waited) ok = __all_sync(0xffffffffu, mbar_wait(acc_full + 8 * buf, phase, &failed));
            if (!ok) break;
            tcgen05_fence_before();
            __syncwarp();
            if (lane == 0) mbar_arrive(acc_empty + 8 * buf);
            phase ^= buf, buf ^= 1;
        }
    } else if (warp == kEpilogueWarps) {
        // ---- products, by one thread
        if (lane == 0) {
            const uint32_t idesc = mma_idesc(p.bn, p.a_mn, p.b_mn);
            const int a_step = p.a_mn ? 2048 >> 4 : 32 >> 4, b_step = p.b_mn ? 2048 >> 4 : 32 >> 4;  // 16 of K further
            int stage = 0, phase = 0, buf = 0, acc_phase = 0;
            bool ok = true;
            for (int w = blockIdx.x; w < total && ok; w += gridDim.x) {
                const Share s = share_of(p, w);
                if (!(ok = mbar_wait(acc_empty + 8 * buf, acc_phase ^ 1, &failed))) break;
                tcgen05_fence_after();
                const uint32_t d = tmem + buf * kParts * p.bn;
                for (int k = s.k; k < s.end; ++k) {
                    if (!(ok = mbar_wait(full + 8 * stage, phase, &failed))) break;
                    tcgen05_fence_after();
                    const uint32_t at = smem_u32(ring) + stage * stage_bytes;
                    const uint64_t a = smem_desc(at, p.a_mn, 8192), b = smem_desc(at + kPieces * a_bytes, p.b_mn, 8192);
                    if constexpr (kPieces == 1) {
#pragma unroll
                        for (int i = 0; i < kBK / 16; ++i) mma_bf16(d, a + i * a_step, b + i * b_step, idesc, k > s.k || i > 0);
                    } else {
                        constexpr int pa[6] = {2, 0, 1, 1, 0, 0}, pb[6] = {0, 2, 1, 0, 1, 0};
#pragma unroll
                        for (int j = 0; j < 6; ++j)
#pragma unroll
                            for (int i = 0; i < kBK / 16; ++i)
                                mma_bf16(j < 5 ? d + p.bn : d, a + pa[j] * (a_bytes >> 4) + i * a_step, b + pb[j] * (b_bytes >> 4) + i * b_step,
                                         idesc, k > s.k || i > 0 || (j > 0 && j < 5));
                    }
                    mma_commit(empty + 8 * stage);
                    if (++stage == p.stages) stage = 0, phase ^= 1;
                }
                if (ok) mma_commit(acc_full + 8 * buf);
                acc_phase ^= buf, buf ^= 1;
            }
            if (!ok) {  // nothing of this CTA may be in flight when it gives its memory back
                mma_commit(last);
                mbar_drain(last, 0);
            }
        }
        __syncwarp();
    } else if constexpr (LOADER == kTma) {
        if (lane == 0) {
            int stage = 0, phase = 0;
            bool ok = true;
            for (int w = blockIdx.x; w < total && ok; w += gridDim.x) {
                const Share s = share_of(p, w);
                for (int k = s.k; k < s.end; ++k) {
                    if (!(ok = mbar_wait(empty + 8 * stage, phase ^ 1, &failed))) break;
                    const uint32_t at = smem_u32(ring) + stage * stage_bytes, bar = full + 8 * stage;
                    mbar_expect(bar, stage_bytes);
                    if (p.a_mn) {
                        for (int i = 0; i < kBM / 64; ++i) tma_load_2d(at + 8192 * i, &p.ta, s.m0 + 64 * i, k * kBK, bar);
                    } else {
                        tma_load_2d(at, &p.ta, k * kBK, s.m0, bar);
                    }
                    if (p.b_mn) {
                        for (int i = 0; i < p.bn / 64; ++i) tma_load_2d(at + a_bytes + 8192 * i, &p.tb, s.n0 + 64 * i, k * kBK, bar);
                    } else {
                        tma_load_2d(at + a_bytes, &p.tb, k * kBK, s.n0, bar);
                    }
                    if (++stage == p.stages) stage = 0, phase ^= 1;
                }
            }
            if (!ok)  // the last load into every stage: the ones before `stage` in this round of the ring, the others in the round before
                for (int i = 0; i < p.stages; ++i) mbar_drain(full + 8 * i, i < stage ? phase : phase ^ 1);
        }
        __syncwarp();
    } else {
        // ---- loads without TMA: a warp brings four rows of 128 bytes (64 elements) at a time; the loads of the next stage are under
        // way while this one is written and the products of the ones before run
        constexpr int kPasses = (kBM + 128) / (4 * kProducerWarps);  // tiles are at most 128 columns wide here
        const int first = (warp - kEpilogueWarps - 1) * 4 + lane / 8, piece = lane % 8;
        const int passes = (kBM + p.bn) / (4 * kProducerWarps);
        int w = blockIdx.x, stage = 0, phase = 0;
        Share s = share_of(p, min(w, total - 1));
        Eight<LOADER> r[kPasses];
        const auto fetch = [&] {
#pragma unroll
            for (int i = 0; i < kPasses; ++i) {
                const int unit = first + 4 * kProducerWarps * i;
                if (i < kBM / (4 * kProducerWarps))
                    r[i] = operand_load<LOADER>(p.a, p.lda, p.a_mn, p.a_vec, s.m0, s.k * kBK, p.M, p.K, unit, piece);
                else if (i < passes)
                    r[i] = operand_load<LOADER>(p.b, p.ldb, p.b_mn, p.b_vec, s.n0, s.k * kBK, p.N, p.K, unit - kBM, piece);
            }
        };
        if (w < total) fetch();
        while (w < total) {
            if (!__all_sync(0xffffffffu, mbar_wait(empty + 8 * stage, phase ^ 1, &failed))) break;
            unsigned char *const at = ring + stage * stage_bytes;
#pragma unroll
            for (int i = 0; i < kPasses; ++i) {
                const int unit = first + 4 * kProducerWarps * i;
                if (i < kBM / (4 * kProducerWarps)) operand_store<LOADER>(r[i], at, a_bytes, unit, piece);
                else if (i < passes) operand_store<LOADER>(r[i], at + kPieces * a_bytes, b_bytes, unit - kBM, piece);
            }
            asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
            __syncwarp();
            if (lane == 0) mbar_arrive(full + 8 * stage);
            if (++stage == p.stages) stage = 0, phase ^= 1;
            if (++s.k == s.end) {
                w += gridDim.x;
                if (w >= total) break;
                s = share_of(p, w);
            }
            fetch();
        }
    }
    tcgen05_fence_before();
    __syncthreads();
    if (warp == kEpilogueWarps) {
        tcgen05_fence_after();
        tmem_free(tmem, columns);
    }
    if (threadIdx.x == 0 && failed && p.error_word) atomicAdd(p.error_word, 1u);
}

// ---- sums that several CTAs shared ----------------------------------------------------------------------------------------

// Adds the shares up in their order and does what the epilogue would have done.  Four columns of a row per thread.
template <typename TIN, typename TOUT>
__global__ void __launch_bounds__(256) join_kernel(const float *__restrict__ partial, long long ld_partial, int splits, int M, int N,
                                                   const TIN *__restrict__ bias, const TOUT *residual, long long ld_res, TOUT *out, long long ld_out,
                                                   TIN *pre, long long ld_pre, int act)
{
    constexpr bool kFast = std::is_same<TOUT, bf16>::value;
    asm volatile("griddepcontrol.wait;" ::: "memory");
    asm volatile("griddepcontrol.launch_dependents;");
    const int quads = (int)(ld_partial / 4);
    const long long all = (long long)M * quads;
    for (long long i = (long long)blockIdx.x * 256 + threadIdx.x; i < all; i += (long long)gridDim.x * 256) {
        const long long row = i / quads;
        const int col = (int)(i - row * quads) * 4;
        const float4 *src = reinterpret_cast<const float4 *>(partial + row * ld_partial + col);
        const long long step = (long long)M * ld_partial / 4;
        float v[4] = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll 8
        for (int s = 0; s < splits; ++s) {
            const float4 q = __ldcs(src + s * step);
            v[0] += q.x, v[1] += q.y, v[2] += q.z, v[3] += q.w;
        }
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            if (col + j >= N) break;
            float z = v[j] + (bias ? to_float(bias[col + j]) : 0.0f);
            if (pre) pre[row * ld_pre + col + j] = from_float<TIN>(z);
            if (act == FLASHBEV_ACT_RELU) z = activate<kFast, FLASHBEV_ACT_RELU>(z);
            else if (act == FLASHBEV_ACT_GELU) z = activate<kFast, FLASHBEV_ACT_GELU>(z);
            else if (act == FLASHBEV_ACT_SILU) z = activate<kFast, FLASHBEV_ACT_SILU>(z);
            if (residual) z += to_float(residual[row * ld_res + col + j]);
            out[row * ld_out + col + j] = from_float<TOUT>(z);
        }
    }
}

// ---- dz = grad_out act'(z), and its column sums ---------------------------------------------------------------------------

constexpr int kSlopeRows = 8;  // warps of a block: each takes every eighth row of the block's

// A lane has VEC neighbouring columns, a warp a stretch of a row, the block `per` rows.  dz may be NULL (column sums only), sums too.
template <typename TG, typename TZ, int VEC>
__global__ void __launch_bounds__(32 * kSlopeRows) slope_kernel(const TG *__restrict__ g, long long ld_g, const TZ *__restrict__ z, long long ld_z,
                                                                TZ *__restrict__ dz, long long ld_dz, float *__restrict__ sums, int M, int N, int per,
                                                                int act)
{
    constexpr bool kFast = std::is_same<TZ, bf16>::value;
    asm volatile("griddepcontrol.wait;" ::: "memory");
    asm volatile("griddepcontrol.launch_dependents;");
    const int warp = threadIdx.x / 32, lane = threadIdx.x % 32;
    const int col = (blockIdx.x * 32 + lane) * VEC;
    const long long row1 = min((long long)M, (long long)(blockIdx.y + 1) * per);
    float acc[VEC];
#pragma unroll
    for (int j = 0; j < VEC; ++j) acc[j] = 0.0f;
    if (col < N)
#pragma unroll 4
        for (long long row = (long long)blockIdx.y * per + warp; row < row1; row += kSlopeRows) {
            TG gv[VEC];
            TZ zv[VEC];
            if constexpr (VEC > 1) {
                constexpr int GQ = VEC * (int)sizeof(TG) / 16, ZQ = VEC * (int)sizeof(TZ) / 16;
                uint4 q[GQ > ZQ ? GQ : ZQ];
#pragma unroll
                for (int i = 0; i < GQ; ++i) q[i] = __ldcs(reinterpret_cast<const uint4 *>(g + row * ld_g + col) + i);
                memcpy(gv, q, sizeof(gv));
                if (z) {
#pragma unroll
                    for (int i = 0; i < ZQ; ++i) q[i] = __ldcs(reinterpret_cast<const uint4 *>(z + row * ld_z + col) + i);
                    memcpy(zv, q, sizeof(zv));
                }
            } else {
                gv[0] = g[row * ld_g + col];
                if (z) zv[0] = z[row * ld_z + col];
            }
            float d[VEC];
#pragma unroll
            for (int j = 0; j < VEC; ++j) {
                d[j] = z ? slope_times<kFast>(to_float(gv[j]), to_float(zv[j]), act) : to_float(gv[j]);
                acc[j] += d[j];
            }
            if (dz) {
                if constexpr (VEC > 1) {
                    constexpr int ZQ = VEC * (int)sizeof(TZ) / 16;
                    TZ o[VEC];
#pragma unroll
                    for (int j = 0; j < VEC; ++j) o[j] = from_float<TZ>(d[j]);
                    uint4 q[ZQ];
                    memcpy(q, o, sizeof(o));
#pragma unroll
                    for (int i = 0; i < ZQ; ++i) reinterpret_cast<uint4 *>(dz + row * ld_dz + col)[i] = q[i];
                } else {
                    dz[row * ld_dz + col] = from_float<TZ>(d[0]);
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

// Column sums of `rows` rows of partial sums: 32 columns per block, its eight warps take every eighth row.
template <typename T>
__global__ void __launch_bounds__(256) column_sum_kernel(const float *__restrict__ sums, int rows, int N, T *__restrict__ out)
{
    asm volatile("griddepcontrol.wait;" ::: "memory");
    asm volatile("griddepcontrol.launch_dependents;");
    __shared__ float part[8][33];
    const int warp = threadIdx.x / 32, lane = threadIdx.x % 32, col = blockIdx.x * 32 + lane;
    float v = 0.0f;
    if (col < N)
#pragma unroll 8
        for (int r = warp; r < rows; r += 8) v += sums[(long long)r * N + col];
    part[warp][lane] = v;
    __syncthreads();
    if (warp == 0 && col < N) {
        v = 0.0f;
#pragma unroll
        for (int w = 0; w < 8; ++w) v += part[w][lane];
        out[col] = from_float<T>(v);
    }
}

// ---- few rows ---------------------------------------------------------------------------------------------------------------

// Up to R rows of x: bound by reading the weights once, so no tensor cores (their tiles would be empty rows).  A warp forms NC
// neighbouring columns of all rows, its lanes 8 elements of the sum each at a time.
template <typename TIN, typename TOUT, int R, int NC, bool VEC>
__global__ void __launch_bounds__(256) rows_kernel(const TIN *__restrict__ x, long long ld_x, const TIN *__restrict__ weight, long long ld_w, int M,
                                                   int N, int K, const TIN *__restrict__ bias, const TOUT *residual, long long ld_res, TOUT *out,
                                                   long long ld_out, TIN *pre, long long ld_pre, int act)
{
    constexpr bool kFast = std::is_same<TOUT, bf16>::value;
    constexpr int Q = 8 * (int)sizeof(TIN) / 16;
    asm volatile("griddepcontrol.wait;" ::: "memory");
    asm volatile("griddepcontrol.launch_dependents;");
    const int lane = threadIdx.x % 32, n0 = (blockIdx.x * 8 + threadIdx.x / 32) * NC;
    if (n0 >= N) return;
    float acc[R][NC];
#pragma unroll
    for (int r = 0; r < R; ++r)
#pragma unroll
        for (int c = 0; c < NC; ++c) acc[r][c] = 0.0f;
    const auto bring = [&](float (&v)[8], const TIN *p, int have) {
        if (VEC && have >= 8) {
            uint4 q[Q];
            TIN t[8];
#pragma unroll
            for (int i = 0; i < Q; ++i) q[i] = __ldg(reinterpret_cast<const uint4 *>(p) + i);
            memcpy(t, q, sizeof(t));
#pragma unroll
            for (int i = 0; i < 8; ++i) v[i] = to_float(t[i]);
        } else {
#pragma unroll
            for (int i = 0; i < 8; ++i) v[i] = i < have ? to_float(p[i]) : 0.0f;
        }
    };
#pragma unroll 2
    for (int k = lane * 8; k < K; k += 256) {
        float wv[NC][8];
#pragma unroll
        for (int c = 0; c < NC; ++c) bring(wv[c], weight + min(n0 + c, N - 1) * ld_w + k, K - k);
#pragma unroll
        for (int r = 0; r < R; ++r) {
            float xv[8];
            bring(xv, x + min(r, M - 1) * ld_x + k, K - k);
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
#pragma unroll
    for (int r = 0; r < R; ++r)
#pragma unroll
        for (int c = 0; c < NC; ++c) {
            if (lane != r * NC + c || r >= M || n0 + c >= N) continue;
            float z = acc[r][c] + (bias ? to_float(bias[n0 + c]) : 0.0f);
            if (pre) pre[r * ld_pre + n0 + c] = from_float<TIN>(z);
            if (act == FLASHBEV_ACT_RELU) z = activate<kFast, FLASHBEV_ACT_RELU>(z);
            else if (act == FLASHBEV_ACT_GELU) z = activate<kFast, FLASHBEV_ACT_GELU>(z);
            else if (act == FLASHBEV_ACT_SILU) z = activate<kFast, FLASHBEV_ACT_SILU>(z);
            if (residual) z += to_float(residual[r * ld_res + n0 + c]);
            out[r * ld_out + n0 + c] = from_float<TOUT>(z);
        }
}

// ---- host -------------------------------------------------------------------------------------------------------------------

constexpr int kMaxFeatures = 1 << 24;
constexpr int kFewRows = 8;

// One of the kernel's operands: rows of `fast` contiguous elements, `slow` of them, ld apart.
struct Operand {
    const void *p;
    long long ld;
    bool mn;  // a row per k
};

bool tma_ok(const Operand &o) { return (uintptr_t)o.p % 16 == 0 && o.ld % 8 == 0; }

int row_vec(const Operand &o, int elem)
{
    const uintptr_t bits = (uintptr_t)o.p | (uintptr_t)(o.ld * elem);
    return bits % 16 == 0 ? 16 : (bits % 4 == 0 ? 4 : 1);
}

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
bool make_map(CUtensorMap &map, const Operand &o, int across, int K, int rows)
{
    const EncodeTiled encode = encode_tiled();
    if (!encode) return false;
    const cuuint64_t size[2] = {(cuuint64_t)(o.mn ? across : K), (cuuint64_t)(o.mn ? K : across)}, pitch[1] = {(cuuint64_t)o.ld * 2};
    const cuuint32_t box[2] = {kBK, (cuuint32_t)(o.mn ? kBK : rows)}, step[2] = {1, 1};
    return encode(&map, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 2, const_cast<void *>(o.p), size, pitch, box, step, CU_TENSOR_MAP_INTERLEAVE_NONE,
                  CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

// Tiles and shares of a product.
struct Plan {
    int loader, bn, stages, tiles_m, tiles_n, kblocks, kshare, splits;
    long long ld_partial;
    size_t partial_bytes;  // 0: every tile's sum belongs to one CTA
};

Plan plan_product(const Operand &a, const Operand &b, bool f32, int M, int N, int K, bool may_split)
{
    Plan q = {};
    q.loader = f32 ? kSplit : (tma_ok(a) && tma_ok(b) ? kTma : kCopy);
    const int sms = sm_count();
    q.tiles_m = (M + kBM - 1) / kBM;
    q.kblocks = (K + kBK - 1) / kBK;
    // The widest tile that does not leave more than a tenth of the SMs' time idle (a wide tile reads A fewer times and feeds the
    // tensor cores better).
    const int widest = q.loader == kTma ? 256 : 128;
    double best = 0.0;
    for (int bn = widest; bn >= 64; bn /= 2) {
        const long long tiles = (long long)q.tiles_m * ((N + bn - 1) / bn);
        const long long waves = (tiles + sms - 1) / sms;
        const double use = (double)M * N / ((double)waves * sms * kBM * bn);
        if (use > 1.1 * best) best = use, q.bn = bn;
    }
    q.tiles_n = (N + q.bn - 1) / q.bn;
    const int stage = (q.loader == kSplit ? 3 : 1) * (kBM + q.bn) * 128;
    q.stages = std::min(8, kRing / stage);
    const long long tiles = (long long)q.tiles_m * q.tiles_n;
    q.splits = 1, q.kshare = q.kblocks;
    if (may_split && tiles * 2 <= sms) {
        const int least = 2;  // blocks of 64 for a share to be worth its partial sums
        int splits = (int)std::min<long long>(sms / tiles, q.kblocks / least);
        if (splits > 1) {
            q.kshare = (q.kblocks + splits - 1) / splits;
            q.splits = (q.kblocks + q.kshare - 1) / q.kshare;
        }
    }
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
};

bool vec_ok(const void *p, long long ld, bool f32)
{
    return ((uintptr_t)p | (uintptr_t)(ld * (f32 ? 4 : 2))) % 16 == 0;
}

template <int LOADER, typename TOUT>
cudaError_t launch_gemm(const GemmParams &g, cudaStream_t stream)
{
    const auto kernel = gemm_kernel<LOADER, TOUT>;
    const cudaError_t e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, kSmem);
    if (e != cudaSuccess) return e;
    const int threads = LOADER == kTma ? 32 * (kEpilogueWarps + 2) : 32 * (kEpilogueWarps + 1 + kProducerWarps);
    const int grid = std::min(g.tiles * g.splits, sm_count());
    return launch_dependent(kernel, dim3((unsigned)grid), dim3((unsigned)threads), kSmem, stream, g);
}

template <typename TIN, typename TOUT>
cudaError_t launch_join(const Plan &q, const float *partial, int M, int N, const Epilogue &e, cudaStream_t stream)
{
    const long long quads = (long long)M * (q.ld_partial / 4);
    const unsigned blocks = (unsigned)std::min<long long>((quads + 255) / 256, 8LL * sm_count());
    return launch_dependent(join_kernel<TIN, TOUT>, dim3(blocks), dim3(256), 0, stream, partial, q.ld_partial, q.splits, M, N,
                            static_cast<const TIN *>(e.bias), static_cast<const TOUT *>(e.residual), e.ld_res, static_cast<TOUT *>(e.out), e.ld_out,
                            static_cast<TIN *>(e.pre), e.ld_pre, e.act);
}

// Enqueues one product; adds the kernels to `launches`.
flashbev_status run_product(const Plan &q, const Operand &a, const Operand &b, bool f32, int M, int N, int K, const Epilogue &e, float *partial,
                            uint32_t *error_word, cudaStream_t stream, int &launches)
{
    GemmParams g = {};
    if (q.loader == kTma && !(make_map(g.ta, a, M, K, kBM) && make_map(g.tb, b, N, K, q.bn))) return FLASHBEV_CUDA_ERROR;
    const int elem = f32 ? 4 : 2;
    g.a = a.p, g.b = b.p, g.lda = a.ld, g.ldb = b.ld, g.a_mn = a.mn, g.b_mn = b.mn;
    g.a_vec = row_vec(a, elem), g.b_vec = row_vec(b, elem);
    g.M = M, g.N = N, g.K = K, g.bn = q.bn, g.stages = q.stages;
    g.tiles_n = q.tiles_n, g.tiles = q.tiles_m * q.tiles_n, g.kblocks = q.kblocks, g.kshare = q.kshare, g.splits = q.splits;
    g.out = e.out, g.pre = e.pre, g.residual = e.residual, g.bias = e.bias, g.act = e.act;
    g.ld_out = e.ld_out, g.ld_pre = e.ld_pre, g.ld_res = e.ld_res;
    g.out_vec = vec_ok(e.out, e.ld_out, e.out_f32), g.pre_vec = vec_ok(e.pre, e.ld_pre, f32), g.res_vec = vec_ok(e.residual, e.ld_res, e.out_f32);
    g.error_word = error_word;
    if (q.splits > 1) g.partial = partial, g.ld_partial = q.ld_partial;
    cudaError_t err;
    if (q.loader == kSplit) err = e.out_f32 ? launch_gemm<kSplit, float>(g, stream) : launch_gemm<kSplit, bf16>(g, stream);
    else if (q.loader == kCopy) err = e.out_f32 ? launch_gemm<kCopy, float>(g, stream) : launch_gemm<kCopy, bf16>(g, stream);
    else err = e.out_f32 ? launch_gemm<kTma, float>(g, stream) : launch_gemm<kTma, bf16>(g, stream);
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
cudaError_t launch_rows(const Operand &x, const Operand &w, int M, int N, int K, const Epilogue &e, cudaStream_t stream)
{
    const bool vec = row_vec(x, sizeof(TIN)) == 16 && row_vec(w, sizeof(TIN)) == 16;
    const auto go = [&](auto kernel, int nc) {
        return launch_dependent(kernel, dim3((unsigned)((N + 8 * nc - 1) / (8 * nc))), dim3(256), 0, stream, static_cast<const TIN *>(x.p), x.ld,
                                static_cast<const TIN *>(w.p), w.ld, M, N, K, static_cast<const TIN *>(e.bias), static_cast<const TOUT *>(e.residual),
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

Operand operand_x(const flashbev_linear_params *p) { return {p->x, dense(p->ld_x, p->in_features), false}; }
Operand operand_w(const flashbev_linear_params *p) { return {p->weight, dense(p->ld_weight, p->in_features), false}; }

// ---- backward

struct BackwardPlan {
    bool need_dz, need_x, need_w, need_b;
    long long ld_dz;
    Plan gx, gw;
    int per, chunks;                                // rows of a block of slope_kernel; blocks along the rows
    size_t dz_at, sums_at, partial_at, total;
    Operand dz;
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
    const auto up = [](size_t v) { return (v + 255) / 256 * 256; };
    q.need_x = p->grad_x, q.need_w = p->grad_weight, q.need_b = p->grad_bias;
    if (!M) return q;
    q.need_dz = (q.need_x || q.need_w) && (p->act != FLASHBEV_ACT_NONE || p->dtype != p->grad_dtype);
    size_t at = 0;
    if (q.need_dz) {
        q.ld_dz = (N + 7) / 8 * 8;
        q.dz_at = at, at += up((size_t)M * q.ld_dz * elem_size(p->dtype));
        q.dz = {static_cast<char *>(p->workspace) + q.dz_at, q.ld_dz, false};
    } else {
        q.dz = {p->grad_out, dense(p->ld_grad_out, N), false};
    }
    if (q.need_dz || q.need_b) {
        // about four blocks per SM, but no fewer than 32 rows for each
        const int across = std::max(1, (N + 255) / 256);
        const long long blocks = std::max(1, 4 * sm_count() / across);
        q.per = (int)std::max<long long>(32, (M + blocks - 1) / blocks);
        q.chunks = (M + q.per - 1) / q.per;
        if (q.chunks > 65535) q.per = (M + 65534) / 65535, q.chunks = (M + q.per - 1) / q.per;
        if (q.need_b) q.sums_at = at, at += up((size_t)q.chunks * N * sizeof(float));
    }
    const Operand w = {p->weight, dense(p->ld_weight, K), true}, x = {p->x, dense(p->ld_x, K), true};
    Operand dzt = q.dz;
    dzt.mn = true;
    if (q.need_x) q.gx = plan_product(q.dz, w, f32, M, K, N, true);
    if (q.need_w) q.gw = plan_product(dzt, x, f32, N, K, M, true);
    q.partial_at = at;  // (the products run one after the other)
    at += up(std::max(q.gx.partial_bytes, q.gw.partial_bytes));
    q.total = at;
    return q;
}

template <typename TG, typename TZ>
cudaError_t launch_slope(const flashbev_linear_backward_params *p, const BackwardPlan &q, cudaStream_t stream)
{
    const int M = (int)p->rows, N = p->out_features;
    char *const ws = static_cast<char *>(p->workspace);
    TZ *const dz = q.need_dz ? reinterpret_cast<TZ *>(ws + q.dz_at) : nullptr;
    float *const sums = q.need_b ? reinterpret_cast<float *>(ws + q.sums_at) : nullptr;
    const TZ *const z = p->act == FLASHBEV_ACT_NONE ? nullptr : static_cast<const TZ *>(p->preact);
    const long long ld_g = dense(p->ld_grad_out, N), ld_z = dense(p->ld_preact, N);
    const bool vec = N % 8 == 0 && vec_ok(p->grad_out, ld_g, sizeof(TG) == 4) && (!z || vec_ok(z, ld_z, sizeof(TZ) == 4));
    const int width = 32 * (vec ? 8 : 1);
    const dim3 grid((unsigned)((N + width - 1) / width), (unsigned)q.chunks);
    return launch_dependent(vec ? slope_kernel<TG, TZ, 8> : slope_kernel<TG, TZ, 1>, grid, dim3(32 * kSlopeRows), 0, stream,
                            static_cast<const TG *>(p->grad_out), ld_g, z, ld_z, dz, q.ld_dz, sums, M, N, q.per, p->act);
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
        const Operand x = operand_x(p), w = operand_w(p);
        Epilogue e;
        e.bias = p->bias, e.residual = p->residual, e.out = p->out, e.pre = p->preact_out, e.act = p->act;
        e.ld_res = dense(p->ld_residual, N), e.ld_out = dense(p->ld_out, N), e.ld_pre = dense(p->ld_preact, N);
        e.out_f32 = p->out_dtype == FLASHBEV_F32;
        if (M <= kFewRows) {
            cudaError_t err;
            if (f32) err = e.out_f32 ? launch_rows<float, float>(x, w, M, N, K, e, stream) : launch_rows<float, bf16>(x, w, M, N, K, e, stream);
            else err = e.out_f32 ? launch_rows<bf16, float>(x, w, M, N, K, e, stream) : launch_rows<bf16, bf16>(x, w, M, N, K, e, stream);
            if (err != cudaSuccess || cudaGetLastError() != cudaSuccess) {
                cudaGetLastError();
                return FLASHBEV_CUDA_ERROR;
            }
            launches = 1;
            t_last_kernel = "linear_rows";
        } else {
            Plan q = plan_product(x, w, f32, M, N, K, true);
            if (q.partial_bytes && (!p->workspace || p->workspace_bytes < q.partial_bytes)) q = plan_product(x, w, f32, M, N, K, false);
            const flashbev_status run =
                run_product(q, x, w, f32, M, N, K, e, static_cast<float *>(p->workspace), p->error_word, stream, launches);
            if (run != FLASHBEV_OK) return run;
            t_last_kernel = q.loader == kTma ? "linear_tma" : (q.loader == kCopy ? "linear_copy" : "linear_f32");
        }
    }
    t_last_launches = launches;
    return FLASHBEV_OK;
}

size_t flashbev_linear_workspace_bytes(const flashbev_linear_params *p)
{
    if (check_linear(p) != FLASHBEV_OK || p->rows <= kFewRows) return 0;
    return plan_product(operand_x(p), operand_w(p), p->dtype == FLASHBEV_F32, (int)p->rows, p->out_features, p->in_features, true).partial_bytes;
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
    if (q.need_dz || q.need_b) {
        if (f32) err = launch_slope<float, float>(p, q, stream);
        else err = p->grad_dtype == FLASHBEV_F32 ? launch_slope<float, bf16>(p, q, stream) : launch_slope<bf16, bf16>(p, q, stream);
        ++launches;
        if (err == cudaSuccess && q.need_b) {
            const float *const sums = reinterpret_cast<const float *>(ws + q.sums_at);
            const dim3 grid((unsigned)((N + 31) / 32));
            if (f32) err = launch_dependent(column_sum_kernel<float>, grid, dim3(256), 0, stream, sums, q.chunks, N, static_cast<float *>(p->grad_bias));
            else err = launch_dependent(column_sum_kernel<bf16>, grid, dim3(256), 0, stream, sums, q.chunks, N, static_cast<bf16 *>(p->grad_bias));
            ++launches;
        }
        if (err != cudaSuccess) {
            cudaGetLastError();
            return FLASHBEV_CUDA_ERROR;
        }
    }
    float *const partial = reinterpret_cast<float *>(ws + q.partial_at);
    Epilogue e;
    e.out_f32 = f32;
    if (q.need_x) {
        const Operand w = {p->weight, dense(p->ld_weight, K), true};
        e.out = p->grad_x, e.ld_out = dense(p->ld_grad_x, K);
        const flashbev_status run = run_product(q.gx, q.dz, w, f32, M, K, N, e, partial, p->error_word, stream, launches);
        if (run != FLASHBEV_OK) return run;
    }
    if (q.need_w) {
        const Operand x = {p->x, dense(p->ld_x, K), true};
        Operand dzt = q.dz;
        dzt.mn = true;
        e.out = p->grad_weight, e.ld_out = dense(p->ld_grad_weight, K);
        const flashbev_status run = run_product(q.gw, dzt, x, f32, N, K, M, e, partial, p->error_word, stream, launches);
        if (run != FLASHBEV_OK) return run;
    }
    t_last_launches = launches;
    t_last_kernel = f32 ? "linear_backward_f32" : "linear_backward_bf16";
    return FLASHBEV_OK;
}

size_t flashbev_linear_backward_workspace_bytes(const flashbev_linear_backward_params *p)
{
    // (the scratch's own address and size do not matter here)
    return check_backward(p) == FLASHBEV_OK ? plan_backward(p).total : 0;
}

}  // extern "C"
