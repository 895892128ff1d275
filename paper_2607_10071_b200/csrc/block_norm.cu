// The norms behind and ahead of a residual block, fused with its gate, its residual scale and the sum (flashbev_block_norm of
// flashbev.h), and their gradients.
//
// All of a row is in the registers of a team of threads, eight elements each: every tensor is read once and written once, and the
// two or three statistics of a row are sums over the team (shuffles; across warps through shared memory).  The floor is memory
// traffic.  A team is the power of two of threads, from 4 to 512, that holds the row, so that narrow rows share a warp; blocks stay
// and walk over the rows with the parameters in shared memory and the gate in registers, and the next row's loads are under way, in
// registers too, while one is worked on.  What each kernel measured stands at it.
#include "flashbev.h"
#include "launch.cuh"

#include <cuda_bf16.h>
#include <math.h>
#include <string.h>

#include <algorithm>
#include <initializer_list>
#include <type_traits>

using namespace flashbev_host;

namespace {

using bf16 = __nv_bfloat16;

constexpr int kE = 8;  // elements of a row per thread

__device__ __forceinline__ float to_float(float v) { return v; }
__device__ __forceinline__ float to_float(bf16 v) { return __bfloat162float(v); }
template <typename T>
__device__ __forceinline__ T from_float(float v)
{
    if constexpr (std::is_same<T, float>::value) return v;
    else return __float2bfloat16_rn(v);
}

struct NormParams {
    const void *x, *y, *gate, *wa, *ba, *wb, *bb;
    void *h, *n;
    const void *gh, *gn;        // backward: gradients at h and n, then those at x, y and (per row) the gate
    void *gx, *gy, *ggate;
    float *sums;                // backward: [array][block][C] partial sums of the parameters' gradients
    int want;                   // which arrays: bit 0 after weight, 1 after bias, 2 before weight, 3 before bias, 4 gate
    unsigned rows, per_gate;    // per_gate: rows that share a gate
    unsigned ld_x, ld_y, ld_h, ld_n, ld_gh, ld_gn, ld_gx, ld_gy;
    int C, after, before, team; // team: threads per row
    int chunks, direct;         // backward: blocks per gate; or `direct`: a team takes whole gates
    long long gates;
    float scale, eps, inv_c;
};

// A thread's eight elements of a row, as four pairs for the two-wide instructions.  VEC 8: eight neighbours, 16-byte accesses; 2:
// every team-th pair of neighbours; 1: every team-th element.
struct Eight {
    float2 p[4];
};

template <typename T>
struct Raw {
    uint32_t w[kE * sizeof(T) / 4];
};

__device__ __forceinline__ float2 both(float v) { return make_float2(v, v); }
__device__ __forceinline__ Eight eight(float v) { return {{both(v), both(v), both(v), both(v)}}; }

// Column of element i
template <int VEC>
__device__ __forceinline__ int column(int i, int t, int team)
{
    return VEC == 8 ? t * 8 + i : (VEC == 2 ? 2 * (t + i / 2 * team) + i % 2 : t + i * team);
}

// Whether it is one of the row's
template <int VEC>
__device__ __forceinline__ bool has(int i, int t, int team, int C)
{
    return VEC == 8 ? t * 8 < C : column<VEC>(VEC == 2 ? i & ~1 : i, t, team) < C;
}

template <typename T, int VEC>
__device__ __forceinline__ void read(Raw<T> &r, const T *row, int t, int team, int C)
{
    constexpr bool kWide = sizeof(T) == 4;
    if constexpr (VEC == 8) {
        if (t * 8 < C) {
#pragma unroll
            for (int i = 0; i < (kWide ? 2 : 1); ++i) {
                const uint4 q = reinterpret_cast<const uint4 *>(row + t * 8)[i];
                r.w[4 * i] = q.x, r.w[4 * i + 1] = q.y, r.w[4 * i + 2] = q.z, r.w[4 * i + 3] = q.w;
            }
        }
    } else if constexpr (VEC == 2) {
#pragma unroll
        for (int i = 0; i < 4; ++i)
            if (has<2>(2 * i, t, team, C)) {
                if constexpr (kWide) {
                    const uint2 q = *reinterpret_cast<const uint2 *>(row + column<2>(2 * i, t, team));
                    r.w[2 * i] = q.x, r.w[2 * i + 1] = q.y;
                } else {
                    r.w[i] = *reinterpret_cast<const uint32_t *>(row + column<2>(2 * i, t, team));
                }
            }
    } else {
#pragma unroll
        for (int i = 0; i < kE; ++i)
            if (has<1>(i, t, team, C)) {
                if constexpr (kWide) r.w[i] = *reinterpret_cast<const uint32_t *>(row + column<1>(i, t, team));
                else if (i % 2) r.w[i / 2] = (r.w[i / 2] & 0xffffu) | (uint32_t)*reinterpret_cast<const unsigned short *>(row + column<1>(i, t, team)) << 16;
                else r.w[i / 2] = *reinterpret_cast<const unsigned short *>(row + column<1>(i, t, team));
            }
    }
}

// The pair 2 i, 2 i + 1
template <typename T>
__device__ __forceinline__ float2 pair_of(const Raw<T> &r, int i)
{
    if constexpr (sizeof(T) == 4) return make_float2(__uint_as_float(r.w[2 * i]), __uint_as_float(r.w[2 * i + 1]));
    else return make_float2(__uint_as_float(r.w[i] << 16), __uint_as_float(r.w[i] & 0xffff0000u));
}

__device__ __forceinline__ uint32_t pack(float2 v)  // two bf16
{
    const __nv_bfloat162 b = __floats2bfloat162_rn(v.x, v.y);
    uint32_t r;
    memcpy(&r, &b, 4);
    return r;
}

template <typename T, int VEC>
__device__ __forceinline__ void write(T *row, const Eight &f, int t, int team, int C)
{
    constexpr bool kWide = sizeof(T) == 4;
    if constexpr (VEC == 8) {
        if (t * 8 >= C) return;
        uint4 *const to = reinterpret_cast<uint4 *>(row + t * 8);
        if constexpr (kWide) {
            to[0] = make_uint4(__float_as_uint(f.p[0].x), __float_as_uint(f.p[0].y), __float_as_uint(f.p[1].x), __float_as_uint(f.p[1].y));
            to[1] = make_uint4(__float_as_uint(f.p[2].x), __float_as_uint(f.p[2].y), __float_as_uint(f.p[3].x), __float_as_uint(f.p[3].y));
        } else {
            to[0] = make_uint4(pack(f.p[0]), pack(f.p[1]), pack(f.p[2]), pack(f.p[3]));
        }
    } else if constexpr (VEC == 2) {
#pragma unroll
        for (int i = 0; i < 4; ++i)
            if (has<2>(2 * i, t, team, C)) {
                if constexpr (kWide) *reinterpret_cast<float2 *>(row + column<2>(2 * i, t, team)) = f.p[i];
                else *reinterpret_cast<uint32_t *>(row + column<2>(2 * i, t, team)) = pack(f.p[i]);
            }
    } else {
#pragma unroll
        for (int i = 0; i < kE; ++i)
            if (has<1>(i, t, team, C)) row[column<1>(i, t, team)] = from_float<T>(i % 2 ? f.p[i / 2].y : f.p[i / 2].x);
    }
}

// To float; with VEC 2 and 1 elements behind the row's end are 0 (with 8 a thread has all of its elements or none, and its sums are masked)
template <typename T, int VEC>
__device__ __forceinline__ void widen(Eight &f, const Raw<T> &r, int t, int team, int C)
{
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        f.p[i] = pair_of<T>(r, i);
        if (VEC != 8 && !has<VEC>(2 * i, t, team, C)) f.p[i].x = 0.0f;
        if (VEC != 8 && !has<VEC>(2 * i + 1, t, team, C)) f.p[i].y = 0.0f;
    }
}

__device__ __forceinline__ Eight operator+(const Eight &a, const Eight &b)
{
    Eight r;
#pragma unroll
    for (int i = 0; i < 4; ++i) r.p[i] = __fadd2_rn(a.p[i], b.p[i]);
    return r;
}

__device__ __forceinline__ Eight operator*(const Eight &a, const Eight &b)
{
    Eight r;
#pragma unroll
    for (int i = 0; i < 4; ++i) r.p[i] = __fmul2_rn(a.p[i], b.p[i]);
    return r;
}

__device__ __forceinline__ Eight fma(const Eight &a, const Eight &b, const Eight &c)
{
    Eight r;
#pragma unroll
    for (int i = 0; i < 4; ++i) r.p[i] = __ffma2_rn(a.p[i], b.p[i], c.p[i]);
    return r;
}

__device__ __forceinline__ float total(const Eight &a)
{
    const float2 s = __fadd2_rn(__fadd2_rn(a.p[0], a.p[1]), __fadd2_rn(a.p[2], a.p[3]));
    return s.x + s.y;
}

// The norms' parameters lie in shared memory as floats, `count` vectors one after another, 1 or 0 where there is none: in registers
// they would be 32 of a thread, and of the gradients' kernel 72 with their sums.
// (VEC 8: the first four of every eight, then the others, so that neighbouring threads read neighbouring 16 bytes)
template <int VEC>
__device__ __forceinline__ int param_at(int c, int C)
{
    return VEC == 8 ? (c / 4 % 2) * (C / 2) + c / 8 * 4 + c % 4 : c;
}

template <typename P, int VEC>
__device__ __forceinline__ void stage_params(float *to, const void *const (&from)[4], int count, int C)
{
    for (int j = 0; j < count; ++j)
        for (int c = threadIdx.x; c < C; c += blockDim.x)
            to[j * C + param_at<VEC>(c, C)] = from[j] ? to_float(static_cast<const P *>(from[j])[c]) : (j % 2 ? 0.0f : 1.0f);
    __syncthreads();
}

template <int VEC>
__device__ __forceinline__ Eight read_param(const float *p, int t, int team, int C)
{
    Eight r;
    if constexpr (VEC == 8) {
        const float *const q = p + (t * 8 < C ? t * 4 : 0);
        const float4 a = *reinterpret_cast<const float4 *>(q), b = *reinterpret_cast<const float4 *>(q + C / 2);
        r.p[0] = make_float2(a.x, a.y), r.p[1] = make_float2(a.z, a.w), r.p[2] = make_float2(b.x, b.y), r.p[3] = make_float2(b.z, b.w);
    } else {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            if constexpr (VEC == 2)  // (C is even, and with it every vector's start)
                r.p[i] = *reinterpret_cast<const float2 *>(p + (has<2>(2 * i, t, team, C) ? column<2>(2 * i, t, team) : 0));
            else
                r.p[i] = make_float2(p[has<1>(2 * i, t, team, C) ? column<1>(2 * i, t, team) : 0],
                                     p[has<1>(2 * i + 1, t, team, C) ? column<1>(2 * i + 1, t, team) : 0]);
        }
    }
    return r;
}

// The gate of row `g` of them, times the scale
template <typename P, int VEC>
__device__ __forceinline__ Eight read_gate(const void *gate, long long g, float scale, int t, int team, int C)
{
    if (!gate) return eight(scale);
    Raw<P> r;
    read<P, VEC>(r, static_cast<const P *>(gate) + g * C, t, team, C);
    Eight f;
    widen<P, VEC>(f, r, t, team, C);
    return f * eight(scale);
}

// Sums over a team.  WIDE: teams of several warps.
template <bool WIDE>
struct Team {
    int threads, t, slot;       // threads of a team; this one's place in it; the team's place in the block
    bool mine;                  // VEC 8: this thread has a part of the row
    float2 *shared;             // WIDE: [2][32] of this team
    int turn;

    __device__ __forceinline__ float2 sum(float a, float b)
    {
        const int most = WIDE ? 16 : threads / 2;
        if (!mine) a = b = 0.0f;
#pragma unroll
        for (int d = 16; d; d /= 2)
            if (d <= most) a += __shfl_xor_sync(0xffffffffu, a, d), b += __shfl_xor_sync(0xffffffffu, b, d);
        if constexpr (WIDE) {
            // (two buffers in turn: who writes the one again has passed the barrier of the other, after everybody read the one)
            float2 *const buf = shared + 32 * turn;
            turn ^= 1;
            const int warps = threads / 32;
            if (t % 32 == 0) buf[t / 32] = make_float2(a, b);
            asm volatile("bar.sync %0, %1;" ::"r"(1 + slot), "r"(threads) : "memory");
            if (warps <= 4) {  // (every thread adds them up: fewer instructions than a tree)
                const float4 u = *reinterpret_cast<const float4 *>(buf);
                a = u.x + u.z, b = u.y + u.w;
                if (warps == 4) {
                    const float4 w = *reinterpret_cast<const float4 *>(buf + 2);
                    a += w.x + w.z, b += w.y + w.w;
                }
                return make_float2(a, b);
            }
            const float2 v = t % 16 < warps ? buf[t % 16] : make_float2(0.0f, 0.0f);  // (both halves of a warp alike)
            a = v.x, b = v.y;
#pragma unroll
            for (int d = 8; d; d /= 2) a += __shfl_xor_sync(0xffffffffu, a, d), b += __shfl_xor_sync(0xffffffffu, b, d);
        }
        return make_float2(a, b);
    }
    __device__ __forceinline__ float sum(float a)
    {
        const int most = WIDE ? 16 : threads / 2;
        if (!mine) a = 0.0f;
#pragma unroll
        for (int d = 16; d; d /= 2)
            if (d <= most) a += __shfl_xor_sync(0xffffffffu, a, d);
        if constexpr (WIDE) {
            float2 *const buf = shared + 32 * turn;
            turn ^= 1;
            if (t % 32 == 0) buf[t / 32].x = a;
            asm volatile("bar.sync %0, %1;" ::"r"(1 + slot), "r"(threads) : "memory");
            if (threads <= 128) {
                a = buf[0].x + buf[1].x;
                if (threads == 128) a += buf[2].x + buf[3].x;
                return a;
            }
            a = t % 16 < threads / 32 ? buf[t % 16].x : 0.0f;
#pragma unroll
            for (int d = 8; d; d /= 2) a += __shfl_xor_sync(0xffffffffu, a, d);
        }
        return a;
    }
};

// Elements behind the row's end, of VEC 2 and 1, back to 0
template <int VEC, bool WIDE>
__device__ __forceinline__ void trim(Eight &v, const Team<WIDE> &team, int C)
{
    if constexpr (VEC != 8) {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            if (!has<VEC>(2 * i, team.t, team.threads, C)) v.p[i].x = 0.0f;
            if (!has<VEC>(2 * i + 1, team.t, team.threads, C)) v.p[i].y = 0.0f;
        }
    }
}

// v becomes (v - mean) / deviation (or v / root mean square); returns 1 / deviation.
template <int VEC, bool WIDE>
__device__ __forceinline__ float whiten(Eight &v, int kind, const NormParams &p, Team<WIDE> &team)
{
    if (kind == FLASHBEV_NORM_LAYER) {
        v = v + eight(-team.sum(total(v)) * p.inv_c);
        trim<VEC>(v, team, p.C);
    }
    const float r = rsqrtf(fmaf(team.sum(total(v * v)), p.inv_c, p.eps));
    v = v * eight(r);
    return r;
}

// Gradient at the input of `whiten` from that at its result t: r (g - mean(g) - t mean(g t)), without mean(g) for root mean squares.
template <int VEC, bool WIDE>
__device__ __forceinline__ void whiten_back(Eight &g, const Eight &t, float r, int kind, const NormParams &p, Team<WIDE> &team)
{
    if (kind == FLASHBEV_NORM_LAYER) {
        const float2 s = team.sum(total(g), total(g * t));
        g = fma(t, eight(-s.y * p.inv_c), g + eight(-s.x * p.inv_c));
        trim<VEC>(g, team, p.C);
    } else {
        g = fma(t, eight(-team.sum(total(g * t)) * p.inv_c), g);
    }
    g = g * eight(r);
}

template <int VEC, bool WIDE>
__device__ __forceinline__ Team<WIDE> make_team(const NormParams &p, float2 *shared)
{
    Team<WIDE> team;
    team.threads = p.team, team.slot = threadIdx.x / p.team, team.t = threadIdx.x % p.team, team.turn = 0;
    team.mine = VEC != 8 || team.t * 8 < p.C;
    team.shared = shared + (WIDE ? 64 * team.slot : 0);
    return team;
}

constexpr int kMostThreads = FLASHBEV_NORM_MAX_CHANNELS / kE;
static_assert(kMostThreads <= 512, "the sums of a team's warps are added up by half a warp");

// Row `row` of a matrix (one 32 x 32 -> 64 bit product)
template <typename T>
__device__ __forceinline__ T *row_of(const void *base, unsigned row, unsigned ld)
{
    return const_cast<T *>(static_cast<const T *>(base)) + (unsigned long long)row * ld;
}

// S, T, P: types of x and h, of y and n, of the parameters.
//
// Measured, 256 columns: 40000 bf16 rows, a norm ahead only, 18 us (4.4 TB/s); with x and h in float32 23 us (5.5 TB/s); 184950 bf16
// rows 68 us (5.6 TB/s); 80000 bf16 rows, two norms and a gate, 33 us (4.9 TB/s, 59 % of the issue slots).  Bound by traffic and, close
// behind, by the instructions of the conversions and shuffles: two-wide arithmetic (Eight) made the last 45 -> 34 us.  Rows of more than
// 2048 columns have one block of 512 threads to an SM (20000 x 4096, bf16, sum and norm: 156 us, 4.2 TB/s).  Rows of an odd C, element by
// element, take twice as long as those of an even one (40000 x 255: 25 us).  A ring of asynchronous copies in place of the prefetch in registers was slower.
template <typename S, typename T, typename P, int VEC, bool WIDE>
__global__ void __launch_bounds__(WIDE ? kMostThreads : 256, WIDE ? 1 : 3) norm_kernel(const __grid_constant__ NormParams p)
{
    __shared__ __align__(16) float2 shared[WIDE ? 64 * 4 : 1];  // (at most four teams of 64 threads in a block)
    asm volatile("griddepcontrol.wait;" ::: "memory");
    asm volatile("griddepcontrol.launch_dependents;");
    Team<WIDE> team = make_team<VEC, WIDE>(p, shared);
    const int t = team.t, threads = p.team, C = p.C, teams = blockDim.x / threads;
    extern __shared__ __align__(16) float params[];  // before weight, before bias, after weight, after bias
    stage_params<P, VEC>(params, {p.wb, p.bb, p.wa, p.ba}, p.after != FLASHBEV_NORM_NONE ? 4 : 2, C);
    // (rows are below 2^31, and so is a step: none of the sums wraps)
    const unsigned step = gridDim.x * teams, first = blockIdx.x * teams + team.slot;
    // (narrow teams share a warp's shuffles: all of them go as long as one has a row)
    const unsigned lead = WIDE ? first : first - (threadIdx.x % 32) / threads;
    Raw<S> xr;
    Raw<T> yr;
    const auto bring = [&](unsigned row) {
        if (row >= p.rows) return;
        read<S, VEC>(xr, row_of<const S>(p.x, row, p.ld_x), t, threads, C);
        if (p.y) read<T, VEC>(yr, row_of<const T>(p.y, row, p.ld_y), t, threads, C);
    };
    bring(first);
    Eight gate = eight(p.scale);
    unsigned gate_end = 0;  // the row behind the last one with this gate
    for (unsigned row = first, at = lead; at < p.rows; row += step, at += step) {
        const bool live = row < p.rows;
        Eight h, m;
        widen<S, VEC>(h, xr, t, threads, C);
        if (p.y) widen<T, VEC>(m, yr, t, threads, C);
        bring(row + step);
        if (p.y) {
            if (p.after != FLASHBEV_NORM_NONE) {
                whiten<VEC, WIDE>(m, p.after, p, team);
                m = fma(m, read_param<VEC>(params + 2 * C, t, threads, C), read_param<VEC>(params + 3 * C, t, threads, C));
            }
            if (p.gate && live && row >= gate_end) {
                const unsigned g = row / p.per_gate;
                gate = read_gate<P, VEC>(p.gate, g, p.scale, t, threads, C);
                gate_end = (g + 1) * p.per_gate;
            }
            h = fma(m, gate, h);
            if (p.h && live) write<S, VEC>(row_of<S>(p.h, row, p.ld_h), h, t, threads, C);
        }
        if (p.before != FLASHBEV_NORM_NONE) {
            trim<VEC>(h, team, C);  // (of the norm's bias)
            whiten<VEC, WIDE>(h, p.before, p, team);
            h = fma(h, read_param<VEC>(params, t, threads, C), read_param<VEC>(params + C, t, threads, C));
            if (live) write<T, VEC>(row_of<T>(p.n, row, p.ld_n), h, t, threads, C);
        }
    }
}

// Gradients.  The rows of a gate are shared by `chunks` blocks, whose teams take every so manieth row; sums over rows stay in
// registers until the block's end, when they are added up over its teams in a fixed order.  `direct`: there are many gates with few
// rows, and a team takes the rows of one gate after another and writes the gate's gradient itself.
//
// Measured, 256 columns: 40000 bf16 rows, a norm ahead only, 37 us (3.3 TB/s); 184950 of them 119 us (4.7 TB/s); 80000 with two norms
// and a gate 71 us (3.4 TB/s, 50 % of the issue slots); 14927 x 936, float32 stream, two norms: 113 us (1.7 TB/s); 20000 x 4096, bf16, a norm
// ahead: 290 us (3.4 TB/s).  Bound by latency: five sums over rows beside this row and the next do not fit the 128 registers that leave 16
// warps on an SM (16 to 280 bytes of them are spilled); in wide rows by the barriers too.
template <typename S, typename T, typename P, int VEC, bool WIDE>
__global__ void __launch_bounds__(WIDE ? kMostThreads : 256, WIDE ? 1 : 2) norm_backward_kernel(const __grid_constant__ NormParams p)
{
    __shared__ __align__(16) float2 shared[WIDE ? 64 * 4 : 1];
    __shared__ float joined[2048];  // [teams (warps, where a warp has several)][C]
    asm volatile("griddepcontrol.wait;" ::: "memory");
    asm volatile("griddepcontrol.launch_dependents;");
    Team<WIDE> team = make_team<VEC, WIDE>(p, shared);
    const int t = team.t, threads = p.team, C = p.C, teams = blockDim.x / threads;
    extern __shared__ __align__(16) float params[];  // before weight, after bias, after weight
    const int vectors = p.after != FLASHBEV_NORM_NONE ? 3 : 1;
    stage_params<P, VEC>(params, {p.wb, p.ba, p.wa, nullptr}, vectors, C);
    Eight dwa = eight(0.0f), dba = dwa, dwb = dwa, dbb = dwa, dg = dwa;

    const int inside = WIDE ? 0 : (threadIdx.x % 32) / threads;  // place of the team in its warp
    long long g, g_step, g_lead;
    if (p.direct) {
        g = (long long)blockIdx.x * teams + team.slot, g_step = (long long)gridDim.x * teams;
        g_lead = g - inside;
    } else {
        g = g_lead = blockIdx.x / p.chunks, g_step = p.gates;
    }
    for (; g_lead < p.gates; g += g_step, g_lead += g_step) {
        unsigned row, end, step;
        const bool mine = g < p.gates;
        if (p.direct) {
            row = (unsigned)(g * p.per_gate), end = mine ? row + p.per_gate : 0, step = 1;
        } else {
            const int chunk = (int)(blockIdx.x - g * p.chunks);
            const unsigned base = (unsigned)(g * p.per_gate), share = (p.per_gate + p.chunks - 1) / p.chunks;
            end = base + min(p.per_gate, (chunk + 1) * share);
            row = base + chunk * share + team.slot, step = teams;
        }
        // every team of a warp goes around as often
        const unsigned warp_row = row - inside, rounds = p.direct ? p.per_gate : (warp_row < end ? (end - warp_row + step - 1) / step : 0);
        const Eight gate = read_gate<P, VEC>(p.gate, mine ? g : 0, p.scale, t, threads, C);
        Raw<S> xr, ghr;
        Raw<T> yr, gnr;
        const auto bring = [&](unsigned at) {
            if (at >= end) return;
            read<S, VEC>(xr, row_of<const S>(p.x, at, p.ld_x), t, threads, C);
            if (p.y) read<T, VEC>(yr, row_of<const T>(p.y, at, p.ld_y), t, threads, C);
            if (p.gn) read<T, VEC>(gnr, row_of<const T>(p.gn, at, p.ld_gn), t, threads, C);
            if (p.gh) read<S, VEC>(ghr, row_of<const S>(p.gh, at, p.ld_gh), t, threads, C);
        };
        bring(row);
        for (unsigned round = 0; round < rounds; ++round, row += step) {
            const bool live = row < end;
            Eight u, v, gn, gh = eight(0.0f);
            widen<S, VEC>(u, xr, t, threads, C);
            if (p.y) widen<T, VEC>(v, yr, t, threads, C);
            if (p.gn) widen<T, VEC>(gn, gnr, t, threads, C);
            if (p.gh) widen<S, VEC>(gh, ghr, t, threads, C);
            bring(row + step);
            // after(y), of which v keeps the part without the parameters
            const auto branch = [&]() -> Eight {
                if (p.after == FLASHBEV_NORM_NONE) return v;
                return fma(v, read_param<VEC>(params + 2 * C, t, threads, C), read_param<VEC>(params + C, t, threads, C));
            };
            float ra = 0.0f;
            if (p.after != FLASHBEV_NORM_NONE) ra = whiten<VEC, WIDE>(v, p.after, p, team);
            if (p.before != FLASHBEV_NORM_NONE) {
                if (p.y) {
                    u = fma(branch(), gate, u);
                    trim<VEC>(u, team, C);
                }
                if constexpr (WIDE) {
                    // The sums over warps cost most: those of the statistics and of the gradient go together.  g (u - mean) gives g
                    // t once the deviation is known, so that two sums over the team are enough, one for root mean squares, instead
                    // of three and two (20000 x 512: 43 us instead of 47; narrow teams would be slower, 41 us instead of 33 at
                    // 36743 x 82, by the instructions).
                    float mean_g = 0.0f;
                    if (p.before == FLASHBEV_NORM_LAYER) {
                        const float2 s = team.sum(total(u), total(gn * read_param<VEC>(params, t, threads, C)));
                        u = u + eight(-s.x * p.inv_c), mean_g = s.y * p.inv_c;
                        trim<VEC>(u, team, C);
                    }
                    const float2 s = team.sum(total(u * u), total(gn * read_param<VEC>(params, t, threads, C) * u));
                    const float rb = rsqrtf(fmaf(s.x, p.inv_c, p.eps));
                    u = u * eight(rb);
                    if (live) dwb = fma(gn, u, dwb), dbb = dbb + gn;
                    gn = fma(u, eight(-s.y * rb * p.inv_c), gn * read_param<VEC>(params, t, threads, C));
                    if (p.before == FLASHBEV_NORM_LAYER) {
                        gn = gn + eight(-mean_g);
                        trim<VEC>(gn, team, C);
                    }
                    gh = fma(gn, eight(rb), gh);
                } else {
                    const float rb = whiten<VEC, WIDE>(u, p.before, p, team);
                    if (live) dwb = fma(gn, u, dwb), dbb = dbb + gn;
                    gn = gn * read_param<VEC>(params, t, threads, C);
                    whiten_back<VEC, WIDE>(gn, u, rb, p.before, p, team);
                    gh = gh + gn;
                }
            }
            if (p.gx && live) write<S, VEC>(row_of<S>(p.gx, row, p.ld_gx), gh, t, threads, C);
            if (!p.y) continue;
            if (live && p.ggate) dg = fma(gh * eight(p.scale), branch(), dg);
            gh = gh * gate;
            if (p.after != FLASHBEV_NORM_NONE) {
                if (live) dwa = fma(gh, v, dwa), dba = dba + gh;
                gh = gh * read_param<VEC>(params + 2 * C, t, threads, C);
                whiten_back<VEC, WIDE>(gh, v, ra, p.after, p, team);
            }
            if (p.gy && live) write<T, VEC>(row_of<T>(p.gy, row, p.ld_gy), gh, t, threads, C);
        }
        if (p.direct) {
            if (p.ggate && mine) write<P, VEC>(static_cast<P *>(p.ggate) + g * C, dg, t, threads, C);
            dg = eight(0.0f);
        }
    }
    // sums over the block's teams, one array after another
    long long array = 0;
    const int slots = WIDE ? teams : blockDim.x / 32, slot = WIDE ? team.slot : threadIdx.x / 32;
    const auto put = [&](Eight &d, int bit) {
        if (!(p.want >> bit & 1)) return;
        float *const out = p.sums + (array++ * gridDim.x + blockIdx.x) * (long long)C;
        if (!WIDE) {
#pragma unroll
            for (int s = 16; s; s /= 2)
                if (s >= threads)
#pragma unroll
                    for (int i = 0; i < 4; ++i)
                        d.p[i].x += __shfl_xor_sync(0xffffffffu, d.p[i].x, s), d.p[i].y += __shfl_xor_sync(0xffffffffu, d.p[i].y, s);
        }
        const auto scatter = [&](float *to) {  // (any alignment)
#pragma unroll
            for (int i = 0; i < kE; ++i)
                if (has<VEC>(i, t, threads, C)) to[column<VEC>(i, t, threads)] = i % 2 ? d.p[i / 2].y : d.p[i / 2].x;
        };
        if (slots == 1) {
            scatter(out);
            return;
        }
        __syncthreads();  // (the array before has been read)
        if (WIDE || inside == 0) scatter(joined + slot * C);
        __syncthreads();
        for (int c = threadIdx.x; c < C; c += blockDim.x) {
            float s = 0.0f;
            for (int w = 0; w < slots; ++w) s += joined[w * C + c];
            out[c] = s;
        }
    };
    put(dwa, 0), put(dba, 1), put(dwb, 2), put(dbb, 3), put(dg, 4);
}

struct SumJobs {
    void *out[5];
    int first[6];               // blocks of job j: first[j] .. first[j + 1], 32 columns of one output row each
    int blocks, per, C;         // partial rows of an array; those of one output row of the gate (job 4 sums every `per` of them)
};

// Adds the blocks' sums up in a fixed order: 16 warps take every sixteenth.  Bound by latency, 3 to 4 us for the sums of 296 blocks.
template <typename P>
__global__ void __launch_bounds__(512) norm_sum_kernel(const float *__restrict__ sums, const __grid_constant__ SumJobs q)
{
    asm volatile("griddepcontrol.wait;" ::: "memory");
    asm volatile("griddepcontrol.launch_dependents;");
    __shared__ float part[16][33];
    int j = 0, array = 0;
    while (j < 4 && (int)blockIdx.x >= q.first[j + 1]) array += q.first[j + 1] > q.first[j], ++j;
    const int across = (q.C + 31) / 32, b = blockIdx.x - q.first[j], line = b / across, warp = threadIdx.x / 32, lane = threadIdx.x % 32;
    const int col = (b - line * across) * 32 + lane, rows = j == 4 ? q.per : q.blocks;
    const float *const src = sums + ((long long)array * q.blocks + (long long)line * rows) * q.C;
    float v = 0.0f;
    if (col < q.C)
#pragma unroll 8
        for (int r = warp; r < rows; r += 16) v += src[(long long)r * q.C + col];
    part[warp][lane] = v;
    __syncthreads();
    if (warp == 0 && col < q.C) {
        v = 0.0f;
#pragma unroll
        for (int w = 0; w < 16; ++w) v += part[w][lane];
        static_cast<P *>(q.out[j])[(long long)line * q.C + col] = from_float<P>(v);
    }
}

// ---- host -------------------------------------------------------------------------------------------------------------------

bool dtype_ok(int d) { return d == FLASHBEV_F32 || d == FLASHBEV_BF16; }
size_t elem_size(int d) { return d == FLASHBEV_F32 ? 4 : 2; }
bool aligned(const void *p, int dtype) { return (uintptr_t)p % elem_size(dtype) == 0; }
unsigned dense(long long ld, int C) { return ld ? (unsigned)ld : (unsigned)C; }  // (below 2^31: check_common)

int team_threads(int C)
{
    int team = 4;
    while (team * kE < C) team *= 2;
    return team;
}

// What the forward and the backward call have in common.
template <typename Q>
flashbev_status check_common(const Q *p, std::initializer_list<int64_t> strides)
{
    if (p->rows < 0 || p->C <= 0) return FLASHBEV_INVALID_ARG;
    if (p->after < 0 || p->after > FLASHBEV_NORM_RMS || p->before < 0 || p->before > FLASHBEV_NORM_RMS) return FLASHBEV_INVALID_ARG;
    if (!dtype_ok(p->dtype) || !dtype_ok(p->branch_dtype) || !dtype_ok(p->param_dtype)) return FLASHBEV_INVALID_ARG;
    if (!isfinite(p->scale) || !isfinite(p->eps) || p->eps < 0.0) return FLASHBEV_INVALID_ARG;
    for (long long ld : strides)
        if (ld != 0 && ld < p->C) return FLASHBEV_INVALID_ARG;
    if (p->gate && (p->gate_groups <= 0 || p->rows % p->gate_groups || (!p->y && p->rows))) return FLASHBEV_INVALID_ARG;
    if (!p->y && p->after != FLASHBEV_NORM_NONE && p->rows) return FLASHBEV_INVALID_ARG;
    if (p->after == FLASHBEV_NORM_NONE && (p->after_weight || p->after_bias)) return FLASHBEV_INVALID_ARG;
    if (p->before == FLASHBEV_NORM_NONE && p->before_weight) return FLASHBEV_INVALID_ARG;
    if (p->dtype == FLASHBEV_BF16 && p->branch_dtype == FLASHBEV_F32) return FLASHBEV_UNSUPPORTED;
    if (p->param_dtype == FLASHBEV_BF16 && p->branch_dtype == FLASHBEV_F32) return FLASHBEV_UNSUPPORTED;
    if (p->C > FLASHBEV_NORM_MAX_CHANNELS || p->rows > 2147483647LL) return FLASHBEV_UNSUPPORTED;
    for (long long ld : strides)
        if (ld > 2147483647LL) return FLASHBEV_UNSUPPORTED;
    const void *const params[] = {p->gate, p->after_weight, p->after_bias, p->before_weight};
    for (const void *v : params)
        if (!aligned(v, p->param_dtype)) return FLASHBEV_MISALIGNED;
    if (!aligned(p->x, p->dtype) || !aligned(p->y, p->branch_dtype)) return FLASHBEV_MISALIGNED;
    return FLASHBEV_OK;
}

flashbev_status check_norm(const flashbev_block_norm_params *p)
{
    if (!p || p->struct_size < sizeof(*p)) return FLASHBEV_INVALID_ARG;
    const flashbev_status st = check_common(p, {p->ld_x, p->ld_y, p->ld_h, p->ld_n});
    if (st != FLASHBEV_OK) return st;
    if (p->before == FLASHBEV_NORM_NONE && p->before_bias) return FLASHBEV_INVALID_ARG;
    if (p->rows) {
        if (!p->x || (p->n != nullptr) != (p->before != FLASHBEV_NORM_NONE)) return FLASHBEV_INVALID_ARG;
        if ((p->h && !p->y) || (!p->h && !p->n)) return FLASHBEV_INVALID_ARG;
    }
    if (!aligned(p->before_bias, p->param_dtype) || !aligned(p->h, p->dtype) || !aligned(p->n, p->branch_dtype)) return FLASHBEV_MISALIGNED;
    return FLASHBEV_OK;
}

flashbev_status check_backward(const flashbev_block_norm_backward_params *p)
{
    if (!p || p->struct_size < sizeof(*p)) return FLASHBEV_INVALID_ARG;
    const flashbev_status st = check_common(p, {p->ld_grad_h, p->ld_grad_n, p->ld_x, p->ld_y, p->ld_grad_x, p->ld_grad_y});
    if (st != FLASHBEV_OK) return st;
    if (p->rows) {
        if (!p->x || (p->grad_n != nullptr) != (p->before != FLASHBEV_NORM_NONE)) return FLASHBEV_INVALID_ARG;
        if ((p->grad_y && !p->y) || (!p->grad_h && !p->grad_n)) return FLASHBEV_INVALID_ARG;
    }
    if (p->grad_gate && !p->gate) return FLASHBEV_INVALID_ARG;
    if ((p->grad_after_weight || p->grad_after_bias) && p->after == FLASHBEV_NORM_NONE) return FLASHBEV_INVALID_ARG;
    if ((p->grad_before_weight || p->grad_before_bias) && p->before == FLASHBEV_NORM_NONE) return FLASHBEV_INVALID_ARG;
    const void *const outs[] = {p->grad_gate, p->grad_after_weight, p->grad_after_bias, p->grad_before_weight, p->grad_before_bias};
    for (const void *v : outs)
        if (!aligned(v, p->param_dtype)) return FLASHBEV_MISALIGNED;
    if (!aligned(p->grad_h, p->dtype) || !aligned(p->grad_x, p->dtype) || !aligned(p->grad_n, p->branch_dtype) || !aligned(p->grad_y, p->branch_dtype) ||
        (uintptr_t)p->workspace % 16)
        return FLASHBEV_MISALIGNED;
    return FLASHBEV_OK;
}

// The instance for the call's types, alignment and width.
template <bool BACKWARD, typename S, typename T, typename P, int VEC>
auto pick(bool wide)
{
    if constexpr (BACKWARD) return wide ? norm_backward_kernel<S, T, P, VEC, true> : norm_backward_kernel<S, T, P, VEC, false>;
    else return wide ? norm_kernel<S, T, P, VEC, true> : norm_kernel<S, T, P, VEC, false>;
}

template <bool BACKWARD, typename S, typename T, typename P>
auto pick(int vec, bool wide)
{
    return vec == 8 ? pick<BACKWARD, S, T, P, 8>(wide) : (vec == 2 ? pick<BACKWARD, S, T, P, 2>(wide) : pick<BACKWARD, S, T, P, 1>(wide));
}

template <bool BACKWARD>
cudaError_t launch_norm(const NormParams &k, int dtype, int branch, int param, int vec, unsigned blocks, int threads, cudaStream_t stream)
{
    const bool wide = k.team > 32;
    void (*kernel)(NormParams);
    if (dtype == FLASHBEV_F32 && branch == FLASHBEV_F32) kernel = pick<BACKWARD, float, float, float>(vec, wide);
    else if (dtype == FLASHBEV_F32 && param == FLASHBEV_F32) kernel = pick<BACKWARD, float, bf16, float>(vec, wide);
    else if (dtype == FLASHBEV_F32) kernel = pick<BACKWARD, float, bf16, bf16>(vec, wide);
    else if (param == FLASHBEV_F32) kernel = pick<BACKWARD, bf16, bf16, float>(vec, wide);
    else kernel = pick<BACKWARD, bf16, bf16, bf16>(vec, wide);
    const size_t vectors = BACKWARD ? (k.after != FLASHBEV_NORM_NONE ? 3 : 1) : (k.after != FLASHBEV_NORM_NONE ? 4 : 2);
    const size_t smem = vectors * k.C * sizeof(float);
    if (smem > 36 * 1024) {  // (beside up to 10 KB that the kernels declare themselves)
        const cudaError_t e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem);
        if (e != cudaSuccess) return e;
    }
    return launch_dependent(kernel, dim3(blocks), dim3((unsigned)threads), smem, stream, k);
}

// Elements that a thread can take at once: 8 or 2 neighbours where every row starts on their boundary, else one.
struct Alignment {
    int vec;
    explicit Alignment(int C) : vec(C % 8 == 0 ? 8 : (C % 2 == 0 ? 2 : 1)) {}
    void rows(const void *p, long long ld, int dtype)
    {
        if (!p) return;
        const uintptr_t bits = (uintptr_t)p | (uintptr_t)(ld * (long long)elem_size(dtype));
        if (vec == 8 && bits % 16) vec = 2;
        if (vec == 2 && bits % (2 * elem_size(dtype))) vec = 1;
    }
};

// Blocks and rows of a backward call.
struct BackwardShape {
    int team, threads, teams, arrays, want;
    long long gates;            // gates whose rows are kept apart (1 without a gate)
    int chunks;
    bool direct;
    long long blocks;
    size_t bytes;
};

BackwardShape backward_shape(const flashbev_block_norm_backward_params *p)
{
    BackwardShape s = {};
    s.team = team_threads(p->C), s.threads = std::max(256, s.team), s.teams = s.threads / s.team;
    s.gates = p->gate ? p->gate_groups : 1;
    const long long per = p->rows / s.gates;
    const long long resident = s.threads >= 512 ? sm_count() : 2LL * sm_count();
    // More gates than teams: a team sums a gate's rows by itself.  More than blocks: whichever takes fewer rows' time, the team, all of the
    // gate's rows one after another, or rounds of blocks, each the rows of a team and three rows' time to begin and end with.  (float32
    // stream, a norm on either side, us by teams and by blocks: 18000 gates of 5 rows of 32: 22 and 420, 3000 of 20: 40 and 77, 1000 of 64: 105
    // and 34; 600 gates of 20 rows of 256: 47 and 48, 2360 of 64: 185 and 269; in 51 such cases the choice is 15 % off at most.)
    s.direct = p->gate && s.gates >= resident &&
               (s.gates >= resident * s.teams || per < (s.gates + resident - 1) / resident * (3 + (per + s.teams - 1) / s.teams));
    const void *const outs[5] = {p->grad_after_weight, p->grad_after_bias, p->grad_before_weight, p->grad_before_bias, p->grad_gate};
    for (int i = 0; i < 5; ++i)
        if (outs[i] && !(i == 4 && s.direct)) s.want |= 1 << i, ++s.arrays;
    if (s.direct) {
        s.chunks = 1;
        s.blocks = std::min(resident, (s.gates + s.teams - 1) / s.teams);
    } else {
        s.chunks = (int)std::max(1LL, std::min(resident / s.gates, (per + s.teams - 1) / s.teams));
        s.blocks = s.gates * s.chunks;
    }
    s.bytes = (size_t)s.arrays * (size_t)s.blocks * (size_t)p->C * sizeof(float);
    return s;
}

}  // namespace

extern "C" {

flashbev_status flashbev_block_norm(const flashbev_block_norm_params *p, void *stream)
{
    const flashbev_status st = check_norm(p);
    if (st != FLASHBEV_OK) return st;
    if (!p->rows) {
        t_last_launches = 0;
        return FLASHBEV_OK;
    }
    NormParams k = {};
    k.x = p->x, k.y = p->y, k.gate = p->gate, k.wa = p->after_weight, k.ba = p->after_bias, k.wb = p->before_weight, k.bb = p->before_bias;
    k.h = p->h, k.n = p->n, k.rows = (unsigned)p->rows, k.per_gate = (unsigned)(p->gate ? p->rows / p->gate_groups : p->rows);
    k.ld_x = dense(p->ld_x, p->C), k.ld_y = dense(p->ld_y, p->C), k.ld_h = dense(p->ld_h, p->C), k.ld_n = dense(p->ld_n, p->C);
    k.C = p->C, k.after = p->after, k.before = p->before, k.scale = (float)p->scale, k.eps = (float)p->eps, k.inv_c = 1.0f / (float)p->C;
    k.team = team_threads(p->C);
    Alignment al(p->C);
    al.rows(p->x, k.ld_x, p->dtype), al.rows(p->h, k.ld_h, p->dtype), al.rows(p->y, k.ld_y, p->branch_dtype), al.rows(p->n, k.ld_n, p->branch_dtype);
    al.rows(p->gate, p->C, p->param_dtype);
    const int threads = std::max(256, k.team), teams = threads / k.team;
    const long long blocks = std::min<long long>((p->rows + teams - 1) / teams, (long long)sm_count() * (threads >= 512 ? 2 : 6));
    const cudaError_t e = launch_norm<false>(k, p->dtype, p->branch_dtype, p->param_dtype, al.vec, (unsigned)blocks, threads, static_cast<cudaStream_t>(stream));
    if (e != cudaSuccess || cudaGetLastError() != cudaSuccess) {
        cudaGetLastError();
        return FLASHBEV_CUDA_ERROR;
    }
    t_last_launches = 1;
    t_last_kernel = al.vec == 8 ? "block_norm" : (al.vec == 2 ? "block_norm_pairs" : "block_norm_scalar");
    return FLASHBEV_OK;
}

size_t flashbev_block_norm_backward_workspace_bytes(const flashbev_block_norm_backward_params *p)
{
    return check_backward(p) == FLASHBEV_OK && p->rows ? backward_shape(p).bytes : 0;
}

flashbev_status flashbev_block_norm_backward(const flashbev_block_norm_backward_params *p, void *stream_)
{
    const flashbev_status st = check_backward(p);
    if (st != FLASHBEV_OK) return st;
    cudaStream_t stream = static_cast<cudaStream_t>(stream_);
    void *const outs[5] = {p->grad_after_weight, p->grad_after_bias, p->grad_before_weight, p->grad_before_bias, p->grad_gate};
    if (!p->rows) {
        for (int i = 0; i < 5; ++i)
            if (outs[i] && cudaMemsetAsync(outs[i], 0, (i == 4 ? p->gate_groups : 1) * p->C * elem_size(p->param_dtype), stream) != cudaSuccess) {
                cudaGetLastError();
                return FLASHBEV_CUDA_ERROR;
            }
        t_last_launches = 0;
        return FLASHBEV_OK;
    }
    const BackwardShape s = backward_shape(p);
    if (s.blocks > 2147483647LL / 256) return FLASHBEV_UNSUPPORTED;
    if (s.bytes && (!p->workspace || p->workspace_bytes < s.bytes)) return FLASHBEV_TOO_SMALL;
    NormParams k = {};
    k.x = p->x, k.y = p->y, k.gate = p->gate, k.wa = p->after_weight, k.ba = p->after_bias, k.wb = p->before_weight;
    k.gh = p->grad_h, k.gn = p->grad_n, k.gx = p->grad_x, k.gy = p->grad_y, k.ggate = p->grad_gate;
    k.sums = static_cast<float *>(p->workspace), k.want = s.want;
    k.rows = (unsigned)p->rows, k.gates = s.gates, k.per_gate = (unsigned)(p->rows / s.gates), k.chunks = s.chunks, k.direct = s.direct;
    k.ld_x = dense(p->ld_x, p->C), k.ld_y = dense(p->ld_y, p->C), k.ld_gh = dense(p->ld_grad_h, p->C), k.ld_gn = dense(p->ld_grad_n, p->C);
    k.ld_gx = dense(p->ld_grad_x, p->C), k.ld_gy = dense(p->ld_grad_y, p->C);
    k.C = p->C, k.after = p->after, k.before = p->before, k.scale = (float)p->scale, k.eps = (float)p->eps, k.inv_c = 1.0f / (float)p->C;
    k.team = s.team;
    Alignment al(p->C);
    al.rows(p->x, k.ld_x, p->dtype), al.rows(p->grad_h, k.ld_gh, p->dtype), al.rows(p->grad_x, k.ld_gx, p->dtype);
    al.rows(p->y, k.ld_y, p->branch_dtype), al.rows(p->grad_n, k.ld_gn, p->branch_dtype), al.rows(p->grad_y, k.ld_gy, p->branch_dtype);
    al.rows(p->gate, p->C, p->param_dtype), al.rows(p->grad_gate, p->C, p->param_dtype);
    cudaError_t e = launch_norm<true>(k, p->dtype, p->branch_dtype, p->param_dtype, al.vec, (unsigned)s.blocks, s.threads, stream);
    int launches = 1;
    if (e == cudaSuccess && s.arrays) {
        SumJobs q = {};
        const long long across = (p->C + 31) / 32;
        long long at = 0;
        for (int i = 0; i < 5; ++i) {
            q.out[i] = outs[i], q.first[i] = (int)at;
            if (s.want >> i & 1) at += across * (i == 4 ? s.gates : 1);
        }
        q.first[5] = (int)at, q.blocks = (int)s.blocks, q.per = s.chunks, q.C = p->C;
        if (p->param_dtype == FLASHBEV_F32) e = launch_dependent(norm_sum_kernel<float>, dim3((unsigned)at), dim3(512), 0, stream, k.sums, q);
        else e = launch_dependent(norm_sum_kernel<bf16>, dim3((unsigned)at), dim3(512), 0, stream, k.sums, q);
        ++launches;
    }
    if (e != cudaSuccess || cudaGetLastError() != cudaSuccess) {
        cudaGetLastError();
        return FLASHBEV_CUDA_ERROR;
    }
    t_last_launches = launches;
    t_last_kernel = al.vec == 8 ? "block_norm_backward" : (al.vec == 2 ? "block_norm_backward_pairs" : "block_norm_backward_scalar");
    return FLASHBEV_OK;
}

}  // extern "C"
