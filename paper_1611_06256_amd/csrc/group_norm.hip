// Group norm with an activation, channels last, and its gradient: of maps, and (one position per sample, a group per head) of
// what an agent's memory reads out.
//
// Bound by memory: what counts is that x (and dy) are read once.  With mean and rstd of a sample's group,
//     xh = (x - mean) rstd,  z = xh gamma + beta,  y = act(z)
//     dz = dy act'(z),  d = dz gamma,  dx = rstd (d - mean(d) - xh mean(d xh)),  dgamma = sum dz xh,  dbeta = sum dz
// Three ways, by size:
//   rows    one position per sample: 64 / LG groups of a sample per wavefront, LG lanes and their registers hold a group
//   tiles   a block holds whole groups of a sample in registers, side by side so that a position's share is a memory line or more
//   chunks  larger samples: partial sums of each chunk of positions, joined, then the result, which reads x a second time
// Means come first and squares are taken around them; chunks are joined by the same rule.
#include <hip/hip_runtime.h>
#include <math.h>

#include <algorithm>
#include <type_traits>

#include "call_error.hpp"
#include "launch.hpp"
#include "tensor_types.hpp"
#include "../../include/ga3c.h"

namespace ga3c {
namespace {

struct NormArgs {
    const void *x, *dy;
    void *y;                         // the result, or dx
    int64_t xs, dys, ys;             // elements from one position to the next
    const float *gamma, *beta;
    float *stats;                    // [samples][groups][2]: mean, 1 / standard deviation
    float *dgamma, *dbeta;
    float *sums;                     // chunks: [samples][chunks][groups][2]
    float *partial;                  // [rows][2][channels]: shares of dgamma and dbeta
    int partial_rows;
    int samples, positions, channels, groups, wide;
    float eps;
    int per_group;                   // vectors of a group's channels
    int tile_groups, tiles;          // groups of a tile, and tiles of a sample
    int chunk, chunks;               // positions of a chunk, and chunks of a sample
};

// 1 / (1 + exp(-z)) from the hardware's power of two and reciprocal, each within a unit in the last place; the exponent's rounding
// moves the result by less than |z| 2^-24 of itself, at most 3 units where it counts; below z = -87 it is 0 in place of numbers
// under 1e-37.  (With the library's exponential and a full
// division the arithmetic of 64 maps of bfloat16 took longer than their way from and to memory.)
__device__ inline float sigmoid(float z) { return __builtin_amdgcn_rcpf(1.f + __builtin_amdgcn_exp2f(z * -1.44269504f)); }
template <int ACT>
__device__ inline float activation(float z) {
    if (ACT == GA3C_ACT_RELU) return z < 0.f ? 0.f : z;      // NaN stays
    if (ACT == GA3C_ACT_SILU) return z * sigmoid(z);
    return z;
}
// dz of dy: nothing of what arrives where the rectifier is closed, whatever it is.
template <int ACT>
__device__ inline float activation_grad(float dy, float z) {
    if (ACT == GA3C_ACT_RELU) return z > 0.f ? dy : 0.f;
    if (ACT == GA3C_ACT_SILU) {
        const float s = sigmoid(z);
        return dy * (s * (1.f + z * (1.f - s)));
    }
    return dy;
}

// VE neighbouring elements as they lie in memory: 16 bytes, two, or a single one.  again(): what was made of them so far is not kept in
// registers for what comes, but made anew.
template <class T, int VE> struct Pack;
template <> struct Pack<float, 4> {
    float4 v;
    __device__ float operator[](int i) const { return i == 0 ? v.x : i == 1 ? v.y : i == 2 ? v.z : v.w; }
    __device__ static Pack of(const float (&f)[4]) { return Pack{float4{f[0], f[1], f[2], f[3]}}; }
    __device__ void again() { asm volatile("" : "+v"(v.x), "+v"(v.y), "+v"(v.z), "+v"(v.w)); }
};
template <> struct Pack<bf16, 8> {
    uint4 v;
    __device__ float operator[](int i) const {
        const uint32_t w = i < 2 ? v.x : i < 4 ? v.y : i < 6 ? v.z : v.w;
        return __uint_as_float(i % 2 ? w & 0xffff0000u : w << 16);
    }
    __device__ static uint32_t two(float a, float b) {
        typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
        typedef float f32x2 __attribute__((ext_vector_type(2)));
        return __builtin_bit_cast(uint32_t, __builtin_convertvector(f32x2{a, b}, bf16x2));
    }
    __device__ static Pack of(const float (&f)[8]) { return Pack{uint4{two(f[0], f[1]), two(f[2], f[3]), two(f[4], f[5]), two(f[6], f[7])}}; }
    __device__ void again() { asm volatile("" : "+v"(v.x), "+v"(v.y), "+v"(v.z), "+v"(v.w)); }
};
template <> struct Pack<float, 2> {
    float2 v;
    __device__ float operator[](int i) const { return i == 0 ? v.x : v.y; }
    __device__ static Pack of(const float (&f)[2]) { return Pack{float2{f[0], f[1]}}; }
    __device__ void again() { asm volatile("" : "+v"(v.x), "+v"(v.y)); }
};
template <> struct Pack<bf16, 2> {
    uint32_t v;
    __device__ float operator[](int i) const { return __uint_as_float(i ? v & 0xffff0000u : v << 16); }
    __device__ static Pack of(const float (&f)[2]) { return Pack{Pack<bf16, 8>::two(f[0], f[1])}; }
    __device__ void again() { asm volatile("" : "+v"(v)); }
};
template <class T> struct Pack<T, 1> {
    T v;
    __device__ float operator[](int) const { return to_f32(v); }
    __device__ static Pack of(const float (&f)[1]) { return Pack{from_f32<T>(f[0])}; }
    __device__ void again() {}
};
template <int VE>
__device__ inline void weights(float (&w)[VE], const float *p) {
    if constexpr (VE < 4)
#pragma unroll
        for (int i = 0; i < VE; ++i) w[i] = p[i];
    else
#pragma unroll
        for (int i = 0; i < VE; i += 4) {
            const float4 v = *(const float4 *)(p + i);
            w[i] = v.x; w[i + 1] = v.y; w[i + 2] = v.z; w[i + 3] = v.w;
        }
}

// Sum over neighbouring `lanes` lanes (a power of two), the same in all of them.
__device__ inline float lanes_sum(float v, int lanes) {
    for (int m = lanes / 2; m > 0; m /= 2) v += __shfl_xor(v, m);
    return v;
}

// ------------------------------------------------------------------------ rows --

// 2560 samples of 4 groups of 32 fp32: 3.4 us (2.6 MB: start and end of a launch).
template <class T, int VE, int NV, int ACT>
__global__ __launch_bounds__(256) void norm_rows_kernel(const NormArgs a, int lg) {
    typedef Pack<T, VE> V;
    const int lane = threadIdx.x % 64, li = lane % lg;
    const int64_t unit = ((int64_t)blockIdx.x * 4 + threadIdx.x / 64) * (64 / lg) + lane / lg;
    const bool there = unit < (int64_t)a.samples * a.groups;
    const int64_t u = there ? unit : 0;
    const int sample = (int)(u / a.groups), group = (int)(u % a.groups);
    const T *x = (const T *)a.x + sample * a.xs + group * a.wide;
    V in[NV];
    float sum = 0.f;
#pragma unroll
    for (int j = 0; j < NV; ++j) {
        const int vi = li + lg * j;
        in[j] = *(const V *)(x + min(vi, a.per_group - 1) * VE);
    }
#pragma unroll
    for (int j = 0; j < NV; ++j)
        if (li + lg * j < a.per_group)
#pragma unroll
            for (int e = 0; e < VE; ++e) sum += in[j][e];
    const float mean = lanes_sum(sum, lg) / (float)a.wide;
    sum = 0.f;
#pragma unroll
    for (int j = 0; j < NV; ++j)
        if (li + lg * j < a.per_group)
#pragma unroll
            for (int e = 0; e < VE; ++e) {
                const float d = in[j][e] - mean;
                sum += d * d;
            }
    const float rstd = 1.f / sqrtf(lanes_sum(sum, lg) / (float)a.wide + a.eps);
    if (!there) return;
    T *y = (T *)a.y + sample * a.ys + group * a.wide;
#pragma unroll
    for (int j = 0; j < NV; ++j) {
        const int vi = li + lg * j;
        if (vi >= a.per_group) break;
        float g[VE], b[VE], z[VE];
        weights<VE>(g, a.gamma + group * a.wide + vi * VE);
        weights<VE>(b, a.beta + group * a.wide + vi * VE);
#pragma unroll
        for (int e = 0; e < VE; ++e) z[e] = activation<ACT>((in[j][e] - mean) * rstd * g[e] + b[e]);
        *(V *)(y + vi * VE) = V::of(z);
    }
    if (a.stats && li == 0) *(float2 *)(a.stats + 2 * u) = float2{mean, rstd};
}

// A wavefront keeps its groups and walks over samples, so that its share of dgamma and dbeta stays in registers.  8192 samples of 16
// groups of 64 bf16: 15.7 us (50 MB, 3.2 TB/s), and 4.2 for dgamma and dbeta from the shares.
template <class T, int VE, int NV, int ACT>
__global__ __launch_bounds__(256) void norm_rows_grad_kernel(const NormArgs a, int lg) {
    typedef Pack<T, VE> V;
    __shared__ float share[4][2][64 * NV * VE];
    const int lane = threadIdx.x % 64, wave = threadIdx.x / 64, li = lane % lg, each = 64 / lg, group = blockIdx.y * each + lane / lg;
    const bool there = group < a.groups;
    const int c0 = (there ? group : 0) * a.wide;
    float g[NV][VE], b[NV][VE], dg[NV][VE], db[NV][VE];
#pragma unroll
    for (int j = 0; j < NV; ++j) {
        const int vi = min(li + lg * j, a.per_group - 1);
        weights<VE>(g[j], a.gamma + c0 + vi * VE);
        weights<VE>(b[j], a.beta + c0 + vi * VE);
#pragma unroll
        for (int e = 0; e < VE; ++e) dg[j][e] = db[j][e] = 0.f;
    }
    for (int sample = blockIdx.x * 4 + wave; sample < a.samples; sample += gridDim.x * 4) {
        const T *x = (const T *)a.x + sample * a.xs + c0, *dy = (const T *)a.dy + sample * a.dys + c0;
        const float2 st = *(const float2 *)(a.stats + 2 * ((int64_t)sample * a.groups + (there ? group : 0)));
        V in[NV], gr[NV];
#pragma unroll
        for (int j = 0; j < NV; ++j) {
            const int vi = min(li + lg * j, a.per_group - 1);
            in[j] = *(const V *)(x + vi * VE);
            gr[j] = *(const V *)(dy + vi * VE);
        }
        float s = 0.f, sx = 0.f, xh[NV][VE], d[NV][VE];
#pragma unroll
        for (int j = 0; j < NV; ++j) {
            if (li + lg * j >= a.per_group) continue;
#pragma unroll
            for (int e = 0; e < VE; ++e) {
                xh[j][e] = (in[j][e] - st.x) * st.y;
                const float dz = activation_grad<ACT>(gr[j][e], xh[j][e] * g[j][e] + b[j][e]);
                dg[j][e] += dz * xh[j][e];
                db[j][e] += dz;
                d[j][e] = dz * g[j][e];
                s += d[j][e]; sx += d[j][e] * xh[j][e];
            }
        }
        const float ma = lanes_sum(s, lg) / (float)a.wide, mb = lanes_sum(sx, lg) / (float)a.wide;
        T *dx = (T *)a.y + sample * a.ys + c0;
#pragma unroll
        for (int j = 0; j < NV; ++j) {
            const int vi = li + lg * j;
            if (!there || vi >= a.per_group) break;
            float r[VE];
#pragma unroll
            for (int e = 0; e < VE; ++e) r[e] = st.y * (d[j][e] - ma - xh[j][e] * mb);
            *(V *)(dx + vi * VE) = V::of(r);
        }
    }
    // the block's four wavefronts together
#pragma unroll
    for (int j = 0; j < NV; ++j)
#pragma unroll
        for (int e = 0; e < VE; ++e) {
            share[wave][0][(j * VE + e) * 64 + lane] = dg[j][e];
            share[wave][1][(j * VE + e) * 64 + lane] = db[j][e];
        }
    __syncthreads();
    for (int i = threadIdx.x; i < 2 * 64 * NV * VE; i += 256) {
        const int which = i / (64 * NV * VE), k = i % (64 * NV * VE), l = k % 64, j = k / 64 / VE, e = k / 64 % VE;
        const int gr = blockIdx.y * each + l / lg, vi = l % lg + lg * j;
        if (gr >= a.groups || vi >= a.per_group) continue;
        const float v = (share[0][which][k] + share[1][which][k]) + (share[2][which][k] + share[3][which][k]);
        a.partial[((int64_t)blockIdx.x * 2 + which) * a.channels + gr * a.wide + vi * VE + e] = v;
    }
}

// ------------------------------------------------------------- tiles and chunks --

// Which vectors a thread of a tile holds: vector `c` of the tile's positions row, row + rows, ... (none: c < 0).
struct Place {
    int c, row, rows, group;
    __device__ Place(const NormArgs &a, int tile, int nt) {
        const int groups = min(a.tile_groups, a.groups - tile * a.tile_groups), all = groups * a.per_group;
        rows = nt / all;
        const int t = threadIdx.x;
        row = t / all;
        c = row < rows ? t % all : -1;
        group = c < 0 ? 0 : c / a.per_group;
    }
};
// Sums of one number per thread over the threads of each group, into `of_group`.
template <int NT>
__device__ inline void group_sums(const NormArgs &a, const Place &w, int groups, float v, float *each, float *of_group) {
    __syncthreads();
    each[threadIdx.x] = v;
    __syncthreads();
    const int lane = threadIdx.x % 64, all = groups * a.per_group;
    for (int g = threadIdx.x / 64; g < groups; g += NT / 64) {
        float s = 0.f;
        for (int e = lane; e < w.rows * a.per_group; e += 64) s += each[e / a.per_group * all + g * a.per_group + e % a.per_group];
        s = lanes_sum(s, 64);
        if (lane == 0) of_group[g] = s;
    }
    __syncthreads();
}

enum { TILE, CHUNK_SUMS, CHUNK_RESULT };
constexpr int MAX_TILE_GROUPS = 128;

// Between the sums of the chunks and the result: a wavefront joins those of one group of one sample, and leaves them in the place of
// the first chunk's.  GRAD: the two sums.  Otherwise from each chunk's mean and its squares around that: mean and 1 / standard
// deviation.  (Where each block of the result joined them for itself, one sample of 4194304 positions of 32 channels fp32 took 5960 us
// instead of 326 and its gradient 38053 instead of 769; a sample of 8192 positions of 64, of few chunks, 13 instead of 17.)
template <bool GRAD>
__global__ __launch_bounds__(256) void norm_join_kernel(const NormArgs a) {
    const int64_t unit = (int64_t)blockIdx.x * 4 + threadIdx.x / 64;
    if (unit >= (int64_t)a.samples * a.groups) return;
    const int lane = threadIdx.x % 64;
    float *s = a.sums + 2 * (unit / a.groups * a.chunks * a.groups + unit % a.groups);
    float first = 0.f, second = 0.f;
    auto numbers = [&](int i) { return (float)min(a.chunk, a.positions - i * a.chunk) * (float)a.wide; };
    for (int i = lane; i < a.chunks; i += 64) {
        const float2 v = *(const float2 *)(s + 2 * (int64_t)i * a.groups);
        first += GRAD ? v.x : v.x * numbers(i);
        if (GRAD) second += v.y;
    }
    const float m = (float)a.positions * (float)a.wide;
    first = lanes_sum(first, 64);
    if (!GRAD) {
        first /= m;
        for (int i = lane; i < a.chunks; i += 64) {
            const float2 v = *(const float2 *)(s + 2 * (int64_t)i * a.groups);
            const float d = v.x - first;
            second += v.y + d * d * numbers(i);
        }
    }
    second = lanes_sum(second, 64);
    if (!GRAD) second = 1.f / sqrtf(second / m + a.eps);
    if (lane == 0) *(float2 *)s = float2{first, second};
}

// Eight wavefronts per SIMD, so that two blocks of 1024 threads share a compute unit and one reads while the other writes (64 maps of
// 1024 positions, 512 channels bf16: 39 us with one, 31 with two: 4.3 TB/s).
template <class T, int VE, int NT, int NV, int MODE, int ACT>
__global__ __launch_bounds__(NT, 8) void norm_tile_kernel(const NormArgs a) {
    typedef Pack<T, VE> V;
    __shared__ float each[NT], mean_of[MAX_TILE_GROUPS], rstd_of[MAX_TILE_GROUPS];
    const int sample = blockIdx.x / a.tiles, tile = blockIdx.x % a.tiles, first = MODE == TILE ? 0 : blockIdx.y * a.chunk;
    const int positions = MODE == TILE ? a.positions : min(a.chunk, a.positions - first);
    const int groups = min(a.tile_groups, a.groups - tile * a.tile_groups), g0 = tile * a.tile_groups;
    const Place w(a, tile, NT);
    const int channel = g0 * a.wide + max(w.c, 0) * VE;
    const int64_t start = (int64_t)sample * a.positions + first;
    const T *x = (const T *)a.x + start * a.xs + channel;
    V in[NV];
#pragma unroll
    for (int j = 0; j < NV; ++j) {
        if (w.rows * j >= positions) continue;               // the same in all threads: nothing is done for positions that are not there
        in[j] = *(const V *)(x + (w.row + w.rows * j < positions ? (w.row + w.rows * j) * a.xs : 0));
    }
    if constexpr (MODE == CHUNK_RESULT) {
        for (int g = threadIdx.x; g < groups; g += NT) {
            const float2 st = *(const float2 *)(a.sums + 2 * ((int64_t)sample * a.chunks * a.groups + g0 + g));
            mean_of[g] = st.x; rstd_of[g] = st.y;
        }
        __syncthreads();
    } else {
        const float m = (float)positions * (float)a.wide;
        float s = 0.f;
#pragma unroll
        for (int j = 0; j < NV; ++j) {
            if (w.rows * j >= positions) continue;
            if (w.c >= 0 && w.row + w.rows * j < positions)
#pragma unroll
                for (int e = 0; e < VE; ++e) s += in[j][e];
        }
        group_sums<NT>(a, w, groups, s, each, mean_of);
        const float mean = mean_of[w.group] / m;
        s = 0.f;
#pragma unroll
        for (int j = 0; j < NV; ++j) {
            if (w.rows * j >= positions) continue;
            in[j].again();
            if (w.c >= 0 && w.row + w.rows * j < positions)
#pragma unroll
                for (int e = 0; e < VE; ++e) {
                    const float d = in[j][e] - mean;
                    s += d * d;
                }
        }
        group_sums<NT>(a, w, groups, s, each, rstd_of);
        if constexpr (MODE == CHUNK_SUMS) {
            for (int g = threadIdx.x; g < groups; g += NT)
                *(float2 *)(a.sums + 2 * (((int64_t)sample * a.chunks + blockIdx.y) * a.groups + g0 + g)) = float2{mean_of[g] / m, rstd_of[g]};
            return;
        }
        for (int g = threadIdx.x; g < groups; g += NT) { mean_of[g] /= m; rstd_of[g] = 1.f / sqrtf(rstd_of[g] / m + a.eps); }
        __syncthreads();
    }
    if (a.stats && (MODE == TILE || blockIdx.y == 0))
        for (int g = threadIdx.x; g < groups; g += NT) *(float2 *)(a.stats + 2 * ((int64_t)sample * a.groups + g0 + g)) = float2{mean_of[g], rstd_of[g]};
    if (w.c < 0) return;
#pragma unroll
    for (int j = 0; j < NV; ++j) {
        if (w.rows * j >= positions) continue;
        in[j].again();
    }
    const float mean = mean_of[w.group], rstd = rstd_of[w.group];
    float g[VE], b[VE];
    weights<VE>(g, a.gamma + channel);
    weights<VE>(b, a.beta + channel);
    T *y = (T *)a.y + start * a.ys + channel;
    int row = w.row;
    asm volatile("" : "+v"(row));                    // places are worked out anew: they are too many to keep
#pragma unroll
    for (int j = 0; j < NV; ++j) {
        if (row + w.rows * j >= positions) break;
        __builtin_amdgcn_sched_barrier(0);
        float z[VE];
#pragma unroll
        for (int e = 0; e < VE; ++e) z[e] = activation<ACT>((in[j][e] - mean) * rstd * g[e] + b[e]);
        *(V *)(y + (row + w.rows * j) * a.ys) = V::of(z);
    }
}

// A block keeps its groups (and its chunk) and walks over samples.  37 samples of 81 positions, 96 channels fp32: 10.5 us (3.5 MB: the
// latency of a block's sums), and 2 for dgamma and dbeta.
template <class T, int VE, int NT, int NV, int MODE, int ACT>
__global__ __launch_bounds__(NT) void norm_tile_grad_kernel(const NormArgs a) {
    typedef Pack<T, VE> V;
    __shared__ float each[NT], d_of[MAX_TILE_GROUPS], dx_of[MAX_TILE_GROUPS];
    const int tile = blockIdx.x % a.tiles, first = MODE == TILE ? 0 : blockIdx.y * a.chunk;
    const int positions = MODE == TILE ? a.positions : min(a.chunk, a.positions - first);
    const int groups = min(a.tile_groups, a.groups - tile * a.tile_groups), g0 = tile * a.tile_groups;
    const Place w(a, tile, NT);
    const int channel = g0 * a.wide + max(w.c, 0) * VE;
    float g[VE], b[VE], dg[VE], db[VE];
    weights<VE>(g, a.gamma + channel);
    weights<VE>(b, a.beta + channel);
#pragma unroll
    for (int e = 0; e < VE; ++e) dg[e] = db[e] = 0.f;
    const float m = (float)a.positions * (float)a.wide;
    for (int sample = blockIdx.x / a.tiles; sample < a.samples; sample += gridDim.x / a.tiles) {
        const int64_t start = (int64_t)sample * a.positions + first;
        const T *x = (const T *)a.x + start * a.xs + channel, *dy = (const T *)a.dy + start * a.dys + channel;
        V in[NV], gr[NV];
        int row = w.row;
        asm volatile("" : "+v"(row));                // places are worked out in each round: they are too many to keep
#pragma unroll
        for (int j = 0; j < NV; ++j) {
            if (w.rows * j >= positions) continue;
            const int pos = min(row + w.rows * j, positions - 1);
            in[j] = *(const V *)(x + pos * a.xs);
            gr[j] = *(const V *)(dy + pos * a.dys);
        }
        const float2 st = *(const float2 *)(a.stats + 2 * ((int64_t)sample * a.groups + g0 + w.group));
        float s = 0.f, sx = 0.f;
#pragma unroll
        for (int j = 0; j < NV; ++j) {
            if (w.rows * j >= positions) continue;
            __builtin_amdgcn_sched_barrier(0);
            if (MODE == CHUNK_RESULT || w.c < 0 || row + w.rows * j >= positions) continue;
#pragma unroll
            for (int e = 0; e < VE; ++e) {
                const float xh = (in[j][e] - st.x) * st.y, dz = activation_grad<ACT>(gr[j][e], xh * g[e] + b[e]), d = dz * g[e];
                dg[e] += dz * xh;
                db[e] += dz;
                s += d;
                sx += d * xh;
            }
        }
        if constexpr (MODE == CHUNK_RESULT) {
            __syncthreads();
            for (int k = threadIdx.x; k < groups; k += NT) {
                const float2 v = *(const float2 *)(a.sums + 2 * ((int64_t)sample * a.chunks * a.groups + g0 + k));
                d_of[k] = v.x; dx_of[k] = v.y;
            }
            __syncthreads();
        } else {
            group_sums<NT>(a, w, groups, s, each, d_of);
            group_sums<NT>(a, w, groups, sx, each, dx_of);
        }
        if constexpr (MODE == CHUNK_SUMS) {
            for (int k = threadIdx.x; k < groups; k += NT)
                *(float2 *)(a.sums + 2 * (((int64_t)sample * a.chunks + blockIdx.y) * a.groups + g0 + k)) = float2{d_of[k], dx_of[k]};
            continue;
        }
        const float ma = d_of[w.group] / m, mb = dx_of[w.group] / m;
#pragma unroll
        for (int j = 0; j < NV; ++j) {
            if (w.rows * j >= positions) continue;
            in[j].again();
            gr[j].again();
        }
        T *dx = (T *)a.y + start * a.ys + channel;
        if (w.c >= 0)
#pragma unroll
            for (int j = 0; j < NV; ++j) {
                if (row + w.rows * j >= positions) break;
                __builtin_amdgcn_sched_barrier(0);
                float r[VE];
#pragma unroll
                for (int e = 0; e < VE; ++e) {
                    const float xh = (in[j][e] - st.x) * st.y, dz = activation_grad<ACT>(gr[j][e], xh * g[e] + b[e]);
                    r[e] = st.y * (dz * g[e] - ma - xh * mb);
                }
                *(V *)(dx + (row + w.rows * j) * a.ys) = V::of(r);
            }
    }
    if constexpr (MODE == CHUNK_RESULT) return;
    // the block's share of dgamma and dbeta: its rows of threads together
    const int row = blockIdx.x / a.tiles + (MODE == TILE ? 0 : blockIdx.y * (gridDim.x / a.tiles)), all = groups * a.per_group;
#pragma unroll
    for (int which = 0; which < 2; ++which)
#pragma unroll
        for (int e = 0; e < VE; ++e) {
            __syncthreads();
            each[threadIdx.x] = which ? db[e] : dg[e];
            __syncthreads();
            for (int c = threadIdx.x; c < all; c += NT) {
                float s = 0.f;
                for (int k = 0; k < w.rows; ++k) s += each[k * all + c];
                a.partial[((int64_t)row * 2 + which) * a.channels + g0 * a.wide + c * VE + e] = s;
            }
        }
}

// ------------------------------------------------------------------ wide groups --
// Groups of more channels than a block has threads for: a block goes over one group of one sample as often as it needs to.  Made for
// being right at sizes that no network here has, not for speed.

__device__ inline float block_sum(float v, float *sh) {
    v = lanes_sum(v, 64);
    __syncthreads();
    if (threadIdx.x % 64 == 0) sh[threadIdx.x / 64] = v;
    __syncthreads();
    return sh[0] + sh[1] + sh[2] + sh[3];
}

template <class T, int ACT>
__global__ __launch_bounds__(256) void norm_wide_kernel(const NormArgs a) {
    __shared__ float sh[4];
    const int sample = blockIdx.x / a.groups, group = blockIdx.x % a.groups, c0 = group * a.wide;
    const T *x = (const T *)a.x + (int64_t)sample * a.positions * a.xs + c0;
    T *y = (T *)a.y + (int64_t)sample * a.positions * a.ys + c0;
    const int64_t m = (int64_t)a.positions * a.wide;
    float s = 0.f;
    for (int64_t e = threadIdx.x; e < m; e += 256) s += to_f32(x[e / a.wide * a.xs + e % a.wide]);
    const float mean = block_sum(s, sh) / (float)m;
    s = 0.f;
    for (int64_t e = threadIdx.x; e < m; e += 256) {
        const float d = to_f32(x[e / a.wide * a.xs + e % a.wide]) - mean;
        s += d * d;
    }
    const float rstd = 1.f / sqrtf(block_sum(s, sh) / (float)m + a.eps);
    for (int64_t e = threadIdx.x; e < m; e += 256) {
        const int64_t p = e / a.wide;
        const int c = (int)(e % a.wide);
        y[p * a.ys + c] = from_f32<T>(activation<ACT>((to_f32(x[p * a.xs + c]) - mean) * rstd * a.gamma[c0 + c] + a.beta[c0 + c]));
    }
    if (a.stats && threadIdx.x == 0) *(float2 *)(a.stats + 2 * ((int64_t)sample * a.groups + group)) = float2{mean, rstd};
}

template <class T, int ACT>
__global__ __launch_bounds__(256) void norm_wide_grad_kernel(const NormArgs a) {
    __shared__ float sh[4];
    const int sample = blockIdx.x / a.groups, group = blockIdx.x % a.groups, c0 = group * a.wide;
    const T *x = (const T *)a.x + (int64_t)sample * a.positions * a.xs + c0, *dy = (const T *)a.dy + (int64_t)sample * a.positions * a.dys + c0;
    T *dx = (T *)a.y + (int64_t)sample * a.positions * a.ys + c0;
    const int64_t m = (int64_t)a.positions * a.wide;
    const float2 st = *(const float2 *)(a.stats + 2 * ((int64_t)sample * a.groups + group));
    float s = 0.f, sx = 0.f;
    for (int64_t e = threadIdx.x; e < m; e += 256) {
        const int64_t p = e / a.wide;
        const int c = (int)(e % a.wide);
        const float xh = (to_f32(x[p * a.xs + c]) - st.x) * st.y, g = a.gamma[c0 + c];
        const float d = activation_grad<ACT>(to_f32(dy[p * a.dys + c]), xh * g + a.beta[c0 + c]) * g;
        s += d; sx += d * xh;
    }
    const float ma = block_sum(s, sh) / (float)m, mb = block_sum(sx, sh) / (float)m;
    for (int64_t e = threadIdx.x; e < m; e += 256) {
        const int64_t p = e / a.wide;
        const int c = (int)(e % a.wide);
        const float xh = (to_f32(x[p * a.xs + c]) - st.x) * st.y, g = a.gamma[c0 + c];
        const float d = activation_grad<ACT>(to_f32(dy[p * a.dys + c]), xh * g + a.beta[c0 + c]) * g;
        dx[p * a.ys + c] = from_f32<T>(st.y * (d - ma - xh * mb));
    }
}

// One row of shares of dgamma and dbeta, a channel per thread.
template <class T, int ACT>
__global__ __launch_bounds__(64) void norm_wide_weights_kernel(const NormArgs a) {
    const int c = blockIdx.x * 64 + threadIdx.x;
    if (c >= a.channels) return;
    const int64_t all = (int64_t)a.samples * a.positions, each = (all + gridDim.y - 1) / gridDim.y, last = min(all, each * (blockIdx.y + 1));
    float s = 0.f, sx = 0.f;
    for (int64_t e = each * blockIdx.y; e < last; ++e) {
        const float2 st = *(const float2 *)(a.stats + 2 * (e / a.positions * a.groups + c / a.wide));
        const float xh = (to_f32(((const T *)a.x)[e * a.xs + c]) - st.x) * st.y;
        const float d = activation_grad<ACT>(to_f32(((const T *)a.dy)[e * a.dys + c]), xh * a.gamma[c] + a.beta[c]);
        s += d; sx += d * xh;
    }
    a.partial[(int64_t)blockIdx.y * 2 * a.channels + c] = sx;
    a.partial[((int64_t)blockIdx.y * 2 + 1) * a.channels + c] = s;
}

// dgamma and dbeta from the shares of the blocks, in a fixed order.  A block takes 64 channels, sixteen threads of each.
__global__ __launch_bounds__(1024) void norm_weights_kernel(const NormArgs a) {
    __shared__ float part[16][64];
    const int64_t all = 2 * (int64_t)a.channels, c = (int64_t)blockIdx.x * 64 + threadIdx.x % 64;
    const int k = threadIdx.x / 64;
    float s = 0.f;
    for (int r = k; r < a.partial_rows; r += 16 * 8) {
        float v[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = a.partial[min(r + 16 * i, a.partial_rows - 1) * all + min(c, all - 1)];
#pragma unroll
        for (int i = 0; i < 8; ++i) s += r + 16 * i < a.partial_rows ? v[i] : 0.f;
    }
    part[k][threadIdx.x % 64] = s;
    __syncthreads();
    if (k == 0 && c < all) {
        s = 0.f;
#pragma unroll
        for (int i = 0; i < 16; ++i) s += part[i][threadIdx.x];
        if (c < a.channels) a.dgamma[c] = s;
        else a.dbeta[c - a.channels] = s;
    }
}

// -------------------------------------------------------------------- host --

int check(const ga3c_norm_desc *d, int samples, int positions, const char *who) {
    if (!d) return call_fail(GA3C_EINVAL, "%s: null description", who);
    if (d->channels < 1 || d->groups < 1 || d->channels % d->groups) return call_fail(GA3C_EINVAL, "%s: %d channels are no %d equal groups", who, d->channels, d->groups);
    if (d->channels > 1 << 20) return call_fail(GA3C_EINVAL, "%s: more than 2^20 channels", who);
    if (d->dtype != GA3C_F32 && d->dtype != GA3C_BF16) return call_fail(GA3C_EINVAL, "%s: dtype must be GA3C_F32 or GA3C_BF16", who);
    if (d->act != GA3C_ACT_NONE && d->act != GA3C_ACT_RELU && d->act != GA3C_ACT_SILU) return call_fail(GA3C_EINVAL, "%s: unknown activation %d", who, d->act);
    if (!(d->eps >= 0.f) || !isfinite(d->eps)) return call_fail(GA3C_EINVAL, "%s: eps must be finite and not negative", who);
    if (samples < 0 || positions < 0) return call_fail(GA3C_EINVAL, "%s: negative count", who);
    if (samples > 0 && positions == 0) return call_fail(GA3C_EINVAL, "%s: samples without a position", who);
    if (samples > 1 << 24 || positions > 1 << 24) return call_fail(GA3C_EINVAL, "%s: more than 2^24 samples or positions", who);
    return GA3C_OK;
}
int check_rows(const void *p, int64_t stride, const ga3c_norm_desc *d, const char *who) {
    if (!p) return call_fail(GA3C_EINVAL, "%s: null tensor", who);
    if ((uintptr_t)p % (d->dtype == GA3C_BF16 ? 2 : 4)) return call_fail(GA3C_EINVAL, "%s: tensor not aligned to its elements", who);
    if (stride < d->channels) return call_fail(GA3C_EINVAL, "%s: positions closer than their channels", who);
    return GA3C_OK;
}

// How a call is cut up.  Decided by the sizes alone, but for the vector's width, which may only be less than they allow: scratch is
// asked for before the tensors are known.
struct Cut {
    int ve;                          // elements of a vector
    bool rows, wide;                 // the kernels for one position per sample, for wide groups
    int lg, nv;                      // rows: lanes per group, vectors per lane
    int threads;                     // tiles: of a block
    int per_group, tile_groups, tiles, chunk, chunks;
    int walkers;                     // gradient: blocks that share the samples out
};
// Vectors of a tensor per thread: the gradient has two tensors, and sums for each channel.  More of them where they are only one or two
// elements (38 samples of 123 positions, groups of 15 channels bf16: 17 us with 8, 10 with 16).
constexpr int tile_vectors(int ve) { return ve >= 4 ? 8 : 16; }
constexpr int GRAD_VECTORS = 4;
constexpr int WIDEST = 1024, GRAD_WIDEST = 512;      // vectors of a group's channels that the threads of a tile's block take
// most: elements of a vector that the tensors allow
Cut cut_of(const ga3c_norm_desc *d, int samples, int positions, int most, bool grad) {
    Cut c{};
    const int size = d->dtype == GA3C_BF16 ? 2 : 4, wide = d->channels / d->groups;
    c.ve = most >= 16 / size && wide % (16 / size) == 0 ? 16 / size : most >= 2 && wide % 2 == 0 ? 2 : 1;
    c.per_group = wide / c.ve;
    c.chunks = 1; c.chunk = positions; c.tiles = 1; c.tile_groups = d->groups;
    // (a lane's shares of dgamma and dbeta are two numbers for each of its channels)
    if (positions == 1 && c.per_group <= 64 * (grad ? 2 : 8)) {
        c.rows = true;
        c.lg = 1;
        while (c.lg < 64 && c.lg < c.per_group) c.lg *= 2;
        c.nv = 1;
        while (c.lg * c.nv < c.per_group) c.nv *= 2;
        const int slabs = (d->groups + 64 / c.lg - 1) / (64 / c.lg);
        c.tiles = slabs;
        c.walkers = std::max(1, std::min((samples + 3) / 4, 1024 / slabs));
        return c;
    }
    const int widest = grad ? GRAD_WIDEST : WIDEST;
    if (c.per_group > widest) {
        c.wide = true;
        c.walkers = (int)std::min<int64_t>(256, (int64_t)samples * positions);
        return c;
    }
    // a memory line of each position, if the groups are small
    int k = std::min({d->groups, MAX_TILE_GROUPS, std::max(1, widest / c.per_group), std::max(1, (128 + wide * size - 1) / (wide * size))});
    c.tile_groups = k;
    c.tiles = (d->groups + k - 1) / k;
    const int all = k * c.per_group;
    const int vectors_each = grad ? GRAD_VECTORS : tile_vectors(c.ve);
    c.threads = 256;
    if (all > 256 || positions > 256 / all * vectors_each) c.threads = widest;
    const int rows = c.threads / all * vectors_each;      // positions that a block holds
    c.chunk = std::min(positions, std::max(rows, 1));
    c.chunks = (positions + c.chunk - 1) / c.chunk;
    c.walkers = (int)std::max<int64_t>(1, std::min<int64_t>(samples, 2048 / ((int64_t)c.tiles * c.chunks)));
    return c;
}
size_t sums_floats(const ga3c_norm_desc *d, const Cut &c, int samples) { return c.chunks > 1 ? 2 * (size_t)samples * c.chunks * d->groups : 0; }
size_t partial_floats(const ga3c_norm_desc *d, const Cut &c) { return 2 * (size_t)c.walkers * c.chunks * d->channels; }

NormArgs args_of(const ga3c_norm_desc *d, const Cut &c, int samples, int positions, void *workspace) {
    NormArgs a{};
    a.samples = samples; a.positions = positions; a.channels = d->channels; a.groups = d->groups; a.eps = d->eps;
    a.wide = d->channels / d->groups;
    a.per_group = c.per_group; a.tile_groups = c.tile_groups; a.tiles = c.tiles; a.chunk = c.chunk; a.chunks = c.chunks;
    a.sums = (float *)workspace;
    a.partial = (float *)workspace + sums_floats(d, c, samples);
    a.partial_rows = c.walkers * c.chunks;
    return a;
}

template <class T, int VE, int ACT, int NV>
void launch_rows(const NormArgs &a, const Cut &c, bool grad, hipStream_t s) {
    if (!grad) {
        const int64_t units = (int64_t)a.samples * a.groups;
        const int each = 4 * (64 / c.lg);
        launch(norm_rows_kernel<T, VE, NV, ACT>, dim3((unsigned)((units + each - 1) / each)), dim3(256), 0, s, a, c.lg);
    } else if constexpr (NV <= 2) launch(norm_rows_grad_kernel<T, VE, NV, ACT>, dim3(c.walkers, c.tiles), dim3(256), 0, s, a, c.lg);
}
template <class K>
void launch_join(K kernel, const NormArgs &a, hipStream_t s) {
    launch(kernel, dim3((unsigned)(((int64_t)a.samples * a.groups + 3) / 4)), dim3(256), 0, s, a);
}
template <class T, int VE, int ACT, int NT>
void launch_tiles(const NormArgs &a, const Cut &c, hipStream_t s) {
    const dim3 block(NT), grid((unsigned)((int64_t)a.samples * c.tiles), c.chunks);
    if (c.chunks == 1) { launch(norm_tile_kernel<T, VE, NT, tile_vectors(VE), TILE, ACT>, grid, block, 0, s, a); return; }
    launch(norm_tile_kernel<T, VE, NT, tile_vectors(VE), CHUNK_SUMS, ACT>, grid, block, 0, s, a);
    launch_join(norm_join_kernel<false>, a, s);
    launch(norm_tile_kernel<T, VE, NT, tile_vectors(VE), CHUNK_RESULT, ACT>, grid, block, 0, s, a);
}
template <class T, int VE, int ACT, int NT>
void launch_tile_grad(const NormArgs &a, const Cut &c, hipStream_t s) {
    const dim3 block(NT), grid(c.walkers * c.tiles, c.chunks);
    if (c.chunks == 1) { launch(norm_tile_grad_kernel<T, VE, NT, GRAD_VECTORS, TILE, ACT>, grid, block, 0, s, a); return; }
    launch(norm_tile_grad_kernel<T, VE, NT, GRAD_VECTORS, CHUNK_SUMS, ACT>, grid, block, 0, s, a);
    launch_join(norm_join_kernel<true>, a, s);
    launch(norm_tile_grad_kernel<T, VE, NT, GRAD_VECTORS, CHUNK_RESULT, ACT>, grid, block, 0, s, a);
}
template <class T, int VE, int ACT>
void launch_kernels(const NormArgs &a, const Cut &c, bool grad, hipStream_t s) {
    if (c.wide) {
        const dim3 grid((unsigned)(a.samples * a.groups)), block(256);
        if (!grad) launch(norm_wide_kernel<T, ACT>, grid, block, 0, s, a);
        else {
            launch(norm_wide_grad_kernel<T, ACT>, grid, block, 0, s, a);
            launch(norm_wide_weights_kernel<T, ACT>, dim3((a.channels + 63) / 64, c.walkers), dim3(64), 0, s, a);
        }
    } else if (c.rows) {
        if (c.nv == 1) launch_rows<T, VE, ACT, 1>(a, c, grad, s);
        else if (c.nv == 2) launch_rows<T, VE, ACT, 2>(a, c, grad, s);
        else if (c.nv == 4) launch_rows<T, VE, ACT, 4>(a, c, grad, s);
        else launch_rows<T, VE, ACT, 8>(a, c, grad, s);
    } else if (c.threads == 256) grad ? launch_tile_grad<T, VE, ACT, 256>(a, c, s) : launch_tiles<T, VE, ACT, 256>(a, c, s);
    else grad ? launch_tile_grad<T, VE, ACT, GRAD_WIDEST>(a, c, s) : launch_tiles<T, VE, ACT, WIDEST>(a, c, s);
}
template <class T, int VE>
void launch_act(const ga3c_norm_desc *d, const NormArgs &a, const Cut &c, bool grad, hipStream_t s) {
    if (d->act == GA3C_ACT_SILU) launch_kernels<T, VE, GA3C_ACT_SILU>(a, c, grad, s);
    else if (d->act == GA3C_ACT_RELU) launch_kernels<T, VE, GA3C_ACT_RELU>(a, c, grad, s);
    else launch_kernels<T, VE, GA3C_ACT_NONE>(a, c, grad, s);
}
void launch_all(const ga3c_norm_desc *d, const NormArgs &a, const Cut &c, bool grad, hipStream_t s) {
    if (d->dtype == GA3C_BF16) c.ve == 1 ? launch_act<bf16, 1>(d, a, c, grad, s) : c.ve == 2 ? launch_act<bf16, 2>(d, a, c, grad, s) : launch_act<bf16, 8>(d, a, c, grad, s);
    else c.ve == 1 ? launch_act<float, 1>(d, a, c, grad, s) : c.ve == 2 ? launch_act<float, 2>(d, a, c, grad, s) : launch_act<float, 4>(d, a, c, grad, s);
}
int hip_result(const char *who) {
    const hipError_t e = hipGetLastError();
    return e == hipSuccess ? GA3C_OK : call_fail(GA3C_EHIP, "%s: %s", who, hipGetErrorString(e));
}
// Elements of a vector that every tensor allows: 16 bytes (and vectors of four weights), two, or one.
int widest_vectors(const ga3c_norm_desc *d, std::initializer_list<const void *> tensors, std::initializer_list<int64_t> strides, const float *gamma, const float *beta) {
    const int size = d->dtype == GA3C_BF16 ? 2 : 4;
    uintptr_t bytes = 0;
    for (const void *p : tensors) bytes |= (uintptr_t)p;
    for (int64_t s : strides) bytes |= (uintptr_t)s * size;
    if (bytes % 16 == 0 && ((uintptr_t)gamma | (uintptr_t)beta) % 16 == 0) return 16 / size;
    return bytes % (2 * size) == 0 ? 2 : 1;
}
int check_cut(const ga3c_norm_desc *d, const Cut &c, int samples, const char *who) {
    if (c.chunks > 65535) return call_fail(GA3C_EINVAL, "%s: samples of too many positions", who);
    // threads of a launch are counted in 32 bits
    const int64_t groups = (int64_t)samples * d->groups, tiles = (int64_t)samples * c.tiles * c.threads;
    if ((c.rows ? groups * c.lg : c.wide ? groups * 256 : std::max(tiles, c.chunks > 1 ? groups * 64 : 0)) > UINT32_MAX - 1024)
        return call_fail(GA3C_EINVAL, "%s: too many samples for one call", who);
    return GA3C_OK;
}

}  // namespace
}  // namespace ga3c

using namespace ga3c;

extern "C" size_t ga3c_group_norm_workspace(const ga3c_norm_desc *d, int n_samples, int n_positions, int grad) {
    if (check(d, n_samples, n_positions, "ga3c_group_norm_workspace") != GA3C_OK || n_samples == 0) return 0;
    size_t most = 0;
    for (int vectors : {1, 2, 8}) {        // what the tensors allow is not known here
        const Cut c = cut_of(d, n_samples, n_positions, vectors, grad != 0);
        most = std::max(most, sums_floats(d, c, n_samples) + (grad ? partial_floats(d, c) : 0));
    }
    return sizeof(float) * most;
}

static int check_workspace(const ga3c_norm_desc *d, int samples, int positions, int grad, void *workspace, size_t bytes, const char *who) {
    const size_t need = ga3c_group_norm_workspace(d, samples, positions, grad);
    if (bytes < need) return call_fail(GA3C_EINVAL, "%s: workspace too small", who);
    if (need && (!workspace || (uintptr_t)workspace % 16)) return call_fail(GA3C_EINVAL, "%s: workspace null or not aligned to 16 bytes", who);
    return GA3C_OK;
}

extern "C" int ga3c_group_norm(const ga3c_norm_desc *d, const void *x, int64_t x_stride, const float *gamma, const float *beta, void *y,
                               int64_t y_stride, float *stats, int n_samples, int n_positions, void *workspace, size_t workspace_bytes,
                               void *stream) {
    const char *who = "ga3c_group_norm";
    int rc = check(d, n_samples, n_positions, who);
    if (rc != GA3C_OK || n_samples == 0) return rc;
    if ((rc = check_rows(x, x_stride, d, who)) != GA3C_OK || (rc = check_rows(y, y_stride, d, who)) != GA3C_OK) return rc;
    if (!gamma || !beta) return call_fail(GA3C_EINVAL, "%s: null gamma or beta", who);
    if ((uintptr_t)stats % 8) return call_fail(GA3C_EINVAL, "%s: stats not aligned to 8 bytes", who);
    if (x == y) return call_fail(GA3C_EINVAL, "%s: the result is the input", who);
    if ((rc = check_workspace(d, n_samples, n_positions, 0, workspace, workspace_bytes, who)) != GA3C_OK) return rc;
    const Cut c = cut_of(d, n_samples, n_positions, widest_vectors(d, {x, y}, {x_stride, y_stride}, gamma, beta), false);
    if ((rc = check_cut(d, c, n_samples, who)) != GA3C_OK) return rc;
    NormArgs a = args_of(d, c, n_samples, n_positions, workspace);
    a.x = x; a.xs = x_stride; a.y = y; a.ys = y_stride; a.gamma = gamma; a.beta = beta; a.stats = stats;
    launch_all(d, a, c, false, (hipStream_t)stream);
    return hip_result(who);
}

extern "C" int ga3c_group_norm_grad(const ga3c_norm_desc *d, const void *x, int64_t x_stride, const void *dy, int64_t dy_stride,
                                    const float *gamma, const float *beta, const float *stats, void *dx, int64_t dx_stride, float *dgamma,
                                    float *dbeta, int n_samples, int n_positions, void *workspace, size_t workspace_bytes, void *stream) {
    const char *who = "ga3c_group_norm_grad";
    int rc = check(d, n_samples, n_positions, who);
    if (rc != GA3C_OK) return rc;
    if (!dgamma || !dbeta) return call_fail(GA3C_EINVAL, "%s: null dgamma or dbeta", who);
    Cut c{};
    if (n_samples > 0) {
        if ((rc = check_rows(x, x_stride, d, who)) != GA3C_OK || (rc = check_rows(dy, dy_stride, d, who)) != GA3C_OK ||
            (rc = check_rows(dx, dx_stride, d, who)) != GA3C_OK) return rc;
        if (!gamma || !beta || !stats) return call_fail(GA3C_EINVAL, "%s: null gamma, beta or stats", who);
        if ((uintptr_t)stats % 8) return call_fail(GA3C_EINVAL, "%s: stats not aligned to 8 bytes", who);
        if (dx == x || dx == dy) return call_fail(GA3C_EINVAL, "%s: the result is an input", who);
        if ((rc = check_workspace(d, n_samples, n_positions, 1, workspace, workspace_bytes, who)) != GA3C_OK) return rc;
        c = cut_of(d, n_samples, n_positions, widest_vectors(d, {x, dy, dx}, {x_stride, dy_stride, dx_stride}, gamma, beta), true);
        if ((rc = check_cut(d, c, n_samples, who)) != GA3C_OK) return rc;
    }
    NormArgs a = args_of(d, c, n_samples, n_positions, workspace);
    a.x = x; a.xs = x_stride; a.dy = dy; a.dys = dy_stride; a.y = dx; a.ys = dx_stride; a.gamma = gamma; a.beta = beta; a.stats = (float *)stats;
    a.dgamma = dgamma; a.dbeta = dbeta;
    const hipStream_t s = (hipStream_t)stream;
    if (n_samples > 0) launch_all(d, a, c, true, s);
    launch(norm_weights_kernel, dim3((unsigned)((2 * (int64_t)a.channels + 63) / 64)), dim3(1024), 0, s, a);
    return hip_result(who);
}
