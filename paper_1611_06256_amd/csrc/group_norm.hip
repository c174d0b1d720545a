// Group norm with an activation, channels last, and its gradient: of maps, and (one position per sample, a group per head) of
// what an agent's memory reads out.
#include <hip/hip_runtime.h>
#include <math.h>

#include <algorithm>

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
    int samples, positions, channels, groups, act;
    float eps;
};

__device__ inline float activation(float z, int act) {
    if (act == GA3C_ACT_RELU) return z > 0.f ? z : 0.f;
    if (act == GA3C_ACT_SILU) return z / (1.f + expf(-z));
    return z;
}
__device__ inline float activation_slope(float z, int act) {
    if (act == GA3C_ACT_RELU) return z > 0.f ? 1.f : 0.f;
    if (act == GA3C_ACT_SILU) {
        const float s = 1.f / (1.f + expf(-z));
        return s * (1.f + z * (1.f - s));
    }
    return 1.f;
}

// Sum over the block's 256 threads, the same in all of them.
__device__ inline float block_sum(float v, float *sh) {
#pragma unroll
    for (int m = 32; m > 0; m /= 2) v += __shfl_xor(v, m);
    __syncthreads();
    if (threadIdx.x % 64 == 0) sh[threadIdx.x / 64] = v;
    __syncthreads();
    return sh[0] + sh[1] + sh[2] + sh[3];
}

// A block takes one group of one sample: mean, then the squares around it, then the result.
template <class T>
__global__ __launch_bounds__(256) void group_norm_kernel(const NormArgs a) {
    __shared__ float sh[4];
    const int sample = blockIdx.x, group = blockIdx.y, wide = a.channels / a.groups, c0 = group * wide;
    const T *x = (const T *)a.x + (int64_t)sample * a.positions * a.xs + c0;
    T *y = (T *)a.y + (int64_t)sample * a.positions * a.ys + c0;
    const int64_t m = (int64_t)a.positions * wide;
    float s = 0.f;
    for (int64_t e = threadIdx.x; e < m; e += 256) s += to_f32(x[e / wide * a.xs + e % wide]);
    const float mean = block_sum(s, sh) / (float)m;
    s = 0.f;
    for (int64_t e = threadIdx.x; e < m; e += 256) {
        const float d = to_f32(x[e / wide * a.xs + e % wide]) - mean;
        s += d * d;
    }
    const float rstd = 1.f / sqrtf(block_sum(s, sh) / (float)m + a.eps);
    for (int64_t e = threadIdx.x; e < m; e += 256) {
        const int64_t p = e / wide;
        const int c = (int)(e % wide);
        const float z = (to_f32(x[p * a.xs + c]) - mean) * rstd * a.gamma[c0 + c] + a.beta[c0 + c];
        y[p * a.ys + c] = from_f32<T>(activation(z, a.act));
    }
    if (a.stats && threadIdx.x == 0) {
        float *st = a.stats + 2 * ((int64_t)sample * a.groups + group);
        st[0] = mean; st[1] = rstd;
    }
}

// dx of one group of one sample.
template <class T>
__global__ __launch_bounds__(256) void group_norm_dx_kernel(const NormArgs a) {
    __shared__ float sh[4];
    const int sample = blockIdx.x, group = blockIdx.y, wide = a.channels / a.groups, c0 = group * wide;
    const T *x = (const T *)a.x + (int64_t)sample * a.positions * a.xs + c0, *dy = (const T *)a.dy + (int64_t)sample * a.positions * a.dys + c0;
    T *dx = (T *)a.y + (int64_t)sample * a.positions * a.ys + c0;
    const int64_t m = (int64_t)a.positions * wide;
    const float *st = a.stats + 2 * ((int64_t)sample * a.groups + group);
    const float mean = st[0], rstd = st[1];
    float s = 0.f, sx = 0.f;
    for (int64_t e = threadIdx.x; e < m; e += 256) {
        const int64_t p = e / wide;
        const int c = (int)(e % wide);
        const float xh = (to_f32(x[p * a.xs + c]) - mean) * rstd, g = a.gamma[c0 + c];
        const float d = to_f32(dy[p * a.dys + c]) * activation_slope(xh * g + a.beta[c0 + c], a.act) * g;
        s += d; sx += d * xh;
    }
    const float ma = block_sum(s, sh) / (float)m, mb = block_sum(sx, sh) / (float)m;
    for (int64_t e = threadIdx.x; e < m; e += 256) {
        const int64_t p = e / wide;
        const int c = (int)(e % wide);
        const float xh = (to_f32(x[p * a.xs + c]) - mean) * rstd, g = a.gamma[c0 + c];
        const float d = to_f32(dy[p * a.dys + c]) * activation_slope(xh * g + a.beta[c0 + c], a.act) * g;
        dx[p * a.ys + c] = from_f32<T>(rstd * (d - ma - xh * mb));
    }
}

// dgamma and dbeta of one channel per block, in a fixed order.
template <class T>
__global__ __launch_bounds__(256) void group_norm_dweights_kernel(const NormArgs a) {
    __shared__ float sh[4];
    const int c = blockIdx.x, group = c / (a.channels / a.groups);
    float s = 0.f, sx = 0.f;
    for (int64_t e = threadIdx.x; e < (int64_t)a.samples * a.positions; e += 256) {
        const float *st = a.stats + 2 * (e / a.positions * a.groups + group);
        const float xh = (to_f32(((const T *)a.x)[e * a.xs + c]) - st[0]) * st[1];
        const float d = to_f32(((const T *)a.dy)[e * a.dys + c]) * activation_slope(xh * a.gamma[c] + a.beta[c], a.act);
        s += d; sx += d * xh;
    }
    s = block_sum(s, sh); sx = block_sum(sx, sh);
    if (threadIdx.x == 0) { a.dbeta[c] = s; a.dgamma[c] = sx; }
}

// -------------------------------------------------------------------- host --

int check(const ga3c_norm_desc *d, int samples, int positions, const char *who) {
    if (!d) return call_fail(GA3C_EINVAL, "%s: null description", who);
    if (d->channels < 1 || d->groups < 1 || d->channels % d->groups) return call_fail(GA3C_EINVAL, "%s: %d channels are no %d equal groups", who, d->channels, d->groups);
    if (d->groups > 65535) return call_fail(GA3C_EINVAL, "%s: more than 65535 groups", who);
    if (d->dtype != GA3C_F32 && d->dtype != GA3C_BF16) return call_fail(GA3C_EINVAL, "%s: dtype must be GA3C_F32 or GA3C_BF16", who);
    if (d->act != GA3C_ACT_NONE && d->act != GA3C_ACT_RELU && d->act != GA3C_ACT_SILU) return call_fail(GA3C_EINVAL, "%s: unknown activation %d", who, d->act);
    if (!(d->eps >= 0.f) || !isfinite(d->eps)) return call_fail(GA3C_EINVAL, "%s: eps must be finite and not negative", who);
    if (samples < 0 || positions < 0) return call_fail(GA3C_EINVAL, "%s: negative count", who);
    if (samples > 0 && positions == 0) return call_fail(GA3C_EINVAL, "%s: samples without a position", who);
    return GA3C_OK;
}
int check_rows(const void *p, int64_t stride, const ga3c_norm_desc *d, const char *who) {
    if (!p) return call_fail(GA3C_EINVAL, "%s: null tensor", who);
    if ((uintptr_t)p % (d->dtype == GA3C_BF16 ? 2 : 4)) return call_fail(GA3C_EINVAL, "%s: tensor not aligned to its elements", who);
    if (stride < d->channels) return call_fail(GA3C_EINVAL, "%s: positions closer than their channels", who);
    return GA3C_OK;
}
NormArgs args_of(const ga3c_norm_desc *d, int samples, int positions) {
    NormArgs a{};
    a.samples = samples; a.positions = positions; a.channels = d->channels; a.groups = d->groups; a.act = d->act; a.eps = d->eps;
    return a;
}
int hip_result(const char *who) {
    const hipError_t e = hipGetLastError();
    return e == hipSuccess ? GA3C_OK : call_fail(GA3C_EHIP, "%s: %s", who, hipGetErrorString(e));
}

}  // namespace
}  // namespace ga3c

using namespace ga3c;

extern "C" size_t ga3c_group_norm_workspace(const ga3c_norm_desc *d, int n_samples, int n_positions) {
    (void)d; (void)n_samples; (void)n_positions;
    return 0;
}

extern "C" int ga3c_group_norm(const ga3c_norm_desc *d, const void *x, int64_t x_stride, const float *gamma, const float *beta, void *y,
                               int64_t y_stride, float *stats, int n_samples, int n_positions, void *workspace, size_t workspace_bytes,
                               void *stream) {
    const char *who = "ga3c_group_norm";
    int rc = check(d, n_samples, n_positions, who);
    if (rc != GA3C_OK || n_samples == 0) return rc;
    if ((rc = check_rows(x, x_stride, d, who)) != GA3C_OK || (rc = check_rows(y, y_stride, d, who)) != GA3C_OK) return rc;
    if (!gamma || !beta) return call_fail(GA3C_EINVAL, "%s: null gamma or beta", who);
    if (x == y) return call_fail(GA3C_EINVAL, "%s: the result is the input", who);
    if (workspace_bytes < ga3c_group_norm_workspace(d, n_samples, n_positions)) return call_fail(GA3C_EINVAL, "%s: workspace too small", who);
    (void)workspace;
    NormArgs a = args_of(d, n_samples, n_positions);
    a.x = x; a.xs = x_stride; a.y = y; a.ys = y_stride; a.gamma = gamma; a.beta = beta; a.stats = stats;
    const dim3 grid(n_samples, d->groups);
    launch(d->dtype == GA3C_BF16 ? group_norm_kernel<bf16> : group_norm_kernel<float>, grid, dim3(256), 0, (hipStream_t)stream, a);
    return hip_result(who);
}

extern "C" int ga3c_group_norm_grad(const ga3c_norm_desc *d, const void *x, int64_t x_stride, const void *dy, int64_t dy_stride,
                                    const float *gamma, const float *beta, const float *stats, void *dx, int64_t dx_stride, float *dgamma,
                                    float *dbeta, int n_samples, int n_positions, void *workspace, size_t workspace_bytes, void *stream) {
    const char *who = "ga3c_group_norm_grad";
    int rc = check(d, n_samples, n_positions, who);
    if (rc != GA3C_OK) return rc;
    if (!dgamma || !dbeta) return call_fail(GA3C_EINVAL, "%s: null dgamma or dbeta", who);
    if (n_samples > 0) {
        if ((rc = check_rows(x, x_stride, d, who)) != GA3C_OK || (rc = check_rows(dy, dy_stride, d, who)) != GA3C_OK ||
            (rc = check_rows(dx, dx_stride, d, who)) != GA3C_OK) return rc;
        if (!gamma || !beta || !stats) return call_fail(GA3C_EINVAL, "%s: null gamma, beta or stats", who);
        if (dx == x || dx == dy) return call_fail(GA3C_EINVAL, "%s: the result is an input", who);
    }
    if (workspace_bytes < ga3c_group_norm_workspace(d, n_samples, n_positions)) return call_fail(GA3C_EINVAL, "%s: workspace too small", who);
    (void)workspace;
    NormArgs a = args_of(d, n_samples, n_positions);
    a.x = x; a.xs = x_stride; a.dy = dy; a.dys = dy_stride; a.y = dx; a.ys = dx_stride; a.gamma = gamma; a.beta = beta; a.stats = (float *)stats;
    a.dgamma = dgamma; a.dbeta = dbeta;
    const hipStream_t s = (hipStream_t)stream;
    const bool b = d->dtype == GA3C_BF16;
    if (n_samples > 0) launch(b ? group_norm_dx_kernel<bf16> : group_norm_dx_kernel<float>, dim3(n_samples, d->groups), dim3(256), 0, s, a);
    launch(b ? group_norm_dweights_kernel<bf16> : group_norm_dweights_kernel<float>, dim3(d->channels), dim3(256), 0, s, a);
    return hip_result(who);
}
