// Attention with a decay for each head over packed segments, its gradient, and its form for single tokens: the memory of an
// agent.  decay_attention.hpp has the recurrence that every pass here computes.
#include <hip/hip_runtime.h>
#include <math.h>
#include <string.h>

#include <algorithm>

#include "call_error.hpp"
#include "decay_attention.hpp"
#include "launch.hpp"
#include "tensor_types.hpp"

namespace ga3c {
namespace {

// Tokens of segment `seg`, kept within the arrays whatever the table says.
__device__ inline void segment_tokens(const DecayPass &p, int seg, int &first, int &end) {
    if (p.seg_start) {
        first = min(max(p.seg_start[seg], 0), p.n_tokens);
        end = min(max(p.seg_start[seg + 1], first), p.n_tokens);
    } else {
        first = seg * p.len;
        end = first + p.len;
    }
}

template <class T>
__device__ inline const T *at(const DecayView &v, int token, int head) { return (const T *)v.data + token * v.token + head * v.head; }

// Token by token.  A block takes DR_ROWS / LPR... rows of one segment's state in one head: LPR lanes share a row, four (or twice
// four) columns each, and a lane has DR_RPL rows.
constexpr int DR_RPL = 4;
template <class T, int LPR, int CV>
__global__ __launch_bounds__(256) void decay_recurrent_kernel(const DecayPass p, int vec) {
    constexpr int RW = 64 / LPR, ROWS = 4 * RW * DR_RPL;
    const int seg = blockIdx.x, head = blockIdx.y, lane = threadIdx.x % 64, wave = threadIdx.x / 64;
    const int heads = gridDim.y, c0 = lane % LPR * 4, r0 = blockIdx.z * ROWS + wave * RW * DR_RPL + lane / LPR;
    const float d = p.decay[head];
    int first, end;
    segment_tokens(p, seg, first, end);
    const size_t state = ((size_t)seg * heads + head) * p.rows * p.cols;
    float4 x[DR_RPL][CV];
#pragma unroll
    for (int i = 0; i < DR_RPL; ++i)
#pragma unroll
        for (int v = 0; v < CV; ++v) {
            const int r = r0 + i * RW, c = c0 + v * 4 * LPR;
            float e[4] = {0.f, 0.f, 0.f, 0.f};
            if (p.x_in && r < p.rows)
#pragma unroll
                for (int k = 0; k < 4; ++k)
                    if (c + k < p.cols) e[k] = p.x_in[state + (p.x_turned ? (size_t)(c + k) * p.rows + r : (size_t)r * p.cols + c + k)];
            x[i][v] = float4{e[0], e[1], e[2], e[3]};
        }
    for (int n = first; n < end; ++n) {
        const int t = p.back ? end - 1 - (n - first) : n;
        const bool start = p.starts && p.starts[t];
        float keep = p.back ? 1.f : start ? 0.f : d;
        float4 col[CV], by[CV];
#pragma unroll
        for (int v = 0; v < CV; ++v) {
            const int c = c0 + v * 4 * LPR;
            col[v] = load4(at<T>(p.col, t, head) + c, p.cols - c, vec);
            by[v] = load4(at<T>(p.by, t, head) + c, p.cols - c, vec);
        }
#pragma unroll
        for (int i = 0; i < DR_RPL; ++i) {
            const int r = r0 + i * RW;
            const float row = r < p.rows ? p.col_scale * to_f32(at<T>(p.row, t, head)[r]) : 0.f;
            float sum = 0.f;
#pragma unroll
            for (int v = 0; v < CV; ++v) {
                float4 &y = x[i][v];
                if (keep == 0.f) y = float4{0.f, 0.f, 0.f, 0.f};        // whatever was in it
                y.x = keep * y.x + row * col[v].x; y.y = keep * y.y + row * col[v].y;
                y.z = keep * y.z + row * col[v].z; y.w = keep * y.w + row * col[v].w;
                sum += y.x * by[v].x + y.y * by[v].y + y.z * by[v].z + y.w * by[v].w;
                if (p.back) {
                    const float f = start ? 0.f : d;
                    y = f == 0.f ? float4{0.f, 0.f, 0.f, 0.f} : float4{f * y.x, f * y.y, f * y.z, f * y.w};
                }
            }
#pragma unroll
            for (int m = LPR / 2; m > 0; m /= 2) sum += __shfl_xor(sum, m);
            if (lane % LPR == 0 && r < p.rows) ((T *)p.out.data)[t * p.out.token + head * p.out.head + r] = from_f32<T>(p.out_scale * sum);
        }
    }
    if (!p.x_out) return;
#pragma unroll
    for (int i = 0; i < DR_RPL; ++i)
#pragma unroll
        for (int v = 0; v < CV; ++v) {
            const int r = r0 + i * RW, c = c0 + v * 4 * LPR;
            const float e[4] = {x[i][v].x, x[i][v].y, x[i][v].z, x[i][v].w};
            if (r < p.rows)
#pragma unroll
                for (int k = 0; k < 4; ++k)
                    if (c + k < p.cols) p.x_out[state + (p.x_turned ? (size_t)(c + k) * p.rows + r : (size_t)r * p.cols + c + k)] = e[k];
        }
}

// One token of each agent.  The state of entry i is row slots[i] of the states (i without slots), read, advanced and written back;
// a slot outside them stands for a state of zeros that is not kept.  Entries that name one slot are consecutive tokens of it, in
// the order of their numbers: the first of them takes the others along, so that nobody else touches the slot.
struct DecayStep {
    DecayView q, k, v, out;
    int key, value;
    const int32_t *slots;
    const uint8_t *starts;
    float *states;
    int n, n_slots;
    float scale;
    float decay[GA3C_MAX_HEADS];
};
// The first entry from `from` on with this slot, n if there is none; the same in all threads of the block.
__device__ inline int next_of_slot(const DecayStep &p, int slot, int from, int to, int *lowest) {
    __syncthreads();
    if (threadIdx.x == 0) *lowest = p.n;
    __syncthreads();
    int mine = p.n;
    for (int j = from + threadIdx.x; j < to; j += 256)
        if (p.slots[j] == slot) { mine = j; break; }
    if (mine < p.n) atomicMin(lowest, mine);
    __syncthreads();
    return *lowest;
}

template <class T, int LPR, int CV>
__global__ __launch_bounds__(256) void decay_step_kernel(const DecayStep p, int vec) {
    constexpr int RW = 64 / LPR, ROWS = 4 * RW * DR_RPL;
    __shared__ int lowest;
    const int head = blockIdx.y, lane = threadIdx.x % 64, wave = threadIdx.x / 64, heads = gridDim.y;
    const int c0 = lane % LPR * 4, r0 = blockIdx.z * ROWS + wave * RW * DR_RPL + lane / LPR;
    const int slot = p.slots ? p.slots[blockIdx.x] : (int)blockIdx.x;
    const bool kept = slot >= 0 && slot < p.n_slots;
    if (p.slots && kept && next_of_slot(p, slot, 0, blockIdx.x, &lowest) < p.n) return;
    const float d = p.decay[head];
    float *state = p.states + ((size_t)(kept ? slot : 0) * heads + head) * p.value * p.key;
    float4 x[DR_RPL][CV];
#pragma unroll
    for (int i = 0; i < DR_RPL; ++i)
#pragma unroll
        for (int v = 0; v < CV; ++v) {
            const int r = r0 + i * RW, c = c0 + v * 4 * LPR;
            x[i][v] = load4(state + (size_t)r * p.key + c, kept && r < p.value ? p.key - c : 0, p.key % 4 == 0 && vec);
        }
    for (int t = blockIdx.x; t < p.n; t = p.slots && kept ? next_of_slot(p, slot, t + 1, p.n, &lowest) : p.n) {
        const float keep = p.starts && p.starts[t] ? 0.f : d;
        float4 col[CV], by[CV];
#pragma unroll
        for (int v = 0; v < CV; ++v) {
            const int c = c0 + v * 4 * LPR;
            col[v] = load4(at<T>(p.k, t, head) + c, p.key - c, vec);
            by[v] = load4(at<T>(p.q, t, head) + c, p.key - c, vec);
        }
#pragma unroll
        for (int i = 0; i < DR_RPL; ++i) {
            const int r = r0 + i * RW;
            const float row = r < p.value ? to_f32(at<T>(p.v, t, head)[r]) : 0.f;
            float sum = 0.f;
#pragma unroll
            for (int v = 0; v < CV; ++v) {
                float4 &y = x[i][v];
                if (keep == 0.f) y = float4{0.f, 0.f, 0.f, 0.f};
                y.x = keep * y.x + row * col[v].x; y.y = keep * y.y + row * col[v].y;
                y.z = keep * y.z + row * col[v].z; y.w = keep * y.w + row * col[v].w;
                sum += y.x * by[v].x + y.y * by[v].y + y.z * by[v].z + y.w * by[v].w;
            }
#pragma unroll
            for (int m = LPR / 2; m > 0; m /= 2) sum += __shfl_xor(sum, m);
            if (lane % LPR == 0 && r < p.value) ((T *)p.out.data)[t * p.out.token + head * p.out.head + r] = from_f32<T>(p.scale * sum);
        }
    }
    if (!kept) return;
#pragma unroll
    for (int i = 0; i < DR_RPL; ++i)
#pragma unroll
        for (int v = 0; v < CV; ++v) {
            const int r = r0 + i * RW, c = c0 + v * 4 * LPR;
            if (r >= p.value) continue;
            float *to = state + (size_t)r * p.key + c;
            if (p.key % 4 == 0 && vec && c + 4 <= p.key) { *(float4 *)to = x[i][v]; continue; }
            const float e[4] = {x[i][v].x, x[i][v].y, x[i][v].z, x[i][v].w};
#pragma unroll
            for (int k = 0; k < 4; ++k)
                if (c + k < p.key) to[k] = e[k];
        }
}

// -------------------------------------------------------------------- host --

// Rows of a view that four elements at a time can be read from.
template <class T>
bool rows_of_four(const DecayView &v) { return (uintptr_t)v.data % (4 * sizeof(T)) == 0 && v.token % 4 == 0 && v.head % 4 == 0; }

template <class F>
hipError_t by_columns(int cols, F go) {      // LPR, CV
    if (cols <= 16) return go(std::integral_constant<int, 4>(), std::integral_constant<int, 1>());
    if (cols <= 32) return go(std::integral_constant<int, 8>(), std::integral_constant<int, 1>());
    if (cols <= 64) return go(std::integral_constant<int, 16>(), std::integral_constant<int, 1>());
    return go(std::integral_constant<int, 16>(), std::integral_constant<int, 2>());
}

template <class T>
hipError_t run_pass(const DecayPass &p, int heads, hipStream_t s) {
    const int vec = rows_of_four<T>(p.col) && rows_of_four<T>(p.by);
    return by_columns(p.cols, [&](auto lpr, auto cv) {
        constexpr int ROWS = 4 * (64 / lpr.value) * DR_RPL;
        launch(decay_recurrent_kernel<T, lpr.value, cv.value>, dim3(p.n_segments, heads, (p.rows + ROWS - 1) / ROWS), dim3(256), 0, s, p, vec);
        return hipGetLastError();
    });
}

int check_desc(const ga3c_decay_desc *d, const char *who) {
    if (!d || !d->decay) return call_fail(GA3C_EINVAL, "%s: null description", who);
    if (d->n_heads < 1 || d->n_heads > GA3C_MAX_HEADS) return call_fail(GA3C_EINVAL, "%s: n_heads must be 1..%d", who, GA3C_MAX_HEADS);
    for (int n : {d->key_dim, d->value_dim})
        if (n < 1 || n > GA3C_MAX_HEAD_DIM) return call_fail(GA3C_EINVAL, "%s: key_dim and value_dim must be 1..%d", who, GA3C_MAX_HEAD_DIM);
    if (d->dtype != GA3C_F32 && d->dtype != GA3C_BF16) return call_fail(GA3C_EINVAL, "%s: dtype must be GA3C_F32 or GA3C_BF16", who);
    if (!isfinite(d->scale)) return call_fail(GA3C_EINVAL, "%s: scale must be finite", who);
    for (int h = 0; h < d->n_heads; ++h)
        if (!(d->decay[h] >= 0.f && d->decay[h] <= 1.f)) return call_fail(GA3C_EINVAL, "%s: decay of head %d outside [0, 1]", who, h);
    return GA3C_OK;
}
// Whether the elements of an output all have places of their own.
bool apart(const ga3c_heads &v, int n, int heads, int dim) {
    const int64_t t = n > 1 ? v.token_stride : INT64_MAX, h = heads > 1 ? v.head_stride : INT64_MAX;
    if (t < dim || h < dim) return false;
    return n <= 1 || heads <= 1 || t >= h * (heads - 1) + dim || h >= t * (n - 1) + dim;
}
int check_views(const ga3c_heads *const *in, int n_in, const ga3c_heads *const *out, const int *out_dims, int n_out, int n, int heads, size_t size, const char *who) {
    for (int i = 0; i < n_in; ++i) {
        if (!in[i] || !in[i]->data) return call_fail(GA3C_EINVAL, "%s: null tensor", who);
        if ((uintptr_t)in[i]->data % size) return call_fail(GA3C_EINVAL, "%s: tensor not aligned to its elements", who);
        if (in[i]->token_stride < 0 || in[i]->head_stride < 0) return call_fail(GA3C_EINVAL, "%s: negative stride", who);
    }
    for (int i = 0; i < n_out; ++i) {
        if (!out[i] || !out[i]->data) return call_fail(GA3C_EINVAL, "%s: null tensor", who);
        if ((uintptr_t)out[i]->data % size) return call_fail(GA3C_EINVAL, "%s: tensor not aligned to its elements", who);
        if (!apart(*out[i], n, heads, out_dims[i])) return call_fail(GA3C_EINVAL, "%s: strides make rows of an output overlap", who);
        for (int k = 0; k < n_in; ++k)
            if (out[i]->data == in[k]->data) return call_fail(GA3C_EINVAL, "%s: an output is one of the inputs", who);
        for (int k = 0; k < i; ++k)
            if (out[i]->data == out[k]->data) return call_fail(GA3C_EINVAL, "%s: two outputs at one place", who);
    }
    return GA3C_OK;
}
int check_segments(const int32_t *seg_start, int n_segments, int n_tokens, const char *who) {
    if (n_segments < 0 || n_tokens < 0) return call_fail(GA3C_EINVAL, "%s: negative count", who);
    if (n_segments == 0 && n_tokens > 0) return call_fail(GA3C_EINVAL, "%s: tokens without a segment", who);
    if (!seg_start && n_segments > 0 && n_tokens % n_segments) return call_fail(GA3C_EINVAL, "%s: %d tokens are no %d equal segments", who, n_tokens, n_segments);
    return GA3C_OK;
}
bool overlap(const void *a, const void *b, size_t bytes) {
    return a && b && (uintptr_t)a < (uintptr_t)b + bytes && (uintptr_t)b < (uintptr_t)a + bytes;
}
DecayView view(const ga3c_heads *h) { return h ? DecayView{h->data, h->token_stride, h->head_stride} : DecayView{nullptr, 0, 0}; }

DecayPass pass_of(const ga3c_decay_desc *d, const int32_t *seg_start, const uint8_t *starts, int n_segments, int n_tokens) {
    DecayPass p;
    memset(&p, 0, sizeof p);
    p.seg_start = seg_start; p.starts = starts; p.n_segments = n_segments; p.n_tokens = n_tokens;
    p.len = n_segments > 0 ? n_tokens / n_segments : 0;
    p.out_scale = d->scale; p.col_scale = 1.f;
    memcpy(p.decay, d->decay, sizeof(float) * d->n_heads);
    return p;
}
hipError_t run(const ga3c_decay_desc *d, const DecayPass &p, hipStream_t s) {
    return d->dtype == GA3C_BF16 ? run_pass<bf16>(p, d->n_heads, s) : run_pass<float>(p, d->n_heads, s);
}
int hip_result(hipError_t e, const char *who) { return e == hipSuccess ? GA3C_OK : call_fail(GA3C_EHIP, "%s: %s", who, hipGetErrorString(e)); }

}  // namespace
}  // namespace ga3c

using namespace ga3c;

extern "C" size_t ga3c_decay_attention_workspace(const ga3c_decay_desc *d, int n_segments, int n_tokens) {
    (void)d; (void)n_segments; (void)n_tokens;
    return 0;
}

extern "C" int ga3c_decay_attention(const ga3c_decay_desc *d, const ga3c_heads *q, const ga3c_heads *k, const ga3c_heads *v,
                                    const ga3c_heads *out, const int32_t *seg_start, const uint8_t *starts, int n_segments, int n_tokens,
                                    const float *state_in, float *state_out, void *workspace, size_t workspace_bytes, void *stream) {
    const char *who = "ga3c_decay_attention";
    int rc = check_desc(d, who);
    if (rc == GA3C_OK) rc = check_segments(seg_start, n_segments, n_tokens, who);
    if (rc != GA3C_OK || n_segments == 0) return rc;
    const size_t size = d->dtype == GA3C_BF16 ? 2 : 4, state = sizeof(float) * n_segments * d->n_heads * d->key_dim * d->value_dim;
    if (n_tokens > 0) {
        const ga3c_heads *in[] = {q, k, v}, *to[] = {out};
        const int dims[] = {d->value_dim};
        rc = check_views(in, 3, to, dims, 1, n_tokens, d->n_heads, size, who);
        if (rc != GA3C_OK) return rc;
    }
    if (overlap(state_in, state_out, state)) return call_fail(GA3C_EINVAL, "%s: state_out lies over state_in", who);
    if (workspace_bytes < ga3c_decay_attention_workspace(d, n_segments, n_tokens)) return call_fail(GA3C_EINVAL, "%s: workspace too small", who);
    (void)workspace;
    DecayPass p = pass_of(d, seg_start, starts, n_segments, n_tokens);
    p.row = view(v); p.col = view(k); p.by = view(q); p.out = view(out);
    p.rows = d->value_dim; p.cols = d->key_dim;
    p.x_in = state_in; p.x_out = state_out;
    return hip_result(run(d, p, (hipStream_t)stream), who);
}

extern "C" int ga3c_decay_attention_grad(const ga3c_decay_desc *d, const ga3c_heads *q, const ga3c_heads *k, const ga3c_heads *v,
                                         const ga3c_heads *dout, const ga3c_heads *dq, const ga3c_heads *dk, const ga3c_heads *dv,
                                         const int32_t *seg_start, const uint8_t *starts, int n_segments, int n_tokens, const float *state_in,
                                         const float *dstate_out, float *dstate_in, void *workspace, size_t workspace_bytes, void *stream) {
    const char *who = "ga3c_decay_attention_grad";
    int rc = check_desc(d, who);
    if (rc == GA3C_OK) rc = check_segments(seg_start, n_segments, n_tokens, who);
    if (rc != GA3C_OK || n_segments == 0) return rc;
    const size_t size = d->dtype == GA3C_BF16 ? 2 : 4, state = sizeof(float) * n_segments * d->n_heads * d->key_dim * d->value_dim;
    if (n_tokens > 0) {
        const ga3c_heads *in[] = {q, k, v, dout}, *to[] = {dq, dk, dv};
        const int dims[] = {d->key_dim, d->key_dim, d->value_dim};
        rc = check_views(in, 4, to, dims, 3, n_tokens, d->n_heads, size, who);
        if (rc != GA3C_OK) return rc;
    }
    if (overlap(state_in, dstate_in, state) || overlap(dstate_out, dstate_in, state)) return call_fail(GA3C_EINVAL, "%s: dstate_in lies over an input", who);
    if (workspace_bytes < ga3c_decay_attention_workspace(d, n_segments, n_tokens)) return call_fail(GA3C_EINVAL, "%s: workspace too small", who);
    (void)workspace;
    const hipStream_t s = (hipStream_t)stream;
    DecayPass p = pass_of(d, seg_start, starts, n_segments, n_tokens);
    // dq: the states in front of the tokens once more, read out by dout
    p.row = view(k); p.col = view(v); p.by = view(dout); p.out = view(dq);
    p.rows = d->key_dim; p.cols = d->value_dim; p.x_turned = 1; p.x_in = state_in; p.x_out = nullptr;
    hipError_t e = run(d, p, s);
    // the gradient of the state behind each token, read out by v and by k
    p.back = 1; p.out_scale = 1.f; p.col_scale = d->scale;
    p.x_in = dstate_out;
    p.row = view(q); p.col = view(dout); p.by = view(v); p.out = view(dk);
    if (e == hipSuccess) e = run(d, p, s);
    p.rows = d->value_dim; p.cols = d->key_dim; p.x_turned = 0; p.x_out = dstate_in;
    p.row = view(dout); p.col = view(q); p.by = view(k); p.out = view(dv);
    if (e == hipSuccess) e = run(d, p, s);
    return hip_result(e, who);
}

extern "C" int ga3c_decay_attention_step(const ga3c_decay_desc *d, const ga3c_heads *q, const ga3c_heads *k, const ga3c_heads *v,
                                         const ga3c_heads *out, const int32_t *slots, const uint8_t *starts, int n, float *states, int n_slots,
                                         void *stream) {
    const char *who = "ga3c_decay_attention_step";
    int rc = check_desc(d, who);
    if (rc != GA3C_OK) return rc;
    if (n < 0 || n_slots < 0) return call_fail(GA3C_EINVAL, "%s: negative count", who);
    if (n == 0) return GA3C_OK;
    if (!slots && n > n_slots) return call_fail(GA3C_EINVAL, "%s: %d tokens for %d states", who, n, n_slots);
    if (!states) return call_fail(GA3C_EINVAL, "%s: null states", who);
    const ga3c_heads *in[] = {q, k, v}, *to[] = {out};
    const int dims[] = {d->value_dim};
    rc = check_views(in, 3, to, dims, 1, n, d->n_heads, d->dtype == GA3C_BF16 ? 2 : 4, who);
    if (rc != GA3C_OK) return rc;
    DecayStep p;
    memset(&p, 0, sizeof p);
    p.q = view(q); p.k = view(k); p.v = view(v); p.out = view(out);
    p.key = d->key_dim; p.value = d->value_dim; p.slots = slots; p.starts = starts; p.states = states; p.n = n; p.n_slots = n_slots;
    p.scale = d->scale;
    memcpy(p.decay, d->decay, sizeof(float) * d->n_heads);
    const hipError_t e = by_columns(p.key, [&](auto lpr, auto cv) {
        constexpr int ROWS = 4 * (64 / lpr.value) * DR_RPL;
        const dim3 grid(n, d->n_heads, (p.value + ROWS - 1) / ROWS);
        const bool states4 = (uintptr_t)states % 16 == 0;
        if (d->dtype == GA3C_BF16)
            launch(decay_step_kernel<bf16, lpr.value, cv.value>, grid, dim3(256), 0, (hipStream_t)stream, p, (int)(states4 && rows_of_four<bf16>(p.k) && rows_of_four<bf16>(p.q)));
        else
            launch(decay_step_kernel<float, lpr.value, cv.value>, grid, dim3(256), 0, (hipStream_t)stream, p, (int)(states4 && rows_of_four<float>(p.k) && rows_of_four<float>(p.q)));
        return hipGetLastError();
    });
    return hip_result(e, who);
}
