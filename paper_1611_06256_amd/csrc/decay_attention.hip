// Attention with a decay for each head over packed segments, its gradient, and its form for single tokens: the memory of an
// agent.  decay_attention.hpp has the recurrence that every pass here computes.
#include <hip/hip_runtime.h>
#include <math.h>
#include <string.h>

#include <algorithm>
#include <type_traits>

#include "call_error.hpp"
#include "decay_attention.hpp"
#include "launch.hpp"
#include "tensor_types.hpp"

namespace ga3c {
namespace {

// Tokens of segment `seg`, kept within the arrays whatever the table says.
__device__ inline void segment_tokens(const DecayJob &p, int seg, int &first, int &end) {
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

// ----------------------------------------------------------------- token by token --
//
// A wavefront takes RPL * 64 / LPR rows of one segment's state in one head: LPR lanes share a row, four columns each (or twice
// four), and a lane has RPL rows.  Bound by the latency of memory: the tokens come eight (or four) at a time, so that those of a
// segment of an update are on their way together.  512 segments of up to 5 tokens, 4 heads of 16 and 32 fp32, states in and out:
// 9.8 us (12 MB, 1.2 TB/s), the three passes of the gradient 22.8 in one launch.
// Sum over LPR neighbouring lanes, the same in all of them: lanes trade within fours, then eight and sixteen mirrored, without LDS.
template <int HOW>
__device__ inline float traded(float v) { return v + __int_as_float(__builtin_amdgcn_mov_dpp(__float_as_int(v), HOW, 0xf, 0xf, true)); }
template <int LPR>
__device__ inline float row_sum(float v) {
    v = traded<0x4e>(traded<0xb1>(v));        // lane ^ 1, lane ^ 2
    if (LPR >= 8) v = traded<0x141>(v);       // 7 - lane of eight
    if (LPR >= 16) v = traded<0x140>(v);      // 15 - lane of sixteen
    return v;
}
template <int RPL, int CV>
struct Rows {
    float4 x[RPL][CV];
    // one token: keep * x + row col^T, read out by `by`; the sums over a row are the same in its LPR lanes
    template <int LPR>
    __device__ void take(float keep, const float (&row)[RPL], const float4 (&col)[CV], const float4 (&by)[CV], float (&sum)[RPL]) {
#pragma unroll
        for (int i = 0; i < RPL; ++i) {
            sum[i] = 0.f;
#pragma unroll
            for (int v = 0; v < CV; ++v) {
                float4 &y = x[i][v];
                if (keep == 0.f) y = float4{0.f, 0.f, 0.f, 0.f};        // whatever was in it
                y.x = keep * y.x + row[i] * col[v].x; y.y = keep * y.y + row[i] * col[v].y;
                y.z = keep * y.z + row[i] * col[v].z; y.w = keep * y.w + row[i] * col[v].w;
                sum[i] += y.x * by[v].x + y.y * by[v].y + y.z * by[v].z + y.w * by[v].w;
            }
            sum[i] = row_sum<LPR>(sum[i]);
        }
    }
    __device__ void fade(float f) {
#pragma unroll
        for (int i = 0; i < RPL; ++i)
#pragma unroll
            for (int v = 0; v < CV; ++v) {
                float4 &y = x[i][v];
                y = f == 0.f ? float4{0.f, 0.f, 0.f, 0.f} : float4{f * y.x, f * y.y, f * y.z, f * y.w};
            }
    }
};

template <class T, int LPR, int CV, int RPL>
__global__ __launch_bounds__(256) void decay_recurrent_kernel(const DecayJob job, int slabs) {
    constexpr int RW = 64 / LPR;
    const DecayPass &p = job.pass[blockIdx.z];
    const int unit = __builtin_amdgcn_readfirstlane(blockIdx.x * 4 + threadIdx.x / 64), lane = threadIdx.x % 64;
    const int seg = unit / slabs, head = blockIdx.y, heads = gridDim.y, c0 = lane % LPR * 4, r0 = unit % slabs * RW * RPL + lane / LPR;
    if (seg >= job.n_segments) return;
    int first, end;
    segment_tokens(job, seg, first, end);
    if (end - first > job.brief) return;
    const int vec = (((uintptr_t)p.col.data | (uintptr_t)p.by.data) % (4 * sizeof(T)) == 0) &&
                    ((p.col.token | p.col.head | p.by.token | p.by.head) % 4 == 0);
    const size_t state = ((size_t)seg * heads + head) * p.rows * p.cols;
    const bool turned = p.turned, back = p.back;
    const int row_step = turned ? 1 : p.cols, col_step = turned ? p.rows : 1;
    const float d = job.decay[head];
    Rows<RPL, CV> s;
    const bool quads = !turned && p.cols % 4 == 0 && ((uintptr_t)p.x_in | (uintptr_t)p.x_out) % 16 == 0;
#pragma unroll
    for (int i = 0; i < RPL; ++i)
#pragma unroll
        for (int v = 0; v < CV; ++v) {
            const int r = r0 + i * RW, c = c0 + v * 4 * LPR;
            float4 e{0.f, 0.f, 0.f, 0.f};
            if (p.x_in && r < p.rows) {
                const float *x = p.x_in + state + (uint32_t)(r * row_step + c * col_step);
                if (quads) {
                    if (c < p.cols) e = load4(x, 4, true);
                } else {
                    if (c < p.cols) e.x = x[0];
                    if (c + 1 < p.cols) e.y = x[col_step];
                    if (c + 2 < p.cols) e.z = x[2 * col_step];
                    if (c + 3 < p.cols) e.w = x[3 * col_step];
                }
            }
            s.x[i][v] = e;
        }
    constexpr int TOGETHER = CV == 1 ? 8 : 4;
    for (int n = first; n < end; n += TOGETHER) {
        float4 col[TOGETHER][CV], by[TOGETHER][CV];
        float row[TOGETHER][RPL];
        int starts = 0;
#pragma unroll
        for (int k = 0; k < TOGETHER; ++k) {
            const int pos = min(n + k, end - 1), t = back ? end - 1 - (pos - first) : pos;
            const T *pc = at<T>(p.col, t, head), *pb = at<T>(p.by, t, head), *pr = at<T>(p.row, t, head);
#pragma unroll
            for (int v = 0; v < CV; ++v) {
                const int c = c0 + v * 4 * LPR;
                col[k][v] = load4(pc + c, p.cols - c, vec);
                by[k][v] = load4(pb + c, p.cols - c, vec);
            }
#pragma unroll
            for (int i = 0; i < RPL; ++i) row[k][i] = r0 + i * RW < p.rows ? to_f32(pr[r0 + i * RW]) : 0.f;
            if (job.starts) starts |= (job.starts[t] != 0) << k;
        }
#pragma unroll
        for (int k = 0; k < TOGETHER; ++k) {
            if (n + k >= end) break;
            const int t = back ? end - 1 - (n + k - first) : n + k;
            const bool start = starts >> k & 1;
            float sum[RPL];
#pragma unroll
            for (int i = 0; i < RPL; ++i) row[k][i] *= p.col_scale;
            s.template take<LPR>(back ? 1.f : start ? 0.f : d, row[k], col[k], by[k], sum);
            if (back) s.fade(start ? 0.f : d);
            T *out = (T *)p.out.data + t * p.out.token + head * p.out.head;
            if (lane % LPR == 0)
#pragma unroll
                for (int i = 0; i < RPL; ++i)
                    if (r0 + i * RW < p.rows) out[r0 + i * RW] = from_f32<T>(p.out_scale * sum[i]);
        }
    }
    if (!p.x_out) return;
#pragma unroll
    for (int i = 0; i < RPL; ++i)
#pragma unroll
        for (int v = 0; v < CV; ++v) {
            const int r = r0 + i * RW, c = c0 + v * 4 * LPR;
            if (r >= p.rows) continue;
            const float4 e = s.x[i][v];
            float *x = p.x_out + state + (uint32_t)(r * row_step + c * col_step);
            if (quads) {
                if (c < p.cols) *(float4 *)x = e;
            } else {
                if (c < p.cols) x[0] = e.x;
                if (c + 1 < p.cols) x[col_step] = e.y;
                if (c + 2 < p.cols) x[2 * col_step] = e.z;
                if (c + 3 < p.cols) x[3 * col_step] = e.w;
            }
        }
}

// ---------------------------------------------------------------- chunked form --
//
// A block takes a span of one segment in one head, tile by tile of C positions (in the order of the pass).  With w(e) = decay^e,
// positions i, j of the tile, n of them, and `fresh` the latest start at or before i:
//     P[i][j] = (by_i . col_j) w(i - j)            for fresh <= j <= i, else 0
//     out_i   = sum_j P[i][j] row_j + w(i + a) X by_i     the second term if no start is at or before i (a = 1, backward 0)
//     X      <- w(n) X + sum_j row_j col_j w(n - j - a)   likewise
// All four products run on the matrix instruction.  X stays in the accumulators, whose layout (four neighbouring columns of a
// row per lane) is that of the left operand of X by_i, so it never passes through LDS; a wavefront has sixteen of its rows.
// The tiles go straight from memory to LDS, the next one while this one is worked on; contractions over positions read them
// across their rows (an instruction of its own for 16 bits, single numbers for 32).
// 16384 tokens bf16, 8 heads of 128, in 32 spans: states of the spans 37 us, states between them 10, outputs 55 (151 MB, 2.7 TB/s; half of
// a wavefront's life is waiting, the matrix units are busy a sixth of the time).  Gradient of 4096 tokens fp32, 4 heads of 128, in 16
// spans: 32, 6 and 59 (the fp32 instruction, on 192 of 256 compute units: 3.6 GFLOP there, 61 TFLOP/s; 16 spans more would cost what
// they bring).
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef __bf16 bf16x4 __attribute__((ext_vector_type(4)));
typedef short s16x4 __attribute__((ext_vector_type(4)));

// A fragment is 16 bytes of one lane: KB numbers of the contraction in the wavefront, VE of them in the lane.  With bfloat16 tensors what
// is computed on the way (weighted scores, rows with their decay, the state) is fp32, and goes into a product as several bfloat16 terms:
// a row with its decay as ROW_TERMS, all of its 24 bits, because states are fp32; a score and a state that is read out as two, which
// miss 2^-16 of it where the result's own rounding misses 2^-8.  (With one term for rows and scores the errors were 2.3e-3 instead of
// the result's rounding, 1.7e-3; 16384 tokens, 8 heads of 128, took 80 us a call, with these 94.)
template <class T> struct Tile;
template <> struct Tile<float> {
    static constexpr int KB = 16, VE = 4, ROW_TERMS = 1, SCORE_TERMS = 1;
    typedef f32x4 Frag;
    typedef f32x4 Quad;
    __device__ static f32x4 mma(Frag a, Frag b, f32x4 c) {
#pragma unroll
        for (int e = 0; e < 4; ++e) c = __builtin_amdgcn_mfma_f32_16x16x4f32(a[e], b[e], c, 0, 0, 0);
        return c;
    }
    __device__ static Quad quad(f32x4 v) { return v; }
};
template <> struct Tile<bf16> {
    static constexpr int KB = 32, VE = 8, ROW_TERMS = 3, SCORE_TERMS = 2;
    typedef bf16x8 Frag;
    typedef bf16x4 Quad;
    __device__ static f32x4 mma(Frag a, Frag b, f32x4 c) { return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0); }
    __device__ static Quad quad(f32x4 v) { return __builtin_convertvector(v, bf16x4); }
};

// One tensor's tile in LDS: C rows of D numbers, 16-byte pieces of a row in another order in each row, so that both ways of
// reading reach all banks: the same piece of sixteen rows, and (16 bits) two neighbouring pieces of rows 0-3, 8-11, 16-19, 24-27,
// (32 bits) four pieces of every fourth row.  The order is an exclusive or, so a lane's place in one step of a contraction gives
// the others with one instruction each: `start` is the lane's, the rest is the same for all lanes.
template <class T, int C, int D>
struct Image {
    typedef Tile<T> W;
    static constexpr int PIECES = D * (int)sizeof(T) / 16, ROW = 16 * PIECES, BYTES = C * ROW;
    __device__ static int order(int row) {
        if (sizeof(T) == 4) return row & 15;
        if (PIECES >= 16) return (row >> 2 & 1) | (row & 3) << 1 | (row & 8);
        return (row >> 2 & 1) | (row & 2) | (row >> 1 & 4);
    }
    // numbers KB step + VE g .. + VE - 1 of row 16 tile + l16
    __device__ static int along_start(int g, int l16) { return l16 * ROW + (g ^ order(l16)) * 16; }
    __device__ static typename W::Frag along(const char *at, int start, int tile, int step) {
        return *(const typename W::Frag *)(at + (start ^ step * 64) + tile * 16 * ROW);
    }
    // (bfloat16) numbers 32 step + 4 g .. + 3 and as many from 16 further on
    __device__ static int fours_start(int g, int l16) { return l16 * ROW + (g / 2 ^ order(l16)) * 16 + g % 2 * 8; }
    __device__ static bf16x8 fours(const char *at, int start, int tile, int step) {
        const bf16x4 a = *(const bf16x4 *)(at + (start ^ step * 64) + tile * 16 * ROW), b = *(const bf16x4 *)(at + (start ^ (step * 64 + 32)) + tile * 16 * ROW);
        return __builtin_shufflevector(a, b, 0, 1, 2, 3, 4, 5, 6, 7);
    }
    // column 16 tile + l16 of rows KB step + VE g .. + VE - 1, as the lanes of an operand hold them
    struct Across { int at[sizeof(T) == 4 ? 4 : 1]; };
    __device__ static Across across_start(int g, int l16) {
        Across r;
        if constexpr (sizeof(T) == 4)
#pragma unroll
            for (int e = 0; e < 4; ++e) r.at[e] = (4 * g + e) * ROW + (l16 / 4 ^ (4 * g + e)) * 16 + l16 % 4 * 4;
        else {
            // lanes 4 t .. 4 t + 3 give the places of a row's four quads, and lane i takes column i of the four rows
            const int row = 8 * g + l16 / 4;
            r.at[0] = row * ROW + (l16 % 4 / 2 ^ order(row)) * 16 + l16 % 2 * 8;
        }
        return r;
    }
    __device__ static typename W::Frag across(const char *at, const Across &start, int tile, int step) {
        typename W::Frag f;
        if constexpr (sizeof(T) == 4) {
#pragma unroll
            for (int e = 0; e < 4; ++e) f[e] = *(const float *)(at + (start.at[e] ^ tile * 64) + step * 16 * ROW);
        } else {
            typedef __attribute__((address_space(3))) s16x4 *Lds;
            const s16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((Lds)(at + (start.at[0] ^ tile * 32) + step * 32 * ROW));
            const s16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((Lds)(at + (start.at[0] ^ (tile * 32 + 16)) + (step * 32 + 4) * ROW));
            f = __builtin_bit_cast(bf16x8, __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7));
        }
        return f;
    }
};

// Positions of a tile, C.  With 16 bits the tile's fixed work asks for 64; where both sizes are 64 or less, outputs take 32, with
// which four blocks have room on a compute unit instead of two (us a call, gradient of 16 segments of 512 tokens, 8 heads of 64: 63 with
// 64, 53 with 32; 16384 tokens of 8 heads of 128: 99 and 113).  With 32 bits 64 would not fit, and 16 is hardly ever faster (16 segments
// of 1000 tokens, 8 heads of 128: 235 us with 32, 271 with 16; 32 such segments, heads of 64: 146 and 142).
constexpr int tile_positions(bool bf, int cols, int rows, bool main) { return bf && !(main && cols <= 64 && rows <= 64) ? 64 : 32; }

template <class T, int CP, int RP, bool MAIN>
struct ChunkLds {
    typedef Tile<T> W;
    static constexpr int C = tile_positions(sizeof(T) == 2, CP, RP, MAIN);
    static constexpr int NT = CP > 64 || RP > 64 ? 512 : 256;                // threads: sixteen rows of the state per wavefront
    static constexpr int COL = 0, ROW = COL + Image<T, C, CP>::BYTES, BY = ROW + Image<T, C, RP>::BYTES, SET = BY + (MAIN ? Image<T, C, CP>::BYTES : 0);
    // P: the rows of tile `it` are as long as the steps of their contraction, and VE more against bank conflicts
    static constexpr int EACH = W::KB / 16;
    __host__ __device__ static constexpr int p_pitch(int it) { return W::KB * (it / EACH + 1) + W::VE; }
    __host__ __device__ static constexpr int p_tile(int it) {
        const int steps = it / EACH;
        return 16 * (W::KB * (EACH * steps * (steps + 1) / 2 + (it - EACH * steps) * (steps + 1)) + W::VE * it);
    }
    static constexpr int P_TERM = p_tile(C / 16);
    static constexpr int P = 2 * SET, PW = P + (MAIN ? W::SCORE_TERMS * P_TERM * (int)sizeof(T) : 0), FW = PW + (C + 4) * 4, ODD = FW + C * 4, BYTES = ODD + 16;
};

// The lane's number as if it were new: places that are made of it are worked out where they are used, not kept in registers from
// one tile to the next.
__device__ inline int fresh_lane() {
    int lane = threadIdx.x % 64;
    asm volatile("" : "+v"(lane));
    return lane;
}
// Nothing is left of what is not kept, whatever it was.
__device__ inline f32x4 scaled(f32x4 v, float w, bool kept) {
    const f32x4 r = v * w;
    return f32x4{kept ? r[0] : 0.f, kept ? r[1] : 0.f, kept ? r[2] : 0.f, kept ? r[3] : 0.f};
}
__device__ inline double power(double d, int e) {
    double r = 1.0;
    for (; e > 0; e >>= 1, d *= d)
        if (e & 1) r *= d;
    return r;
}

// The item that a block takes: eight neighbours change places, by one more in the next eight and in the next head.  Blocks go to the
// eight dies in turn, and places without a span (one behind each segment that is whole spans long) would fall to some of them only
// (gradient of 64 segments of 512 tokens in spans of 512, 8 heads of 64 and 128 bf16: 464 us a call without this, 313 with).
__device__ inline int item_of(int i, int head) { return (i & ~7) | ((i + (i >> 3) + head) & 7); }

// (The state that span k of a segment makes of nothing, if it is not its last one, has place first token / span + k.  That is less than
// the place of the next segment's first: scratch is n_tokens / span places, however many segments there are.)
//
// Which segment and which span of it the item is; false: none.  A wavefront looks at 64 places of the table at a time.
// Where short segments are left to the other kernel there are no spans, and item i is the segment that token i * (brief + 1) lies
// in, if no smaller one does: a segment that is longer than `brief` holds one of these.
__device__ inline bool find_item(const DecayJob &p, int item, int &seg, int &span) {
    if (!p.seg_start) {
        const int each = p.len / p.span + 1;
        seg = item / each; span = item % each;
        return seg < p.n_segments;
    }
    const int lane = threadIdx.x % 64, place = p.brief >= 0 ? item * (p.brief + 1) : item;
    int lo = 0, hi = p.n_segments;                         // the last segment whose items begin at or before this one
    while (hi - lo > 1) {
        const int step = (hi - lo + 63) / 64, i = lo + lane * step;
        const int begins = min(max(p.seg_start[min(i, p.n_segments)], 0), p.n_tokens);
        const bool before = i < hi && (p.brief >= 0 ? begins : begins / p.span + i) <= place;
        const int k = max(1, __popcll(__ballot(before)));
        lo += (k - 1) * step;
        hi = min(hi, lo + step);
    }
    seg = lo;
    const int begins = min(max(p.seg_start[seg], 0), p.n_tokens);
    if (p.brief >= 0) {          // the item is the first of its segment
        span = 0;
        return begins <= place && place - begins <= p.brief;
    }
    span = item - (begins / p.span + seg);
    return span >= 0;
}

// Pieces of rows that are not there.
__device__ const uint4 decay_nothing[1] = {{0, 0, 0, 0}};

// A pointer that is the same in all lanes, in scalar registers.
__device__ inline const void *uniform(const void *p) {
    const uint64_t u = (uint64_t)p;
    return (const void *)((uint64_t)(uint32_t)__builtin_amdgcn_readfirstlane((int)(u >> 32)) << 32 | (uint32_t)__builtin_amdgcn_readfirstlane((int)u));
}
// 16 bytes per lane to lds + 16 * lane; lds is the same for the whole wavefront.  The caller waits for vmcnt itself: the compiler,
// which would wait for every such load in front of the next LDS read, does not see it.  m0 needs a wait state between its scalar
// write and the load, which the compiler does not put into inline assembly.
__device__ inline void piece_to_lds(const void *from, uint32_t lds) {
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, off" ::"s"(lds), "v"(from) : "memory", "m0");
}
__device__ inline void piece_to_lds(const void *base, uint32_t off, uint32_t lds) {
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, %2" ::"s"(lds), "v"(off), "s"(base) : "memory", "m0");
}
// The same with 4 bytes per lane.
__device__ inline void word_to_lds(const void *from, uint32_t lds) {
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dword %1, off" ::"s"(lds), "v"(from) : "memory", "m0");
}
// VE elements of a row from element `i` on, zero behind its `dim` elements; rows begin anywhere.
template <class T>
__device__ inline uint4 loose_piece(const T *row, int i, int dim) {
    constexpr int VE = Tile<T>::VE;
    union { uint4 u; T e[VE]; } r;
    r.u = uint4{0, 0, 0, 0};
#pragma unroll
    for (int k = 0; k < VE; ++k)
        if (i + k < dim) r.e[k] = row[i + k];
    return r.u;
}
template <class T>
__device__ inline bool whole_pieces(const DecayView &v, int dim) {
    return (uintptr_t)v.data % 16 == 0 && ((v.token | v.head | dim) % Tile<T>::VE) == 0;
}
// The tile of one tensor: n positions of the span, `lowest` the first of their tokens in memory, zeros behind them.
// off: of this thread's piece in a whole tile (tile_offset).
template <class T, int C, int D, int NT>
__device__ inline uint32_t tile_offset(const DecayView &v, bool back, int tid) {
    typedef Image<T, C, D> I;
    const int pos = tid / I::PIECES, piece = tid % I::PIECES ^ I::order(pos);
    return (uint32_t)(back ? C - 1 - pos : pos) * (uint32_t)v.token * (uint32_t)sizeof(T) + piece * 16;
}
template <class T, int C, int D, int NT>
__device__ inline void stage(const DecayView &v, int dim, bool whole, uint32_t off, int lowest, int n, bool back, int head, char *to, int wave) {
    typedef Image<T, C, D> I;
    constexpr int ALL = I::BYTES / 16, STEP = NT / I::PIECES;        // positions from one piece of a thread to the next
    static_assert(ALL % 64 == 0 && STEP % 16 == 0, "whole wavefronts, and a thread's rows in one order");
    const char *rows = (const char *)at<T>(v, lowest, head);
    const uint32_t step = (uint32_t)v.token * (uint32_t)sizeof(T);
    const uint32_t lds = __builtin_amdgcn_readfirstlane((uint32_t)(uintptr_t)(const __attribute__((address_space(3))) void *)to + wave * 1024);
    const bool full = whole && n == C && dim == D;
    // rows of whole words (any of 32 bits) come word by word, on their way like the pieces (gradient of 16 segments, 8190 tokens, 8 heads
    // of 62 bf16: 148 us a call if they pass registers, 115; 8 heads of 64: 62)
    if (!whole && (sizeof(T) == 4 || ((uintptr_t)v.data % 4 == 0 && ((v.token | v.head | dim) % 2) == 0))) {
        constexpr int WORDS = 4 * ALL, EACH = 4 / (int)sizeof(T);
        static_assert(WORDS % NT == 0, "whole blocks of words");
#pragma unroll 2
        for (int k = 0; k < WORDS / NT; ++k) {
            const int s = 64 * wave + NT * k + fresh_lane(), pos = s / (4 * I::PIECES), w = s % (4 * I::PIECES), i = ((w / 4 ^ I::order(pos)) * 4 + w % 4) * EACH;
            const char *row = rows + (uint64_t)(uint32_t)(back ? n - 1 - pos : pos) * step;
            word_to_lds(pos < n && i < dim ? (const void *)(row + i * sizeof(T)) : (const void *)decay_nothing, lds - wave * 768 + NT * 4 * k);
        }
        return;
    }
#pragma unroll
    for (int k = 0; k < (ALL + NT - 1) / NT; ++k) {
        if (ALL % NT && 64 * wave + NT * k >= ALL) break;
        if (full) {
            const int64_t further = (int64_t)(STEP * k) * step;
            piece_to_lds(uniform(rows + (back ? -further : further)), off, lds + NT * 16 * k);
            continue;
        }
        const int s = 64 * wave + NT * k + fresh_lane(), pos = s / I::PIECES, piece = (s % I::PIECES) ^ I::order(pos), i = piece * Tile<T>::VE;
        const char *row = rows + (uint64_t)(uint32_t)(back ? n - 1 - pos : pos) * step;
        if (whole)
            piece_to_lds(pos < n && i < dim ? (const void *)(row + piece * 16) : (const void *)decay_nothing, lds + NT * 16 * k);
        else {
            uint4 u{0, 0, 0, 0};
            if (pos < n && i < dim) u = loose_piece((const T *)row, i, dim);
            *(uint4 *)(to + s * 16) = u;
        }
    }
}

// Whether one of the numbers in 16 bytes has an exponent of ones.
template <class T>
__device__ inline bool not_finite(uint4 v) {
    typedef unsigned short u16x2 __attribute__((ext_vector_type(2)));
    uint32_t most = 0;
    for (uint32_t w : {v.x, v.y, v.z, v.w}) {
        if constexpr (sizeof(T) == 4) most = max(most, w & 0x7fffffffu);
        else most = __builtin_bit_cast(uint32_t, __builtin_elementwise_max(__builtin_bit_cast(u16x2, most), __builtin_bit_cast(u16x2, w & 0x7fff7fffu)));
    }
    if constexpr (sizeof(T) == 4) return most >= 0x7f800000u;
    return (most >> 16) >= 0x7f80u || (most & 0xffffu) >= 0x7f80u;
}

// MAIN: outputs, and the state behind the segment.  Otherwise the state that each span but a segment's last one makes of nothing,
// which decay_spans_kernel turns into the states between the spans.
template <class T, int CP, int RP, bool MAIN>
__global__ __launch_bounds__((ChunkLds<T, CP, RP, MAIN>::NT), 2) void decay_chunk_kernel(const DecayJob job) {
    typedef Tile<T> W;
    typedef ChunkLds<T, CP, RP, MAIN> L;
    typedef Image<T, L::C, CP> IC;
    typedef Image<T, L::C, RP> IR;
    constexpr int C = L::C, KB = W::KB, VE = W::VE, IT = C / 16, CT = CP / 16, KT = C / KB, NT = L::NT, WAVES = NT / 64;
    extern __shared__ uint4 lds4[];
    char *const lds = (char *)lds4;
    T *const P = (T *)(lds + L::P);
    float *const pw = (float *)(lds + L::PW), *const fw = (float *)(lds + L::FW);
    int *const odd = (int *)(lds + L::ODD);
    const DecayPass &p = job.pass[blockIdx.z];
    const int tid = threadIdx.x, lane = tid % 64, wave = __builtin_amdgcn_readfirstlane(tid / 64), g = lane / 16, l16 = lane % 16;
    const int head = blockIdx.y, heads = gridDim.y, item = item_of(blockIdx.x, head);
    int seg, nth, first, end;
    if (item >= job.items || !find_item(job, item, seg, nth)) return;
    segment_tokens(job, seg, first, end);
    first = __builtin_amdgcn_readfirstlane(first); end = __builtin_amdgcn_readfirstlane(end);
    const int whole = end - first;
    if (whole <= job.brief || nth > whole / job.span) return;
    const int from = __builtin_amdgcn_readfirstlane(nth * job.span);
    if (nth > 0 && from >= whole) return;
    if (!MAIN && from + job.span >= whole) return;
    const int to = min(whole, from + job.span);                     // positions of the segment
    const bool back = p.back, turned = p.turned, last = to == whole;
    const int rows = p.rows, cols = p.cols, a = back ? 0 : 1;
    const float d = job.decay[head];
    // With a decay of zero a token sees its own only, as if each began an episode.  (A power of another decay that is too small to be
    // a number is a factor of zero, which takes finite numbers away and leaves the others.)
    const bool none = d == 0.f;
    const bool pieces = whole_pieces<T>(p.col, cols) && whole_pieces<T>(p.row, rows) && whole_pieces<T>(p.by, cols);
    const uint32_t col_off = tile_offset<T, C, CP, NT>(p.col, back, tid), row_off = tile_offset<T, C, RP, NT>(p.row, back, tid),
                   by_off = MAIN ? tile_offset<T, C, CP, NT>(p.by, back, tid) : 0;
    int flag = 0;
    auto fetch = [&](int base, int n, char *set) {
        const int lowest = back ? end - base - n : first + base;
        stage<T, C, CP, NT>(p.col, cols, pieces, col_off, lowest, n, back, head, set + L::COL, wave);
        stage<T, C, RP, NT>(p.row, rows, pieces, row_off, lowest, n, back, head, set + L::ROW, wave);
        if (MAIN) stage<T, C, CP, NT>(p.by, cols, pieces, by_off, lowest, n, back, head, set + L::BY, wave);
        if (job.starts) {
            // backward, the cut lies between a token and the one behind it
            const int pos = min(lane, n - 1), t = lowest + (back ? n - pos : pos);
            flag = job.starts[min(t, end - 1)];
        }
    };
    int base = from, single = 0, set = 0;
    if (base < to) fetch(base, min(C, to - base), lds);
    if (tid <= C) pw[tid] = (float)power((double)d, tid);
    if (tid == 0) *odd = 0;

    // the state: tile ct holds X[r][.] of row r = 16 wave + l16 and the four columns from 16 ct + 4 g on
    const size_t size = (size_t)rows * cols;
    const int row_step = turned ? 1 : cols, col_step = turned ? rows : 1;
    const size_t place = (size_t)(first / job.span + nth) * heads + head;      // of the span's state
    const float *x_in = nth > 0 && MAIN ? p.spans + (place - heads) * size
                                        : MAIN && p.x_in ? p.x_in + ((size_t)seg * heads + head) * size : nullptr;
    f32x4 x[CT];
    const int r = 16 * wave + l16;
    const bool quads = !turned && cols % 4 == 0 && (uintptr_t)x_in % 16 == 0;
#pragma unroll
    for (int ct = 0; ct < CT; ++ct) {
        f32x4 v{0.f, 0.f, 0.f, 0.f};
        const int c = 16 * ct + 4 * g;
        if (x_in && quads) v = r < rows && c < cols ? *(const f32x4 *)(x_in + (uint32_t)(r * cols + c)) : v;
        else if (x_in)
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const bool there = r < rows && c + e < cols;
                const float w = x_in[there ? (uint32_t)(r * row_step + (c + e) * col_step) : 0u];
                v[e] = there ? w : 0.f;
            }
        x[ct] = v;
    }

    const bool vec_out = (uintptr_t)p.out.data % (4 * sizeof(T)) == 0 && ((p.out.token | p.out.head | rows) % 4) == 0;
    bool passes = true;                                             // whether the state in front of the span reaches its end
    const bool mine = MAIN ? 16 * wave < rows : RP / 16 == WAVES || wave < RP / 16;      // the wavefront has rows
    const int along = IC::along_start(g, l16), fours = IC::fours_start(g, l16);
    const auto row_across = IR::across_start(g, l16);
    const auto col_across = IC::across_start(g, l16);
    __syncthreads();                                                // pw
    while (base < to) {
        const int n = single ? 1 : min(C, to - base);
        const uint64_t cuts = job.starts ? __ballot(lane < n && flag && !(back && base + lane == 0)) : 0;
        const int cut = cuts ? 63 - __clzll(cuts) : -1;             // the tile's last start
        const bool whole_tile = cuts == 0 && !none;                // every position sees the state, and it stays
        asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
        __syncthreads();
        const char *const now = lds + set;
        char *const then = lds + (L::SET - set);
        if (base + n < to) fetch(base + n, single > 1 ? 1 : min(C, to - base - n), then);

        if (tid < C) fw[tid] = tid < n && tid >= cut ? pw[n - tid - a] * p.col_scale : 0.f;
        typename W::Frag rowf[KT], colf;
        bool wrong = false;
        if (mine)
#pragma unroll
            for (int k = 0; k < KT; ++k) {
                rowf[k] = IR::across(now + L::ROW, row_across, wave, k);
                wrong = wrong || not_finite<T>(__builtin_bit_cast(uint4, rowf[k]));
            }
        if (!whole_tile)
            for (int s = tid; s < IC::BYTES / 16; s += NT) wrong = wrong || not_finite<T>(*(const uint4 *)(now + L::COL + 16 * s));
        if (wrong && !single) *odd = 1;
        f32x4 acc[IT];
        if constexpr (MAIN) {
            // scores, a 16x16 tile at a time: tile (jt, it) with jt <= it
#pragma unroll
            for (int k = 0; k < (IT * (IT + 1) / 2 + WAVES - 1) / WAVES; ++k) {
                const int t = wave + WAVES * k;
                if (t >= IT * (IT + 1) / 2) break;
                const int it = t >= 6 ? 3 : t >= 3 ? 2 : t >= 1 ? 1 : 0, jt = t - it * (it + 1) / 2;
                f32x4 s{0.f, 0.f, 0.f, 0.f};
#pragma unroll
                for (int c = 0; c < CP / KB; ++c)
                    s = W::mma(IC::along(now + L::COL, along, jt, c), IC::along(now + L::BY, along, it, c), s);
                const int i = 16 * it + l16;
                const uint64_t before = cuts & (~0ull >> (63 - i));
                const int fresh = before ? 63 - __clzll(before) : -1;
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const int j = 16 * jt + 4 * g + e;
                    const float w = pw[max(i - j, 0)] * p.col_scale;
                    s[e] = j <= i && j >= fresh && (j == i || !none) ? s[e] * w : 0.f;
                }
                T *const pi = P + L::p_tile(it) + l16 * L::p_pitch(it) + 16 * jt + 4 * g;
#pragma unroll
                for (int term = 0; term < W::SCORE_TERMS; ++term) {
                    const typename W::Quad w = W::quad(s);
                    *(typename W::Quad *)(pi + term * L::P_TERM) = w;
                    if (term + 1 < W::SCORE_TERMS) s -= __builtin_convertvector(w, f32x4);
                    // the fragment above the diagonal that shares a contraction step with this tile
                    if (it == jt && KB > 16 && it % 2 == 0) *(typename W::Quad *)(pi + term * L::P_TERM + 16) = W::quad(f32x4{0.f, 0.f, 0.f, 0.f});
                }
            }
            // what the state says
            if (mine) {
#pragma unroll
                for (int it = 0; it < IT; ++it) acc[it] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
                for (int c = 0; c < CP / KB; ++c) {
                    __builtin_amdgcn_sched_barrier(0);      // loads of all steps at once would not fit the registers
                    if constexpr (KB == 16) {
#pragma unroll
                        for (int it = 0; it < IT; ++it) acc[it] = W::mma(x[c], IC::along(now + L::BY, along, it, c), acc[it]);
                    } else {       // two terms of the state
                        const f32x4 x0 = x[2 * c % CT], x1 = x[(2 * c + 1) % CT];
                        const bf16x4 h0 = W::quad(x0), h1 = W::quad(x1);
                        const bf16x4 l0 = W::quad(x0 - __builtin_convertvector(h0, f32x4)), l1 = W::quad(x1 - __builtin_convertvector(h1, f32x4));
                        const bf16x8 h = __builtin_shufflevector(h0, h1, 0, 1, 2, 3, 4, 5, 6, 7), l = __builtin_shufflevector(l0, l1, 0, 1, 2, 3, 4, 5, 6, 7);
#pragma unroll
                        for (int it = 0; it < IT; ++it) {
                            const bf16x8 fb = IC::fours(now + L::BY, fours, it, c);
                            acc[it] = W::mma(h, fb, acc[it]);
                            acc[it] = W::mma(l, fb, acc[it]);
                        }
                    }
                }
#pragma unroll
                for (int it = 0; it < IT; ++it) {
                    const int i = 16 * it + l16;
                    const float w = pw[min(i + a, C)];
                    if (whole_tile) acc[it] = acc[it] * w;
                    else acc[it] = scaled(acc[it], w, !(cuts & (~0ull >> (63 - i))) && (i + a == 0 || !none));
                }
            }
        }
        __syncthreads();
        // A product with zero does not hide a number that is not finite from the positions that must not see it: one position at
        // a time then.
        if (!single && n > 1 && __builtin_amdgcn_readfirstlane(*odd)) {
            asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
            __syncthreads();
            if (tid == 0) *odd = 0;
            single = n;
            fetch(base, 1, then);
        } else {
            if (mine) {
                if constexpr (MAIN) {
                    char *const out_tile = (char *)at<T>(p.out, back ? end - base - n : first + base, head);
                    const uint32_t out_step = (uint32_t)p.out.token * (uint32_t)sizeof(T);
#pragma unroll
                    for (int it = 0; it < IT; ++it) {
                        __builtin_amdgcn_sched_barrier(0);
#pragma unroll
                        for (int k = 0; k * KB <= 16 * it; ++k)
#pragma unroll
                            for (int term = 0; term < W::SCORE_TERMS; ++term)
                                acc[it] = W::mma(rowf[k], *(const typename W::Frag *)(P + term * L::P_TERM + L::p_tile(it) + l16 * L::p_pitch(it) + k * KB + g * VE), acc[it]);
                        const int pos = 16 * it + l16, o = 16 * wave + 4 * g;
                        const typename W::Quad w = W::quad(acc[it] * p.out_scale);
                        T *out = (T *)(out_tile + (uint32_t)(back ? n - 1 - pos : pos) * out_step);
                        if (pos < n && vec_out) {
                            if (o < rows) *(typename W::Quad *)(out + o) = w;
                        } else if (pos < n) {
#pragma unroll
                            for (int e = 0; e < 4; ++e)
                                if (o + e < rows) out[o + e] = w[e];
                        }
                    }
                }
                // rows with their decay, in place of the keys: a wavefront needs its own rows only
                typename W::Frag rs[W::ROW_TERMS][KT];
#pragma unroll
                for (int k = 0; k < KT; ++k) {
                    float v[VE];
#pragma unroll
                    for (int e = 0; e < VE; ++e) v[e] = (float)rowf[k][e] * fw[KB * k + VE * g + e];
#pragma unroll
                    for (int term = 0; term < W::ROW_TERMS; ++term)
#pragma unroll
                        for (int e = 0; e < VE; ++e) {
                            rs[term][k][e] = from_f32<T>(v[e]);
                            if (term + 1 < W::ROW_TERMS) v[e] -= (float)rs[term][k][e];
                        }
                }
                const float carry = pw[n];
                if (whole_tile) {
#pragma unroll
                    for (int ct = 0; ct < CT; ++ct) x[ct] = x[ct] * carry;
                } else {
#pragma unroll
                    for (int ct = 0; ct < CT; ++ct) x[ct] = f32x4{0.f, 0.f, 0.f, 0.f};
                }
                if (!(none && back))                                // nothing of a tile stays then
#pragma unroll
                for (int ct = 0; ct < CT; ++ct) {
                    if (ct % (MAIN ? 4 : 2) == 0) __builtin_amdgcn_sched_barrier(0);
#pragma unroll
                    for (int k = 0; k < KT; ++k) {
                        colf = IC::across(now + L::COL, col_across, ct, k);
#pragma unroll
                        for (int term = 0; term < W::ROW_TERMS; ++term) x[ct] = W::mma(colf, rs[term][k], x[ct]);
                    }
                }
            }
            passes = passes && cuts == 0;
            base += n;
            single = max(single - 1, 0);
        }
        set = L::SET - set;
    }
    float *x_out = !MAIN ? p.spans + place * size : last && p.x_out ? p.x_out + ((size_t)seg * heads + head) * size : nullptr;
    if (!MAIN && tid == 0) p.passes[place] = passes ? 1.f : 0.f;
    if (!x_out || !mine) return;
    const bool quads_out = !turned && cols % 4 == 0 && (uintptr_t)x_out % 16 == 0;
    const bool nothing = MAIN && back && whole > 0 && job.starts && job.starts[first];      // the first token knows of no state
#pragma unroll
    for (int ct = 0; ct < CT; ++ct) {
        const int c = 16 * ct + 4 * g;
        if (quads_out) {
            if (r < rows && c < cols) *(f32x4 *)(x_out + (uint32_t)(r * cols + c)) = nothing ? f32x4{0.f, 0.f, 0.f, 0.f} : x[ct];
        } else if (r < rows)
#pragma unroll
            for (int e = 0; e < 4; ++e)
                if (c + e < cols) x_out[(uint32_t)(r * row_step + (c + e) * col_step)] = nothing ? 0.f : x[ct][e];
    }
}

// The states between the spans of a segment, from the segment's first state and what each span made of nothing: in place.
// QUAD: four numbers per thread.  Bound by memory: 32 spans of 8 heads of 128 and 128 10.7 us (33 MB, 3.0 TB/s).  With 16 or 32 spans'
// numbers under way together instead of 8: 16 segments 7.4 and 9.2 us, the 32 spans 10.7 and 10.8.
template <bool QUAD>
__global__ __launch_bounds__(256) void decay_spans_kernel(const DecayJob job, int parts) {
    typedef typename std::conditional<QUAD, f32x4, float>::type V;
    const DecayPass &p = job.pass[blockIdx.z / parts];
    const int seg = blockIdx.x, head = blockIdx.y, heads = gridDim.y;
    int first, end;
    segment_tokens(job, seg, first, end);
    const int spans = (end - first + job.span - 1) / job.span;
    if (spans < 2) return;
    const int e = ((blockIdx.z % parts) * 256 + threadIdx.x) * (QUAD ? 4 : 1);
    const size_t size = (size_t)p.rows * p.cols;
    if (e >= (int)size) return;
    const size_t place = (size_t)(first / job.span) * heads + head;
    float *at_span = p.spans + place * size + e;
    const float *passes = p.passes + place;
    const float w = (float)power((double)job.decay[head], job.span);
    const bool none = job.decay[head] == 0.f;
    V x{};
    if (p.x_in) __builtin_memcpy(&x, p.x_in + ((size_t)seg * heads + head) * size + e, sizeof x);
    constexpr int AHEAD = 8;                              // spans whose numbers are under way together
    for (int i = 0; i + 1 < spans; i += AHEAD) {
        float f[AHEAD];
        V v[AHEAD];
#pragma unroll
        for (int k = 0; k < AHEAD; ++k) {
            const size_t at = (size_t)min(i + k, spans - 2) * heads;
            f[k] = passes[at];
            v[k] = *(const V *)(at_span + at * size);
        }
#pragma unroll
        for (int k = 0; k < AHEAD; ++k)
            if (i + k + 1 < spans) {
                if (f[k] == 0.f || none) x = V{};         // whatever was in it
                x = w * x + v[k];
                *(V *)(at_span + (size_t)(i + k) * heads * size) = x;
            }
    }
}

// One token of each agent.  The state of entry i is row slots[i] of the states (i without slots), read, advanced and written back;
// a slot outside them stands for a state of zeros that is not kept.  Entries that name one slot are consecutive tokens of it, in
// the order of their numbers: the first of them takes the others along, so that nobody else touches the slot.
// Bound by memory: a state is read and written once.  512 agents, 16 heads of 64 and 64: 59 us (270 MB, 4.6 TB/s); one agent 4.
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
// The first entry behind `entry` with this slot, p.n if there is none, -1 if there is one in front of it (looked for only where
// `first`); the same in all lanes of the wavefront.
__device__ inline int next_of_slot(const DecayStep &p, int slot, int entry, bool first) {
    const int lane = threadIdx.x % 64;
    for (int j = first ? 0 : entry + 1; j < p.n; j += 512) {
        bool is[8];
#pragma unroll
        for (int k = 0; k < 8; ++k) {
            const int at = j + 64 * k + lane;
            is[k] = p.slots[min(at, p.n - 1)] == slot && at < p.n && at != entry;
        }
#pragma unroll
        for (int k = 0; k < 8; ++k) {
            const uint64_t m = __ballot(is[k]);
            if (m) {
                const int found = j + 64 * k + __ffsll((unsigned long long)m) - 1;
                return found < entry ? -1 : found;
            }
        }
    }
    return p.n;
}

// Four numbers that the caches need not keep.
typedef float f32x4_once __attribute__((ext_vector_type(4)));
__device__ inline float4 load_once(const float *p) {
    const f32x4_once v = __builtin_nontemporal_load((const f32x4_once *)p);
    return float4{v.x, v.y, v.z, v.w};
}
__device__ inline void store_once(float *p, float4 v) { __builtin_nontemporal_store(f32x4_once{v.x, v.y, v.z, v.w}, (f32x4_once *)p); }

// STREAM: the states of a call are more than the caches hold, and may be moved four numbers at a time.
template <class T, int LPR, int CV, int RPL, bool STREAM>
__global__ __launch_bounds__(256) void decay_step_kernel(const DecayStep p, int slabs, int vec) {
    constexpr int RW = 64 / LPR;
    const int unit = __builtin_amdgcn_readfirstlane(blockIdx.x * 4 + threadIdx.x / 64), lane = threadIdx.x % 64;
    const int entry = unit / slabs, head = blockIdx.y, heads = gridDim.y, c0 = lane % LPR * 4, r0 = unit % slabs * RW * RPL + lane / LPR;
    if (entry >= p.n) return;
    const int slot = p.slots ? __builtin_amdgcn_readfirstlane(p.slots[entry]) : entry;
    const bool kept = slot >= 0 && slot < p.n_slots, shared = p.slots && kept;
    const float d = p.decay[head];
    float *state = p.states + ((size_t)(kept ? slot : 0) * heads + head) * p.value * p.key;
    const bool quads = p.key % 4 == 0 && (uintptr_t)p.states % 16 == 0;
    Rows<RPL, CV> s;
#pragma unroll
    for (int i = 0; i < RPL; ++i)
#pragma unroll
        for (int v = 0; v < CV; ++v) {
            const int r = r0 + i * RW, c = c0 + v * 4 * LPR;
            const float *x = state + (uint32_t)(r * p.key + c);
            if (STREAM) s.x[i][v] = r < p.value && c < p.key && kept ? load_once(x) : float4{0.f, 0.f, 0.f, 0.f};
            else s.x[i][v] = load4(x, kept && r < p.value ? p.key - c : 0, quads);
        }
    float4 col[CV], by[CV];
    float row[RPL], sum[RPL];
    int start;
    auto fetch = [&](int t) {
        const T *q = at<T>(p.q, t, head), *k = at<T>(p.k, t, head), *w = at<T>(p.v, t, head);
#pragma unroll
        for (int v = 0; v < CV; ++v) {
            const int c = c0 + v * 4 * LPR;
            col[v] = load4(k + c, p.key - c, vec);
            by[v] = load4(q + c, p.key - c, vec);
        }
#pragma unroll
        for (int i = 0; i < RPL; ++i) row[i] = r0 + i * RW < p.value ? to_f32(w[r0 + i * RW]) : 0.f;
        start = p.starts ? p.starts[t] : 0;
    };
    fetch(entry);
    // (all of that is on its way meanwhile)
    int next = shared ? next_of_slot(p, slot, entry, true) : p.n;
    if (next < 0) return;
    for (int t = entry;;) {
        s.template take<LPR>(start ? 0.f : d, row, col, by, sum);
        T *out = (T *)p.out.data + t * p.out.token + head * p.out.head;
        if (lane % LPR == 0)
#pragma unroll
            for (int i = 0; i < RPL; ++i)
                if (r0 + i * RW < p.value) out[r0 + i * RW] = from_f32<T>(p.scale * sum[i]);
        if (next >= p.n) break;
        t = next;
        fetch(t);
        next = next_of_slot(p, slot, t, false);
    }
    if (!kept) return;
#pragma unroll
    for (int i = 0; i < RPL; ++i)
#pragma unroll
        for (int v = 0; v < CV; ++v) {
            const int r = r0 + i * RW, c = c0 + v * 4 * LPR;
            if (r >= p.value) continue;
            const float4 e = s.x[i][v];
            float *x = state + (uint32_t)(r * p.key + c);
            if (STREAM) {
                if (c < p.key) store_once(x, e);
            } else if (quads) {
                if (c < p.key) *(float4 *)x = e;
            } else {
                if (c < p.key) x[0] = e.x;
                if (c + 1 < p.key) x[1] = e.y;
                if (c + 2 < p.key) x[2] = e.z;
                if (c + 3 < p.key) x[3] = e.w;
            }
        }
}

// -------------------------------------------------------------------- host --

// Rows of a view that four elements at a time can be read from.
template <class T>
bool rows_of_four(const DecayView &v) { return (uintptr_t)v.data % (4 * sizeof(T)) == 0 && v.token % 4 == 0 && v.head % 4 == 0; }

// go(LPR, CV, RPL) of the token-by-token kernels: as few lanes per row as its columns need, and no more rows per lane than there are.
template <class F>
hipError_t by_shape(int rows, int cols, F go) {
    auto with = [&](auto lpr, auto cv) {
        constexpr int RW = 64 / lpr.value;
        if (rows <= RW) return go(lpr, cv, std::integral_constant<int, 1>());
        if (rows <= 2 * RW) return go(lpr, cv, std::integral_constant<int, 2>());
        return go(lpr, cv, std::integral_constant<int, 4>());
    };
    if (cols <= 16) return with(std::integral_constant<int, 4>(), std::integral_constant<int, 1>());
    if (cols <= 32) return with(std::integral_constant<int, 8>(), std::integral_constant<int, 1>());
    if (cols <= 64) return with(std::integral_constant<int, 16>(), std::integral_constant<int, 1>());
    return with(std::integral_constant<int, 16>(), std::integral_constant<int, 2>());
}

// States of a call from which on they pass the caches by (they would not be there any more at the next call; 270 MB of states 77 us
// through the caches, 59 past them).
constexpr size_t STREAM_BYTES = (size_t)64 << 20;

// Token by token: the passes of the job.
template <class T>
hipError_t launch_recurrent(const DecayJob &job, int passes, int heads, hipStream_t s) {
    int rows = 0, cols = 0;
    for (int i = 0; i < passes; ++i) { rows = std::max(rows, job.pass[i].rows); cols = std::max(cols, job.pass[i].cols); }
    return by_shape(rows, cols, [&](auto lpr, auto cv, auto rpl) {
        constexpr int ROWS = 64 / lpr.value * rpl.value;
        const int slabs = (rows + ROWS - 1) / ROWS;
        const int64_t units = (int64_t)job.n_segments * slabs;
        launch(decay_recurrent_kernel<T, lpr.value, cv.value, rpl.value>, dim3((unsigned)((units + 3) / 4), heads, passes), dim3(256), 0, s, job, slabs);
        return hipGetLastError();
    });
}

template <class T, int CP, int RP, bool MAIN>
hipError_t launch_chunk_kernel(const DecayJob &job, int passes, int heads, hipStream_t s) {
    static size_t lds_set = 0;
    const auto kernel = decay_chunk_kernel<T, CP, RP, MAIN>;
    constexpr size_t lds = ChunkLds<T, CP, RP, MAIN>::BYTES;
    if (lds > 64 * 1024 && lds_set == 0) {
        const hipError_t e = hipFuncSetAttribute((const void *)kernel, hipFuncAttributeMaxDynamicSharedMemorySize, (int)lds);
        if (e != hipSuccess) return e;
        lds_set = lds;
    }
    launch(kernel, dim3((job.items + 7) / 8 * 8, heads, passes), dim3(ChunkLds<T, CP, RP, MAIN>::NT), lds, s, job);
    return hipGetLastError();
}
template <class T, bool MAIN>
hipError_t launch_chunk(const DecayJob &job, int passes, int heads, hipStream_t s) {
    const bool wide_rows = job.pass[0].rows > 64;
    if (job.pass[0].cols > 64) return wide_rows ? launch_chunk_kernel<T, 128, 128, MAIN>(job, passes, heads, s) : launch_chunk_kernel<T, 128, 64, MAIN>(job, passes, heads, s);
    return wide_rows ? launch_chunk_kernel<T, 64, 128, MAIN>(job, passes, heads, s) : launch_chunk_kernel<T, 64, 64, MAIN>(job, passes, heads, s);
}

// Calls go(job, passes) for each group of passes that one launch can take: those that `together` says of.
template <class Together, class F>
hipError_t by_sizes(const DecayJob &job, int passes, Together together, F go) {
    bool done[3] = {false, false, false};
    for (int i = 0; i < passes; ++i) {
        if (done[i]) continue;
        DecayJob some = job;
        int n = 0;
        for (int k = i; k < passes; ++k)
            if (!done[k] && together(job.pass[i], job.pass[k])) { some.pass[n++] = job.pass[k]; done[k] = true; }
        const hipError_t e = go(some, n);
        if (e != hipSuccess) return e;
    }
    return hipSuccess;
}
// Token by token: passes of small states share a launch, with room for the larger sizes (gradient of 32 segments of 5 tokens, 4 heads
// of 16 and 32: 22 us apart, 16 together; of 512 such segments 29 and 25, with heads of 32 and 64 56 and 96).
bool recurrent_together(const DecayPass &a, const DecayPass &b) {
    return (a.rows == b.rows && a.cols == b.cols) || std::max({a.rows, a.cols, b.rows, b.cols}) <= 32;
}
// Chunked: passes of one kernel (gradient of 64 segments of 256 tokens bf16, 4 heads of 64 and 32: 77 us a call apart, 35 together).
bool chunk_together(const DecayPass &a, const DecayPass &b) { return (a.rows > 64) == (b.rows > 64) && (a.cols > 64) == (b.cols > 64); }

// Tokens of a segment that a block of the chunked kernels takes: a power of two of SHORTEST_SPAN, the one that takes least time by this
// count.  A block's time is its tiles and three more for its beginning; blocks take turns on as many places as the compute units have.
// Two more kernels, two tiles' time, are launched unless no segment can be longer than the span; if the longest segment (by guess,
// twice the average) is longer, they take half of the time of the outputs and as long again for what lies between.  Over 120 calls of
// 1 to 100 segments, equal, uneven and cut at random, of 200 to 64000 tokens this is 4% behind the best of 128 to 1024 each time, 99%
// at most (random cuts, whose longest segment is longer than guessed; profiles/memory_operators_span_choice.txt); us a call with 128 /
// 256 / 512 / 1024 tokens: 16384 tokens bf16, 8 heads of 128: 129 / 105 / 98 / 144 (512 taken); gradient of 4096 tokens fp32, 4 heads of
// 128: 93 / 96 / 168 / 316 (256); gradient of 64 segments of 512 tokens bf16, 8 heads of 64 and 128: 496 / 396 / 313 / 308 (none split: 228).
constexpr int SHORTEST_SPAN = 128;
int span_of(int heads, int n_segments, int n_tokens, int key, int value, int passes, bool bf) {
    const bool small = key <= 64 && value <= 64;
    const int tile = tile_positions(bf, key, value, true);
    const int64_t slots = small && bf ? 1024 : key > 64 && value > 64 ? 256 : 512,
                  longest = n_segments == 1 ? n_tokens : std::min<int64_t>(n_tokens, 2 * ((int64_t)n_tokens / n_segments));
    int best = 0;
    int64_t least = INT64_MAX;
    for (int span = SHORTEST_SPAN; span <= 1 << 20; span *= 2) {
        const bool split = span < longest;
        auto rounds = [&](int64_t items) { return std::max<int64_t>(1, (items * heads + slots - 1) / slots); };
        // half of a segment's last span is not there
        int64_t time = 2 * rounds((split ? n_tokens / span + n_segments / 2 : n_segments) * (int64_t)passes) * (std::min<int64_t>(span, longest) / tile + 3);
        if (n_tokens > span) time += 4;
        if (split) time += rounds(std::max(1, n_tokens / span - n_segments / 2) * (int64_t)(passes > 1 ? 2 : 1)) * (span / tile + 3) + 4;
        if (time < least) { least = time; best = span; }
    }
    return best;
}
// The average length up to which segments take the token-by-token kernel (those of up to twice that, the rest are chunked).  What that
// kernel does for a token grows with the state, the chunked one has its fixed work per segment, which takes longer with 32 bits.  us a
// call, token by token (with the launch that finds no long segment) / chunked, 768 segments of 4 heads, states in and out: fp32 16 and 32,
// 15 tokens 20 / 40; 32 and 32, 10 tokens 24 / 40; 64 and 64, 4 tokens 53 / 49, 7 tokens 60 / 50 (without states 31 / 39 and 39 / 39);
// 128 and 128, 5 tokens 175 / 174 (91 / 117); bf16 16 and 16, 10 tokens 17 / 22; 32 and 32, 4.5 tokens 22 / 25, 10 tokens 30 / 24; 64 and
// 64, 2 tokens 57 / 33 (33 / 22); 128 and 128, 1 token 136 / 162 (46 / 107), 3 tokens 180 / 163 (85 / 108).  (bf16 states of
// 64 and 64 would be faster chunked from one token on.)  128 segments take 12 to 16 us either way, the host's time and one launch more or less.
int brief_average(int key, int value, bool bf) {
    const int size = key * value;
    if (bf) return size <= 256 ? 12 : size <= 1024 ? 5 : 3;
    return size <= 512 ? 16 : size <= 1024 ? 10 : 7;
}

void plan(DecayJob &job, const ga3c_decay_desc *d, bool grad) {
    const bool bf = d->dtype == GA3C_BF16;
    const int average = brief_average(d->key_dim, d->value_dim, bf);
    job.brief = job.n_tokens <= average * (int64_t)job.n_segments ? 2 * average : -1;
    job.span = job.brief >= 0 ? 1 << 30 : span_of(d->n_heads, job.n_segments, job.n_tokens, d->key_dim, d->value_dim, grad ? 3 : 1, bf);
    job.items = job.brief >= 0 ? job.n_tokens / (job.brief + 1) + 1
                               : job.seg_start ? job.n_tokens / job.span + job.n_segments : job.n_segments * (job.len / job.span + 1);
}
// Scratch: the states between the spans of each direction, and behind all of them a number for each state.  (The states of a second
// direction behind the first one's numbers would lie anywhere, and be read and written one element at a time.)
size_t span_places(const DecayJob &job, int heads) { return (size_t)(job.n_tokens / job.span) * heads; }

// passes: of outputs; sources: those of them whose spans' states are made (one forward, one backward)
template <class T>
hipError_t run_job(DecayJob &job, int passes, const int *sources, int n_sources, int heads, hipStream_t s) {
    const int longest = job.seg_start ? job.n_tokens : job.len;
    hipError_t e = hipSuccess;
    if (job.brief >= 0 && (job.seg_start || longest <= job.brief))
        e = by_sizes(job, passes, recurrent_together, [&](const DecayJob &some, int n) { return launch_recurrent<T>(some, n, heads, s); });
    if (e != hipSuccess || longest <= job.brief) return e;
    if (longest > job.span) {
        DecayJob made = job;
        for (int i = 0; i < n_sources; ++i) made.pass[i] = job.pass[sources[i]];
        e = by_sizes(made, n_sources, chunk_together, [&](const DecayJob &some, int n) { return launch_chunk<T, false>(some, n, heads, s); });
        if (e != hipSuccess) return e;
        // four numbers per thread where that leaves enough blocks (one segment of 16384 tokens: 10 us, with four 16)
        const int size = job.pass[0].rows * job.pass[0].cols;
        const bool quad = size % 4 == 0 && (int64_t)job.n_segments * heads * n_sources * size >= 1 << 20;
        const int each = quad ? 1024 : 256, parts = (size + each - 1) / each;
        launch(quad ? decay_spans_kernel<true> : decay_spans_kernel<false>, dim3(job.n_segments, heads, parts * n_sources), dim3(256), 0, s, made, parts);
        if ((e = hipGetLastError()) != hipSuccess) return e;
    }
    return by_sizes(job, passes, chunk_together, [&](const DecayJob &some, int n) { return launch_chunk<T, true>(some, n, heads, s); });
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
constexpr int64_t MAX_STRIDE = 1 << 24;      // the 64 positions of a tile are 32-bit numbers of bytes apart
int check_views(const ga3c_heads *const *in, int n_in, const ga3c_heads *const *out, const int *out_dims, int n_out, int n, int heads, size_t size, const char *who) {
    for (int i = 0; i < n_in; ++i) {
        if (!in[i] || !in[i]->data) return call_fail(GA3C_EINVAL, "%s: null tensor", who);
        if ((uintptr_t)in[i]->data % size) return call_fail(GA3C_EINVAL, "%s: tensor not aligned to its elements", who);
        if (in[i]->token_stride < 0 || in[i]->head_stride < 0) return call_fail(GA3C_EINVAL, "%s: negative stride", who);
        if (n > 1 && in[i]->token_stride >= MAX_STRIDE) return call_fail(GA3C_EINVAL, "%s: token_stride of 2^24 or more", who);
    }
    for (int i = 0; i < n_out; ++i) {
        if (!out[i] || !out[i]->data) return call_fail(GA3C_EINVAL, "%s: null tensor", who);
        if ((uintptr_t)out[i]->data % size) return call_fail(GA3C_EINVAL, "%s: tensor not aligned to its elements", who);
        if (n > 1 && out[i]->token_stride >= MAX_STRIDE) return call_fail(GA3C_EINVAL, "%s: token_stride of 2^24 or more", who);
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
    // threads of a launch are counted in 32 bits
    if (n_segments > 1 << 22 || n_tokens > 1 << 28) return call_fail(GA3C_EINVAL, "%s: more than 2^22 segments or 2^28 tokens", who);
    if (n_segments == 0 && n_tokens > 0) return call_fail(GA3C_EINVAL, "%s: tokens without a segment", who);
    if (!seg_start && n_segments > 0 && n_tokens % n_segments) return call_fail(GA3C_EINVAL, "%s: %d tokens are no %d equal segments", who, n_tokens, n_segments);
    return GA3C_OK;
}
bool overlap(const void *a, const void *b, size_t bytes) {
    return a && b && (uintptr_t)a < (uintptr_t)b + bytes && (uintptr_t)b < (uintptr_t)a + bytes;
}
DecayView view(const ga3c_heads *h) { return h ? DecayView{h->data, h->token_stride, h->head_stride} : DecayView{nullptr, 0, 0}; }

DecayJob job_of(const ga3c_decay_desc *d, const int32_t *seg_start, const uint8_t *starts, int n_segments, int n_tokens, bool grad) {
    DecayJob j;
    memset(&j, 0, sizeof j);
    j.seg_start = seg_start; j.starts = starts; j.n_segments = n_segments; j.n_tokens = n_tokens;
    j.len = n_tokens / n_segments;
    memcpy(j.decay, d->decay, sizeof(float) * d->n_heads);
    plan(j, d, grad);
    return j;
}
DecayPass pass_of(const ga3c_heads *row, const ga3c_heads *col, const ga3c_heads *by, const ga3c_heads *out, int rows, int cols, int turned, int back,
                  float out_scale, float col_scale, const float *x_in, float *x_out, float *spans, float *passes) {
    return DecayPass{view(row), view(col), view(by), view(out), rows, cols, turned, back, out_scale, col_scale, x_in, x_out, spans, passes};
}
hipError_t run(const ga3c_decay_desc *d, DecayJob &j, int passes, const int *sources, int n_sources, hipStream_t s) {
    return d->dtype == GA3C_BF16 ? run_job<bf16>(j, passes, sources, n_sources, d->n_heads, s) : run_job<float>(j, passes, sources, n_sources, d->n_heads, s);
}
int hip_result(hipError_t e, const char *who) { return e == hipSuccess ? GA3C_OK : call_fail(GA3C_EHIP, "%s: %s", who, hipGetErrorString(e)); }

}  // namespace
}  // namespace ga3c

using namespace ga3c;

extern "C" size_t ga3c_decay_attention_workspace(const ga3c_decay_desc *d, int n_segments, int n_tokens, int grad) {
    if (check_desc(d, "ga3c_decay_attention_workspace") != GA3C_OK || n_segments < 1 || n_tokens < 1) return 0;
    // the gradient has states of both directions
    const DecayJob j = job_of(d, (const int32_t *)1, nullptr, n_segments, n_tokens, grad);
    return (grad ? 2 : 1) * sizeof(float) * span_places(j, d->n_heads) * ((size_t)d->key_dim * d->value_dim + 1);
}

size_t ga3c::decay_workspace_most(const ga3c_decay_desc *d, int n_tokens) {
    return 2 * sizeof(float) * (n_tokens / SHORTEST_SPAN) * d->n_heads * ((size_t)d->key_dim * d->value_dim + 1);
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
    const size_t need = ga3c_decay_attention_workspace(d, n_segments, n_tokens, 0);
    if (workspace_bytes < need) return call_fail(GA3C_EINVAL, "%s: workspace too small", who);
    if (need && (!workspace || (uintptr_t)workspace % 16)) return call_fail(GA3C_EINVAL, "%s: workspace null or not aligned to 16 bytes", who);
    DecayJob j = job_of(d, seg_start, starts, n_segments, n_tokens, false);
    float *const spans = (float *)workspace, *const passes = spans + span_places(j, d->n_heads) * d->key_dim * d->value_dim;
    j.pass[0] = pass_of(v, k, q, out, d->value_dim, d->key_dim, 0, 0, d->scale, 1.f, state_in, state_out, spans, passes);
    const int sources[] = {0};
    return hip_result(run(d, j, 1, sources, 1, (hipStream_t)stream), who);
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
    const size_t need = ga3c_decay_attention_workspace(d, n_segments, n_tokens, 1);
    if (workspace_bytes < need) return call_fail(GA3C_EINVAL, "%s: workspace too small", who);
    if (need && (!workspace || (uintptr_t)workspace % 16)) return call_fail(GA3C_EINVAL, "%s: workspace null or not aligned to 16 bytes", who);
    DecayJob j = job_of(d, seg_start, starts, n_segments, n_tokens, true);
    const int key = d->key_dim, value = d->value_dim;
    const size_t places = span_places(j, d->n_heads), states = places * key * value;
    float *const forward = (float *)workspace, *const backward = forward + states, *const passes = backward + states, *const passes_back = passes + places;
    // the states in front of the tokens once more, read out by dout; the gradient of the state behind each token, read out by v and k
    j.pass[0] = pass_of(k, v, dout, dq, key, value, 1, 0, d->scale, 1.f, state_in, nullptr, forward, passes);
    j.pass[1] = pass_of(q, dout, v, dk, key, value, 1, 1, 1.f, d->scale, dstate_out, nullptr, backward, passes_back);
    j.pass[2] = pass_of(dout, q, k, dv, value, key, 0, 1, 1.f, d->scale, dstate_out, dstate_in, backward, passes_back);
    const int sources[] = {0, 2};         // one of each direction
    return hip_result(run(d, j, 3, sources, 2, (hipStream_t)stream), who);
}

extern "C" int ga3c_decay_attention_step(const ga3c_decay_desc *d, const ga3c_heads *q, const ga3c_heads *k, const ga3c_heads *v,
                                         const ga3c_heads *out, const int32_t *slots, const uint8_t *starts, int n, float *states, int n_slots,
                                         void *stream) {
    const char *who = "ga3c_decay_attention_step";
    int rc = check_desc(d, who);
    if (rc != GA3C_OK) return rc;
    if (n < 0 || n_slots < 0) return call_fail(GA3C_EINVAL, "%s: negative count", who);
    if (n > 1 << 22) return call_fail(GA3C_EINVAL, "%s: more than 2^22 tokens", who);
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
    const hipStream_t s = (hipStream_t)stream;
    const hipError_t e = by_shape(p.value, p.key, [&](auto lpr, auto cv, auto rpl) {
        constexpr int ROWS = 64 / lpr.value * rpl.value;
        const int slabs = (p.value + ROWS - 1) / ROWS;
        const dim3 grid((unsigned)(((int64_t)n * slabs + 3) / 4), d->n_heads);
        const bool bf = d->dtype == GA3C_BF16;
        const int vec = bf ? rows_of_four<bf16>(p.k) && rows_of_four<bf16>(p.q) : rows_of_four<float>(p.k) && rows_of_four<float>(p.q);
        const bool stream_states = p.key % 4 == 0 && (uintptr_t)states % 16 == 0 && (size_t)n * d->n_heads * p.key * p.value * sizeof(float) >= STREAM_BYTES;
        typedef void (*Kernel)(DecayStep, int, int);
        static const Kernel kernels[4] = {decay_step_kernel<float, lpr.value, cv.value, rpl.value, false>, decay_step_kernel<float, lpr.value, cv.value, rpl.value, true>,
                                          decay_step_kernel<bf16, lpr.value, cv.value, rpl.value, false>, decay_step_kernel<bf16, lpr.value, cv.value, rpl.value, true>};
        launch(kernels[2 * bf + stream_states], grid, dim3(256), 0, s, p, slabs, vec);
        return hipGetLastError();
    });
    return hip_result(e, who);
}
