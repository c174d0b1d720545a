// What the passes of decay_attention.hip compute, and how they are described to the kernels.
#pragma once
#include <hip/hip_runtime.h>

#include "../../include/ga3c.h"

namespace ga3c {

// One pass over the segments.  Forward in time (back == 0), with a state X of [rows][cols] per segment and head:
//     X = start ? 0 : X;  X = decay X + row_t col_t^T;  out_t = out_scale X by_t
// and backward (back == 1), from the last token of a segment to its first:
//     Y = X + col_scale row_t col_t^T;  out_t = out_scale Y by_t;  X = start ? 0 : decay Y
// `row` has the output's width, `col` and `by` the other one.  The output of the operator and each of its three gradients are
// passes of this kind: (row, col, by) = (v, k, q) gives out, (k, v, dout) dq, backward (dout, q, k) dv, and (q, dout, v) dk.
struct DecayView { void *data; int64_t token, head; };      // strides in elements
struct DecayPass {
    DecayView row, col, by, out;
    int rows, cols;
    int turned;                      // states lie in memory as [cols][rows]
    int back;
    float out_scale, col_scale;
    const float *x_in;               // nullptr: zero
    float *x_out;                    // nullptr: not wanted
    float *spans;                    // states between the spans of a segment
    float *passes;                   // whether a span passes the state in front of it on: 1, or 0
};
struct DecayJob {
    DecayPass pass[3];               // one grid: a pass per z
    const int32_t *seg_start;        // nullptr: segments of `len` tokens each
    const uint8_t *starts;           // nullptr: none
    int n_segments, n_tokens, len;
    int span;                        // tokens of a segment that one block of the chunked kernels takes
    int items;                       // blocks' places for spans: those of segment i begin at seg_start[i] / span + i
    int brief;                       // segments of up to so many tokens go to the token-by-token kernel, longer ones to the chunked,
                                     // in one span each; -1: all to the chunked
    float decay[GA3C_MAX_HEADS];
};

// Scratch for a call on up to n_tokens tokens, in whatever segments, in bytes.
size_t decay_workspace_most(const ga3c_decay_desc *d, int n_tokens);

}  // namespace ga3c
