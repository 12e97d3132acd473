// delta.hpp -- host-side launchers of the gated delta rule's kernels, called by the C ABI after argument
// validation.  Each returns hipSuccess or the launch error.
#pragma once

#include "linear.hpp"

namespace pm {

// What a chunk's preparation (delta_prep.hip) leaves for the walks, per batch row, head and chunk: products of
// 64 x 64 tokens as the 10 tiles of 16 x 16 on and below the diagonal, tile (i, j) at i (i + 1) / 2 + j, in the
// order of a matrix operand: lane l, values 4 (l / 16) .. + 3 of row l % 16.
constexpr int kDeltaTiles = 10;
constexpr int64_t kDeltaProduct = (int64_t)kDeltaTiles * 64 * 4;       // values of one product
// and its tokens' weights: in, up, beta, hi, lo, start (linear_walk.hpp), then a and whether k or q is not finite
enum : int { kCoefIn = 0, kCoefUp = 64, kCoefBeta = 128, kCoefHi = 192, kCoefLo = 256, kCoefStart = 320, kCoefA = 384, kDeltaCoef = 448 };

struct DeltaArgs {
    const void* q;              // (batch, groups, dk, seqlen)
    const void* k;
    const void* v;              // (batch, heads, dv, seqlen)
    const void* dout;
    const float* beta;          // (batch, heads, seqlen)
    const float* decay;         // per head or per token, or null
    const int32_t* pos;
    const float* entry;         // state that enters the row, or null (zeros); reverse: the final state's gradient
    float* leave;               // state that leaves it, or null; reverse: the initial state's gradient
    void* out;                  // forward: out; reverse: dv
    float* products;            // H, then P, of every chunk
    float* coef;
    // split rows: (batch, heads, nseg) of
    float* seg;                 // the state that enters a segment (first what it adds), dk x dv
    float* seg_m;               // what it multiplies the state with, dk x dk padded to tiles
    int32_t* seg_cut;           // whether a sequence starts in it
    // the backward's: per chunk the states before and the gradients after it, (dv, dk) padded to tiles; bf16: also the row's last state
    float* states;
    float* grads;
    float* bound;               // fp32: the states at every bound_chunks chunks' end again, in the threads' order
    float* dot;                 // their products with the gradients there, (batch, heads, nb + 1)
    void* e;                    // the errors, (batch, heads, dv, seqlen) in the inputs' type, rounded half up
    uint16_t* e_low;            // bf16: the lower halves of their fp32 patterns, as e
    void* w;                    // dv, rounded, where the out is of another type; else null
    uint16_t* w_low;            // bf16: what the rounding leaves of it, as e_low
    float* rq;                  // out . dout and -(v . dv) of every token
    float* rk;
    float* dbeta;
    void* dq;                   // (batch, groups, dk, seqlen), or fp32 of `parts` pieces a group
    void* dk_out;
    float scale;
    int64_t seqlen;
    int32_t batch, heads, groups, dk, dv;
    int32_t decay_mode;         // 0 none, 1 per head, 2 per token
    int32_t chunks, nseg, seg_chunks, bound_chunks, nb, bound_end;
    int32_t sum_segs;           // segments summed in time: all but the last, in the backward all
    int32_t heads_per;          // heads of a group that a block of the preparation takes
    int32_t grad_per;           // and one of the gradients of q and k
    int32_t dtype;              // 0 fp32, 1 bf16, 2 bf16 with fp32 out
};

inline int32_t delta_pad(int32_t n) { return n <= 64 ? 64 : 128; }

hipError_t launch_delta_prep(const DeltaArgs& a, hipStream_t s);
hipError_t launch_delta_fwd(const DeltaArgs& a, bool split, hipStream_t s);     // split: the states that enter the segments first
hipError_t launch_delta_states(const DeltaArgs& a, hipStream_t s);          // the backward's walk in time
hipError_t launch_delta_rev(const DeltaArgs& a, hipStream_t s);
hipError_t launch_delta_segments(const DeltaArgs& a, bool rev, hipStream_t s);
hipError_t launch_delta_grads(const DeltaArgs& a, bool f32, hipStream_t s);    // f32: dq and dk in 32 bits

struct DeltaStepArgs {
    const void* q;
    const void* k;
    const void* v;
    const float* beta;
    const float* decay;
    const int32_t* pos;
    float* state;
    void* out;
    float scale;
    int32_t batch, heads, groups, dk, dv, decay_mode, dtype;
};
hipError_t launch_delta_step(const DeltaStepArgs& a, hipStream_t s);

}  // namespace pm
