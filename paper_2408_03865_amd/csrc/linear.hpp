// linear.hpp -- host-side launchers of the linear-attention kernels and the gated RMSNorm,
// called by the C ABI after argument validation.  Each returns hipSuccess or the launch error.
#pragma once

#include <hip/hip_runtime.h>
#include <stddef.h>
#include <stdint.h>

#include "launch.hpp"

namespace pm {

constexpr int64_t kLinChunk = 64;       // tokens of a chunk
constexpr int32_t kLinMaxHead = 128;    // features of a head, dk and dv

// A tensor in one of a walk's roles: (batch, heads, rows, seqlen); head h of the walk reads
// its head h / (walk's heads / heads).
struct WalkTensor {
    const void* p;
    int32_t rows, heads;
};

// One walk over the chunks of every row and head (linear_walk.hpp says what it computes).
struct WalkArgs {
    WalkTensor x, y, z;
    WalkTensor e;           // MODE dq and dk: what the out is multiplied with for the decay's gradient
    void* out;              // (batch, heads, z.rows, seqlen)
    const float* decay;     // per head or per token, or null
    const int32_t* pos;     // (batch, seqlen)
    const float* entry;     // state that enters the row, or null (zeros)
    float* leave;           // state that leaves it, or null
    float* seg;             // split rows: the state that enters each segment, (batch, heads, nseg, x.rows z.rows)
    float* seg_a;           // and what a segment multiplies it by, -1 where it is cut, (batch, heads, nseg)
    float* bound;           // dq writes, dk reads: the states at the boundaries, in the threads' order
    float* dot;             // dk writes: (batch, heads, nb + 1) products of the two states at the boundaries
    float* r;               // dq, dk: (batch, heads, seqlen), their parts of the decay's gradient
    float pscale, iscale, uscale;   // of the products inside a chunk, of the entering state's, of the update
    int64_t seqlen;
    int32_t batch, heads;
    int32_t decay_mode;     // 0 none, 1 per head, 2 per token
    int32_t rev;            // from the last token to the first
    int32_t nseg, seg_chunks;
    int32_t bound_chunks, nb;       // chunks between boundaries, boundaries of a row (the last: its end)
    int32_t bound_end;      // the row's end is a boundary too
    int32_t s_x, s_z;       // strides of the state's x and z features in entry, leave and seg
    int32_t dtype;          // 0 fp32, 1 bf16, 2 bf16 with fp32 out
};

enum WalkMode : int { kWalkPlain = 0, kWalkDq = 1, kWalkDk = 2 };

// exact: the state that leaves is an output, or a gradient is taken from the states: the update's
// operands are split so that the state keeps 32-bit accuracy (else 16 bits of the weighted values).
hipError_t launch_walk(const WalkArgs& a, WalkMode mode, bool exact, hipStream_t s);
hipError_t launch_walk_segments(const WalkArgs& a, hipStream_t s);
// floats of one stored state, in the threads' order
inline int64_t walk_bound_floats(int32_t x_rows, int32_t z_rows) {
    return (int64_t)(x_rows <= 64 ? 64 : 128) * (z_rows <= 64 ? 64 : 128);
}

// Split of the rows into segments of whole chunks, each walked by its own block, with the states that enter them
// from two launches more (aggregate and chain): where rows and heads give the CUs less than a block each, and
// rows are long enough.  Two blocks a CU are aimed at.  Us of a walk of 4096 tokens, dk 128 and dv 64, bf16:
// 512 (row, head) pairs 330, 128 pairs unsplit 217, so that a chunk takes 8100 cycles alone and 12300 with another
// block on its CU; 128 pairs in four segments 105 with the two launches.  256 pairs gain nothing by it.
constexpr int64_t kWalkBlocks = 512;
// Rows of fewer chunks are walked whole: the launches take as long as the chunks (256 tokens, 2 heads, fp32, the
// whole backward: 65 us split, 126 unsplit).
constexpr int64_t kSplitChunks = 4;
// Chunks between the boundaries at which the backward takes the product of the two states.
constexpr int32_t kBoundChunks = 8;

struct LinPlan {
    int32_t nseg, seg_chunks;
    int32_t bound_chunks, nb;
};
inline LinPlan linear_plan(int64_t batch, int64_t heads, int64_t seqlen) {
    const int64_t chunks = (seqlen + kLinChunk - 1) / kLinChunk, blocks = batch * heads;
    int64_t nseg = blocks >= kWalkBlocks / 2 || chunks < kSplitChunks ? 1 : (kWalkBlocks + blocks - 1) / blocks;
    if (nseg > chunks) nseg = chunks;
    int64_t per = (chunks + nseg - 1) / nseg;
    if (nseg > 1 && per > kBoundChunks) per = (per + kBoundChunks - 1) / kBoundChunks * kBoundChunks;
    LinPlan p;
    p.seg_chunks = (int32_t)per;
    p.nseg = (int32_t)((chunks + per - 1) / per);
    p.bound_chunks = p.nseg > 1 && per < kBoundChunks ? (int32_t)per : kBoundChunks;
    p.nb = (int32_t)((chunks + p.bound_chunks - 1) / p.bound_chunks);
    return p;
}

struct LinDecayArgs {
    const float* rq;        // (batch, heads, seqlen)
    const float* rk;
    const float* dot;       // (batch, heads, nb + 1)
    const float* decay;
    const int32_t* pos;
    float* ddecay;          // per head or per token
    float* partial;         // per head: (heads, batch, nb)
    int64_t seqlen;
    int32_t batch, heads, decay_mode, bound_tokens, nb, bound_end;
};
hipError_t launch_linear_ddecay(const LinDecayArgs& a, hipStream_t s);

// out[b, g, i] = sum over the heads of group g of part[b, h, i], i < n, in the heads' order
hipError_t launch_linear_group_sum(const float* part, void* out, int64_t batch, int32_t heads, int32_t groups, int64_t n,
                                   bool f32, hipStream_t s);

struct LinStepArgs {
    const void* q;
    const void* k;
    const void* v;
    const float* decay;
    const int32_t* pos;
    float* state;
    void* out;
    float scale;
    int32_t batch, heads, groups, dk, dv, decay_mode, dtype;
};
hipError_t launch_linear_step(const LinStepArgs& a, hipStream_t s);

struct GatedArgs {
    const void* x;
    const void* z;
    const float* w;
    const float* rstd;      // bwd: saved by the forward, (batch, groups, seqlen)
    const void* dout;       // bwd only
    void* out;              // fwd: out; bwd: dx
    void* dz;               // bwd only
    float* rstd_out;        // fwd
    float* dw;              // bwd only
    float* partial;         // bwd only
    float eps;
    int64_t batch, dim, seqlen;
    int32_t groups, gate_first, dtype;
};
// rows of dweight's partial sums: one for each kRmsTile tokens of a batch row
inline int64_t gated_bwd_partial_rows(int64_t batch, int64_t seqlen) {
    return batch * ((seqlen + kRmsTile - 1) / kRmsTile);
}
hipError_t launch_gated_fwd(const GatedArgs& a, hipStream_t s);
hipError_t launch_gated_bwd(const GatedArgs& a, hipStream_t s);

}  // namespace pm
