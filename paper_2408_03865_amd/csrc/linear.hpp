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
// from two launches more (aggregate and chain).  The plan is the cheapest in units of a chunk walked alone on a CU:
//   - a CU holds two blocks (one where dk and dv are both above 64), and a chunk in company takes 1.5 (8100 and
//     12300 cycles, dk 128, dv 64, bf16); blocks beyond a round follow as others end, with half a block's wait;
//   - an aggregate takes 0.45 of a walk; the backward has two for its three walks;
//   - a block costs three chunks besides its own, the two launches two (forward calls of 4 and 5 chunks: bf16 25 us
//     for 16 and 18 unsplit, fp32 25 for 32 and 38).
// These are bf16's numbers, and fp32 rows are split alike: the plan does not look at the type.  fp32 walks hold one
// block a CU in every form but the plain one of 64 x 64 (85 to 154 KB of LDS), so that 257 to 511 blocks of them are
// two rounds where it counts one.
// Us of a bf16 call, dk and dv 64, planned and unsplit (batch x heads x tokens, forward then the whole backward):
//   4 x 24 x 2048 56, 83; 188, 376   2 x 64 x 4096 (dk 128) 132, 206; 576, 1000   1 x 300 x 4096 222, 220; 1046, 1225
//   1 x 32 x 16384 103, 623; 398, 2670   1 x 8 x 320 24, 18; 58, 79   1 x 150 x 2048 (dk 128) 105, 108; 471, 565
// and 1 x 100 x 4096 with dk and dv 128 227, 259; 892, 1213.  More segments to use the four blocks a CU of one part
// (below) gain nothing: 1 x 32 x 65536 forward in 16 a row 455, in 32 492.
constexpr int64_t kSplitChunks = 4;     // rows of fewer are walked whole
// Blocks from which plain bf16 walks of heads of up to 64 features take one part (linear_walk.hpp).
constexpr int64_t kManyWalks = 768;
// Chunks between the boundaries at which the backward takes the product of the two states.
constexpr int32_t kBoundChunks = 8;

struct LinPlan {
    int32_t nseg, seg_chunks;
    int32_t bound_chunks, nb;
};
inline LinPlan linear_plan(int64_t batch, int64_t heads, int64_t dk, int64_t dv, int64_t seqlen, bool backward) {
    const int64_t chunks = (seqlen + kLinChunk - 1) / kLinChunk, blocks = batch * heads;
    const int64_t cus = 256, slots = dk > 64 && dv > 64 ? cus : 2 * cus;
    const double company = slots > cus ? 1.5 : 1.0, walk = backward ? 1.3 : 1.45;
    const auto load = [&](int64_t n) { return n <= cus ? 1.0 : n <= slots ? company : company * (double)n / (double)slots + 0.5; };
    int64_t best = chunks;
    if (blocks < slots && chunks >= kSplitChunks) {
        double least = load(blocks) * (double)chunks + 3.0;
        for (int64_t per = 1; per < chunks; ++per) {
            if (per > kBoundChunks) per = (per + kBoundChunks - 1) / kBoundChunks * kBoundChunks;
            if (per >= chunks) break;
            const int64_t n = blocks * ((chunks + per - 1) / per);
            if (n > 4 * slots) continue;
            const double rounds = n <= slots ? 1.0 : (double)n / (double)slots;
            const double cost = walk * load(n) * (double)per + 3.0 * rounds + 2.0;
            if (cost < least) {
                least = cost;
                best = per;
            }
        }
    }
    LinPlan p;
    p.seg_chunks = (int32_t)best;
    p.nseg = (int32_t)((chunks + best - 1) / best);
    p.bound_chunks = p.nseg > 1 && best < kBoundChunks ? (int32_t)best : kBoundChunks;
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
hipError_t launch_linear_group_sums(const float* part, void* out, const float* part1, void* out1, int64_t batch, int32_t heads,
                                    int32_t groups, int64_t n, bool f32, hipStream_t s);     // two tensors'

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
// Tokens of a block's tile: 64 (the fp32 forward 32) where that makes more than 64 tiles of them, 16 where fewer
// leave CUs idle, 8 for rows of no more.  Fewer tokens are more slices of the features, and shorter pieces of lines.
// Us of the bf16 forward and backward, tiles of 16 against 64 (batch x tokens x features, groups):
//   1 x 64 x 4096, 1 (1 tile of 64) 19, 48; 26, 73     1 x 512 x 4096, 1 (8) 19, 49; 27, 73    2 x 1024 x 4096, 1 (32) 29, 51; 54, 86
//   1 x 256 x 4096, 8 (32) 7.9, 10.3; 10.7, 16.6       1 x 512 x 4096, 8 (64) 9.0, 10.3; 13, 17    4 x 1024 x 4096, 1 (64) 49, 58; 94, 87
//   2 x 1024 x 4096, 4 (128) 24, 18; 39, 31            8 x 1024 x 4096, 1 (128) 91, 64; 166, 99
// and in fp32 4 x 1024 x 4096, 1 57, 56; 94, 131, 2 x 1024 x 4096, 4 24, 19; 46, 47.
// Rows of 4 and 8 tokens (4 x 4096, 1 group, bf16): tiles of 8 18 and 10 us, of 64 78 and 54.
constexpr int64_t kGatedFewTokens = 8, kGatedFewTiles = 64, kGatedNarrow = 16;
inline int64_t gated_tile(int64_t batch, int64_t seqlen, int64_t groups) {
    if (seqlen <= kGatedFewTokens) return kGatedFewTokens;
    return batch * groups * ((seqlen + kRmsTile - 1) / kRmsTile) <= kGatedFewTiles ? kGatedNarrow : kRmsTile;
}
// rows of dweight's partial sums: one for each tile of a batch row
inline int64_t gated_bwd_partial_rows(int64_t batch, int64_t seqlen, int64_t groups) {
    const int64_t tile = gated_tile(batch, seqlen, groups);
    return batch * ((seqlen + tile - 1) / tile);
}
hipError_t launch_gated_fwd(const GatedArgs& a, hipStream_t s);
hipError_t launch_gated_bwd(const GatedArgs& a, hipStream_t s);

}  // namespace pm
