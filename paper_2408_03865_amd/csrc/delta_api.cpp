// delta_api.cpp -- the C ABI of packmamba_delta.h: argument validation (before anything is
// enqueued), workspace layout and the order of the launches.
#include <hip/hip_runtime.h>

#include <cstdint>

#include "delta.hpp"
#include "norms.hpp"
#include "packmamba_delta.h"

namespace {

constexpr size_t kAlign = 256;
constexpr int64_t kMaxSeqlen = (int64_t)1 << 22;    // 128 rows of it in fp32 are an offset of 32 bits in the walks
// Chunks of all rows and heads: up to 382 KB of workspace each in a backward of two heads that share keys, some hundred tokens and
// segments of two chunks, 215 KB in the largest calls.
constexpr int64_t kMaxUnits = (int64_t)1 << 20;

inline size_t align_up(size_t v) { return (v + kAlign - 1) / kAlign * kAlign; }
inline size_t floats(int64_t n) { return align_up(sizeof(float) * (size_t)n); }
inline int launch_status(hipError_t e) { return e == hipSuccess ? PACKMAMBA_OK : PACKMAMBA_ERR_LAUNCH; }

template <typename... P>
bool aligned16(P... p) {
    return ((((uintptr_t)p & 15u) == 0) && ...);
}

int check_dtype(int32_t dtype) {
    return (dtype == PACKMAMBA_F32 || dtype == PACKMAMBA_BF16 || dtype == PACKMAMBA_BF16_F32OUT) ? PACKMAMBA_OK
                                                                                                 : PACKMAMBA_ERR_UNSUPPORTED;
}

int check_heads(int64_t batch, int64_t heads, int64_t groups, int64_t dk, int64_t dv, int64_t seqlen) {
    if (batch <= 0 || heads <= 0 || groups <= 0 || dk <= 0 || dv <= 0 || seqlen <= 0) return PACKMAMBA_ERR_SHAPE;
    if (heads > kMaxUnits || batch > kMaxUnits / heads || heads % groups) return PACKMAMBA_ERR_SHAPE;
    if (dk > PACKMAMBA_DELTA_MAX_HEAD || dv > PACKMAMBA_DELTA_MAX_HEAD) return PACKMAMBA_ERR_UNSUPPORTED;
    if (seqlen > kMaxSeqlen || (seqlen + pm::kLinChunk - 1) / pm::kLinChunk > kMaxUnits / (batch * heads)) return PACKMAMBA_ERR_SHAPE;
    return PACKMAMBA_OK;
}

constexpr int64_t kMaxNormRows = (int64_t)1 << 20;
constexpr int64_t kMaxNormTiles = ((int64_t)1 << 22) - 1;   // tiles of 16 tokens, a block of up to 1024 threads each
constexpr int64_t kMaxNormDim = ((int64_t)1 << 26) - 32;    // the sums over tokens take 64 threads a feature, 2^32 in all
constexpr int64_t kMaxElems = (int64_t)1 << 33;

int check_norm(int64_t batch, int64_t dim, int64_t seqlen, int64_t groups) {
    if (batch <= 0 || dim <= 0 || seqlen <= 0 || groups <= 0 || dim % groups) return PACKMAMBA_ERR_SHAPE;
    if (groups > kMaxNormRows || batch > kMaxNormRows / groups) return PACKMAMBA_ERR_SHAPE;
    if (dim > kMaxNormDim || seqlen > INT32_MAX / 2) return PACKMAMBA_ERR_SHAPE;
    if (batch * dim > kMaxElems / seqlen) return PACKMAMBA_ERR_SHAPE;
    if (batch * groups > kMaxNormTiles / ((seqlen + 15) / 16)) return PACKMAMBA_ERR_SHAPE;
    return PACKMAMBA_OK;
}

pm::NormArgs norm_args(const void* x, int64_t rows, int64_t dim, int64_t seqlen, int32_t dtype) {
    pm::NormArgs a{};
    a.x = x; a.rows = rows; a.dim = dim; a.seqlen = seqlen; a.dtype = dtype;
    return a;
}

// Split of the rows into segments of whole chunks, each walked by its own block.
struct Plan {
    int64_t chunks, units;
    int32_t nseg, seg_chunks, bound, nb, heads_per, grad_per, grad_parts;
};
// Chunks between the boundaries at which the backward multiplies the two states.  A decay's gradient is a sum over the tokens up
// to the next, of terms that cancel: its error grows with their number.  In bf16 every chunk ends at one, whose state the gradients
// keep anyway; in fp32 boundaries have a copy of it, which moves memory.  Us with 1, 2 and 4 chunks (batch x heads x tokens, dk x dv;
// the chunks of all heads):
//   fp32   1 x 16 x 2048, 64 x 64 (512) 221, 217, 216    2 x 16 x 2048 (1024) 283, 279, 278    4 x 16 x 2048 (2048) 480, 471, 470
//          8 x 16 x 2048 (4096) 888, 868, 865, of 128 x 128 2445, 2367, 2328    16 x 16 x 2048, 64 x 64 (8192) 1413, 1363, 1338
//          8 x 32 x 4096, 128 x 128 (16384) 6950, 6750, 6670: 1 costs 2% to 1024 chunks, 2 1% or less to 4096 but for 128 x 128.  Errors in the
//          2-norm 5.0e-7 to 5.8e-7, 6.1e-7 to 8.1e-7, 8.0e-7 to 1.1e-6
//   bf16   4 x 24 x 2048, 64 x 64 397, 391, 393    8 x 16 x 2048, 128 x 128 1119, 1091, 1080    8 x 32 x 4096 3328, 3241, 3209; errors of the
//          last 4.5e-7, 6.0e-7, 7.9e-7 (the plain form 5.6e-7)
int32_t bound_chunks(int64_t units, bool f32) { return !f32 || units <= 1024 ? 1 : units <= 4096 ? 2 : 4; }
// Heads of a group that one block takes: all, or fewer where that leaves the GPU's CUs without blocks.  Us with this rule, with
// all heads of a group in a block and with one (batch x heads in groups x tokens, dk x dv; bf16):
//   the preparation, forward    1 x 32 in 1 x 512, 128 x 128: 63, 175, 63    2 x 64 in 4 x 2048, 128 x 128: 245, 270, 246
//                               8 x 32 in 16 x 4096, 128 x 128: 610, 610, 637    1 x 24 in 8 x 30001, 128 x 64: 597, 597, 629
//   gradients of q, k, backward 1 x 32 in 1 x 512, 128 x 128: 165, 579, 157    1 x 16 in 1 x 4096, 64 x 64: 196, 286, 194
//                               8 x 32 in 16 x 4096, 128 x 128: 3018, 3018, 3330    4 x 24 in 8 x 2048, 64 x 64: 368, 368, 405
int32_t heads_for(int64_t blocks, int64_t rep, int64_t target) {
    int64_t per = rep;
    while (per > 1 && blocks * ((rep + per - 1) / per) < target) per = (per + 1) / 2;
    return (int32_t)per;
}

// The cheapest split, in units of a chunk walked alone on a CU (4.4 us forward, 3.5 in one of the backward's walks; with these, the
// figures below to within 10%):
//   - a CU holds two blocks of heads with up to 64 features of v, one with more; a chunk in company takes 1.35, and
//     blocks beyond a round add to it, in the walks that end a call with a quarter of a block's wait besides;
//   - a sum walk takes 0.55 of one forward and 0.7 in the backward (0.3 backwards) and needs a block more for every 64 or 128
//     columns of the multiplier; the chain of the segments' states 0.4 (0.5) a segment;
//   - a block costs a chunk besides its own, the launches 1.6 (2).
// Us of a bf16 call by chunks a segment (batch x heads x tokens, dk x dv):
//   forward   1 x 24 x 30001, 128 x 64: unsplit 2535, 20 757, 22 742, 27 689, 36 736    1 x 8 x 16384, 64 x 64: 1004, 4 143, 8 121, 16 152
//             1 x 64 x 8192, 128 x 128: 888, 16 656, 32 593, 43 577, 64 775    2 x 24 x 4096, 64 x 64: 279, 4 133, 8 127, 16 161
//             1 x 4 x 1024, 64 x 64: 72, 2 37, 4 46, 8 70    1 x 4 x 512: 41, 2 34, 4 44    4 x 32 x 4096, 128 x 128: 498, 16 580, 32 466
//             2 x 64 x 4096, 64 x 64: 338, 8 294, 16 261, 32 311
//   backward  4 x 24 x 2048, 64 x 64: 497, 4 411, 8 397, 16 473    1 x 32 x 4096, 128 x 128: 1439, 4 678, 8 613, 16 759
//             1 x 4 x 1024, 64 x 64: 199, 2 94, 4 121, 8 183    4 x 32 x 4096, 128 x 128: 2149, 16 2185, 32 2092
//             1 x 24 x 30001, 128 x 64: 8781, 20 2427, 27 2234, 36 2455
int64_t segment_chunks(int64_t rows, int64_t dk, int64_t dv, int64_t chunks, bool backward) {
    const double slots = dv <= 64 ? 512 : 256, company = dv <= 64 ? 1.35 : 1.0;
    const int64_t columns = 1 + ((dk <= 64 ? 64 : 128) + (dv <= 64 ? 64 : 128) - 1) / (dv <= 64 ? 64 : 128);
    const auto load = [&](int64_t n) { return n <= 256 ? 1.0 : (double)n <= slots ? company : company * (double)n / slots; };
    const double walks = backward ? 2.0 : 1.0, sums = backward ? 0.7 : 0.55, chain = backward ? 0.5 : 0.4, launches = backward ? 2.0 : 1.6;
    int64_t best = chunks;
    double least = walks * load(rows) * (double)(chunks + 1);
    if (rows > 256) return best;
    for (int64_t per = 2; per < chunks; per += (per + 2) / 3) {      // 2, 3, 4, 6, 8, 11, 15, 20, 27, ...
        const int64_t nseg = (chunks + per - 1) / per;
        const double block = (double)(per + 1);
        const double walk = load(rows * nseg) + ((double)(rows * nseg) > slots ? 0.25 : 0.0);
        double cost = walks * block * walk + sums * block * load(rows * (backward ? nseg : nseg - 1) * columns) + chain * (double)nseg + launches;
        if (backward) cost += 0.3 * block * load(rows * (nseg - 1)) + chain * (double)nseg + launches;
        if (cost < least) {
            least = cost;
            best = per;
        }
    }
    return best;
}

Plan make_plan(int64_t batch, int64_t heads, int64_t groups, int64_t dk, int64_t dv, int64_t seqlen, bool backward, bool f32 = false) {
    Plan p;
    p.chunks = (seqlen + pm::kLinChunk - 1) / pm::kLinChunk;
    const int64_t rows = batch * heads, per = segment_chunks(rows, dk, dv, p.chunks, backward);
    p.units = rows * p.chunks;
    p.seg_chunks = (int32_t)per;
    p.nseg = (int32_t)((p.chunks + per - 1) / per);
    p.bound = bound_chunks(p.units, f32);
    p.nb = (int32_t)((p.chunks + p.bound - 1) / p.bound);
    const int64_t rep = heads / groups, blocks = batch * p.chunks * groups;
    p.heads_per = heads_for(blocks, rep, 1024);
    p.grad_per = heads_for(blocks * (dk <= 64 ? 1 : 2), rep, 256);
    p.grad_parts = (int32_t)((rep + p.grad_per - 1) / p.grad_per);
    return p;
}

// Hands out pieces of the workspace, or with none sums them up.
struct Taker {
    char* base;
    size_t at = 0;
    void* take(size_t bytes) {
        void* got = base ? base + at : nullptr;
        at += align_up(bytes);
        return got;
    }
    float* floats(int64_t n) { return static_cast<float*>(take(sizeof(float) * (size_t)n)); }
};

void take_common(Taker& t, pm::DeltaArgs& a, const Plan& p, int64_t rows, int64_t dk, int64_t dv) {
    a.products = t.floats(p.units * 2 * pm::kDeltaProduct);
    a.coef = t.floats(p.units * pm::kDeltaCoef);
    if (p.nseg > 1) {
        const int64_t pad = pm::delta_pad((int32_t)dk);
        a.seg = t.floats(rows * p.nseg * dk * dv);
        a.seg_m = t.floats(rows * p.nseg * pad * pad);
        a.seg_cut = static_cast<int32_t*>(t.take(sizeof(int32_t) * (size_t)(rows * p.nseg)));
    }
}

struct BwdExtra {
    float *pieces, *dq, *dk;
};
BwdExtra take_bwd(Taker& t, pm::DeltaArgs& a, const Plan& p, int64_t batch, int64_t heads, int64_t groups, int64_t dk, int64_t dv,
                  int64_t seqlen, int32_t dtype) {
    const int64_t rows = batch * heads, state = (int64_t)pm::delta_pad((int32_t)dk) * pm::delta_pad((int32_t)dv);
    const bool f32 = dtype == PACKMAMBA_F32;
    const size_t size = f32 ? 4 : 2;
    take_common(t, a, p, rows, dk, dv);
    a.states = t.floats((f32 ? p.units : p.units + rows) * state);
    a.grads = t.floats(p.units * state);
    a.bound = f32 ? t.floats(rows * p.nb * state) : nullptr;
    a.dot = t.floats(rows * (p.nb + 1));
    a.e = t.take(size * (size_t)(rows * dv * seqlen));
    if (!f32) {
        a.e_low = static_cast<uint16_t*>(t.take(size * (size_t)(rows * dv * seqlen)));
        a.w_low = static_cast<uint16_t*>(t.take(size * (size_t)(rows * dv * seqlen)));
    }
    a.w = dtype == PACKMAMBA_BF16_F32OUT ? t.take(size * (size_t)(rows * dv * seqlen)) : nullptr;
    a.rq = t.floats(rows * seqlen);
    a.rk = t.floats(rows * seqlen);
    BwdExtra x{};
    x.pieces = t.floats(rows * p.nb);
    if (p.grad_parts > 1) {
        x.dq = t.floats(batch * groups * p.grad_parts * dk * seqlen);
        x.dk = t.floats(batch * groups * p.grad_parts * dk * seqlen);
    }
    return x;
}

void set_plan(pm::DeltaArgs& a, const Plan& p) {
    a.chunks = (int32_t)p.chunks;
    a.nseg = p.nseg;
    a.seg_chunks = p.seg_chunks;
    a.bound_chunks = p.bound;
    a.nb = p.nb;
    a.heads_per = p.heads_per;
    a.grad_per = p.grad_per;
}

}  // namespace

extern "C" {

size_t packmamba_delta_rule_fwd_workspace_size(int64_t batch, int64_t heads, int64_t groups, int64_t dk, int64_t dv,
                                               int64_t seqlen) {
    if (check_heads(batch, heads, groups, dk, dv, seqlen)) return 0;
    Taker t{nullptr};
    pm::DeltaArgs a{};
    take_common(t, a, make_plan(batch, heads, groups, dk, dv, seqlen, false), batch * heads, dk, dv);
    return t.at;
}

int packmamba_delta_rule_fwd(const void* q, const void* k, const void* v, const float* beta, const float* decay,
                             const int32_t* position_indices, const float* initial_state, float scale, void* out,
                             float* final_state, void* workspace, size_t workspace_bytes, int64_t batch, int64_t heads,
                             int64_t groups, int64_t dk, int64_t dv, int64_t seqlen, int32_t decay_per_token,
                             int32_t dtype, void* stream) {
    if (!q || !k || !v || !beta || !position_indices || !out) return PACKMAMBA_ERR_NULL;
    if (int e = check_heads(batch, heads, groups, dk, dv, seqlen)) return e;
    if (int e = check_dtype(dtype)) return e;
    if (!aligned16(q, k, v, beta, decay, position_indices, initial_state, out, final_state, workspace)) return PACKMAMBA_ERR_ALIGN;
    const Plan p = make_plan(batch, heads, groups, dk, dv, seqlen, false);
    Taker t{static_cast<char*>(workspace)};
    pm::DeltaArgs a{};
    take_common(t, a, p, batch * heads, dk, dv);
    if (!workspace || workspace_bytes < t.at) return PACKMAMBA_ERR_WORKSPACE;
    a.q = q; a.k = k; a.v = v; a.beta = beta; a.decay = decay; a.pos = position_indices;
    a.entry = initial_state; a.leave = final_state; a.out = out; a.scale = scale;
    a.seqlen = seqlen; a.batch = (int32_t)batch; a.heads = (int32_t)heads; a.groups = (int32_t)groups;
    a.dk = (int32_t)dk; a.dv = (int32_t)dv; a.dtype = dtype;
    a.decay_mode = decay ? (decay_per_token ? 2 : 1) : 0;
    set_plan(a, p);
    a.sum_segs = p.nseg - 1;
    const hipStream_t s = (hipStream_t)stream;
    if (int e = launch_status(pm::launch_delta_prep(a, s))) return e;
    return launch_status(pm::launch_delta_fwd(a, p.nseg > 1, s));
}

size_t packmamba_delta_rule_bwd_workspace_size(int64_t batch, int64_t heads, int64_t groups, int64_t dk, int64_t dv,
                                               int64_t seqlen, int32_t dtype) {
    if (check_heads(batch, heads, groups, dk, dv, seqlen) || check_dtype(dtype)) return 0;
    Taker t{nullptr};
    pm::DeltaArgs a{};
    take_bwd(t, a, make_plan(batch, heads, groups, dk, dv, seqlen, true, dtype == PACKMAMBA_F32), batch, heads, groups, dk, dv, seqlen, dtype);
    return t.at;
}

int packmamba_delta_rule_bwd(const void* q, const void* k, const void* v, const float* beta, const float* decay,
                             const int32_t* position_indices, const float* initial_state, float scale, const void* dout,
                             const float* dfinal_state, void* dq, void* dk, void* dv, float* dbeta, float* ddecay,
                             float* dinitial_state, void* workspace, size_t workspace_bytes, int64_t batch,
                             int64_t heads, int64_t groups, int64_t dk_size, int64_t dv_size, int64_t seqlen,
                             int32_t decay_per_token, int32_t dtype, void* stream) {
    if (!q || !k || !v || !beta || !position_indices || !dout || !dq || !dk || !dv || !dbeta) return PACKMAMBA_ERR_NULL;
    if (ddecay && !decay) return PACKMAMBA_ERR_NULL;
    if ((initial_state == nullptr) != (dinitial_state == nullptr)) return PACKMAMBA_ERR_NULL;
    if (int e = check_heads(batch, heads, groups, dk_size, dv_size, seqlen)) return e;
    if (int e = check_dtype(dtype)) return e;
    if (!aligned16(q, k, v, beta, decay, position_indices, initial_state, dout, dfinal_state) ||
        !aligned16(dq, dk, dv, dbeta, ddecay, dinitial_state, workspace))
        return PACKMAMBA_ERR_ALIGN;
    const Plan p = make_plan(batch, heads, groups, dk_size, dv_size, seqlen, true, dtype == PACKMAMBA_F32);
    Taker t{static_cast<char*>(workspace)};
    pm::DeltaArgs a{};
    const BwdExtra x = take_bwd(t, a, p, batch, heads, groups, dk_size, dv_size, seqlen, dtype);
    if (!workspace || workspace_bytes < t.at) return PACKMAMBA_ERR_WORKSPACE;
    a.q = q; a.k = k; a.v = v; a.dout = dout; a.beta = beta; a.decay = decay; a.pos = position_indices;
    a.scale = scale; a.dbeta = dbeta;
    a.seqlen = seqlen; a.batch = (int32_t)batch; a.heads = (int32_t)heads; a.groups = (int32_t)groups;
    a.dk = (int32_t)dk_size; a.dv = (int32_t)dv_size; a.dtype = dtype;
    a.decay_mode = decay ? (decay_per_token ? 2 : 1) : 0;
    a.bound_end = dfinal_state != nullptr;
    set_plan(a, p);
    a.sum_segs = p.nseg;                // the reverse walk takes the last segment's multiplier too
    const hipStream_t s = (hipStream_t)stream;
    if (int e = launch_status(pm::launch_delta_prep(a, s))) return e;
    a.entry = initial_state;
    if (p.nseg > 1)
        if (int e = launch_status(pm::launch_delta_segments(a, false, s))) return e;
    if (int e = launch_status(pm::launch_delta_states(a, s))) return e;

    a.entry = dfinal_state;
    a.leave = dinitial_state;
    a.out = dv;
    if (p.nseg > 1)
        if (int e = launch_status(pm::launch_delta_segments(a, true, s))) return e;
    if (int e = launch_status(pm::launch_delta_rev(a, s))) return e;

    if (!a.w) a.w = dv;
    const bool pieces = p.grad_parts > 1;
    a.dq = pieces ? x.dq : dq;
    a.dk_out = pieces ? x.dk : dk;
    if (int e = launch_status(pm::launch_delta_grads(a, pieces || dtype != PACKMAMBA_BF16, s))) return e;
    if (pieces) {
        if (int e = launch_status(pm::launch_linear_group_sums(x.dq, dq, x.dk, dk, batch, (int32_t)groups * p.grad_parts, (int32_t)groups,
                                                               dk_size * seqlen, dtype != PACKMAMBA_BF16, s)))
            return e;
    }
    if (!ddecay) return PACKMAMBA_OK;
    pm::LinDecayArgs d{};
    d.rq = a.rq; d.rk = a.rk; d.dot = a.dot; d.decay = decay; d.pos = position_indices; d.ddecay = ddecay; d.partial = x.pieces;
    d.seqlen = seqlen; d.batch = a.batch; d.heads = a.heads; d.decay_mode = a.decay_mode;
    d.bound_tokens = p.bound * (int32_t)pm::kLinChunk; d.nb = p.nb; d.bound_end = a.bound_end;
    return launch_status(pm::launch_linear_ddecay(d, s));
}

int packmamba_delta_rule_step(const void* q, const void* k, const void* v, const float* beta, const float* decay,
                              const int32_t* position_indices, float* state, float scale, void* out, int64_t batch,
                              int64_t heads, int64_t groups, int64_t dk, int64_t dv, int32_t decay_per_token,
                              int32_t dtype, void* stream) {
    if (!q || !k || !v || !beta || !state || !out) return PACKMAMBA_ERR_NULL;
    if (int e = check_heads(batch, heads, groups, dk, dv, 1)) return e;
    if (int e = check_dtype(dtype)) return e;
    if (!aligned16(q, k, v, beta, decay, position_indices, state, out)) return PACKMAMBA_ERR_ALIGN;
    pm::DeltaStepArgs a{};
    a.q = q; a.k = k; a.v = v; a.beta = beta; a.decay = decay; a.pos = position_indices; a.state = state; a.out = out; a.scale = scale;
    a.batch = (int32_t)batch; a.heads = (int32_t)heads; a.groups = (int32_t)groups;
    a.dk = (int32_t)dk; a.dv = (int32_t)dv;
    a.decay_mode = decay ? (decay_per_token ? 2 : 1) : 0;
    a.dtype = dtype;
    return launch_status(pm::launch_delta_step(a, (hipStream_t)stream));
}

int packmamba_head_l2norm_fwd(const void* x, float eps, void* out, float* rnorm, int64_t batch, int64_t dim,
                              int64_t seqlen, int64_t groups, int32_t dtype, void* stream) {
    if (!x || !out || !rnorm) return PACKMAMBA_ERR_NULL;
    if (int e = check_norm(batch, dim, seqlen, groups)) return e;
    if (int e = check_dtype(dtype)) return e;
    if (!(eps >= 0.0f)) return PACKMAMBA_ERR_SHAPE;
    if (!aligned16(x, out, rnorm)) return PACKMAMBA_ERR_ALIGN;
    pm::NormArgs a = norm_args(x, batch * groups, dim / groups, seqlen, dtype);
    a.eps = eps; a.out = out; a.rstd_out = rnorm;
    return launch_status(pm::launch_l2norm_fwd(a, (hipStream_t)stream));
}

int packmamba_head_l2norm_bwd(const void* x, const float* rnorm, const void* dout, void* dx, int64_t batch, int64_t dim,
                              int64_t seqlen, int64_t groups, int32_t dtype, void* stream) {
    if (!x || !rnorm || !dout || !dx) return PACKMAMBA_ERR_NULL;
    if (int e = check_norm(batch, dim, seqlen, groups)) return e;
    if (int e = check_dtype(dtype)) return e;
    if (!aligned16(x, rnorm, dout, dx)) return PACKMAMBA_ERR_ALIGN;
    pm::NormArgs a = norm_args(x, batch * groups, dim / groups, seqlen, dtype);
    a.rstd = rnorm; a.dout = dout; a.out = dx;
    return launch_status(pm::launch_l2norm_bwd(a, (hipStream_t)stream));
}

int packmamba_layernorm_fwd(const void* x, const float* weight, const float* bias, float eps, void* out, float* mean,
                            float* rstd, int64_t batch, int64_t dim, int64_t seqlen, int32_t dtype, void* stream) {
    if (!x || !weight || !out || !mean || !rstd) return PACKMAMBA_ERR_NULL;
    if (int e = check_norm(batch, dim, seqlen, 1)) return e;
    if (int e = check_dtype(dtype)) return e;
    if (!(eps >= 0.0f)) return PACKMAMBA_ERR_SHAPE;
    if (!aligned16(x, weight, bias, out, mean, rstd)) return PACKMAMBA_ERR_ALIGN;
    pm::NormArgs a = norm_args(x, batch, dim, seqlen, dtype);
    a.w = weight; a.b = bias; a.eps = eps; a.out = out; a.mean_out = mean; a.rstd_out = rstd;
    return launch_status(pm::launch_layernorm_fwd(a, (hipStream_t)stream));
}

size_t packmamba_layernorm_bwd_workspace_size(int64_t batch, int64_t dim, int64_t seqlen, int32_t dtype) {
    if (check_norm(batch, dim, seqlen, 1) || check_dtype(dtype)) return 0;
    return floats(pm::norm_tiles(batch, seqlen, dtype == PACKMAMBA_F32) * 2 * dim);
}

int packmamba_layernorm_bwd(const void* x, const float* weight, const float* mean, const float* rstd, const void* dout,
                            const void* dresidual, void* dx, float* dweight, float* dbias, void* workspace,
                            size_t workspace_bytes, int64_t batch, int64_t dim, int64_t seqlen, int32_t dtype,
                            void* stream) {
    if (!x || !weight || !mean || !rstd || !dout || !dx || !dweight) return PACKMAMBA_ERR_NULL;
    if (int e = check_norm(batch, dim, seqlen, 1)) return e;
    if (int e = check_dtype(dtype)) return e;
    if (!aligned16(x, weight, mean, rstd, dout, dresidual, dx, dweight, dbias, workspace)) return PACKMAMBA_ERR_ALIGN;
    if (!workspace || workspace_bytes < packmamba_layernorm_bwd_workspace_size(batch, dim, seqlen, dtype)) return PACKMAMBA_ERR_WORKSPACE;
    pm::NormArgs a = norm_args(x, batch, dim, seqlen, dtype);
    a.w = weight; a.mean = mean; a.rstd = rstd; a.dout = dout; a.dres = dresidual; a.out = dx; a.dw = dweight; a.db = dbias;
    a.partial = static_cast<float*>(workspace);
    return launch_status(pm::launch_layernorm_bwd(a, (hipStream_t)stream));
}

}  // extern "C"
