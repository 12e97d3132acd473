// linear_api.cpp -- the C ABI of packmamba_linear.h: argument validation (before anything is
// enqueued), workspace layout and the order of the launches.
#include <hip/hip_runtime.h>

#include <cstdint>

#include "linear.hpp"
#include "packmamba_linear.h"

namespace {

constexpr size_t kAlign = 256;
constexpr int64_t kMaxRows = (int64_t)1 << 21;      // (batch, head) pairs: a block of up to 1024 threads each, 2^32 in all
constexpr int64_t kMaxNormTiles = ((int64_t)1 << 22) - 1;   // tiles of 32 tokens, a block each
// features: counted in 32 bits with strides of some thousands; dweight's sum takes 32 threads each, 2^32 in all
constexpr int64_t kMaxNormDim = ((int64_t)1 << 27) - 32;
constexpr int64_t kMaxSeqlen = (int64_t)1 << 22;    // 64 rows of it in fp32 are an offset of 32 bits in the walks
constexpr int64_t kMaxElems = (int64_t)1 << 33;     // of a tensor, heads' copies of q and k included

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
    if (heads > kMaxRows || batch > kMaxRows / heads || heads % groups) return PACKMAMBA_ERR_SHAPE;
    if (dk > PACKMAMBA_LINEAR_MAX_HEAD || dv > PACKMAMBA_LINEAR_MAX_HEAD) return PACKMAMBA_ERR_UNSUPPORTED;
    if (seqlen > kMaxSeqlen || seqlen > kMaxElems / (batch * heads * (dk > dv ? dk : dv))) return PACKMAMBA_ERR_SHAPE;
    return PACKMAMBA_OK;
}

// What split rows need: the states that enter the segments and what each multiplies its by.
struct SegWs {
    size_t states, total;
};
SegWs seg_ws(const pm::LinPlan& p, int64_t rows, int64_t dk, int64_t dv) {
    if (p.nseg <= 1) return {0, 0};
    const size_t states = floats(rows * p.nseg * dk * dv);
    return {states, states + floats(rows * p.nseg)};
}

// Backward: the segments' states (one walk after another uses them), the states at the boundaries
// and their products, the tokens' parts of ddecay, the pieces of a head's, and each head's dq or dk.
struct BwdWs {
    SegWs seg;
    size_t bound, dot, r, pieces, heads, total;
};
BwdWs bwd_ws(const pm::LinPlan& p, int64_t batch, int64_t heads, int64_t groups, int64_t dk, int64_t dv, int64_t seqlen) {
    const int64_t rows = batch * heads;
    BwdWs w;
    w.seg = seg_ws(p, rows, dk, dv);
    w.bound = floats(rows * p.nb * pm::walk_bound_floats((int32_t)dv, (int32_t)dk));
    w.dot = floats(rows * (p.nb + 1));
    w.r = floats(rows * seqlen);
    w.pieces = floats(rows * p.nb);
    w.heads = heads > groups ? floats(rows * dk * seqlen) : 0;
    w.total = w.seg.total + w.bound + w.dot + 2 * w.r + w.pieces + w.heads;
    return w;
}

int check_norm(int64_t batch, int64_t dim, int64_t seqlen, int64_t groups) {
    if (batch <= 0 || dim <= 0 || seqlen <= 0 || groups <= 0 || dim % groups) return PACKMAMBA_ERR_SHAPE;
    if (groups > (1 << 20) || batch > (1 << 20) / groups) return PACKMAMBA_ERR_SHAPE;
    if (dim > kMaxNormDim || seqlen > INT32_MAX / 2) return PACKMAMBA_ERR_SHAPE;
    if (batch * dim > kMaxElems / seqlen) return PACKMAMBA_ERR_SHAPE;
    if (batch * groups > kMaxNormTiles / ((seqlen + 31) / 32)) return PACKMAMBA_ERR_SHAPE;
    return PACKMAMBA_OK;
}

}  // namespace

extern "C" {

size_t packmamba_linear_attention_fwd_workspace_size(int64_t batch, int64_t heads, int64_t groups, int64_t dk, int64_t dv,
                                                     int64_t seqlen) {
    if (check_heads(batch, heads, groups, dk, dv, seqlen)) return 0;
    return seg_ws(pm::linear_plan(batch, heads, dk, dv, seqlen, false), batch * heads, dk, dv).total;
}

int packmamba_linear_attention_fwd(const void* q, const void* k, const void* v, const float* decay,
                                   const int32_t* position_indices, const float* initial_state, float scale, void* out,
                                   float* final_state, void* workspace, size_t workspace_bytes, int64_t batch,
                                   int64_t heads, int64_t groups, int64_t dk, int64_t dv, int64_t seqlen,
                                   int32_t decay_per_token, int32_t dtype, void* stream) {
    if (!q || !k || !v || !position_indices || !out) return PACKMAMBA_ERR_NULL;
    if (int e = check_heads(batch, heads, groups, dk, dv, seqlen)) return e;
    if (int e = check_dtype(dtype)) return e;
    if (!aligned16(q, k, v, decay, position_indices, initial_state, out, final_state, workspace)) return PACKMAMBA_ERR_ALIGN;
    const pm::LinPlan p = pm::linear_plan(batch, heads, dk, dv, seqlen, false);
    const SegWs w = seg_ws(p, batch * heads, dk, dv);
    if (w.total && (!workspace || workspace_bytes < w.total)) return PACKMAMBA_ERR_WORKSPACE;
    pm::WalkArgs a{};
    a.x = {q, (int32_t)dk, (int32_t)groups};
    a.y = {k, (int32_t)dk, (int32_t)groups};
    a.z = {v, (int32_t)dv, (int32_t)heads};
    a.out = out; a.decay = decay; a.pos = position_indices;
    a.entry = initial_state; a.leave = final_state;
    a.pscale = a.iscale = scale; a.uscale = 1.0f;
    a.seqlen = seqlen; a.batch = (int32_t)batch; a.heads = (int32_t)heads;
    a.decay_mode = decay ? (decay_per_token ? 2 : 1) : 0;
    a.nseg = p.nseg; a.seg_chunks = p.seg_chunks; a.bound_chunks = p.bound_chunks; a.nb = p.nb;
    a.s_x = (int32_t)dv; a.s_z = 1; a.dtype = dtype;
    const hipStream_t s = (hipStream_t)stream;
    if (p.nseg > 1) {
        a.seg = static_cast<float*>(workspace);
        a.seg_a = reinterpret_cast<float*>(static_cast<char*>(workspace) + w.states);
        if (int e = launch_status(pm::launch_walk_segments(a, s))) return e;
    }
    return launch_status(pm::launch_walk(a, pm::kWalkPlain, final_state != nullptr, s));
}

size_t packmamba_linear_attention_bwd_workspace_size(int64_t batch, int64_t heads, int64_t groups, int64_t dk, int64_t dv,
                                                     int64_t seqlen) {
    if (check_heads(batch, heads, groups, dk, dv, seqlen)) return 0;
    return bwd_ws(pm::linear_plan(batch, heads, dk, dv, seqlen, true), batch, heads, groups, dk, dv, seqlen).total;
}

int packmamba_linear_attention_bwd(const void* q, const void* k, const void* v, const float* decay,
                                   const int32_t* position_indices, const float* initial_state, float scale,
                                   const void* dout, const float* dfinal_state, void* dq, void* dk, void* dv,
                                   float* ddecay, float* dinitial_state, void* workspace, size_t workspace_bytes,
                                   int64_t batch, int64_t heads, int64_t groups, int64_t dk_size, int64_t dv_size,
                                   int64_t seqlen, int32_t decay_per_token, int32_t dtype, void* stream) {
    if (!q || !k || !v || !position_indices || !dout || !dq || !dk || !dv) return PACKMAMBA_ERR_NULL;
    if (ddecay && !decay) return PACKMAMBA_ERR_NULL;
    if ((initial_state == nullptr) != (dinitial_state == nullptr)) return PACKMAMBA_ERR_NULL;
    if (int e = check_heads(batch, heads, groups, dk_size, dv_size, seqlen)) return e;
    if (int e = check_dtype(dtype)) return e;
    if (!aligned16(q, k, v, decay, position_indices, initial_state, dout, dfinal_state) ||
        !aligned16(dq, dk, dv, ddecay, dinitial_state, workspace))
        return PACKMAMBA_ERR_ALIGN;
    const pm::LinPlan p = pm::linear_plan(batch, heads, dk_size, dv_size, seqlen, true);
    const BwdWs w = bwd_ws(p, batch, heads, groups, dk_size, dv_size, seqlen);
    if (!workspace || workspace_bytes < w.total) return PACKMAMBA_ERR_WORKSPACE;
    const hipStream_t s = (hipStream_t)stream;
    char* at = static_cast<char*>(workspace);
    const auto take = [&](size_t bytes) {
        char* got = at;
        at += bytes;
        return reinterpret_cast<float*>(got);
    };
    pm::WalkArgs a{};
    a.seg = take(w.seg.states);
    a.seg_a = take(w.seg.total - w.seg.states);
    a.bound = take(w.bound);
    a.dot = take(w.dot);
    float* rq = take(w.r);
    float* rk = take(w.r);
    float* pieces = take(w.pieces);
    float* part = take(w.heads);
    a.decay = decay; a.pos = position_indices;
    a.seqlen = seqlen; a.batch = (int32_t)batch; a.heads = (int32_t)heads;
    a.decay_mode = decay ? (decay_per_token ? 2 : 1) : 0;
    a.nseg = p.nseg; a.seg_chunks = p.seg_chunks; a.bound_chunks = p.bound_chunks; a.nb = p.nb;
    a.bound_end = dfinal_state != nullptr;
    const pm::WalkTensor tq{q, (int32_t)dk_size, (int32_t)groups}, tk{k, (int32_t)dk_size, (int32_t)groups};
    const pm::WalkTensor tv{v, (int32_t)dv_size, (int32_t)heads}, tdo{dout, (int32_t)dv_size, (int32_t)heads};
    const bool shared = heads > groups;
    const auto walk = [&](pm::WalkMode mode, bool exact, bool segments = true) {
        if (p.nseg > 1 && segments)
            if (int e = launch_status(pm::launch_walk_segments(a, s))) return e;
        return launch_status(pm::launch_walk(a, mode, exact, s));
    };
    // dq and dk: each head's own, in 32 bits, where heads share them
    const auto sum = [&](void* to) {
        return shared ? launch_status(pm::launch_linear_group_sum(part, to, batch, (int32_t)heads, (int32_t)groups,
                                                                  dk_size * seqlen, dtype != PACKMAMBA_BF16, s))
                      : PACKMAMBA_OK;
    };
    const int32_t head_dtype = shared && dtype == PACKMAMBA_BF16 ? PACKMAMBA_BF16_F32OUT : dtype;

    a.x = tdo; a.y = tv; a.z = tk; a.e = tq;
    a.out = shared ? part : dq;
    a.dtype = head_dtype;
    a.entry = initial_state;
    a.s_x = 1; a.s_z = (int32_t)dv_size;                     // the state transposed: dv x dk
    a.pscale = a.iscale = scale; a.uscale = 1.0f;
    a.r = rq;
    if (int e = walk(ddecay ? pm::kWalkDq : pm::kWalkPlain, false)) return e;
    if (int e = sum(dq)) return e;

    a.rev = 1;
    a.x = tv; a.y = tdo; a.z = tq; a.e = tk;
    a.out = shared ? part : dk;
    a.entry = dfinal_state;
    a.pscale = a.uscale = scale; a.iscale = 1.0f;
    a.r = rk;
    if (int e = walk(ddecay ? pm::kWalkDk : pm::kWalkPlain, false)) return e;
    if (int e = sum(dk)) return e;

    a.x = tk; a.y = tq; a.z = tdo; a.e = {};
    a.out = dv;
    a.dtype = dtype;
    a.leave = dinitial_state;
    a.s_x = (int32_t)dv_size; a.s_z = 1;
    // the states that enter the segments are those of dk, which lie in memory the same way
    if (int e = walk(pm::kWalkPlain, dinitial_state != nullptr, false)) return e;
    if (!ddecay) return PACKMAMBA_OK;

    pm::LinDecayArgs d{};
    d.rq = rq; d.rk = rk; d.dot = a.dot; d.decay = decay; d.pos = position_indices; d.ddecay = ddecay; d.partial = pieces;
    d.seqlen = seqlen; d.batch = a.batch; d.heads = a.heads; d.decay_mode = a.decay_mode;
    d.bound_tokens = p.bound_chunks * (int32_t)pm::kLinChunk; d.nb = p.nb; d.bound_end = a.bound_end;
    return launch_status(pm::launch_linear_ddecay(d, s));
}

int packmamba_linear_attention_step(const void* q, const void* k, const void* v, const float* decay,
                                    const int32_t* position_indices, float* state, float scale, void* out, int64_t batch,
                                    int64_t heads, int64_t groups, int64_t dk, int64_t dv, int32_t decay_per_token,
                                    int32_t dtype, void* stream) {
    if (!q || !k || !v || !state || !out) return PACKMAMBA_ERR_NULL;
    if (int e = check_heads(batch, heads, groups, dk, dv, 1)) return e;
    if (int e = check_dtype(dtype)) return e;
    if (!aligned16(q, k, v, decay, position_indices, state, out)) return PACKMAMBA_ERR_ALIGN;
    pm::LinStepArgs a{};
    a.q = q; a.k = k; a.v = v; a.decay = decay; a.pos = position_indices; a.state = state; a.out = out; a.scale = scale;
    a.batch = (int32_t)batch; a.heads = (int32_t)heads; a.groups = (int32_t)groups;
    a.dk = (int32_t)dk; a.dv = (int32_t)dv;
    a.decay_mode = decay ? (decay_per_token ? 2 : 1) : 0;
    a.dtype = dtype;
    return launch_status(pm::launch_linear_step(a, (hipStream_t)stream));
}

int packmamba_gated_rmsnorm_fwd(const void* x, const void* z, const float* weight, float eps, void* out, float* rstd,
                                int64_t batch, int64_t dim, int64_t seqlen, int64_t groups, int32_t gate_first,
                                int32_t dtype, void* stream) {
    if (!x || !z || !weight || !out || !rstd) return PACKMAMBA_ERR_NULL;
    if (int e = check_norm(batch, dim, seqlen, groups)) return e;
    if (int e = check_dtype(dtype)) return e;
    if (!(eps >= 0.0f)) return PACKMAMBA_ERR_SHAPE;
    if (!aligned16(x, z, weight, out, rstd)) return PACKMAMBA_ERR_ALIGN;
    pm::GatedArgs a{};
    a.x = x; a.z = z; a.w = weight; a.out = out; a.rstd_out = rstd; a.eps = eps;
    a.batch = batch; a.dim = dim; a.seqlen = seqlen; a.groups = (int32_t)groups; a.gate_first = gate_first ? 1 : 0;
    a.dtype = dtype;
    return launch_status(pm::launch_gated_fwd(a, (hipStream_t)stream));
}

size_t packmamba_gated_rmsnorm_bwd_workspace_size(int64_t batch, int64_t dim, int64_t seqlen, int64_t groups) {
    if (check_norm(batch, dim, seqlen, groups)) return 0;
    return floats(pm::gated_bwd_partial_rows(batch, seqlen, groups) * dim);
}

int packmamba_gated_rmsnorm_bwd(const void* x, const void* z, const float* weight, const float* rstd, const void* dout,
                                void* dx, void* dz, float* dweight, void* workspace, size_t workspace_bytes,
                                int64_t batch, int64_t dim, int64_t seqlen, int64_t groups, int32_t gate_first,
                                int32_t dtype, void* stream) {
    if (!x || !z || !weight || !rstd || !dout || !dx || !dz || !dweight) return PACKMAMBA_ERR_NULL;
    if (int e = check_norm(batch, dim, seqlen, groups)) return e;
    if (int e = check_dtype(dtype)) return e;
    if (!aligned16(x, z, weight, rstd, dout, dx, dz, dweight, workspace)) return PACKMAMBA_ERR_ALIGN;
    const size_t need = packmamba_gated_rmsnorm_bwd_workspace_size(batch, dim, seqlen, groups);
    if (!workspace || workspace_bytes < need) return PACKMAMBA_ERR_WORKSPACE;
    pm::GatedArgs a{};
    a.x = x; a.z = z; a.w = weight; a.rstd = rstd; a.dout = dout; a.out = dx; a.dz = dz; a.dw = dweight;
    a.partial = static_cast<float*>(workspace);
    a.batch = batch; a.dim = dim; a.seqlen = seqlen; a.groups = (int32_t)groups; a.gate_first = gate_first ? 1 : 0;
    a.dtype = dtype;
    return launch_status(pm::launch_gated_bwd(a, (hipStream_t)stream));
}

}  // extern "C"
