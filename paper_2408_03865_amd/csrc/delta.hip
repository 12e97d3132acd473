// delta.hip -- the gated delta rule beside its walks (delta_walk.hpp): which kernel a walk takes, the states of split
// rows, and the gradients of q and k.
#include "delta_walk.hpp"

namespace pm {

extern template hipError_t launch_delta_kc<float, float, 64>(const DeltaArgs&, DeltaWalk, hipStream_t);
extern template hipError_t launch_delta_kc<float, float, 128>(const DeltaArgs&, DeltaWalk, hipStream_t);
extern template hipError_t launch_delta_kc<bf16_t, bf16_t, 64>(const DeltaArgs&, DeltaWalk, hipStream_t);
extern template hipError_t launch_delta_kc<bf16_t, bf16_t, 128>(const DeltaArgs&, DeltaWalk, hipStream_t);
extern template hipError_t launch_delta_kc<bf16_t, float, 64>(const DeltaArgs&, DeltaWalk, hipStream_t);
extern template hipError_t launch_delta_kc<bf16_t, float, 128>(const DeltaArgs&, DeltaWalk, hipStream_t);

namespace {

template <typename T, typename TO>
hipError_t walk_t(const DeltaArgs& a, DeltaWalk which, hipStream_t s) {
    return a.dk <= 64 ? launch_delta_kc<T, TO, 64>(a, which, s) : launch_delta_kc<T, TO, 128>(a, which, s);
}
hipError_t walk(const DeltaArgs& a, DeltaWalk which, hipStream_t s) {
    switch (a.dtype) {
        case 1: return walk_t<bf16_t, bf16_t>(a, which, s);
        case 2: return walk_t<bf16_t, float>(a, which, s);
        default: return walk_t<float, float>(a, which, s);
    }
}

// --------------------------------------------------------------------------------------------
// split rows: the state that enters each segment, cur <- M cur + added (nothing of cur where a sequence starts in
// the segment), in place of what is added; backwards with M's transpose.  A block takes 16 columns of the state of one
// row and head, its waves 16 rows each; products in 32 bits.
// --------------------------------------------------------------------------------------------
template <int KC, bool REV>
__global__ __launch_bounds__(256) void delta_chain(DeltaArgs a) {
    constexpr int KF = KC / 16, kMine = KF / 4;
    __shared__ f32x4 cur[KF][64];
    const int l = lane_id(), w = wave_id(), col = l & 15, g4 = (l >> 4) * 4;
    const int cols = (a.dv + 15) / 16;
    const int64_t bh = blockIdx.x / cols;
    const int z = (int)(blockIdx.x - bh * cols) * 16 + col;
    const int64_t sz = (int64_t)a.dk * a.dv;
    const auto at = [&](const float* p, int x) { return p && x < a.dk && z < a.dv ? p[(int64_t)x * a.dv + z] : 0.0f; };
#pragma unroll
    for (int m = 0; m < kMine; ++m) {
        const int k = w + m * 4;
        f32x4 v;
#pragma unroll
        for (int r = 0; r < 4; ++r) v[r] = at(a.entry ? a.entry + bh * sz : nullptr, k * 16 + g4 + r);
        cur[k][l] = v;
    }
    __syncthreads();
    for (int n = 0; n < a.nseg; ++n) {
        const int64_t seg = bh * a.nseg + (REV ? a.nseg - 1 - n : n);
        float* p = a.seg + seg * sz;
        const float* M = a.seg_m + seg * KC * KC;
        const bool more = n + 1 < a.nseg, cut = more && a.seg_cut[seg] != 0;
        f32x4 next[kMine];
#pragma unroll
        for (int m = 0; m < kMine; ++m) {
            const int k = w + m * 4;
#pragma unroll
            for (int r = 0; r < 4; ++r) next[m][r] = more ? at(p, k * 16 + g4 + r) : 0.0f;
            if (more && !cut) {
#pragma unroll
                for (int j = 0; j < KF; ++j) {
                    f32x4 f;
                    if constexpr (REV) {
#pragma unroll
                        for (int r = 0; r < 4; ++r) f[r] = M[(j * 16 + g4 + r) * KC + k * 16 + col];
                    } else {
                        f = *reinterpret_cast<const f32x4*>(M + (k * 16 + col) * KC + j * 16 + g4);
                    }
                    const f32x4 c = cur[j][l];
#pragma unroll
                    for (int e = 0; e < 4; ++e) next[m] = __builtin_amdgcn_mfma_f32_16x16x4f32(f[e], c[e], next[m], 0, 0, 0);
                }
            }
        }
        __syncthreads();
#pragma unroll
        for (int m = 0; m < kMine; ++m) {
            const int k = w + m * 4;
            const f32x4 c = cur[k][l];
#pragma unroll
            for (int r = 0; r < 4; ++r)
                if (k * 16 + g4 + r < a.dk && z < a.dv) p[(int64_t)(k * 16 + g4 + r) * a.dv + z] = c[r];
            cur[k][l] = next[m];
        }
        __syncthreads();
    }
}

// --------------------------------------------------------------------------------------------
// dq and dk of a chunk, from the states before and the gradients after it.  With Mo = scale (dout . u) D (pairs s <= t)
// and Mv = -(dv . u) D (s < t), D the decay between the two tokens:
//   dq = Mo k + scale in (S dout),   dk = Mo^T q + Mv k + Mv^T k - in (S dv) + up (D u)
// One block a chunk, 64 features and grad_per heads of a group, whose sums stay in registers; wave w owns 16 tokens.  Mo and Mv
// are made in both directions by the wave that needs them, as the operands they are next.
// In bf16 u, dv and the states are rounded once; Mo and Mv are split into two terms.
// --------------------------------------------------------------------------------------------
template <typename T>
struct GradSmem {
    __attribute__((aligned(16))) T k[64 * kC];
    __attribute__((aligned(16))) T q[64 * kC];
    __attribute__((aligned(16))) T dout[64 * kC];
    __attribute__((aligned(16))) T u[64 * kC];
    __attribute__((aligned(16))) T w[64 * kC];
    __attribute__((aligned(16))) T s[64 * 64];       // the state before, features of v by features of k
    __attribute__((aligned(16))) T d[64 * 64];       // the gradient after
    __attribute__((aligned(16))) float coef[kDeltaCoef];
};

template <typename T, typename TO, int KC>
__global__ __launch_bounds__(256, 2) void delta_grads_kernel(DeltaArgs a) {
    using M = Mat<T>;
    using Frag = typename M::Frag;
    using Regs = TileRegs<T, 64, 256>;
    constexpr int NM = M::kSplit ? 2 : 1, kHalves = KC / 64;
    __shared__ GradSmem<T> sm;
    const int l = lane_id(), w = wave_id(), col = l & 15, g4 = (l >> 4) * 4, tid = threadIdx.x;
    const int64_t L = a.seqlen;
    const int rep = a.heads / a.groups, parts = (rep + a.grad_per - 1) / a.grad_per;
    const uint32_t id = blockIdx.x, n_in = (uint32_t)(a.groups * parts * kHalves);
    const uint32_t bc = id / n_in, in_id = id - bc * n_in;
    const int64_t b = bc / (uint32_t)a.chunks, chunk = bc - b * a.chunks;
    const int half = (int)(in_id % kHalves), gp = (int)(in_id / kHalves), part = gp % parts;
    const int64_t grp = gp / parts, t0 = chunk * kC;
    const int f0 = half * 64, frows = min(64, a.dk - f0);
    const int vpad = a.dv <= 64 ? 64 : 128, vhalves = vpad / 64;
    const int h0 = (int)grp * rep + part * a.grad_per, h1 = min((int)(grp + 1) * rep, h0 + a.grad_per);
    if (frows <= 0) return;
    const T* kp = static_cast<const T*>(a.k) + ((b * a.groups + grp) * a.dk + f0) * L;
    const T* qp = static_cast<const T*>(a.q) + ((b * a.groups + grp) * a.dk + f0) * L;
    const uint32_t at = Regs::offset_of(tid, (int)t0, (int)L), sat = Regs::offset_of(tid, 0, KC);

    {
        Regs kr, qr;
        kr.load(tid, at, kp, frows, (int)L);
        qr.load(tid, at, qp, frows, (int)L);
        kr.settle(tid, kp, frows, t0, L);
        qr.settle(tid, qp, frows, t0, L);
        kr.store(tid, sm.k);
        qr.store(tid, sm.q);
    }
    f32x4 dq[4], dk[4];
#pragma unroll
    for (int f = 0; f < 4; ++f) dq[f] = dk[f] = f32x4{0, 0, 0, 0};

    Regs dor, ur, wr, sr, gr;
    float cr[2];
    const int steps = (h1 - h0) * vhalves;
    const auto base = [&](const void* p, int step) {
        const int h = h0 + step / vhalves, v0 = step % vhalves * 64;
        return static_cast<const T*>(p) + ((b * a.heads + h) * a.dv + v0) * L;
    };
    const auto load = [&](int step) {
        const int h = h0 + step / vhalves, v0 = step % vhalves * 64, rows = min(64, a.dv - v0);
        const int64_t unit = (b * a.heads + h) * a.chunks + chunk;
        dor.load(tid, at, base(a.dout, step), rows, (int)L);
        ur.load(tid, at, base(a.u, step), rows, (int)L);
        wr.load(tid, at, base(a.w, step), rows, (int)L);
        sr.load(tid, sat, static_cast<const T*>(a.states) + (unit * vpad + v0) * KC + f0, 64, KC);
        gr.load(tid, sat, static_cast<const T*>(a.grads) + (unit * vpad + v0) * KC + f0, 64, KC);
        cr[0] = a.coef[unit * kDeltaCoef + tid];
        cr[1] = a.coef[unit * kDeltaCoef + min(tid + 256, kDeltaCoef - 1)];
    };
    load(0);
    f32x4 o1[4], o2[4], v1[4], v2[4], sq[4], sk[4], gk[4];
    for (int step = 0; step < steps; ++step) {
        const bool first = step % vhalves == 0, done = step % vhalves == vhalves - 1;
        const int v0 = step % vhalves * 64, rows = min(64, a.dv - v0);
        __syncthreads();
        dor.settle(tid, base(a.dout, step), rows, t0, L);
        ur.settle(tid, base(a.u, step), rows, t0, L);
        wr.settle(tid, base(a.w, step), rows, t0, L);
        dor.store(tid, sm.dout);
        ur.store(tid, sm.u);
        wr.store(tid, sm.w);
        sr.store(tid, sm.s);
        gr.store(tid, sm.d);
        sm.coef[tid] = cr[0];
        if (tid + 256 < kDeltaCoef) sm.coef[tid + 256] = cr[1];
        __syncthreads();
        if (step + 1 < steps) load(step + 1);
        if (first) {
#pragma unroll
            for (int i = 0; i < 4; ++i) o1[i] = o2[i] = v1[i] = v2[i] = sq[i] = sk[i] = gk[i] = f32x4{0, 0, 0, 0};
        }
#pragma unroll
        for (int n = 0; n < 4; n += 2) {                        // 32 features of v
            const auto tok = [&](const T* tile, int k, int i) { return M::transposed(l, tile + k * 16 * kC, i); };
            const Frag d0 = tok(sm.dout, n, w), d1 = tok(sm.dout, n + 1, w), u0 = tok(sm.u, n, w), u1 = tok(sm.u, n + 1, w);
            const Frag w0 = tok(sm.w, n, w), w1 = tok(sm.w, n + 1, w);
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                if (i <= w) {
                    const Frag x0 = tok(sm.u, n, i), x1 = tok(sm.u, n + 1, i);
                    o1[i] = M::mma(x0, x1, d0, d1, o1[i]);
                    v1[i] = M::mma(x0, x1, w0, w1, v1[i]);
                }
                if (i >= w) {
                    o2[i] = M::mma(tok(sm.dout, n, i), tok(sm.dout, n + 1, i), u0, u1, o2[i]);
                    v2[i] = M::mma(tok(sm.w, n, i), tok(sm.w, n + 1, i), u0, u1, v2[i]);
                }
                const Frag s0 = tok(sm.s, n, i), s1 = tok(sm.s, n + 1, i);
                sq[i] = M::mma(d0, d1, s0, s1, sq[i]);
                sk[i] = M::mma(w0, w1, s0, s1, sk[i]);
                gk[i] = M::mma(u0, u1, tok(sm.d, n, i), tok(sm.d, n + 1, i), gk[i]);
            }
        }
        if (!done) continue;
        // weights between the tokens
        const auto c4 = [&](int which, int i) { return *reinterpret_cast<const f32x4*>(&sm.coef[which + i * 16 + g4]); };
        {
            const int t = w * 16 + col;
            const float hi = sm.coef[kCoefHi + t], lo = sm.coef[kCoefLo + t];
            const int start = __float_as_int(sm.coef[kCoefStart + t]);
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const f32x4 hi4 = c4(kCoefHi, i), lo4 = c4(kCoefLo, i), st4 = c4(kCoefStart, i);
#pragma unroll
                for (int r = 0; r < 4; ++r) {
                    const int s = i * 16 + g4 + r;
                    if (i <= w) {                                // t is the later one
                        const float d = pair_decay(hi, lo, hi4[r], lo4[r]);
                        const bool on = s <= t && start <= s;
                        o1[i][r] = on ? o1[i][r] * (d * a.scale) : 0.0f;
                        v1[i][r] = on && s < t ? -v1[i][r] * d : 0.0f;
                    }
                    if (i >= w) {                                // s is
                        const float d = pair_decay(hi4[r], lo4[r], hi, lo);
                        const bool on = t <= s && __float_as_int(st4[r]) <= t;
                        o2[i][r] = on ? o2[i][r] * (d * a.scale) : 0.0f;
                        v2[i][r] = on && t < s ? -v2[i][r] * d : 0.0f;
                    }
                }
            }
        }
        const f32x4 in = c4(kCoefIn, w), up = c4(kCoefUp, w);
#pragma unroll
        for (int f = 0; f < 4; ++f) {
            dq[f] += weighted(sq[f], in) * a.scale;
            dk[f] += weighted(gk[f], up) - weighted(sk[f], in);
        }
        if (__builtin_amdgcn_readfirstlane(__float_as_int(sm.coef[kCoefA + 1])) == 0) {
#pragma unroll
            for (int p = 0; p < 2; ++p) {                        // pairs of token tiles
                const auto terms = [&](const f32x4& v, Frag (&to)[NM]) { M::template split<NM>(v, to); };
                Frag a0[NM], a1[NM], b0[NM], b1[NM], e0[NM], e1[NM], g0[NM], g1[NM];
                terms(o1[2 * p], a0);
                terms(o1[2 * p + 1], a1);
                terms(o2[2 * p], b0);
                terms(o2[2 * p + 1], b1);
                terms(v1[2 * p] + v2[2 * p], e0);               // v1 and v2 meet only on the diagonal tile, where each is 0 at the other's
                terms(v1[2 * p + 1] + v2[2 * p + 1], e1);
#pragma unroll
                for (int f = 0; f < 4; ++f) {
                    const Frag k0 = M::direct(l, sm.k + f * 16 * kC, 2 * p), k1 = M::direct(l, sm.k + f * 16 * kC, 2 * p + 1);
                    const Frag q0 = M::direct(l, sm.q + f * 16 * kC, 2 * p), q1 = M::direct(l, sm.q + f * 16 * kC, 2 * p + 1);
#pragma unroll
                    for (int n = NM - 1; n >= 0; --n) {
                        dq[f] = M::mma(a0[n], a1[n], k0, k1, dq[f]);
                        dk[f] = M::mma(b0[n], b1[n], q0, q1, dk[f]);
                        dk[f] = M::mma(e0[n], e1[n], k0, k1, dk[f]);
                    }
                }
            }
        } else {                                                 // k or q not finite: pair by pair
#pragma unroll
            for (int i = 0; i < 4; ++i)
#pragma unroll
                for (int r = 0; r < 4; ++r)
#pragma unroll 1
                    for (int g = 0; g < 4; ++g) {
                        const int s = i * 16 + g * 4 + r;
#pragma unroll
                        for (int x = 0; x < 4; ++x) {
                            const int from = (g << 4) | (g4 + x);
                            const float mo = __shfl(o1[i][r], from), mt = __shfl(o2[i][r], from), mv = __shfl(v1[i][r] + v2[i][r], from);
#pragma unroll
                            for (int f = 0; f < 4; ++f) {
                                const float ks = tile_value(sm.k + f * 16 * kC, col, s), qs = tile_value(sm.q + f * 16 * kC, col, s);
                                if (mo != 0.0f) dq[f][x] = fmaf(mo, ks, dq[f][x]);
                                if (mt != 0.0f) dk[f][x] = fmaf(mt, qs, dk[f][x]);
                                if (mv != 0.0f) dk[f][x] = fmaf(mv, ks, dk[f][x]);
                            }
                        }
                    }
        }
    }
    const int64_t out = ((b * a.groups + grp) * parts + part) * a.dk + f0;
#pragma unroll
    for (int f = 0; f < 4; ++f) {
        if (f * 16 + col >= frows) continue;
        const int64_t at_row = (out + f * 16 + col) * L;
        store_tokens(static_cast<TO*>(a.dq) + at_row, t0 + w * 16 + g4, L, dq[f]);
        store_tokens(static_cast<TO*>(a.dk_out) + at_row, t0 + w * 16 + g4, L, dk[f]);
    }
}

template <typename T, typename TO>
hipError_t grads_t(const DeltaArgs& a, hipStream_t s) {
    const int64_t parts = (a.heads / a.groups + a.grad_per - 1) / a.grad_per, units = (int64_t)a.batch * a.chunks * a.groups * parts;
    if (a.dk <= 64) hipLaunchKernelGGL((delta_grads_kernel<T, TO, 64>), dim3((unsigned)units), dim3(256), 0, s, a);
    else hipLaunchKernelGGL((delta_grads_kernel<T, TO, 128>), dim3((unsigned)(units * 2)), dim3(256), 0, s, a);
    return hipGetLastError();
}

template <int KC>
hipError_t chain_kc(const DeltaArgs& a, bool rev, hipStream_t s) {
    const dim3 grid((unsigned)((int64_t)a.batch * a.heads * ((a.dv + 15) / 16)));
    if (rev) hipLaunchKernelGGL((delta_chain<KC, true>), grid, dim3(256), 0, s, a);
    else hipLaunchKernelGGL((delta_chain<KC, false>), grid, dim3(256), 0, s, a);
    return hipGetLastError();
}

}  // namespace

hipError_t launch_delta_fwd(const DeltaArgs& a, bool exact, hipStream_t s) { return walk(a, exact ? kWalkOutExact : kWalkOut, s); }
hipError_t launch_delta_states(const DeltaArgs& a, hipStream_t s) { return walk(a, kWalkStates, s); }
hipError_t launch_delta_rev(const DeltaArgs& a, hipStream_t s) { return walk(a, kWalkRev, s); }

hipError_t launch_delta_segments(const DeltaArgs& a, bool rev, hipStream_t s) {
    if (hipError_t e = walk(a, rev ? kWalkSumRev : kWalkSum, s)) return e;
    return a.dk <= 64 ? chain_kc<64>(a, rev, s) : chain_kc<128>(a, rev, s);
}

hipError_t launch_delta_grads(const DeltaArgs& a, bool f32, hipStream_t s) {
    if (a.dtype == 0) return grads_t<float, float>(a, s);
    return f32 ? grads_t<bf16_t, float>(a, s) : grads_t<bf16_t, bf16_t>(a, s);
}

}  // namespace pm
