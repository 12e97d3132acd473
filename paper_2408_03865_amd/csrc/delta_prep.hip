// delta_prep.hip -- what every chunk of 64 tokens of the gated delta rule needs of its keys and queries, for all
// chunks at once; the walks (delta_walk.hpp) then do the rest in order.
//
// With D_ts = exp(G_t - G_s) for tokens s <= t of one sequence (else 0) and A_ts = D_ts k_t . k_s below the diagonal,
// the errors of a chunk are e = (I + A diag(beta))^-1 x.  H = (I + A diag(beta))^-1 A gives e = x - H (beta x), and
// its transpose does the same for the gradients: (I + (diag(beta) A)^T)^-1 x = x - H^T (beta x).  The identity stays
// exact, and beta = 0 needs no care.  H comes by forward substitution: blocks of 16 tokens on the diagonal row by row,
// those below by products of blocks,
//   Y = A_ij - sum over j <= k < i of A_ik (beta_k H_kj),   H_ij = Y - H_ii (beta_i Y),
// all in 32 bits: A's inverse can be far larger than A where keys repeat.  P = scale D_ts q_t . k_s, on the diagonal too.
#include "linear_walk.hpp"
#include "delta.hpp"

namespace pm {
namespace {

__host__ __device__ constexpr int tile_at(int i, int j) { return i * (i + 1) / 2 + j; }

__device__ __forceinline__ f32x4 mma16(const f32x4& a, const f32x4& b, f32x4 c) {
#pragma unroll
    for (int e = 0; e < 4; ++e) c = __builtin_amdgcn_mfma_f32_16x16x4f32(a[e], b[e], c, 0, 0, 0);
    return c;
}

template <typename T, int KC>
struct PrepSmem {
    __attribute__((aligned(16))) T k[KC * kC];
    __attribute__((aligned(16))) T q[KC * kC];
    f32x4 a[kDeltaTiles][64];           // A as operands
    f32x4 hd[4][64];                    // H's diagonal blocks as operands
    __attribute__((aligned(16))) float rows[4][16][16];     // A's diagonal blocks
    __attribute__((aligned(16))) float turn[4][16][20];
    ChunkDecay c;
    __attribute__((aligned(16))) float beta[kC];
    int bad;
};

// One block a chunk and heads_per heads of one group.  Wave j takes the tiles of column j.
template <typename T, int KC, bool BOTH>
__global__ __launch_bounds__(256) void delta_prep_kernel(DeltaArgs a) {
    using M = Mat<T>;
    using Frag = typename M::Frag;
    constexpr int KT = KC / 16;
    __shared__ PrepSmem<T, KC> sm;
    const int l = lane_id(), w = wave_id(), g4 = (l >> 4) * 4, col = l & 15;
    const int64_t L = a.seqlen;
    const int rep = a.heads / a.groups, parts = (rep + a.heads_per - 1) / a.heads_per;
    const uint32_t id = blockIdx.x, per = (uint32_t)(a.groups * parts);
    const uint32_t bc = id / per, gp = id - bc * per;
    const int64_t b = bc / (uint32_t)a.chunks, chunk = bc - b * a.chunks, grp = gp / (uint32_t)parts;
    const int part = (int)(gp - grp * parts);
    const int64_t t0 = chunk * kC;
    const T* kp = static_cast<const T*>(a.k) + (b * a.groups + grp) * a.dk * L;
    const T* qp = static_cast<const T*>(a.q) + (b * a.groups + grp) * a.dk * L;
    const int h0 = (int)grp * rep + part * a.heads_per, h1 = min((int)(grp + 1) * rep, h0 + a.heads_per);

    if (threadIdx.x == 0) sm.bad = 0;
    {
        TileRegs<T, KC, 256> kr, qr;
        const uint32_t at = TileRegs<T, KC, 256>::offset_of(threadIdx.x, (int)t0, (int)L);
        kr.load(threadIdx.x, at, kp, a.dk, (int)L);
        qr.load(threadIdx.x, at, qp, a.dk, (int)L);
        kr.settle(threadIdx.x, kp, a.dk, t0, L);
        qr.settle(threadIdx.x, qp, a.dk, t0, L);
        kr.store(threadIdx.x, sm.k);
        qr.store(threadIdx.x, sm.q);
        __syncthreads();
        if (qr.zero_sum(kr.zero_sum(0.0f)) != 0.0f) sm.bad = 1;
    }
    // products of column w's tokens with the later ones: as operands (f: lane = later token) and as results (c)
    f32x4 kf[4], kc[4], qf[4], qc[4];
    {
        Frag ks[KT];
#pragma unroll
        for (int k = 0; k < KT; ++k) ks[k] = M::transposed(l, sm.k + k * 16 * kC, w);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            kf[i] = kc[i] = qf[i] = qc[i] = f32x4{0, 0, 0, 0};
            if (i < w) continue;
#pragma unroll
            for (int k = 0; k < KT; k += 2) {
                const Frag k0 = M::transposed(l, sm.k + k * 16 * kC, i), k1 = M::transposed(l, sm.k + (k + 1) * 16 * kC, i);
                const Frag q0 = M::transposed(l, sm.q + k * 16 * kC, i), q1 = M::transposed(l, sm.q + (k + 1) * 16 * kC, i);
                kf[i] = M::mma(ks[k], ks[k + 1], k0, k1, kf[i]);
                kc[i] = M::mma(k0, k1, ks[k], ks[k + 1], kc[i]);
                qf[i] = M::mma(ks[k], ks[k + 1], q0, q1, qf[i]);
                if (BOTH) qc[i] = M::mma(q0, q1, ks[k], ks[k + 1], qc[i]);
            }
        }
    }
    for (int h = h0; h < h1; ++h) {
        const int64_t unit = (b * a.heads + h) * a.chunks + chunk;
        f32x4* hf = reinterpret_cast<f32x4*>(a.h[0] + unit * kDeltaProduct) + l;
        f32x4* ht = BOTH ? reinterpret_cast<f32x4*>(a.h[1] + unit * kDeltaProduct) + l : nullptr;
        f32x4* pf = reinterpret_cast<f32x4*>(a.p[0] + unit * kDeltaProduct) + l;
        f32x4* pt = BOTH ? reinterpret_cast<f32x4*>(a.p[1] + unit * kDeltaProduct) + l : nullptr;
        float* cf = a.coef + unit * kDeltaCoef;
        __syncthreads();                                // the head before is done with the tiles
        if (w == 0) {
            TokenDecay d{0.0f, 1};
            float beta = 0.0f;
            const int64_t t = t0 + l;
            if (t < L) {
                d.pos = a.pos[b * L + t];
                if (a.decay_mode == 2) d.g = a.decay[(b * a.heads + h) * L + t];
                else if (a.decay_mode == 1) d.g = a.decay[h];
                beta = a.beta[(b * a.heads + h) * L + t];
            }
            chunk_decay<false>(d, sm.c, 1.0f, 1.0f);
            sm.beta[l] = beta;
        }
        __syncthreads();
        if (w == 1) {
            cf[kCoefIn + l] = sm.c.in[l];
            cf[kCoefUp + l] = sm.c.up[l];
            cf[kCoefBeta + l] = sm.beta[l];
            cf[kCoefHi + l] = sm.c.hi[l];
            cf[kCoefLo + l] = sm.c.lo[l];
            cf[kCoefStart + l] = __int_as_float(sm.c.start[l]);
            if (l == 0) {
                cf[kCoefA] = sm.c.a;
                cf[kCoefA + 1] = __int_as_float(sm.bad);
            }
        }
        // weighted: A and P
        f32x4 ac[4];
        {
            const int s1 = w * 16 + col, s4 = w * 16 + g4;
            const float hi1 = sm.c.hi[s1], lo1 = sm.c.lo[s1];
            const f32x4 hi4 = *reinterpret_cast<const f32x4*>(&sm.c.hi[s4]), lo4 = *reinterpret_cast<const f32x4*>(&sm.c.lo[s4]);
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                ac[i] = f32x4{0, 0, 0, 0};
                if (i < w) continue;
                const int t1 = i * 16 + col, t4 = i * 16 + g4;
                const float thi = sm.c.hi[t1], tlo = sm.c.lo[t1];
                const f32x4 thi4 = *reinterpret_cast<const f32x4*>(&sm.c.hi[t4]), tlo4 = *reinterpret_cast<const f32x4*>(&sm.c.lo[t4]);
                f32x4 af, pv, pc;
#pragma unroll
                for (int r = 0; r < 4; ++r) {
                    const float d = pair_decay(thi, tlo, hi4[r], lo4[r]);
                    const bool on = takes<false>(sm.c, t1, s4 + r);
                    af[r] = on && s4 + r < t1 ? kf[i][r] * d : 0.0f;
                    pv[r] = on ? qf[i][r] * (d * a.scale) : 0.0f;
                    const float d4 = pair_decay(thi4[r], tlo4[r], hi1, lo1);
                    const bool on4 = takes<false>(sm.c, t4 + r, s1);
                    ac[i][r] = on4 && s1 < t4 + r ? kc[i][r] * d4 : 0.0f;
                    pc[r] = on4 ? qc[i][r] * (d4 * a.scale) : 0.0f;
                }
                sm.a[tile_at(i, w)][l] = af;
                pf[tile_at(i, w) * 64] = pv;
                if (BOTH) pt[tile_at(i, w) * 64] = pc;
                if (i == w) *reinterpret_cast<f32x4*>(&sm.rows[w][col][g4]) = af;
            }
        }
        __syncthreads();
        // H's diagonal block, column col in every lane, row by row
        f32x4 hc[4], nb[4];             // H as results, and -beta H
        const auto beta4 = [&](int i) { return *reinterpret_cast<const f32x4*>(&sm.beta[i * 16 + g4]); };
        const auto turned = [&](const f32x4& v) {           // a result as an operand
            *reinterpret_cast<f32x4*>(&sm.turn[w][col][g4]) = v;
            __builtin_amdgcn_wave_barrier();
            f32x4 o;
#pragma unroll
            for (int r = 0; r < 4; ++r) o[r] = sm.turn[w][g4 + r][col];
            __builtin_amdgcn_wave_barrier();
            return o;
        };
        f32x4 own;
        {
            float x[16], xb[16];
#pragma unroll
            for (int i = 0; i < 16; ++i) {
                float v = sm.rows[w][i][col];
#pragma unroll
                for (int m = 0; m < i; ++m) v = fmaf(-sm.rows[w][i][m], xb[m], v);
                x[i] = v;
                xb[i] = v * sm.beta[w * 16 + i];
            }
            const int g = l >> 4;
#pragma unroll
            for (int r = 0; r < 4; ++r) own[r] = g == 0 ? x[r] : g == 1 ? x[4 + r] : g == 2 ? x[8 + r] : x[12 + r];
        }
        {
            const f32x4 f = turned(own);
            sm.hd[w][l] = f;
            hf[tile_at(w, w) * 64] = f;
            if (BOTH) ht[tile_at(w, w) * 64] = own;
        }
        __syncthreads();
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            hc[i] = nb[i] = f32x4{0, 0, 0, 0};
            if (i < w) continue;
            if (i == w) {
                hc[i] = own;
            } else {
                f32x4 y = ac[i];
#pragma unroll
                for (int k = 0; k < i; ++k)
                    if (k >= w) y = mma16(sm.a[tile_at(i, k)][l], nb[k], y);
                hc[i] = mma16(sm.hd[i][l], y * -beta4(i), y);
                hf[tile_at(i, w) * 64] = turned(hc[i]);
                if (BOTH) ht[tile_at(i, w) * 64] = hc[i];
            }
            nb[i] = hc[i] * -beta4(i);
        }
    }
}

template <typename T, int KC>
hipError_t prep_kc(const DeltaArgs& a, bool both, hipStream_t s) {
    const int64_t parts = (a.heads / a.groups + a.heads_per - 1) / a.heads_per;
    const dim3 grid((unsigned)((int64_t)a.batch * a.chunks * a.groups * parts));
    if (both) hipLaunchKernelGGL((delta_prep_kernel<T, KC, true>), grid, dim3(256), 0, s, a);
    else hipLaunchKernelGGL((delta_prep_kernel<T, KC, false>), grid, dim3(256), 0, s, a);
    return hipGetLastError();
}
template <typename T>
hipError_t prep_t(const DeltaArgs& a, bool both, hipStream_t s) {
    return a.dk <= 64 ? prep_kc<T, 64>(a, both, s) : prep_kc<T, 128>(a, both, s);
}

}  // namespace

hipError_t launch_delta_prep(const DeltaArgs& a, bool both, hipStream_t s) {
    return a.dtype == 0 ? prep_t<float>(a, both, s) : prep_t<bf16_t>(a, both, s);
}

}  // namespace pm
