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
// What bounds it: a step's way through LDS, 32 matrix instructions in 32 bits (16 with keys of 64) and a block's 64 KB of M, on their
// way for one step: 24 heads of 128 x 64 in 18 segments 54 us (the sums one after the other, M loaded after the products: 66),
// 96 of 64 x 64 in four 8.6.
// --------------------------------------------------------------------------------------------
template <int KC, bool REV>
__global__ __launch_bounds__(KC * 4) void delta_chain(DeltaArgs a) {
    constexpr int KF = KC / 16;
    __shared__ f32x4 cur[2][KF][64];
    const int l = lane_id(), w = wave_id(), col = l & 15, g4 = (l >> 4) * 4;
    const uint32_t cols = (uint32_t)(a.dv + 15) / 16, id = walk_block(gridDim.x);      // a state's blocks on one XCD: they read the same M
    const int64_t bh = id / cols;
    const int z = (int)(id % cols) * 16 + col;
    const int64_t sz = (int64_t)a.dk * a.dv;
    const auto seg = [&](int n) { return bh * a.nseg + (REV ? a.nseg - 1 - n : n); };
    bool live[4];
    int place[4];                                       // in the state, of a row and column that it has
#pragma unroll
    for (int r = 0; r < 4; ++r) {
        live[r] = w * 16 + g4 + r < a.dk && z < a.dv;
        place[r] = min(w * 16 + g4 + r, a.dk - 1) * a.dv + min(z, a.dv - 1);
    }
    const auto at = [&](const float* p) {
        f32x4 v;
#pragma unroll
        for (int r = 0; r < 4; ++r) v[r] = p[place[r]];
        return v;
    };
    const auto lives = [&](f32x4 v) {
#pragma unroll
        for (int r = 0; r < 4; ++r) v[r] = live[r] ? v[r] : 0.0f;
        return v;
    };
    f32x4 m[2][KF], added[2];                           // the segment's and the next one's, on their way
    int cut[2];
    const auto load = [&](auto slot, int n) {           // without a branch, which would have all loads waited for at once
        constexpr int i = decltype(slot)::value;
        n = min(n, a.nseg - 2);                         // the last segment adds to nothing
        const float* M = a.seg_m + seg(n) * KC * KC;
        cut[i] = a.seg_cut[seg(n)];
        added[i] = at(a.seg + seg(n) * sz);
#pragma unroll
        for (int j = 0; j < KF; ++j) {
            if constexpr (REV) {
#pragma unroll
                for (int r = 0; r < 4; ++r) m[i][j][r] = M[(j * 16 + g4 + r) * KC + w * 16 + col];
            } else {
                m[i][j] = *reinterpret_cast<const f32x4*>(M + (w * 16 + col) * KC + j * 16 + g4);
            }
        }
    };
    f32x4 own = {0, 0, 0, 0};
    if (a.entry) own = lives(at(a.entry + bh * sz));
    using std::integral_constant;
    const auto step = [&](auto slot, int n) {
        constexpr int i = decltype(slot)::value;
        const f32x4 before = own;
        load(integral_constant<int, 1 - i>{}, n + 1);
        cur[i][w][l] = own;
        __syncthreads();
        f32x4 c[KF], sum[4];
#pragma unroll
        for (int j = 0; j < KF; ++j) c[j] = cur[i][j][l];
#pragma unroll
        for (int j = 0; j < 4; ++j) sum[j] = f32x4{0, 0, 0, 0};
        if (!cut[i]) {
            f32x4 zero = {0, 0, 0, 0};
#pragma unroll
            for (int j = 0; j < KF; ++j)
#pragma unroll
                for (int e = 0; e < 4; ++e) zero[e] = fmaf(m[i][j][e], 0.0f, zero[e]);
            // the sums in turns: a matrix instruction waits for the one whose result it takes
            if (__ballot(!((zero.x + zero.y) + (zero.z + zero.w) == 0.0f)) == 0) {
#pragma unroll
                for (int j = 0; j < KF; j += 4)
#pragma unroll
                    for (int e = 0; e < 4; ++e)
#pragma unroll
                        for (int q = 0; q < 4; ++q) sum[q] = __builtin_amdgcn_mfma_f32_16x16x4f32(m[i][j + q][e], c[j + q][e], sum[q], 0, 0, 0);
            } else {                                    // decays above 0, or k is not finite: what is 0 stays 0 whatever it is multiplied with
                const float* M = a.seg_m + seg(min(n, a.nseg - 2)) * KC * KC;
#pragma unroll 1
                for (int x = 0; x < KC; ++x) {
                    const float v = reinterpret_cast<const float*>(&cur[i][x >> 4][((x >> 2) & 3) * 16 + col])[x & 3];
#pragma unroll
                    for (int r = 0; r < 4; ++r) {
                        const int y = w * 16 + g4 + r;
                        sum[0][r] += v == 0.0f ? 0.0f : (REV ? M[x * KC + y] : M[y * KC + x]) * v;
                    }
                }
            }
        }
        own = lives(added[i]) + ((sum[0] + sum[1]) + (sum[2] + sum[3]));
        float* p = a.seg + seg(n) * sz;
#pragma unroll
        for (int r = 0; r < 4; ++r)
            if (live[r]) p[place[r]] = before[r];
    };
    load(integral_constant<int, 0>{}, 0);
    for (int n = 0; n < a.nseg; n += 2) {               // what follows the last segment is left
        step(integral_constant<int, 0>{}, n);
        if (n + 1 < a.nseg) step(integral_constant<int, 1>{}, n + 1);
    }
}

// --------------------------------------------------------------------------------------------
// dq and dk of a chunk, from the states before and the gradients after it.  With Mo = scale (dout . u) D (pairs s <= t)
// and Mv = -(dv . u) D (s < t), D the decay between the two tokens:
//   dq = Mo k + scale in (S dout),   dk = Mo^T q + Mv k + Mv^T k - in (S dv) + up (D u)
// One block a chunk, 64 features of k and grad_per heads of a group, whose sums stay in registers; wave w owns 16 tokens.  Mo
// and Mv are made in both directions by the wave that needs them, as the operands they are next.  u is beta e: the
// errors are what lies in memory.
// In bf16 all but the inputs is in three terms, as in the walks: what the state before the chunk holds and the chunk's tokens
// replace cancels between (S dout) and Mo k, and between (S dv), (D u) and Mv.  32 features of v a step, so that two blocks of 70 KB of
// LDS fit a CU.
// What bounds it: VALU 59%, nearly a third of it splitting, and matrix 36% with two waves a SIMD (LDS 28%): 8 x 4096 tokens, 32 heads of
// 128 x 128 in 16 groups, 1521 us for 4.1 GB, 2.7 TB/s.  States and dv rounded to bf16, e in two terms: 806 us, but dk as far off as it is
// large where the gradient of the final state is 100 times dout's, and 1.8e-3 off and not 1.7e-3 elsewhere.
// --------------------------------------------------------------------------------------------
// 0 where the weight is, which an infinity or NaN must not pass
__device__ __forceinline__ f32x4 masked(const f32x4& v, const f32x4& weight) {
    f32x4 o;
#pragma unroll
    for (int r = 0; r < 4; ++r) o[r] = weight[r] == 0.0f ? 0.0f : v[r];
    return o;
}

template <typename T>
struct GradSmem {
    static constexpr int kTerms = Mat<T>::kSplit ? 3 : 1, kRows = Mat<T>::kSplit ? 32 : 64;      // features of v a step
    __attribute__((aligned(16))) T k[64 * kC];
    __attribute__((aligned(16))) T q[64 * kC];
    __attribute__((aligned(16))) T dout[kRows * kC];
    __attribute__((aligned(16))) T e[kTerms][kRows * kC];
    __attribute__((aligned(16))) T w[kTerms][kRows * kC];
    struct {
        __attribute__((aligned(16))) T s[kTerms][kRows * 64];      // the state before, features of v by features of k
        __attribute__((aligned(16))) T d[kTerms][kRows * 64];      // the gradient after
    } st;
    __attribute__((aligned(16))) float coef[kDeltaCoef];
};

// Values of 32 bits on their way into LDS as T's terms.
template <int ROWS>
__device__ __forceinline__ void store_terms(int tid, const TileRegs<float, ROWS, 256>& r, float (*tiles)[ROWS * 64]) {
    r.store(tid, tiles[0]);
}
template <int ROWS>
__device__ __forceinline__ void store_terms(int tid, const TileRegs<float, ROWS, 256>& r, bf16_t (*tiles)[ROWS * 64]) {
    using Regs = TileRegs<float, ROWS, 256>;
    const int row0 = tid / Regs::kLanes, c = tid % Regs::kLanes;                 // four values of a row, half a piece of 16 bytes
    const int at = row0 * 64 + ((c >> 1) ^ Mat<bf16_t>::swz(row0)) * 8 + (c & 1) * 4;
#pragma unroll
    for (int i = 0; i < Regs::kPasses; ++i) {
        u32x2 f[3];
        Mat<bf16_t>::split<3>(__builtin_bit_cast(f32x4, r.w[i]), f);
#pragma unroll
        for (int n = 0; n < 3; ++n) *reinterpret_cast<u32x2*>(&tiles[n][at + i * Regs::kRowsPass * 64]) = f[n];
    }
}
// The same of halves, upper ones rounded and lower (delta_walk.hpp); in 32 bits `hi` is all.
template <typename T, int ROWS>
__device__ __forceinline__ void store_halves(int tid, const TileRegs<T, ROWS, 256>& hi, const TileRegs<T, ROWS, 256>& lo, T (*tiles)[ROWS * kC]) {
    if constexpr (Mat<T>::kSplit) {
        TileRegs<T, ROWS, 256> f[3];
#pragma unroll
        for (int i = 0; i < TileRegs<T, ROWS, 256>::kPasses; ++i)
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                float a = whole(hi.w[i][r], lo.w[i][r], 0), b = whole(hi.w[i][r], lo.w[i][r], 1);
#pragma unroll
                for (int n = 0; n < 3; ++n) {
                    f[n].w[i][r] = Mat<T>::high2(a, b);
                    a -= Mat<T>::cut1(a);
                    b -= Mat<T>::cut1(b);
                }
            }
#pragma unroll
        for (int n = 0; n < 3; ++n) f[n].store(tid, tiles[n]);
    } else {
        hi.store(tid, tiles[0]);
    }
}

template <typename T, typename TO, int KC>
__global__ __launch_bounds__(256, (sizeof(T) == 2 ? 2 : 1)) void delta_grads_kernel(DeltaArgs a) {
    using M = Mat<T>;
    using Frag = typename M::Frag;
    constexpr int NM = GradSmem<T>::kTerms, VR = GradSmem<T>::kRows, NV = VR / 16, kHalves = KC / 64;
    using Regs = TileRegs<T, VR, 256>;
    using Wide = TileRegs<float, VR, 256>;
    __shared__ GradSmem<T> sm;
    const int l = lane_id(), w = wave_id(), col = l & 15, g4 = (l >> 4) * 4, tid = threadIdx.x;
    const int64_t L = a.seqlen;
    const int rep = a.heads / a.groups, parts = (rep + a.grad_per - 1) / a.grad_per;
    const uint32_t id = chunk_block(kHalves), unit_id = id / kHalves, row = unit_id / (uint32_t)a.chunks;
    const uint32_t bg = row / (uint32_t)parts, bat = bg / (uint32_t)a.groups;
    const int64_t b = bat, chunk = unit_id - row * (uint32_t)a.chunks, grp = bg - bat * (uint32_t)a.groups, t0 = chunk * kC;
    const int half = (int)(id % kHalves), part = (int)(row - bg * (uint32_t)parts);
    const int f0 = half * 64, frows = min(64, a.dk - f0);
    const bool few_k = !M::kSplit && frows <= 32;       // in 32 bits, where matrix instructions are slow: tiles without features are left out
    const int vpad = a.dv <= 64 ? 64 : 128, vsteps = (a.dv + VR - 1) / VR;
    const int h0 = (int)grp * rep + part * a.grad_per, h1 = min((int)(grp + 1) * rep, h0 + a.grad_per);
    const T* kp = static_cast<const T*>(a.k) + ((b * a.groups + grp) * a.dk + f0) * L;
    const T* qp = static_cast<const T*>(a.q) + ((b * a.groups + grp) * a.dk + f0) * L;
    const uint32_t at = Regs::offset_of(tid, (int)t0, (int)L), sat = Wide::offset_of(tid, 0, KC);
    const int slots = delta_slots<T>(a.chunks);

    f32x4 dq[4], dk[4];
#pragma unroll
    for (int f = 0; f < 4; ++f) dq[f] = dk[f] = f32x4{0, 0, 0, 0};

    Regs dor, er, lr, wr, xr;
    Wide sr, gr;
    float cr[2];
    const int steps = (h1 - h0) * vsteps;
    const auto rows_of_step = [&](int step) { return min(VR, a.dv - step % vsteps * VR); };
    const auto base = [&](const void* p, int step) {
        const int h = h0 + step / vsteps, v0 = step % vsteps * VR;
        return static_cast<const T*>(p) + ((b * a.heads + h) * a.dv + v0) * L;
    };
    const auto load = [&](int step) {
        const int h = h0 + step / vsteps, v0 = step % vsteps * VR, rows = rows_of_step(step);
        const int64_t bh = b * a.heads + h;
        dor.load(tid, at, base(a.dout, step), rows, (int)L);
        er.load(tid, at, base(a.e, step), rows, (int)L);
        wr.load(tid, at, base(a.w, step), rows, (int)L);
        if constexpr (M::kSplit) {
            lr.load(tid, at, base(a.e_low, step), rows, (int)L);
            xr.load(tid, at, base(a.w_low, step), rows, (int)L);
        }
        sr.load(tid, sat, a.states + ((bh * slots + chunk) * vpad + v0) * KC + f0, VR, KC);
        gr.load(tid, sat, a.grads + ((bh * a.chunks + chunk) * vpad + v0) * KC + f0, VR, KC);
        const float* cf = a.coef + (bh * a.chunks + chunk) * kDeltaCoef;
        cr[0] = cf[tid];
        cr[1] = cf[min(tid + 256, kDeltaCoef - 1)];
    };
    {
        using Keys = TileRegs<T, 64, 256>;
        Keys kr, qr;
        const uint32_t kat = Keys::offset_of(tid, (int)t0, (int)L);
        kr.load(tid, kat, kp, frows, (int)L);
        qr.load(tid, kat, qp, frows, (int)L);
        load(0);                                        // blocks are short: all their first loads at once
        kr.settle(tid, kp, frows, t0, L);
        qr.settle(tid, qp, frows, t0, L);
        kr.store(tid, sm.k);
        qr.store(tid, sm.q);
    }
    // Mo's tiles of the wave's 16 tokens: with the earlier ones (and its own) as rows of dq, with the later ones of dk; the
    // diagonal tile a second time for dk.  Mv's the same way.
    f32x4 mo[4], mv[4], mo_d, mv_d;
    for (int step = 0; step < steps; ++step) {
        const bool first = step % vsteps == 0, done = step % vsteps == vsteps - 1;
        const int rows = rows_of_step(step);
        const bool few_v = !M::kSplit && rows <= 32;
        __syncthreads();
        dor.settle(tid, base(a.dout, step), rows, t0, L);
        er.settle(tid, base(a.e, step), rows, t0, L);
        wr.settle(tid, base(a.w, step), rows, t0, L);
        if constexpr (M::kSplit) {
            lr.settle(tid, base(a.e_low, step), rows, t0, L);
            xr.settle(tid, base(a.w_low, step), rows, t0, L);
        }
        dor.store(tid, sm.dout);
        store_halves<T, VR>(tid, er, lr, sm.e);
        store_halves<T, VR>(tid, wr, xr, sm.w);
        store_terms<VR>(tid, sr, sm.st.s);
        store_terms<VR>(tid, gr, sm.st.d);
        sm.coef[tid] = cr[0];
        if (tid + 256 < kDeltaCoef) sm.coef[tid + 256] = cr[1];
        __syncthreads();
        load(min(step + 1, steps - 1));
        const int l = here(lane_id()), col = l & 15, g4 = (l >> 4) * 4;
        const auto c4 = [&](int which, int i) { return *reinterpret_cast<const f32x4*>(&sm.coef[which + i * 16 + g4]); };
        const auto tok = [&](const T* tile, int k, int i) { return M::transposed(l, tile + k * 16 * kC, i); };
        if (first) {
            mo_d = mv_d = f32x4{0, 0, 0, 0};
#pragma unroll
            for (int i = 0; i < 4; ++i) mo[i] = mv[i] = f32x4{0, 0, 0, 0};
        }
        Frag dw[NV], uw[NM][NV], ww[NM][NV];
#pragma unroll
        for (int n = 0; n < NV; ++n) {
            dw[n] = tok(sm.dout, n, w);
#pragma unroll
            for (int p = 0; p < NM; ++p) {
                uw[p][n] = tok(sm.e[p], n, w);
                ww[p][n] = tok(sm.w[p], n, w);
            }
        }
        // terms' products below the last term's size are left out, the small ones come first
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            if (i <= w) {
#pragma unroll
                for (int n = 0; n < NV; n += 2) {
                    if (n >= 2 && few_v) break;
#pragma unroll
                    for (int p = NM - 1; p >= 0; --p) {
                        const Frag x0 = tok(sm.e[p], n, i), x1 = tok(sm.e[p], n + 1, i);
                        mo[i] = M::mma(x0, x1, dw[n], dw[n + 1], mo[i]);
#pragma unroll
                        for (int m = NM - 1 - p; m >= 0; --m) mv[i] = M::mma(x0, x1, ww[m][n], ww[m][n + 1], mv[i]);
                    }
                }
            } else {
#pragma unroll
                for (int n = 0; n < NV; n += 2) {
                    if (n >= 2 && few_v) break;
                    const Frag x0 = tok(sm.dout, n, i), x1 = tok(sm.dout, n + 1, i);
#pragma unroll
                    for (int p = NM - 1; p >= 0; --p) {
                        mo[i] = M::mma(x0, x1, uw[p][n], uw[p][n + 1], mo[i]);
                        const Frag y0 = tok(sm.w[p], n, i), y1 = tok(sm.w[p], n + 1, i);
#pragma unroll
                        for (int m = NM - 1 - p; m >= 0; --m) mv[i] = M::mma(y0, y1, uw[m][n], uw[m][n + 1], mv[i]);
                    }
                }
            }
        }
#pragma unroll
        for (int n = 0; n < NV; n += 2) {
            if (n >= 2 && few_v) break;
#pragma unroll
            for (int p = NM - 1; p >= 0; --p) {
                mo_d = M::mma(dw[n], dw[n + 1], uw[p][n], uw[p][n + 1], mo_d);
#pragma unroll
                for (int m = NM - 1 - p; m >= 0; --m) mv_d = M::mma(ww[p][n], ww[p][n + 1], uw[m][n], uw[m][n + 1], mv_d);
            }
        }
        {
            const f32x4 in = c4(kCoefIn, w), up = c4(kCoefUp, w) * c4(kCoefBeta, w), scaled = in * a.scale;
            float least = 1.0f;                             // a NaN among them does not count
#pragma unroll
            for (int r = 0; r < 4; ++r) least = fminf(least, fminf(fabsf(in[r]), fabsf(up[r])));
            const bool zeros = __ballot(least == 0.0f) != 0;
            const auto states = [&](auto some) {
#pragma unroll
                for (int f = 0; f < 4; ++f) {
                    if (f >= 2 && few_k) break;
                    f32x4 q = {0, 0, 0, 0}, g = q, x = q;
#pragma unroll
                    for (int n = 0; n < NV; n += 2) {
                        if (n >= 2 && few_v) break;
#pragma unroll
                        for (int p = NM - 1; p >= 0; --p) {
                            const Frag s0 = tok(sm.st.s[p], n, f), s1 = tok(sm.st.s[p], n + 1, f);
                            const Frag d0 = tok(sm.st.d[p], n, f), d1 = tok(sm.st.d[p], n + 1, f);
                            q = M::mma(dw[n], dw[n + 1], s0, s1, q);
#pragma unroll
                            for (int m = NM - 1 - p; m >= 0; --m) {
                                x = M::mma(ww[m][n], ww[m][n + 1], s0, s1, x);
                                g = M::mma(uw[m][n], uw[m][n + 1], d0, d1, g);
                            }
                        }
                    }
                    if constexpr (decltype(some)::value) {
                        q = masked(q, in);
                        x = masked(x, in);
                        g = masked(g, up);
                    }
                    dq[f] += q * scaled;
                    dk[f] += g * up - x * in;
                }
            };
            if (zeros) states(std::true_type{});            // sequences start here, or betas are 0
            else states(std::false_type{});
        }
        if (!done) continue;
        // weights between the tokens
        {
            const int t = w * 16 + col;
            const float hi = sm.coef[kCoefHi + t], lo = sm.coef[kCoefLo + t];
            const float beta = sm.coef[kCoefBeta + t];
            const int start = __float_as_int(sm.coef[kCoefStart + t]);
            // tile i's pairs, whose tokens are the later ones or the earlier: no condition is a branch
            const auto weigh = [&](auto side, int i, f32x4& o, f32x4& v) {
                constexpr bool kLater = decltype(side)::value;
                const f32x4 hi4 = c4(kCoefHi, i), lo4 = c4(kCoefLo, i), st4 = c4(kCoefStart, i), b4 = c4(kCoefBeta, i);
#pragma unroll
                for (int r = 0; r < 4; ++r) {
                    const int s = i * 16 + g4 + r;
                    const float d = kLater ? pair_decay(hi4[r], lo4[r], hi, lo) * beta : pair_decay(hi, lo, hi4[r], lo4[r]) * b4[r];    // the earlier one's beta
                    const int on = kLater ? (int)(t <= s) & (int)(__float_as_int(st4[r]) <= t) : (int)(s <= t) & (int)(start <= s);
                    const float od = o[r] * (d * a.scale), vd = -v[r] * d;
                    o[r] = on ? od : 0.0f;
                    v[r] = on & (int)(s != t) ? vd : 0.0f;
                }
            };
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                if (i <= w) weigh(std::false_type{}, i, mo[i], mv[i]);
                else weigh(std::true_type{}, i, mo[i], mv[i]);
            }
            weigh(std::true_type{}, w, mo_d, mv_d);
#pragma unroll
            for (int i = 0; i < 4; ++i)
                if (i == w) mv[i] += mv_d;               // each is 0 where the other is not
        }
        if (__builtin_amdgcn_readfirstlane(__float_as_int(sm.coef[kCoefA + 1])) == 0) {
            Frag diag[NM];
            M::template split<NM>(mo_d, diag);
#pragma unroll
            for (int p = 0; p < 2; ++p) {                        // pairs of token tiles
                Frag a0[NM], a1[NM], b0[NM], b1[NM], e0[NM], e1[NM];
                const auto rows_of = [&](int i, Frag (&q)[NM], Frag (&k)[NM], Frag (&v)[NM]) {
                    Frag o[NM];
                    M::template split<NM>(mo[i], o);
                    M::template split<NM>(mv[i], v);
#pragma unroll
                    for (int n = 0; n < NM; ++n) {
                        q[n] = i <= w ? o[n] : Frag{};
                        k[n] = i == w ? diag[n] : i > w ? o[n] : Frag{};
                    }
                };
                rows_of(2 * p, a0, b0, e0);
                rows_of(2 * p + 1, a1, b1, e1);
#pragma unroll
                for (int f = 0; f < 4; ++f) {
                    if (f >= 2 && few_k) break;
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
        } else {                                                 // k or q not finite: pair by pair, a wave's rows of M in LDS
            float* rows16 = reinterpret_cast<float*>(&sm.st) + w * 16 * kC;
            __syncthreads();
#pragma unroll
            for (int which = 0; which < 3; ++which) {            // dq from k, dk from q, dk from k
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const f32x4 none = {0, 0, 0, 0};
                    const f32x4 v = which == 0 ? (i <= w ? mo[i] : none) : which == 1 ? (i == w ? mo_d : i > w ? mo[i] : none) : mv[i];
                    *reinterpret_cast<f32x4*>(rows16 + col * kC + i * 16 + g4) = v;
                }
                __builtin_amdgcn_wave_barrier();
#pragma unroll 1
                for (int s = 0; s < kC; ++s)
#pragma unroll 1
                    for (int x = 0; x < 4; ++x) {
                        const float m = rows16[(g4 + x) * kC + s];
#pragma unroll
                        for (int f = 0; f < 4; ++f) {
                            const float v = m == 0.0f ? 0.0f : m * tile_value((which == 1 ? sm.q : sm.k) + f * 16 * kC, col, s);
#pragma unroll
                            for (int r = 0; r < 4; ++r) {
                                if (which == 0) dq[f][r] += x == r ? v : 0.0f;
                                else dk[f][r] += x == r ? v : 0.0f;
                            }
                        }
                    }
                __builtin_amdgcn_wave_barrier();
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
    if (rev) hipLaunchKernelGGL((delta_chain<KC, true>), grid, dim3(KC * 4), 0, s, a);
    else hipLaunchKernelGGL((delta_chain<KC, false>), grid, dim3(KC * 4), 0, s, a);
    return hipGetLastError();
}

}  // namespace

hipError_t launch_delta_fwd(const DeltaArgs& a, bool split, hipStream_t s) {
    if (split)
        if (hipError_t e = launch_delta_segments(a, false, s)) return e;
    return walk(a, kWalkOut, s);
}
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
