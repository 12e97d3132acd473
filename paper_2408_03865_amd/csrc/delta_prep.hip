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
// A block takes a chunk and the heads of a group in turn, whose keys' products it makes once.
// What bounds it: 8 x 4096 tokens, 32 heads in 16 groups of 128 features, 181 us for 630 MB, 3.5 TB/s, with the waves at the barriers
// between weights, diagonal blocks and the others half the time (VALU 38%, LDS 34%, matrix 13%); four blocks a CU and not three
// change calls by less than 1%.  Blocks that start with the same column on each SIMD: 230; the 32-bit products kept as three bf16 terms, as the
// walks take them: 205, and 20 KB more of memory a chunk and walk.
#include "linear_walk.hpp"
#include "delta.hpp"

namespace pm {
namespace {

__host__ __device__ constexpr int tile_at(int i, int j) { return i * (i + 1) / 2 + j; }

// A product of blocks, added to two sums in turns: an instruction that takes the result of the one before waits for it.
__device__ __forceinline__ void mma16(const f32x4& a, const f32x4& b, f32x4 (&c)[2]) {
#pragma unroll
    for (int e = 0; e < 4; ++e) c[e & 1] = __builtin_amdgcn_mfma_f32_16x16x4f32(a[e], b[e], c[e & 1], 0, 0, 0);
}

// The keys and queries are done with once their products are in registers.
template <typename T, int KC>
struct PrepSmem {
    struct Inputs {
        __attribute__((aligned(16))) T k[KC * kC];
        __attribute__((aligned(16))) T q[KC * kC];
    };
    struct Solve {
        f32x4 a[kDeltaTiles][64];           // A as operands
        f32x4 hd[4][64];                    // H's diagonal blocks as operands
        __attribute__((aligned(16))) float cols[4][16][20];     // A's diagonal blocks by columns
        __attribute__((aligned(16))) float turn[4][16][20];
    };
    union {
        Inputs in;
        Solve at;
    };
    ChunkDecay c[2];                        // the head's, and the next one's
    __attribute__((aligned(16))) float beta[2][kC];
    int bad;
};

// A tile of one of the two products.
__device__ __forceinline__ void put_tile(const DeltaArgs& a, int64_t unit, int which, int tile, const f32x4& v) {
    reinterpret_cast<f32x4*>(a.products)[(unit * 2 + which) * (kDeltaProduct / 4) + tile * 64 + lane_id()] = v;
}

// One block a chunk and heads_per heads of one group.  Wave j takes the tiles of column j.
template <typename T, int KC>
__global__ __launch_bounds__(256, 3) void delta_prep_kernel(DeltaArgs a) {
    using M = Mat<T>;
    using Frag = typename M::Frag;
    constexpr int KT = KC / 16;
    __shared__ PrepSmem<T, KC> sm;
    // the columns have four to one tiles: blocks of a CU start with different ones, so that no SIMD has all the long ones
    const int l = lane_id(), w = (wave_id() + (int)blockIdx.x) & 3, g4 = (l >> 4) * 4, col = l & 15;
    const int64_t L = a.seqlen;
    const int rep = a.heads / a.groups, parts = (rep + a.heads_per - 1) / a.heads_per;
    const uint32_t id = chunk_block(1), row = id / (uint32_t)a.chunks;
    const uint32_t bg = row / (uint32_t)parts, bat = bg / (uint32_t)a.groups;
    const int64_t b = bat, chunk = id - row * (uint32_t)a.chunks, grp = bg - bat * (uint32_t)a.groups, t0 = chunk * kC;
    const int part = (int)(row - bg * (uint32_t)parts);
    const T* kp = static_cast<const T*>(a.k) + (b * a.groups + grp) * a.dk * L;
    const T* qp = static_cast<const T*>(a.q) + (b * a.groups + grp) * a.dk * L;
    const int h0 = (int)grp * rep + part * a.heads_per, h1 = min((int)(grp + 1) * rep, h0 + a.heads_per);

    if (threadIdx.x == 0) sm.bad = 0;
    // a head's weights, by the wave that has the fewest products
    TokenDecay td{0.0f, 1};
    float tb = 0.0f;
    const auto load_weights = [&](int h) {
        const int64_t t = t0 + l;
        td = TokenDecay{0.0f, 1};
        tb = 0.0f;
        if (t < L) {
            td.pos = a.pos[b * L + t];
            if (a.decay_mode == 2) td.g = a.decay[(b * a.heads + h) * L + t];
            else if (a.decay_mode == 1) td.g = a.decay[h];
            tb = a.beta[(b * a.heads + h) * L + t];
        }
    };
    if (w == 3) load_weights(h0);
    {
        TileRegs<T, KC, 256> kr, qr;
        const uint32_t at = TileRegs<T, KC, 256>::offset_of(threadIdx.x, (int)t0, (int)L);
        kr.load(threadIdx.x, at, kp, a.dk, (int)L);
        qr.load(threadIdx.x, at, qp, a.dk, (int)L);
        kr.settle(threadIdx.x, kp, a.dk, t0, L);
        qr.settle(threadIdx.x, qp, a.dk, t0, L);
        kr.store(threadIdx.x, sm.in.k);
        qr.store(threadIdx.x, sm.in.q);
        __syncthreads();
        if (qr.zero_sum(kr.zero_sum(0.0f)) != 0.0f) sm.bad = 1;
    }
    // products of column w's tokens with the later ones, as operands (a lane is a later token)
    f32x4 kf[4], qf[4];
    {
        Frag ks[KT];
#pragma unroll
        for (int k = 0; k < KT; ++k) ks[k] = M::transposed(l, sm.in.k + k * 16 * kC, w);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            kf[i] = qf[i] = f32x4{0, 0, 0, 0};
            if (i < w) continue;
#pragma unroll
            for (int k = 0; k < KT; k += 2) {
                if (!M::kSplit && KT == 4 && k >= 2 && a.dk <= 32) break;
                const Frag k0 = M::transposed(l, sm.in.k + k * 16 * kC, i), k1 = M::transposed(l, sm.in.k + (k + 1) * 16 * kC, i);
                const Frag q0 = M::transposed(l, sm.in.q + k * 16 * kC, i), q1 = M::transposed(l, sm.in.q + (k + 1) * 16 * kC, i);
                kf[i] = M::mma(ks[k], ks[k + 1], k0, k1, kf[i]);
                qf[i] = M::mma(ks[k], ks[k + 1], q0, q1, qf[i]);
            }
        }
    }
    const auto weigh = [&](int which) {
        chunk_decay<false>(td, sm.c[which], 1.0f, 1.0f);
        sm.beta[which][l] = tb;
    };
    if (w == 3) {
        weigh(0);
        if (h0 + 1 < h1) load_weights(h0 + 1);
    }
    for (int h = h0; h < h1; ++h) {
        const int64_t unit = (b * a.heads + h) * a.chunks + chunk;
        float* cf = a.coef + unit * kDeltaCoef;
        const ChunkDecay& c = sm.c[(h - h0) & 1];
        const float* betas = sm.beta[(h - h0) & 1];
        __syncthreads();                                // the weights are there, and the head before is done with the tiles
        if (w == 1) {
            cf[kCoefIn + l] = c.in[l];
            cf[kCoefUp + l] = c.up[l];
            cf[kCoefBeta + l] = betas[l];
            cf[kCoefHi + l] = c.hi[l];
            cf[kCoefLo + l] = c.lo[l];
            cf[kCoefStart + l] = __int_as_float(c.start[l]);
            if (l == 0) {
                cf[kCoefA] = c.a;
                cf[kCoefA + 1] = __int_as_float(sm.bad);
            }
        }
        // weighted: A and P
        {
            const int s4 = w * 16 + g4;
            const f32x4 hi4 = *reinterpret_cast<const f32x4*>(&c.hi[s4]), lo4 = *reinterpret_cast<const f32x4*>(&c.lo[s4]);
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                if (i < w) continue;
                const int t1 = i * 16 + col, start = c.start[t1];
                const float thi = c.hi[t1], tlo = c.lo[t1];
                f32x4 af, pv;
#pragma unroll
                for (int r = 0; r < 4; ++r) {
                    const float d = pair_decay(thi, tlo, hi4[r], lo4[r]);
                    const bool on = s4 + r <= t1 && start <= s4 + r;
                    af[r] = on && s4 + r < t1 ? kf[i][r] * d : 0.0f;
                    pv[r] = on ? qf[i][r] * (d * a.scale) : 0.0f;
                }
                sm.at.a[tile_at(i, w)][l] = af;
                put_tile(a, unit, 1, tile_at(i, w), pv);
                if (i == w) {
#pragma unroll
                    for (int r = 0; r < 4; ++r) sm.at.cols[w][g4 + r][col] = af[r];
                }
            }
        }
        __syncthreads();
        // H's diagonal block, column col in every lane, row by row
        f32x4 nb[4];                    // -beta H, as results
        const auto beta4 = [&](int i) { return *reinterpret_cast<const f32x4*>(&betas[i * 16 + g4]); };
        const auto turned = [&](const f32x4& v) {           // a result as an operand
            *reinterpret_cast<f32x4*>(&sm.at.turn[w][col][g4]) = v;
            __builtin_amdgcn_wave_barrier();
            f32x4 o;
#pragma unroll
            for (int r = 0; r < 4; ++r) o[r] = sm.at.turn[w][g4 + r][col];
            __builtin_amdgcn_wave_barrier();
            return o;
        };
        f32x4 own;
        {
            float x[16];
#pragma unroll
            for (int i = 0; i < 16; i += 4) {
                const f32x4 v = *reinterpret_cast<const f32x4*>(&sm.at.cols[w][col][i]);
#pragma unroll
                for (int r = 0; r < 4; ++r) x[i + r] = v[r];
            }
            // a row that is done leaves those below it: what waits for the row before is one product a row
#pragma unroll
            for (int i = 0; i < 15; ++i) {
                const float xb = x[i] * betas[w * 16 + i];
#pragma unroll
                for (int q = i / 4 * 4; q < 16; q += 4) {
                    const f32x4 below = *reinterpret_cast<const f32x4*>(&sm.at.cols[w][i][q]);
#pragma unroll
                    for (int r = 0; r < 4; ++r)
                        if (q + r > i) x[q + r] = fmaf(-below[r], xb, x[q + r]);
                }
            }
            const int g = l >> 4;
#pragma unroll
            for (int r = 0; r < 4; ++r) own[r] = g == 0 ? x[r] : g == 1 ? x[4 + r] : g == 2 ? x[8 + r] : x[12 + r];
        }
        {
            const f32x4 f = turned(own);
            sm.at.hd[w][l] = f;
            put_tile(a, unit, 0, tile_at(w, w), f);
        }
        __syncthreads();
        if (w == 3 && h + 1 < h1) {                     // this wave has no blocks below its diagonal one
            weigh((h + 1 - h0) & 1);
            if (h + 2 < h1) load_weights(h + 2);
        }
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            nb[i] = f32x4{0, 0, 0, 0};
            if (i < w) continue;
            f32x4 hc = own;
            if (i != w) {
                f32x4 y[2] = {{0, 0, 0, 0}, {0, 0, 0, 0}};      // A_ij as a result: the operand turned
                const float* at = reinterpret_cast<const float*>(&sm.at.a[tile_at(i, w)][(col >> 2) * 16 + g4]) + (col & 3);
#pragma unroll
                for (int r = 0; r < 4; ++r) y[0][r] = at[r * 4];
#pragma unroll
                for (int k = 0; k < i; ++k)
                    if (k >= w) mma16(sm.at.a[tile_at(i, k)][l], nb[k], y);
                y[0] += y[1];
                y[1] = f32x4{0, 0, 0, 0};
                mma16(sm.at.hd[i][l], y[0] * -beta4(i), y);
                hc = y[0] + y[1];
                put_tile(a, unit, 0, tile_at(i, w), turned(hc));
            }
            nb[i] = hc * -beta4(i);
        }
    }
}

template <typename T>
hipError_t prep_t(const DeltaArgs& a, hipStream_t s) {
    const int64_t parts = (a.heads / a.groups + a.heads_per - 1) / a.heads_per;
    const dim3 grid((unsigned)((int64_t)a.batch * a.chunks * a.groups * parts));
    if (a.dk <= 64) hipLaunchKernelGGL((delta_prep_kernel<T, 64>), grid, dim3(256), 0, s, a);
    else hipLaunchKernelGGL((delta_prep_kernel<T, 128>), grid, dim3(256), 0, s, a);
    return hipGetLastError();
}

}  // namespace

hipError_t launch_delta_prep(const DeltaArgs& a, hipStream_t s) {
    return a.dtype == 0 ? prep_t<float>(a, s) : prep_t<bf16_t>(a, s);
}

}  // namespace pm
