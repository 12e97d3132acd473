// linear_walk.hpp -- the walk that every linear-attention pass is made of.
//
// With a_t = exp(g_t), 0 at a sequence start, and S_t = a_t S_{t-1} + y_t z_t^T, a walk gives
// out_t = S_t^T x_t for every token of a row and head.  In chunks of 64 tokens, with G the sum
// of the log decays since the chunk's or the sequence's start, whichever is later:
//   out_i = in_i S^T x_i + sum_{j <= i, same sequence} exp(G_i - G_j) (x_i . y_j) z_j
//   S    <- A S + sum_j up_j y_j z_j^T
//   in_i = exp(G_i) where no sequence starts in the chunk up to i, up_j = exp(G_end - G_j) where
//   none starts after j, A = exp(G_end) where none starts at all; otherwise the term is left out.
// A reverse walk runs from the last token (i >= j in place of j <= i, `in` and `up` change
// places): its state at a chunk is what the tokens after it make.  All passes are such walks:
//   forward  x, y, z = q, k, v      dq  dout, v, k     (forward in time)
//   dk       v, dout, q             dv  k, q, dout     (reverse)
// The gradient of a log decay at t is the sum of W_ij = exp(G_i - G_j)(q_i . k_j)(dout_i . v_j) over
// i >= t > j, and with r_s = sum_{j <= s} W_sj - sum_{i >= s} W_is that is what r sums to over the tokens
// s >= t up to a boundary, plus <dS, S> there (W over pairs on both sides of the boundary).  The
// pairs inside a chunk are summed from the 32-bit products; a pair's contributions to r_i and r_j
// cancel to rounding.  Boundaries every 512 tokens keep those sums short.
//
// Mapping.  One block of 4 waves walks a row (or a segment of it) of one head; activations are
// (features, tokens), tokens innermost.  A chunk's tiles sit in LDS as they do in memory.  Products
// over tokens (z and the update) read their operands directly, four tokens a lane; products over
// features (x . y and x . S) read them transposed (ds_read_b64_tr_b16 in bf16).  The waves share the
// 64 x 64 products of x and y by strips of 16 x's and pass them, weighted and rounded to T, through
// LDS.  Each wave owns 16 or 32 of z's features: its part of S stays in registers, in the layout
// that an MFMA result has and, four rows of it a lane, an MFMA operand takes.
// Rounding in bf16: the weighted products x . y and, in plain walks, the copy of S that is
// multiplied with x are rounded to bf16 once (each enters bf16 outputs only); what S itself adds is
// split into two or three bf16 terms that hold 16 or all 24 bits of it, and in the walks that feed
// the decay's gradient so is the copy of S.
//
// Infinities and NaN stay in their sequence and do not pass to earlier tokens: masks select, and a
// chunk whose y or z holds one takes plain loops over the unmasked pairs in place of the matrix
// products over tokens, where 0 times it would spread.
#pragma once

#include "common.hpp"
#include "linear.hpp"

namespace pm {

typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));

constexpr int kWalkThreads = 256, kWalkWaves = 4, kC = (int)kLinChunk;

__device__ __forceinline__ int wave_id() { return __builtin_amdgcn_readfirstlane((int)(threadIdx.x >> 6)); }

// A decay below this multiplies by 0 in 32 bits (exp(-104) < 2^-150): the token is taken for a start.
constexpr float kDecayCut = -104.0f;

// --------------------------------------------------------------------------------------------
// matrix operands: four values of the contracted index a lane, 4 (lane / 16) .. + 3 of 16, for
// row or column lane % 16 -- also the layout of a 16 x 16 result, contracted along its rows
// --------------------------------------------------------------------------------------------
template <typename T> struct Mat;

template <> struct Mat<bf16_t> {
    typedef u32x2 Frag;
    static constexpr int kStride = kC + 8;          // of a tile's rows: 144 bytes spread 16 rows over all banks
    static constexpr bool kSplit = true;
    __device__ static Frag direct(const bf16_t* p) { return *reinterpret_cast<const u32x2*>(p); }
    // rows 0..15 of p (kStride apart), token lane % 16 of 16
    __device__ static Frag transposed(const bf16_t* p) {
        const int l = lane_id();
        const bf16_t* q = p + ((l >> 4) * 4 + ((l & 15) >> 2)) * kStride + (l & 3) * 4;
        const s16x4 v = __builtin_amdgcn_ds_read_tr16_b64_v4i16(
            (__attribute__((address_space(3))) s16x4*)(const_cast<bf16_t*>(q)));
        return __builtin_bit_cast(u32x2, v);
    }
    __device__ static Frag round(const f32x4& v) { return Frag{pack_bf16x2(v.x, v.y), pack_bf16x2(v.z, v.w)}; }
    __device__ static f32x4 mma(const Frag& a0, const Frag& a1, const Frag& b0, const Frag& b1, const f32x4& c) {
        const u32x4 a = {a0.x, a0.y, a1.x, a1.y}, b = {b0.x, b0.y, b1.x, b1.y};
        return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), c, 0, 0, 0);
    }
    __device__ static f32x4 widen(const Frag& f) { return f32x4{bf16_lo(f.x), bf16_hi(f.x), bf16_lo(f.y), bf16_hi(f.y)}; }
    // v as a sum of N bf16 values: truncations of what is left, exact for N = 3; the last of two is rounded
    template <int N>
    __device__ static void split(const f32x4& v, Frag* out) {
        if constexpr (N == 1) {
            out[0] = round(v);
        } else {
            out[0] = high(v);
            f32x4 r = v - cut(v);
            if constexpr (N == 3) {
                out[1] = high(r);
                out[2] = high(r - cut(r));
            } else {
                out[1] = round(r);
            }
        }
    }
    __device__ static f32x4 cut(const f32x4& v) {
        return f32x4{cut1(v.x), cut1(v.y), cut1(v.z), cut1(v.w)};
    }
    __device__ static float cut1(float v) { return __uint_as_float(__float_as_uint(v) & 0xffff0000u); }
    __device__ static Frag high(const f32x4& v) { return Frag{high2(v.x, v.y), high2(v.z, v.w)}; }
    __device__ static uint32_t high2(float a, float b) {
        return __builtin_amdgcn_perm(__float_as_uint(b), __float_as_uint(a), 0x07060302u);
    }
    __device__ static bool finite(const u32x4& w) {
        uint32_t t = 0;
#pragma unroll
        for (int i = 0; i < 4; ++i) t |= (w[i] & 0x7f807f80u) + 0x00800080u;
        return (t & 0x80008000u) == 0;
    }
};

template <> struct Mat<float> {
    typedef f32x4 Frag;
    static constexpr int kStride = kC + 4;
    static constexpr bool kSplit = false;
    __device__ static Frag direct(const float* p) { return *reinterpret_cast<const f32x4*>(p); }
    __device__ static Frag transposed(const float* p) {
        const int l = lane_id();
        const float* q = p + (l >> 4) * 4 * kStride + (l & 15);
        return Frag{q[0], q[kStride], q[2 * kStride], q[3 * kStride]};
    }
    __device__ static Frag round(const f32x4& v) { return v; }
    __device__ static f32x4 mma(const Frag& a0, const Frag& a1, const Frag& b0, const Frag& b1, f32x4 c) {
#pragma unroll
        for (int e = 0; e < 4; ++e) c = __builtin_amdgcn_mfma_f32_16x16x4f32(a0[e], b0[e], c, 0, 0, 0);
#pragma unroll
        for (int e = 0; e < 4; ++e) c = __builtin_amdgcn_mfma_f32_16x16x4f32(a1[e], b1[e], c, 0, 0, 0);
        return c;
    }
    __device__ static f32x4 widen(const Frag& f) { return f; }
    template <int N>
    __device__ static void split(const f32x4& v, Frag* out) { out[0] = v; }
    __device__ static bool finite(const u32x4& w) {
        bool ok = true;
#pragma unroll
        for (int i = 0; i < 4; ++i) ok = ok && (w[i] & 0x7f800000u) != 0x7f800000u;
        return ok;
    }
};

// --------------------------------------------------------------------------------------------
// a chunk's decays
// --------------------------------------------------------------------------------------------
struct __attribute__((aligned(16))) ChunkDecay {
    float hi[kC], lo[kC];       // G in log2 units, as a sum of two floats
    float in[kC], up[kC];       // -1: left out
    int32_t start[kC];          // the last start up to the token, -1: none in the chunk
    float a;                    // -1: cut
    int32_t bad[1];             // an infinity or a NaN in y or z
};

struct TokenDecay {
    float g;
    int32_t pos;
};

__device__ __forceinline__ TokenDecay load_decay(const WalkArgs& a, int64_t b, int64_t h, int64_t t) {
    TokenDecay d{0.0f, 1};
    if (t < a.seqlen) {
        d.pos = a.pos[b * a.seqlen + t];
        if (a.decay_mode == 2) d.g = a.decay[(b * a.heads + h) * a.seqlen + t];
        else if (a.decay_mode == 1) d.g = a.decay[h];
    }
    return d;
}

// exp2 of (hi_i + lo_i) - (hi_j + lo_j)
__device__ __forceinline__ float pair_decay(float hi, float lo, float hj, float lj) {
    return fast_exp2((hi - hj) + (lo - lj));
}

// One wave, lane = token.  The sum is kept in 64 bits and starts anew at each start, so that no
// sequence's decays reach another's.
__device__ __forceinline__ void chunk_decay(const TokenDecay& d, bool rev, ChunkDecay& c) {
    const int l = lane_id();
    bool cut = d.pos == 0 || d.g <= kDecayCut;
    double v = cut ? 0.0 : (double)d.g * 1.4426950408889634;
    int start = cut ? l : -1;
#pragma unroll
    for (int m = 1; m < 64; m *= 2) {
        const double pv = __shfl_up(v, m);
        const int ps = __shfl_up(start, m);
        if (l >= m && start < 0) {      // no start in the lanes summed so far
            v += pv;
            start = ps;
        }
    }
    const float hi = (float)v, lo = (float)(v - (double)hi);
    const float ehi = __shfl(hi, 63), elo = __shfl(lo, 63);
    const int estart = __shfl(start, 63);
    const float first = start < 0 ? fast_exp2(hi + lo) : -1.0f;
    const float last = l >= estart ? pair_decay(ehi, elo, hi, lo) : -1.0f;
    c.hi[l] = hi;
    c.lo[l] = lo;
    c.start[l] = start;
    c.in[l] = rev ? last : first;
    c.up[l] = rev ? first : last;
    if (l == 63) c.a = first;
}

// --------------------------------------------------------------------------------------------
// tiles: ROWS features x 64 tokens through registers into LDS; features and tokens that the tensor
// lacks are 0
// --------------------------------------------------------------------------------------------
template <typename T, int ROWS>
struct TileRegs {
    static constexpr int kPer = Storage<T>::kPerVec, kLanes = kC / kPer, kRowsPass = kWalkThreads / kLanes;
    static constexpr int kPasses = ROWS / kRowsPass;
    u32x4 w[kPasses];

    __device__ void load(const T* p, int rows, int64_t t0, int64_t L) {
        const int tok = (threadIdx.x % kLanes) * kPer, row0 = threadIdx.x / kLanes;
        const bool whole = t0 + kC <= L;
#pragma unroll
        for (int i = 0; i < kPasses; ++i) {
            const int row = row0 + i * kRowsPass;
            w[i] = u32x4{0, 0, 0, 0};
            if (row < rows) {
                const T* src = p + (int64_t)row * L + t0 + tok;
                if (whole || t0 + tok + kPer <= L) {
                    w[i] = load_vec<T, kPer>(src);
                } else {
                    float v[kPer];
#pragma unroll
                    for (int k = 0; k < kPer; ++k) v[k] = t0 + tok + k < L ? Storage<T>::load1(src + k) : 0.0f;
                    w[i] = Storage<T>::pack(v);
                }
            }
        }
    }
    __device__ void store(T* tile) const {
        const int tok = (threadIdx.x % kLanes) * kPer, row0 = threadIdx.x / kLanes;
#pragma unroll
        for (int i = 0; i < kPasses; ++i)
            *reinterpret_cast<u32x4*>(tile + (row0 + i * kRowsPass) * Mat<T>::kStride + tok) = w[i];
    }
    __device__ bool finite() const {
        bool ok = true;
#pragma unroll
        for (int i = 0; i < kPasses; ++i) ok = Mat<T>::finite(w[i]) && ok;
        return ok;
    }
};

template <typename T>
__device__ __forceinline__ const T* head_base(const WalkTensor& t, int64_t b, int64_t h, int heads, int64_t L) {
    return static_cast<const T*>(t.p) + ((b * t.heads + h / (heads / t.heads)) * t.rows) * L;
}

// The block's place: heads that share tensors run on one XCD, whose L2 then holds them (blocks go to
// the 8 XCDs in turn).
__device__ __forceinline__ int64_t walk_block(int64_t n) {
    const int64_t id = blockIdx.x, per = n / 8;
    return id < per * 8 ? (id % 8) * per + id / 8 : id;
}

// --------------------------------------------------------------------------------------------
// the state: KT x DT tiles of 16 x features by 16 z features; wave w owns z features 16 DT w .. + 16 DT - 1
// --------------------------------------------------------------------------------------------
template <int KT, int DT>
struct State {
    f32x4 s[KT][DT];

    template <typename F>
    __device__ void each(F f) {         // f(x feature of the tile's row 0, z feature, its four values)
        const int l = lane_id(), w = wave_id();
#pragma unroll
        for (int k = 0; k < KT; ++k)
#pragma unroll
            for (int d = 0; d < DT; ++d) f(k * 16 + (l >> 4) * 4, (w * DT + d) * 16 + (l & 15), s[k][d]);
    }
    __device__ void load(const float* p, const WalkArgs& a) {
        each([&](int xf, int zf, f32x4& v) {
#pragma unroll
            for (int r = 0; r < 4; ++r)
                v[r] = p && xf + r < a.x.rows && zf < a.z.rows ? p[(int64_t)(xf + r) * a.s_x + (int64_t)zf * a.s_z] : 0.0f;
        });
    }
    __device__ void store(float* p, const WalkArgs& a) {
        each([&](int xf, int zf, f32x4& v) {
#pragma unroll
            for (int r = 0; r < 4; ++r)
                if (xf + r < a.x.rows && zf < a.z.rows) p[(int64_t)(xf + r) * a.s_x + (int64_t)zf * a.s_z] = v[r];
        });
    }
    __device__ void decay(float a) {
#pragma unroll
        for (int k = 0; k < KT; ++k)
#pragma unroll
            for (int d = 0; d < DT; ++d)
                s[k][d] = a < 0.0f ? f32x4{0, 0, 0, 0} : s[k][d] * a;
    }
};

// S <- A S + sum_j up_j y_j z_j^T; zf: the wave's z, four tokens a lane, for each of the four token tiles
template <typename T, int NS, int KT, int DT>
__device__ __forceinline__ void update(State<KT, DT>& S, const T* ys, const T* zs, const ChunkDecay& c, float uscale) {
    using M = Mat<T>;
    const int l = lane_id(), w = wave_id(), row = l & 15, tok = (l >> 4) * 4;
    S.decay(c.a);
    if (c.bad[0]) {
#pragma unroll 1
        for (int j = 0; j < kC; ++j) {
            const float up = c.up[j];
            if (up < 0.0f) continue;
#pragma unroll
            for (int k = 0; k < KT; ++k)
#pragma unroll
                for (int d = 0; d < DT; ++d) {
                    const float zv = Storage<T>::load1(zs + ((w * DT + d) * 16 + row) * M::kStride + j) * (up * uscale);
#pragma unroll
                    for (int r = 0; r < 4; ++r)
                        S.s[k][d][r] = fmaf(Storage<T>::load1(ys + (k * 16 + tok + r) * M::kStride + j), zv, S.s[k][d][r]);
                }
        }
        return;
    }
#pragma unroll
    for (int p = 0; p < 2; ++p) {                               // 32 tokens
        typename M::Frag zw[2][DT][NS];
#pragma unroll
        for (int q = 0; q < 2; ++q) {
            const int t0 = (2 * p + q) * 16 + tok;
            f32x4 up = *reinterpret_cast<const f32x4*>(&c.up[t0]);
#pragma unroll
            for (int r = 0; r < 4; ++r) up[r] = up[r] < 0.0f ? 0.0f : up[r] * uscale;
#pragma unroll
            for (int d = 0; d < DT; ++d)
                M::template split<NS>(M::widen(M::direct(zs + ((w * DT + d) * 16 + row) * M::kStride + t0)) * up, zw[q][d]);
        }
#pragma unroll
        for (int k = 0; k < KT; ++k) {
            const T* y = ys + (k * 16 + row) * M::kStride + 2 * p * 16 + tok;
            const typename M::Frag y0 = M::direct(y), y1 = M::direct(y + 16);
#pragma unroll
            for (int d = 0; d < DT; ++d)
#pragma unroll
                for (int n = 0; n < NS; ++n) S.s[k][d] = M::mma(y0, y1, zw[0][d][n], zw[1][d][n], S.s[k][d]);
        }
    }
}

__device__ __forceinline__ float sum16(float v) {       // over the 16 lanes of a row, to all of them
#pragma unroll
    for (int m = 1; m < 16; m *= 2) v += __shfl_xor(v, m, 16);
    return v;
}

template <typename T, int KC, int VP, int MODE>
struct WalkSmem {
    static constexpr int kS = Mat<T>::kStride;
    __attribute__((aligned(16))) T x[KC * kS];
    __attribute__((aligned(16))) T y[KC * kS];
    __attribute__((aligned(16))) T z[VP * kS];
    __attribute__((aligned(16))) T e[MODE != kWalkPlain ? VP * kS : 8];
    __attribute__((aligned(16))) T p[kC * kS];          // x's rows
    ChunkDecay c[2];
    __attribute__((aligned(16))) float rsum[MODE == kWalkDq ? kC : 4];
    __attribute__((aligned(16))) float csum[MODE == kWalkDq ? kWalkWaves : 1][kC];
    __attribute__((aligned(16))) float dot[MODE != kWalkPlain ? kWalkWaves : 1][kC];
    float xdot[kWalkWaves];
};

template <typename T, typename TO, int KC, int VP, int MODE, int NS, int NO>
__global__ __launch_bounds__(kWalkThreads) void walk_kernel(WalkArgs a) {
    using M = Mat<T>;
    using Frag = typename M::Frag;
    constexpr int KT = KC / 16, DT = VP / (16 * kWalkWaves), VT = VP / 16, kS = M::kStride;
    constexpr bool kAhead = sizeof(T) == 2;             // the next chunk's tiles are loaded during a chunk
    __shared__ WalkSmem<T, KC, VP, MODE> sm;
    const int l = lane_id(), w = wave_id(), col = l & 15, four = (l >> 4) * 4;
    const int64_t L = a.seqlen;
    const int64_t id = walk_block((int64_t)a.batch * a.heads * a.nseg);
    const int64_t bh = id / a.nseg, seg = id - bh * a.nseg;
    const int64_t b = bh / a.heads, h = bh - b * a.heads;
    const bool rev = a.rev != 0;
    const int chunks = (int)((L + kC - 1) / kC);
    const int first = (int)seg * a.seg_chunks, last = min(chunks, first + a.seg_chunks) - 1;
    const T* xp = head_base<T>(a.x, b, h, a.heads, L);
    const T* yp = head_base<T>(a.y, b, h, a.heads, L);
    const T* zp = head_base<T>(a.z, b, h, a.heads, L);
    const T* ep = MODE != kWalkPlain ? head_base<T>(a.e, b, h, a.heads, L) : nullptr;
    TO* op = static_cast<TO*>(a.out) + bh * a.z.rows * L;

    State<KT, DT> S;
    const int64_t sz = (int64_t)a.x.rows * a.z.rows;
    S.load(a.nseg > 1 ? a.seg + (bh * a.nseg + seg) * sz : a.entry ? a.entry + bh * sz : nullptr, a);

    constexpr int64_t kBound = (int64_t)KT * DT * 4 * kWalkThreads;
    // boundary n of the row: the state there, stored (dq) or multiplied with the one that dq stored (dk)
    const auto bound_store = [&](int64_t n) {
        float* p = a.bound + (bh * (a.nb + 1) + n) * kBound + threadIdx.x * 4;
#pragma unroll
        for (int k = 0; k < KT; ++k)
#pragma unroll
            for (int d = 0; d < DT; ++d) *reinterpret_cast<f32x4*>(p + (k * DT + d) * 4 * kWalkThreads) = S.s[k][d];
    };
    const auto bound_dot = [&](int64_t n) {              // block-uniform
        const float* p = a.bound + (bh * (a.nb + 1) + n) * kBound + threadIdx.x * 4;
        float v = 0.0f;
#pragma unroll
        for (int k = 0; k < KT; ++k)
#pragma unroll
            for (int d = 0; d < DT; ++d) {
                const f32x4 o = *reinterpret_cast<const f32x4*>(p + (k * DT + d) * 4 * kWalkThreads);
#pragma unroll
                for (int r = 0; r < 4; ++r) v = fmaf(o[r], S.s[k][d][r], v);
            }
#pragma unroll
        for (int m = 1; m < 64; m *= 2) v += __shfl_xor(v, m);
        __syncthreads();
        if (l == 0) sm.xdot[w] = v;
        __syncthreads();
        if (threadIdx.x == 0)
            a.dot[bh * (a.nb + 1) + n] = (sm.xdot[0] + sm.xdot[1]) + (sm.xdot[2] + sm.xdot[3]);
    };

    TileRegs<T, KC> xr, yr;
    TileRegs<T, VP> zr, er;
    TokenDecay td{0.0f, 1};
    const int coef_wave = rev ? kWalkWaves - 1 : 0;     // the wave with the fewest products of x and y
    const auto load = [&](int chunk) {
        const int64_t t0 = (int64_t)chunk * kC;
        xr.load(xp, a.x.rows, t0, L);
        yr.load(yp, a.y.rows, t0, L);
        zr.load(zp, a.z.rows, t0, L);
        if constexpr (MODE != kWalkPlain) er.load(ep, a.e.rows, t0, L);
    };
    const auto load_td = [&](int chunk) {
        if (w == coef_wave) td = load_decay(a, b, h, (int64_t)chunk * kC + l);
    };
    // the decay's part of a finished chunk, from the waves' sums
    const auto flush_r = [&](int chunk) {
        if constexpr (MODE != kWalkPlain) {
            const int64_t t = (int64_t)chunk * kC + threadIdx.x;
            if (threadIdx.x < kC && t < L) {
                float v = (sm.dot[0][threadIdx.x] + sm.dot[1][threadIdx.x]) + (sm.dot[2][threadIdx.x] + sm.dot[3][threadIdx.x]);
                if constexpr (MODE == kWalkDq) {
                    const int i = threadIdx.x;
                    v += sm.rsum[i] - ((sm.csum[0][i] + sm.csum[1][i]) + (sm.csum[2][i] + sm.csum[3][i]));
                }
                a.r[bh * L + t] = v;
            }
        }
    };

    const int step = rev ? -1 : 1, begin = rev ? last : first, n = last - first + 1;
    if (threadIdx.x == 0) sm.c[0].bad[0] = sm.c[1].bad[0] = 0;
    load_td(begin);
    if (kAhead) load(begin);
    if (w == coef_wave) chunk_decay(td, rev, sm.c[0]);
    if (n > 1) load_td(begin + step);
    for (int it = 0; it < n; ++it) {
        const int chunk = begin + it * step;
        ChunkDecay& c = sm.c[it & 1];
        __syncthreads();                                // the tiles of the chunk before are read
        if (it > 0) flush_r(chunk - step);
        if (!kAhead) load(chunk);
        xr.store(sm.x);
        yr.store(sm.y);
        zr.store(sm.z);
        if constexpr (MODE != kWalkPlain) er.store(sm.e);
        if (!(yr.finite() && zr.finite())) c.bad[0] = 1;
        if constexpr (MODE == kWalkDq) {
            if (chunk > 0 && chunk % a.bound_chunks == 0) bound_store(chunk / a.bound_chunks);
        }
        if constexpr (MODE == kWalkDk) {
            const int next = chunk + 1;
            if (next < chunks ? next % a.bound_chunks == 0 : a.bound_end != 0)
                bound_dot((next + a.bound_chunks - 1) / a.bound_chunks);
        }
        __syncthreads();
        if (kAhead && it + 1 < n) load(chunk + step);

        // products of x and y, weighted: strip w of 16 x's
        {
            if (w == coef_wave && it + 1 < n) {
                ChunkDecay& cn = sm.c[(it + 1) & 1];
                chunk_decay(td, rev, cn);
                if (l == 0) cn.bad[0] = 0;
                if (it + 2 < n) load_td(chunk + 2 * step);
            }
            Frag xf[KT];
#pragma unroll
            for (int k = 0; k < KT; ++k) xf[k] = M::transposed(sm.x + k * 16 * kS + w * 16);
            const int xt = w * 16 + col;
            const float xhi = c.hi[xt], xlo = c.lo[xt];
            const int xstart = c.start[xt];
            float rs = 0.0f;
#pragma unroll
            for (int yt = 0; yt < 4; ++yt) {
                f32x4 d = {0, 0, 0, 0};
                T* pp = sm.p + xt * kS + yt * 16 + four;
                const bool needed = rev ? yt >= w : yt <= w;
                float cs[4] = {0, 0, 0, 0};
                if (needed) {
#pragma unroll
                    for (int k = 0; k < KT; k += 2)
                        d = M::mma(M::transposed(sm.y + k * 16 * kS + yt * 16), M::transposed(sm.y + (k + 1) * 16 * kS + yt * 16),
                                   xf[k], xf[k + 1], d);
                    const int y0 = yt * 16 + four;
                    const f32x4 yhi = *reinterpret_cast<const f32x4*>(&c.hi[y0]), ylo = *reinterpret_cast<const f32x4*>(&c.lo[y0]);
                    f32x4 p;
                    bool on[4];
#pragma unroll
                    for (int r = 0; r < 4; ++r) {
                        const int y = y0 + r;
                        on[r] = rev ? xt <= y && c.start[y] <= xt : y <= xt && xstart <= y;
                        const float dec = rev ? pair_decay(yhi[r], ylo[r], xhi, xlo) : pair_decay(xhi, xlo, yhi[r], ylo[r]);
                        p[r] = on[r] ? d[r] * (dec * a.pscale) : 0.0f;
                    }
                    if constexpr (MODE == kWalkDq) {
                        f32x4 d2 = {0, 0, 0, 0};
#pragma unroll
                        for (int k = 0; k < VT; k += 2)
                            d2 = M::mma(M::transposed(sm.z + k * 16 * kS + yt * 16), M::transposed(sm.z + (k + 1) * 16 * kS + yt * 16),
                                        M::transposed(sm.e + k * 16 * kS + w * 16), M::transposed(sm.e + (k + 1) * 16 * kS + w * 16), d2);
#pragma unroll
                        for (int r = 0; r < 4; ++r) {
                            const float wv = on[r] ? p[r] * d2[r] : 0.0f;
                            rs += wv;
                            cs[r] = sum16(wv);
                        }
                    }
                    *reinterpret_cast<Frag*>(pp) = M::round(p);
                } else if (rev ? (w & 1) && yt == w - 1 : !(w & 1) && yt == w + 1) {
                    *reinterpret_cast<Frag*>(pp) = M::round(d);      // the other half of a step of 32 tokens
                }
                if constexpr (MODE == kWalkDq) {
                    if (col == 0) *reinterpret_cast<f32x4*>(&sm.csum[w][yt * 16 + four]) = f32x4{cs[0], cs[1], cs[2], cs[3]};
                }
            }
            if constexpr (MODE == kWalkDq) {
                rs += __shfl_xor(rs, 16);
                rs += __shfl_xor(rs, 32);
                if (l < 16) sm.rsum[xt] = rs;
            }
        }
        __syncthreads();

        // out, from the state that enters the chunk and from the chunk's own products
        {
            f32x4 o[4][DT];
#pragma unroll
            for (int xt = 0; xt < 4; ++xt)
#pragma unroll
                for (int d = 0; d < DT; ++d) o[xt][d] = f32x4{0, 0, 0, 0};
#pragma unroll
            for (int k = 0; k < KT; k += 2) {
                Frag s0[DT][NO], s1[DT][NO];
#pragma unroll
                for (int d = 0; d < DT; ++d) {
                    M::template split<NO>(S.s[k][d], s0[d]);
                    M::template split<NO>(S.s[k + 1][d], s1[d]);
                }
#pragma unroll
                for (int xt = 0; xt < 4; ++xt) {
                    const Frag x0 = M::transposed(sm.x + k * 16 * kS + xt * 16), x1 = M::transposed(sm.x + (k + 1) * 16 * kS + xt * 16);
#pragma unroll
                    for (int d = 0; d < DT; ++d)
#pragma unroll
                        for (int q = 0; q < NO; ++q) o[xt][d] = M::mma(x0, x1, s0[d][q], s1[d][q], o[xt][d]);
                }
            }
            const bool bad = c.bad[0] != 0;
            const int64_t t0 = (int64_t)chunk * kC;
#pragma unroll
            for (int xt = 0; xt < 4; ++xt) {
                const int x0 = xt * 16 + four;
                const f32x4 in = *reinterpret_cast<const f32x4*>(&c.in[x0]);
                float rd[4] = {0, 0, 0, 0};
#pragma unroll
                for (int d = 0; d < DT; ++d) {
#pragma unroll
                    for (int r = 0; r < 4; ++r) o[xt][d][r] = in[r] < 0.0f ? 0.0f : o[xt][d][r] * (in[r] * a.iscale);
                    if constexpr (MODE != kWalkPlain) {
                        const f32x4 ev = M::widen(M::direct(sm.e + ((w * DT + d) * 16 + col) * kS + x0));
#pragma unroll
                        for (int r = 0; r < 4; ++r) rd[r] = in[r] < 0.0f ? 0.0f : fmaf(o[xt][d][r], ev[r], rd[r]);
                    }
                }
                if constexpr (MODE != kWalkPlain) {
#pragma unroll
                    for (int r = 0; r < 4; ++r) rd[r] = sum16(rd[r]);
                    if (col == 0)
                        *reinterpret_cast<f32x4*>(&sm.dot[w][x0]) = MODE == kWalkDk ? f32x4{-rd[0], -rd[1], -rd[2], -rd[3]}
                                                                                    : f32x4{rd[0], rd[1], rd[2], rd[3]};
                }
                if (!bad) {
#pragma unroll
                    for (int q = 0; q < 2; ++q) {
                        if (rev ? 2 * q + 1 < xt : 2 * q > xt) continue;
                        const T* pp = sm.p + (xt * 16 + col) * kS + q * 32 + four;
                        const Frag p0 = M::direct(pp), p1 = M::direct(pp + 16);
#pragma unroll
                        for (int d = 0; d < DT; ++d) {
                            const T* zz = sm.z + ((w * DT + d) * 16 + col) * kS + q * 32 + four;
                            o[xt][d] = M::mma(p0, p1, M::direct(zz), M::direct(zz + 16), o[xt][d]);
                        }
                    }
                } else {
#pragma unroll 1
                    for (int y = 0; y < kC; ++y)
#pragma unroll
                        for (int r = 0; r < 4; ++r) {
                            const int x = x0 + r;
                            if (!(rev ? x <= y && c.start[y] <= x : y <= x && c.start[x] <= y)) continue;
                            const float pv = Storage<T>::load1(sm.p + x * kS + y);
#pragma unroll
                            for (int d = 0; d < DT; ++d)
                                o[xt][d][r] = fmaf(pv, Storage<T>::load1(sm.z + ((w * DT + d) * 16 + col) * kS + y), o[xt][d][r]);
                        }
                }
#pragma unroll
                for (int d = 0; d < DT; ++d) {
                    const int zf = (w * DT + d) * 16 + col;
                    if (zf >= a.z.rows) continue;
                    float v[4] = {o[xt][d].x, o[xt][d].y, o[xt][d].z, o[xt][d].w};
                    TO* dst = op + (int64_t)zf * L;
                    if (t0 + x0 + 4 <= L) {
                        if constexpr (sizeof(TO) == 2)
                            *reinterpret_cast<u32x2_a2*>(dst + t0 + x0) = Mat<bf16_t>::round(o[xt][d]);
                        else
                            *reinterpret_cast<u32x4_a4*>(dst + t0 + x0) = Storage<float>::pack(v);
                    } else {
#pragma unroll
                        for (int r = 0; r < 4; ++r)
                            if (t0 + x0 + r < L) Storage<TO>::store1(dst + t0 + x0 + r, v[r]);
                    }
                }
            }
        }
        update<T, NS>(S, sm.y, sm.z, c, a.uscale);
    }
    if constexpr (MODE != kWalkPlain) {
        __syncthreads();
        flush_r(begin + (n - 1) * step);
    }
    const bool ends = rev ? seg == 0 : seg == a.nseg - 1;       // the state leaves the row
    if constexpr (MODE == kWalkDq) {
        if (ends && a.bound_end) bound_store(a.nb);
    }
    if (ends && a.leave) S.store(a.leave + bh * sz, a);
}

// --------------------------------------------------------------------------------------------
// split rows: what each segment adds to the state (aggregate), then the states that enter the
// segments one after another (chain)
// --------------------------------------------------------------------------------------------
template <typename T, int KC, int VP>
struct AggSmem {
    __attribute__((aligned(16))) T y[KC * Mat<T>::kStride];
    __attribute__((aligned(16))) T z[VP * Mat<T>::kStride];
    ChunkDecay c[2];
};

template <typename T, int KC, int VP, int NS>
__global__ __launch_bounds__(kWalkThreads) void walk_aggregate(WalkArgs a) {
    constexpr int KT = KC / 16, DT = VP / (16 * kWalkWaves);
    __shared__ AggSmem<T, KC, VP> sm;
    const int l = lane_id(), w = wave_id();
    const int64_t L = a.seqlen;
    // the segment that nothing enters after it is left out
    const int64_t id = walk_block((int64_t)a.batch * a.heads * (a.nseg - 1));
    const int64_t bh = id / (a.nseg - 1);
    const bool rev = a.rev != 0;
    const int64_t seg = id - bh * (a.nseg - 1) + (rev ? 1 : 0);
    const int64_t b = bh / a.heads, h = bh - b * a.heads;
    const int chunks = (int)((L + kC - 1) / kC);
    const int first = (int)seg * a.seg_chunks, last = min(chunks, first + a.seg_chunks) - 1;
    const T* yp = head_base<T>(a.y, b, h, a.heads, L);
    const T* zp = head_base<T>(a.z, b, h, a.heads, L);
    State<KT, DT> S;
    S.load(nullptr, a);
    float all = 1.0f;
    TileRegs<T, KC> yr;
    TileRegs<T, VP> zr;
    const int step = rev ? -1 : 1, begin = rev ? last : first, n = last - first + 1;
    if (threadIdx.x == 0) sm.c[0].bad[0] = sm.c[1].bad[0] = 0;
    TokenDecay td{0.0f, 1};
    if (w == 0) {
        td = load_decay(a, b, h, (int64_t)begin * kC + l);
        chunk_decay(td, rev, sm.c[0]);
        if (n > 1) td = load_decay(a, b, h, (int64_t)(begin + step) * kC + l);
    }
    yr.load(yp, a.y.rows, (int64_t)begin * kC, L);
    zr.load(zp, a.z.rows, (int64_t)begin * kC, L);
    for (int it = 0; it < n; ++it) {
        const int chunk = begin + it * step;
        ChunkDecay& c = sm.c[it & 1];
        __syncthreads();
        yr.store(sm.y);
        zr.store(sm.z);
        if (!(yr.finite() && zr.finite())) c.bad[0] = 1;
        __syncthreads();
        if (it + 1 < n) {
            yr.load(yp, a.y.rows, (int64_t)(chunk + step) * kC, L);
            zr.load(zp, a.z.rows, (int64_t)(chunk + step) * kC, L);
            if (w == 0) {
                ChunkDecay& cn = sm.c[(it + 1) & 1];
                chunk_decay(td, rev, cn);
                if (l == 0) cn.bad[0] = 0;
                if (it + 2 < n) td = load_decay(a, b, h, (int64_t)(chunk + 2 * step) * kC + l);
            }
        }
        update<T, NS>(S, sm.y, sm.z, c, a.uscale);
        all = c.a < 0.0f || all < 0.0f ? -1.0f : all * c.a;
    }
    const int64_t sz = (int64_t)a.x.rows * a.z.rows;
    S.store(a.seg + (bh * a.nseg + seg) * sz, a);
    if (threadIdx.x == 0) a.seg_a[bh * a.nseg + seg] = all;
}

// --------------------------------------------------------------------------------------------
// launches: one T, TO and KC in each translation unit
// --------------------------------------------------------------------------------------------
template <typename T, typename TO, int KC, int VP, int MODE, int NS, int NO>
hipError_t launch_walk_one(const WalkArgs& a, hipStream_t s) {
    const int64_t blocks = (int64_t)a.batch * a.heads * a.nseg;
    hipLaunchKernelGGL((walk_kernel<T, TO, KC, VP, MODE, NS, NO>), dim3((unsigned)blocks), dim3(kWalkThreads), 0, s, a);
    return hipGetLastError();
}

template <typename T, typename TO, int KC, int VP>
hipError_t launch_walk_vp(const WalkArgs& a, WalkMode mode, bool exact, hipStream_t s) {
    constexpr int kAll = Mat<T>::kSplit ? 3 : 1, kSome = Mat<T>::kSplit ? 2 : 1;
    switch (mode) {
        case kWalkDq: return launch_walk_one<T, TO, KC, VP, kWalkDq, kAll, kAll>(a, s);
        case kWalkDk: return launch_walk_one<T, TO, KC, VP, kWalkDk, kAll, kAll>(a, s);
        default:
            if (exact) return launch_walk_one<T, TO, KC, VP, kWalkPlain, kAll, 1>(a, s);
            return launch_walk_one<T, TO, KC, VP, kWalkPlain, kSome, 1>(a, s);
    }
}

template <typename T, typename TO, int KC>
hipError_t launch_walk_kc(const WalkArgs& a, WalkMode mode, bool exact, hipStream_t s) {
    return a.z.rows <= 64 ? launch_walk_vp<T, TO, KC, 64>(a, mode, exact, s)
                          : launch_walk_vp<T, TO, KC, 128>(a, mode, exact, s);
}

}  // namespace pm
